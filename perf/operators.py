"""Timed calls of the paged-cache attention operators: inputs, a plain form, an fp64 reference.

Five operators of a serving program that keeps the keys and values of its
requests in pages of a shared cache:

  tables   block tables and slots of the new tokens from the request lengths
  append   the new tokens' K and V rows written into their slots, with the 8-bit
           summary (mean key) of every page that they touch
  attend   attention of the new tokens over the cached rows of their request
  select   per query and KV head, the pages with the best 8-bit score
  sparse   attention of every query over its selected pages

`own` chooses between the library's entry points and the plain form, which is
made of elementary torch operations in fp32 (sums whose rounding decides whole
numbers are taken in fp64 and rounded once, so that their order does not
matter).  A case's lengths follow from its values alone (`mix` seeds them);
tensors and the pages' order follow from the seed.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BIG = torch.finfo(torch.float32).max


def listed():
    cases = [
        # one decode step of a batch: every request one token further
        dict(name="tables_decode_64", op="tables", mix=1, R=64, ctx=[1, 8192], new=[1, 1], P=64),
        # a step that admits new requests beside running ones, small pages
        dict(name="tables_admit_1024", op="tables", mix=2, R=1024, ctx=[0, 16384], new=[0, 40], P=16),
        # K and V of one decode step
        dict(name="append_decode_64", op="append", mix=3, R=64, ctx=[1, 2048], new=[1, 1], P=64, Hq=32, Hkv=8, D=128, dtype="bf16"),
        # K and V of chunks of prompts, of odd lengths
        dict(name="append_chunk_8k", op="append", mix=4, R=9, ctx=[0, 4001], new=[501, 1501], P=32, Hq=16, Hkv=4, D=64, dtype="fp16"),
        # a small model in fp32 answers four users
        dict(name="attend_small_fp32", op="attend", mix=5, R=4, ctx=[300, 1000], new=[1, 1], P=16, Hq=8, Hkv=2, D=64, dtype="fp32", window=0, lse=False),
        # one decode step of a batch of ragged contexts
        dict(name="attend_decode_64", op="attend", mix=6, R=64, ctx=[512, 16384], new=[1, 1], P=64, Hq=32, Hkv=8, D=128, dtype="bf16", window=0, lse=False),
        # two long prompts in chunks
        dict(name="attend_chunk_4k", op="attend", mix=7, R=2, ctx=[6000, 14000], new=[2001, 2100], P=64, Hq=32, Hkv=8, D=128, dtype="bf16", window=0, lse=False),
        # chunks and single tokens in one batch, sliding window with the pages behind it given back, parts to be joined later
        dict(name="attend_mixed_window", op="attend", mix=8, R=24, ctx=[1, 4096], new=[1, 512], P=32, Hq=16, Hkv=4, D=64, dtype="fp16", window=1024, lse=True),
        # one decode step: pages of long contexts
        dict(name="select_decode_32", op="select", mix=9, R=32, ctx=[8192, 65536], new=[1, 1], P=64, Hq=32, Hkv=8, D=128, dtype="bf16", top=32, first=1, local=2),
        # a chunk behind a long context
        dict(name="select_chunk_2k", op="select", mix=10, R=2, ctx=[20000, 70000], new=[1001, 1024], P=64, Hq=32, Hkv=8, D=128, dtype="bf16", top=16, first=1, local=2),
        # the attention of the two selections above
        dict(name="sparse_decode_32", op="sparse", mix=9, R=32, ctx=[8192, 65536], new=[1, 1], P=64, Hq=32, Hkv=8, D=128, dtype="bf16", top=32, lse=False),
        dict(name="sparse_chunk_2k", op="sparse", mix=10, R=2, ctx=[20000, 70000], new=[1001, 1024], P=64, Hq=32, Hkv=8, D=128, dtype="bf16", top=16, lse=False),
    ]
    return [_case(c) for c in cases]


def _spread(rng, lo, hi):
    """Log-uniform whole number of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 0.5)), math.log(max(hi, 0.5))))))))


def _case(c):
    """The case with the ends of its ranges as values of their own."""
    c = dict(c)
    for key in ("ctx", "new"):
        c[key + "_lo"], c[key + "_hi"] = c.pop(key)
    return c


def draw(rng):
    op = rng.choice(["tables", "append", "attend", "attend", "select", "sparse"])
    c = dict(op=op, mix=rng.randrange(1 << 30), P=rng.choice([16, 32, 64, 128]))
    if op == "tables":
        c["R"] = _spread(rng, 1, 1024)
        c["ctx"] = [rng.choice([0, 1]), _spread(rng, 64, 16384)]
        c["new"] = rng.choice([[1, 1], [0, 7], [0, 40]]) if c["R"] >= 8 else [1, 40]
        return _case(c)
    c["D"] = rng.choice([64, 128])
    c["Hkv"] = rng.choice([1, 2, 4, 8])
    c["Hq"] = c["Hkv"] * rng.choice([1, 2, 4, 5, 7, 8])
    c["dtype"] = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "append":
        c["R"] = _spread(rng, 1, 64)
        c["ctx"] = [0, _spread(rng, 16, 2048)]
        c["new"] = [1, 1] if rng.random() < 0.4 else [1, max(2, 8000 // c["R"])]
        return _case(c)
    decode = rng.random() < 0.5
    if op == "attend":
        most = _spread(rng, 16, 8192)
        c["R"] = _spread(rng, 1, 48) if decode else _spread(rng, 1, 16)
        c["ctx"] = [rng.choice([0, 1, most // 4]), most]
        c["new"] = [1, rng.choice([1, 1, 3])] if decode else [1, max(2, _spread(rng, 32, 1600) // c["R"])]
        c["window"] = rng.choice([0, 0, 0, 100, 1024])
        c["lse"] = rng.random() < 0.5
        return _case(c)
    most = _spread(rng, 1024, 65536)
    c["R"] = _spread(rng, 1, 32) if decode else _spread(rng, 1, 4)
    c["ctx"] = [most // 8, most]
    c["new"] = [1, 1] if decode else [1, max(2, _spread(rng, 64, 1800) // c["R"])]
    c["top"] = rng.choice([4, 8, 16])
    if op == "select":
        c["first"], c["local"] = rng.choice([0, 1]), rng.choice([1, 2])
        c["ctx"] = [max(2 * c["top"] * c["P"], most // 8), max(3 * c["top"] * c["P"], most)]  # there is something to choose from
    else:
        c["P"] = min(c["P"], 64)
        c["lse"] = rng.random() < 0.5
    return _case(c)


def _lengths(c):
    """Cached and new tokens of every request."""
    rng = random.Random(c["mix"])
    ctx = [_spread(rng, c["ctx_lo"], c["ctx_hi"]) for _ in range(c["R"])]
    new = [_spread(rng, c["new_lo"], c["new_hi"]) for _ in range(c["R"])]
    return ctx, new


# ---------------------------------------------------------------- inputs


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ctx, new = _lengths(case)
    R, P, op = case["R"], case["P"], case["op"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    have = [-(-c // P) if op in ("tables", "append") else -(-(c + n) // P) for c, n in zip(ctx, new)]
    want = [-(-(c + n) // P) for c, n in zip(ctx, new)]
    T, W, pages = sum(new), max(want) + 3, sum(want) + 5
    order = torch.randperm(pages, device="cuda", generator=g, dtype=torch.int32)
    col = torch.arange(W, device="cuda")
    begin = ints(have).cumsum(0) - ints(have)
    held = col < ints(have)[:, None]
    table = torch.where(held, order[(begin[:, None] + col).clamp(max=pages - 1)], -1).contiguous()
    s = dict(case=case, T=T, table=table, ctx=ints(ctx), new=ints(new))
    free = order[sum(have):].contiguous()
    if op == "tables":
        s["free"] = free
        return s
    n = ints(new)
    s["seq"] = ints([c + k for c, k in zip(ctx, new)])
    s["qptr"] = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), n.cumsum(0).to(torch.int32)])
    Hq, Hkv, D, t = case["Hq"], case["Hkv"], case["D"], TYPES[case["dtype"]]
    # one projection gives q, k and v side by side
    qkv = torch.randn(T, Hq + 2 * Hkv, D, device="cuda", generator=g).mul_(1.5).to(t)
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    if op != "select":
        s["kc"] = torch.randn(pages, P, Hkv, D, device="cuda", generator=g, dtype=t)
        s["vc"] = torch.randn(pages, P, Hkv, D, device="cuda", generator=g, dtype=t)
    if op in ("append", "select"):
        s["kq"] = torch.randn(pages, Hkv, D, device="cuda", generator=g).mul_(45).round_().clamp_(-127, 127).to(torch.int8)
        s["ks"] = torch.rand(pages, Hkv, device="cuda", generator=g).mul_(0.004).add_(0.001)
    if op == "append":
        r = torch.repeat_interleave(torch.arange(R, device="cuda"), n)
        pos = s["ctx"][r] + torch.arange(T, device="cuda") - s["qptr"][r]
        grow = ints(want) - ints(have)
        at = (grow.cumsum(0) - grow - ints(have))[:, None] + col
        full = torch.where(held, table, free[at.clamp(0, free.numel() - 1)])
        s["slots"] = full[r, pos // P].long() * P + pos % P
        return s
    if op in ("attend", "sparse"):
        # rows past a request's end hold whatever was there before
        last = (s["seq"] - 1).clamp(min=0)
        page = table[torch.arange(R, device="cuda"), last // P].long()
        stale = (torch.arange(P, device="cuda") > (last % P)[:, None]) & (s["seq"] > 0)[:, None]
        for x in (s["kc"], s["vc"]):
            x[page] = torch.where(stale[:, :, None, None], torch.full((), float("nan"), device="cuda", dtype=t), x[page])
    if case.get("window"):
        behind = (s["ctx"] - case["window"] + 1).clamp(min=0) // P  # pages that no new token sees
        s["table"] = torch.where(col < behind[:, None], -1, table).contiguous()
    if op == "sparse":
        top = case["top"]
        r = torch.repeat_interleave(torch.arange(R, device="cuda"), n)
        p = s["ctx"][r] + torch.arange(T, device="cuda") - s["qptr"][r]
        near = p // P
        rank = torch.rand(T, Hkv, W, device="cuda", generator=g)
        rank = torch.where(col[None, None] <= near[:, None, None], rank, -1.0)
        rank = torch.where(col[None, None] == near[:, None, None], 2.0, rank)
        val, at = rank.topk(min(top, W), dim=2)
        at = torch.where(val >= 0, at, W).sort(dim=2).values
        s["sel"] = torch.full((T, Hkv, top), -1, dtype=torch.int32, device="cuda")
        s["sel"][:, :, :at.shape[2]] = torch.where(at < W, at, -1).to(torch.int32)
    return s


# ---------------------------------------------------------------- the calls


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2205_11622_amd as slnr

    c = s["case"]
    if c["op"] == "tables":
        return *slnr.sparselnr_page_tables(s["ctx"], s["new"], s["table"], s["free"], s["T"], c["P"]), s["table"]
    if c["op"] == "append":
        slnr.sparselnr_cache_append(s["k"], s["v"], s["slots"], s["kc"], s["vc"], s["kq"], s["ks"])
        return s["kc"], s["vc"], s["kq"].float() * s["ks"][:, :, None]
    if c["op"] == "attend":
        lse = torch.empty(s["T"], c["Hq"], device="cuda") if c["lse"] else None
        out = slnr.sparselnr_paged_attention(s["q"], s["kc"], s["vc"], s["table"], s["seq"], s["qptr"], window=c["window"], max_new=c["new_hi"], lse=lse)
        return (out, lse) if c["lse"] else out
    if c["op"] == "select":
        return slnr.sparselnr_block_select(s["q"], s["kq"], s["ks"], s["table"], s["seq"], s["qptr"], c["P"], c["top"], first=c["first"], local=c["local"])
    lse = torch.empty(s["T"], c["Hq"], device="cuda") if c["lse"] else None
    out = slnr.sparselnr_block_attention(s["q"], s["kc"], s["vc"], s["table"], s["seq"], s["qptr"], s["sel"], lse=lse)
    return (out, lse) if c["lse"] else out


def _run_plain(s):
    return {"tables": _tables, "append": _append, "attend": _attend, "select": _select, "sparse": _sparse}[s["case"]["op"]](s)


# ---------------------------------------------------------------- plain forms


def _tables(s):
    ctx, new, table, free, P, T = s["ctx"], s["new"], s["table"], s["free"], s["case"]["P"], s["T"]
    R, W = table.shape
    seq = ctx + new
    qptr = torch.cat([ctx.new_zeros(1), new.cumsum(0).to(torch.int32)])
    have, want = (ctx + P - 1) // P, (seq + P - 1) // P
    taken = (want - have).cumsum(0)
    j = torch.arange(W, device="cuda")
    at = (taken - (want - have) - have)[:, None] + j
    fresh = (j >= have[:, None]) & (j < want[:, None])
    given = torch.where(at < free.numel(), free[at.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where(fresh, given, table))
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(qptr[1:], t, right=True).clamp(max=R - 1)
    pos = ctx[r] + t - qptr[r]
    page = torch.where(pos // P < W, table[r, (pos // P).clamp(max=W - 1)], -1).long()
    slots = torch.where((page >= 0) & (t < qptr[R]), page * P + pos % P, -1)
    lost = ((slots < 0) & (t < qptr[R])).sum()
    counts = torch.stack([qptr[R].long(), taken[-1], lost]).to(torch.int32)
    return qptr, seq, slots, counts, table


def _append(s):
    k, v, slots, kc, vc, kq, ks, P = s["k"], s["v"], s["slots"], s["kc"], s["vc"], s["kq"], s["ks"], s["case"]["P"]
    page, row = slots // P, slots % P
    kc[page, row] = k
    vc[page, row] = v
    after = torch.cat([slots[1:], slots.new_full((1,), -1)])
    done = ((after != slots + 1) | (row == P - 1)).nonzero()[:, 0]  # the last new row of each page
    page, row = page[done], row[done]
    seen = torch.arange(P, device="cuda") <= row[:, None]
    total = torch.where(seen[:, :, None, None], kc[page].float(), 0.0).double().sum(1)
    mean = (total / (row + 1).double()[:, None, None]).float()
    most = mean.abs().amax(2)
    fine = torch.isfinite(most)
    step = torch.where(fine, most / 127, math.inf)
    whole = (mean / step[:, :, None]).round().clamp(-127, 127)
    kq[page] = torch.where((fine & (step > 0))[:, :, None], whole, 0.0).to(torch.int8)
    ks[page] = step
    return kc, vc, kq.float() * ks[:, :, None]


def _padded(s):
    """Token of every place of a rectangle R x longest chunk, its position, and whether there is one."""
    n = s["qptr"][1:] - s["qptr"][:-1]
    at = torch.arange(max(_lengths(s["case"])[1]), device="cuda")
    there = at < n[:, None]
    token = torch.where(there, s["qptr"][:-1, None] + at, 0)
    return token, (s["seq"] - n)[:, None] + at, there


def _attend(s):
    c, q, table = s["case"], s["q"], s["table"]
    P, Hq, Hkv, D, window = c["P"], c["Hq"], c["Hkv"], c["D"], c["window"]
    token, pos, there = _padded(s)
    R, N = token.shape
    longest = max(a + b for a, b in zip(*_lengths(c)))
    j = torch.arange(longest, device="cuda")
    page = table[:, j // P].long()
    live = (page >= 0) & (j < s["seq"][:, None])  # R, S
    rows = page.clamp(min=0), (j % P).expand_as(page)
    K = torch.where(live[:, :, None, None], s["kc"][rows].float(), 0.0)  # R, S, Hkv, D
    V = torch.where(live[:, :, None, None], s["vc"][rows].float(), 0.0)
    Q = q[token].float().view(R, N, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(R, Hkv, -1, D)
    x = (Q @ K.permute(0, 2, 3, 1).contiguous()).mul_(1 / math.sqrt(D)).view(R, Hkv, -1, N, longest)
    seen = live[:, None] & (j <= pos[:, :, None])  # R, N, S
    if window:
        seen &= j > pos[:, :, None] - window
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(4, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    x.sub_(top).exp_()
    total = x.sum(4, keepdim=True)
    o = (x.view(R, Hkv, -1, longest) @ V.permute(0, 2, 1, 3).contiguous()).view(R, Hkv, -1, N, D)
    o = torch.where(total == 0, 0.0, o / total).permute(0, 3, 1, 2, 4).reshape(R, N, Hq, D)[there].to(q.dtype)
    if not c["lse"]:
        return o
    return o, (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(R, N, Hq)[there]


def _select(s):
    c, q, table = s["case"], s["q"], s["table"]
    P, Hkv, D, top = c["P"], c["Hkv"], c["D"], c["top"]
    token, pos, there = _padded(s)
    R, N = token.shape
    W = table.shape[1]
    u = q.view(s["T"], Hkv, -1, D).double().sum(2).float()
    most = u.abs().amax(2, keepdim=True)
    step = most / 127
    q8 = torch.where((step > 0) & torch.isfinite(most), (u / step).round().clamp(-127, 127), 0.0)[token]  # R, N, Hkv, D
    page = table.long().clamp(min=0)
    k8 = s["kq"][page].float().permute(0, 2, 3, 1).contiguous()  # R, Hkv, D, W
    score = q8.permute(0, 2, 1, 3) @ k8  # whole numbers below 2^24
    score = score * s["ks"][page].permute(0, 2, 1)[:, :, None]
    score = score.nan_to_num(nan=BIG, posinf=BIG, neginf=-BIG)
    b, near = torch.arange(W, device="cuda"), (pos // P)[:, None, :, None]
    score = torch.where((b < c["first"]) | (b > near - c["local"]), math.inf, score)
    score = torch.where((b <= near) & (table >= 0)[:, None, None], score, -math.inf)
    val, at = score.sort(dim=3, descending=True, stable=True)
    at = torch.where(val[..., :top] > -math.inf, at[..., :top], W).sort(dim=3).values
    sel = torch.full((R, N, Hkv, top), -1, dtype=torch.int32, device="cuda")
    sel[..., :at.shape[3]] = torch.where(at < W, at, -1).permute(0, 2, 1, 3).to(torch.int32)
    return sel[there]


def _sparse(s):
    c, q, sel = s["case"], s["q"], s["sel"].long()
    P, Hq, Hkv, D, T = c["P"], c["Hq"], c["Hkv"], c["D"], s["T"]
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(s["qptr"][1:], t, right=True)
    pos = s["seq"][r] - s["qptr"][r + 1] + t
    page = s["table"][r[:, None, None], sel.clamp(min=0)].long()
    page = torch.where(sel >= 0, page, -1)
    i = torch.arange(P, device="cuda")
    live = ((page >= 0)[..., None] & (sel[..., None] * P + i <= pos[:, None, None, None])).view(T, Hkv, -1)
    h = torch.arange(Hkv, device="cuda")[:, None, None]
    rows = page.clamp(min=0)[..., None], i, h
    K = torch.where(live[..., None], s["kc"][rows].view(T, Hkv, -1, D).float(), 0.0)
    Q = q.float().view(T, Hkv, -1, D)
    x = (Q @ K.transpose(2, 3).contiguous()) * (1 / math.sqrt(D))
    x = torch.where(live[:, :, None], x, -math.inf)
    top = x.amax(3, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    x = (x - top).exp()
    total = x.sum(3, keepdim=True)
    V = torch.where(live[..., None], s["vc"][rows].view(T, Hkv, -1, D).float(), 0.0)
    o = torch.where(total == 0, 0.0, (x @ V) / total).view(T, Hq, D).to(q.dtype)
    return (o, (top + total.log()).view(T, Hq)) if c["lse"] else o


# ---------------------------------------------------------------- work and reference


def _seen(c, ctx, new):
    """Pairs of query and key, and keys that some query sees, of one request."""
    w = c.get("window") or ctx + new
    if ctx + 1 >= w:
        return new * w, min(ctx + new, new + w - 1)
    grow = min(new, w - ctx)  # queries that still see every key
    return grow * ctx + grow * (grow + 1) // 2 + (new - grow) * w, ctx + new


def work(case):
    """Every input that the results depend on read once, every output written once; the multiplications and additions of the definition."""
    ctx, new = _lengths(case)
    op, P, R, T = case["op"], case["P"], case["R"], sum(_lengths(case)[1])
    fresh = sum(-(-(c + n) // P) - -(-c // P) for c, n in zip(ctx, new))
    if op == "tables":
        return {"bytes": 8 * R + 4 * fresh + 4 * R + 4 * (R + 1) + 4 * R + 8 * T + 4 * fresh + 12, "flops": 4 * R + 4 * T}
    e, Hq, Hkv, D = 4 if case["dtype"] == "fp32" else 2, case["Hq"], case["Hkv"], case["D"]
    row = Hkv * D * e
    if op == "append":
        touched = sum(-(-(c + n) // P) - c // P for c, n in zip(ctx, new) if n)
        old = sum(c % P for c, n in zip(ctx, new) if n)
        return {"bytes": 4 * T * row + 8 * T + old * row + touched * Hkv * (D + 4), "flops": (T + old) * Hkv * D + 4 * touched * Hkv * D}
    pages = sum(-(-(c + n) // P) for c, n in zip(ctx, new))
    ids = 4 * (2 * R + 1) + 4 * pages
    if op == "attend":
        pairs, keys = (sum(x) for x in zip(*(_seen(case, c, n) for c, n in zip(ctx, new))))
        return {"bytes": ids + 2 * T * Hq * D * e + 2 * keys * row + (4 * T * Hq if case["lse"] else 0), "flops": 4 * pairs * Hq * D}
    if op == "select":
        pairs = sum((c + i) // P + 1 for c, n in zip(ctx, new) for i in range(n))
        return {"bytes": ids + T * Hq * D * e + pages * Hkv * (D + 4) + 4 * T * Hkv * case["top"], "flops": (2 * pairs * Hkv + T * Hq) * D}
    top = case["top"]
    picked = sum(min(top, (c + i) // P + 1) * P for c, n in zip(ctx, new) for i in range(n))
    keys = sum(min(c + n, top * P * n) for c, n in zip(ctx, new))  # a row that two queries select need be read once only
    return {"bytes": ids + 4 * T * Hkv * top + 2 * T * Hq * D * e + 2 * keys * row + (4 * T * Hq if case["lse"] else 0), "flops": 4 * picked * Hq * D}


def exact(case, seed):
    """fp64, one request and one head after the other; whole numbers have no such value."""
    op = case["op"]
    if op in ("tables", "select"):
        return None
    s = prepare(case, seed)
    P, Hq, Hkv, D, T = case["P"], case["Hq"], case["Hkv"], case["D"], s["T"]
    kc, vc = s["kc"], s["vc"]
    if op == "append":
        kc, vc, stand = kc.double(), vc.double(), s["kq"].double() * s["ks"].double()[:, :, None]
        ctx, new = _lengths(case)
        at = 0
        for c, n in zip(ctx, new):
            slots = s["slots"][at:at + n]
            kc.view(-1, Hkv, D)[slots], vc.view(-1, Hkv, D)[slots] = s["k"][at:at + n].double(), s["v"][at:at + n].double()
            for b in range(c // P, -(-(c + n) // P)):
                page = int(slots[max(0, b * P - c)]) // P
                mean = kc[page, :min(P, c + n - b * P)].mean(0).float().double()
                step = mean.abs().amax(1, keepdim=True) / 127
                stand[page] = torch.where(step > 0, (mean / step).round(), 0.0) * step
            at += n
        return kc, vc, stand
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    qptr, seq, G = s["qptr"].tolist(), s["seq"].tolist(), Hq // Hkv
    for r in range(case["R"]):
        a, b, S = qptr[r], qptr[r + 1], seq[r]
        p = torch.arange(S - (b - a), S, device="cuda")[:, None]
        if op == "attend":
            j = torch.arange(S, device="cuda")
            page = s["table"][r].long().repeat_interleave(P)[:S]
            ok = (page >= 0) & (j <= p)
            if case["window"]:
                ok = ok & (p - j < case["window"])
            rows = page.clamp(min=0) * P + j % P
            for h in range(Hkv):
                k, v = (torch.where((page >= 0)[:, None], x.reshape(-1, Hkv, D)[rows, h], 0).double() for x in (kc, vc))
                for g in range(h * G, (h + 1) * G):
                    x = (s["q"][a:b, g].double() @ k.t().contiguous() / D ** 0.5).masked_fill(~ok, -math.inf)
                    lse[a:b, g] = torch.logsumexp(x, 1)
                    out[a:b, g] = (x - lse[a:b, g, None]).exp().nan_to_num(0.0) @ v
            continue
        for t0 in range(a, b, 128):
            t1 = min(b, t0 + 128)
            sel = s["sel"][t0:t1].long()
            j = (sel[..., None] * P + torch.arange(P, device="cuda")).flatten(2)  # t, Hkv, keys
            page = torch.where(sel >= 0, s["table"][r].long()[sel.clamp(min=0)], -1).repeat_interleave(P, dim=2)
            ok = (page >= 0) & (j <= p[t0 - a:t1 - a, :, None])
            rows = page.clamp(min=0) * P + j.clamp(min=0) % P
            for h in range(Hkv):
                k, v = (torch.where(ok[:, h, :, None], x.reshape(-1, Hkv, D)[rows[:, h], h], 0).double() for x in (kc, vc))
                for g in range(h * G, (h + 1) * G):
                    x = ((k * s["q"][t0:t1, g, None].double()).sum(2) / D ** 0.5).masked_fill(~ok[:, h], -math.inf)
                    lse[t0:t1, g] = torch.logsumexp(x, 1)
                    out[t0:t1, g] = ((x - lse[t0:t1, g, None]).exp().nan_to_num(0.0)[..., None] * v).sum(1)
    return (out, lse) if case["lse"] else out
