"""Timed calls of a paged cache in 4 bits and of its pages' life: inputs, a plain form, an fp64 reference.

Five operators of a serving program that keeps the keys and values of its
requests in pages of a shared cache:

  append   the new tokens' K and V rows into their slots in 4 bits, and the values
           that these then stand for
  attend   attention of the new tokens over the 4-bit rows of their requests
  fork     block table rows that share the pages of others, and the copies of the
           pages that are not full
  free     rows given up, and the list of pages that no row holds any more
  compact  the pages in use moved to the front of the cache, and the tables after them

A row of 4-bit values is groups of 32 along the head dimension (the last one filled
up with zeros), each with a power of two: two values of {0, 0.5, 1, 1.5, 2, 3, 4, 6}
with a sign to a byte, the first in the low half, and a byte e + 127 for each group.

`own` chooses between the library's entry points and the plain form, which is made
of elementary torch operations in fp32.  A case's lengths follow from its values
alone (`mix` seeds them); tensors and the pages' order follow from the seed.  Table
rows, lengths and shares that a call changes lie in one array, which each pass
begins by setting back, so that every pass has the same to do.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# exponents of a group by type: 0.5 * 2^e and 6 * 2^e are values of the type
LEAST = {"bf16": -125, "fp16": -23, "fp32": -125}
MOST = {"bf16": 125, "fp16": 13, "fp32": 125}


def listed():
    cases = [
        # K and V of one decode step of a batch
        dict(name="append_decode_64", op="append", mix=21, R=64, ctx=[1, 2048], new=[1, 1], P=64, Hq=32, Hkv=8, D=128, dtype="bf16", by_head=True),
        # K and V of chunks of prompts, a head dimension that does not fill its groups, small pages in the order of tokens
        dict(name="append_chunk_5k", op="append", mix=22, R=7, ctx=[0, 3001], new=[301, 1499], P=16, Hq=16, Hkv=4, D=80, dtype="fp16", by_head=False),
        # a small model in fp32 answers three users
        dict(name="attend_small_fp32", op="attend", mix=23, R=3, ctx=[200, 900], new=[1, 1], P=16, Hq=8, Hkv=2, D=64, dtype="fp32", window=0, lse=False, by_head=True),
        # one decode step of a batch of ragged contexts
        dict(name="attend_decode_96", op="attend", mix=24, R=96, ctx=[400, 20000], new=[1, 1], P=64, Hq=32, Hkv=8, D=128, dtype="bf16", window=0, lse=False, by_head=True),
        # two long prompts in chunks
        dict(name="attend_chunk_4k", op="attend", mix=25, R=2, ctx=[5000, 13000], new=[1901, 2100], P=64, Hq=32, Hkv=8, D=128, dtype="bf16", window=0, lse=False, by_head=True),
        # chunks and single tokens in one batch, sliding window with the pages behind it given back, parts to be joined later
        dict(name="attend_mixed_window", op="attend", mix=26, R=20, ctx=[1, 6000], new=[1, 400], P=32, Hq=16, Hkv=4, D=96, dtype="fp16", window=1000, lse=True, by_head=False),
        # a few beams go on from some of the running ones
        dict(name="fork_beams_12", op="fork", mix=27, R=32, n=12, parents=4, ctx=[100, 2000], P=32, Hkv=8, D=64, dtype="bf16"),
        # many answers to each of some prompts
        dict(name="fork_samples_256", op="fork", mix=28, R=300, n=256, parents=8, ctx=[1000, 9000], P=64, Hkv=8, D=128, dtype="bf16"),
        # requests that are done, of a small batch
        dict(name="free_few_6", op="free", mix=29, R=48, n=6, group=3, ctx=[50, 3000], P=64),
        # a large batch ends, much of it over shared prompts
        dict(name="free_many_700", op="free", mix=30, R=1000, n=700, group=5, ctx=[500, 8192], P=16),
        # a small cache is tidied up
        dict(name="compact_small", op="compact", mix=31, R=24, group=2, ctx=[10, 1200], P=16, Hkv=2, D=64, dtype="fp32", used=0.3),
        # the free part of a large cache is to be given back
        dict(name="compact_large", op="compact", mix=32, R=80, group=4, ctx=[200, 8000], P=64, Hkv=8, D=128, dtype="bf16", used=0.4),
    ]
    return [_case(c) for c in cases]


def _spread(rng, lo, hi):
    """Log-uniform whole number of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 0.5)), math.log(max(hi, 0.5))))))))


def _case(c):
    """The case with the ends of its ranges as values of their own."""
    c = dict(c)
    for key in ("ctx", "new"):
        if key in c:
            c[key + "_lo"], c[key + "_hi"] = c.pop(key)
    return c


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "fork", "free", "compact"])
    c = dict(op=op, mix=rng.randrange(1 << 30), P=rng.choice([16, 32, 64, 128]))
    if op == "free":
        c["R"] = _spread(rng, 2, 1000)
        c["n"] = _spread(rng, 1, c["R"])
        c["group"] = rng.choice([1, 2, 5])
        c["ctx"] = [_spread(rng, 1, 64), _spread(rng, 64, 8192)]
        return _case(c)
    c["D"] = rng.choice([64, 80, 96, 128, 128])
    c["Hkv"] = rng.choice([1, 2, 4, 8])
    c["dtype"] = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("fork", "compact"):
        c["ctx"] = [_spread(rng, 1, 64), _spread(rng, 64, 4096)]
        c["R"] = _spread(rng, 4, 64)
        if op == "fork":
            c["n"] = _spread(rng, 1, c["R"] - 1)
            c["parents"] = _spread(rng, 1, c["R"] - c["n"])
        else:
            c["group"] = rng.choice([1, 2, 4])
            c["used"] = rng.choice([0.25, 0.5, 0.8])
        return _case(c)
    c["by_head"] = rng.random() < 0.6
    c["Hq"] = c["Hkv"] * rng.choice([1, 2, 4, 5, 7, 8])
    if op == "append":
        c["R"] = _spread(rng, 1, 64)
        c["ctx"] = [0, _spread(rng, 16, 2048)]
        c["new"] = [1, 1] if rng.random() < 0.4 else [1, max(2, 6000 // c["R"])]
        return _case(c)
    decode = rng.random() < 0.5
    most = _spread(rng, 16, 8192)
    c["R"] = _spread(rng, 1, 64) if decode else _spread(rng, 1, 16)
    c["ctx"] = [rng.choice([0, 1, most // 4]), most]
    c["new"] = [1, rng.choice([1, 1, 3])] if decode else [1, max(2, _spread(rng, 32, 1600) // c["R"])]
    c["window"] = rng.choice([0, 0, 0, 100, 1000])
    c["lse"] = rng.random() < 0.5
    return _case(c)


def _lengths(c):
    """Cached and new tokens of every request."""
    rng = random.Random(c["mix"])
    ctx = [_spread(rng, c["ctx_lo"], c["ctx_hi"]) for _ in range(c["R"])]
    new = [_spread(rng, c["new_lo"], c["new_hi"]) for _ in range(c["R"])] if "new_lo" in c else [0] * c["R"]
    return ctx, new


def _ends(c):
    """What the calls on tables start from: lengths, pages of each row, how many of them its group's first row has, pages in use."""
    ctx, P, rng = _lengths(c)[0], c["P"], random.Random(c["mix"] + 1)
    have = [-(-x // P) for x in ctx]
    if c["op"] == "fork":  # the children's rows are empty
        empty = _family(c)[1]
        ctx = [0 if r in empty else x for r, x in enumerate(ctx)]
        return ctx, [-(-x // P) for x in ctx], [0] * c["R"]
    first = [r - r % c["group"] for r in range(c["R"])]
    same = [0 if f == r else min(ctx[f] // P, ctx[r] // P, rng.randrange(1 + ctx[f] // P)) for r, f in enumerate(first)]
    return ctx, have, same


def _family(c):
    """A fork's parents, in any order, and its children."""
    rng = random.Random(c["mix"] + 2)
    rows = list(range(c["R"]))
    rng.shuffle(rows)
    some, children = rows[:c["parents"]], rows[c["parents"]:c["parents"] + c["n"]]
    return [rng.choice(some) for _ in children], children


def _pages(c):
    """Pages in use and in all."""
    _, have, same = _ends(c)
    used = sum(have) - sum(same)
    if c["op"] == "compact":
        return used, int(used / c["used"]) + 1
    return used, used + (c["n"] + 3 if c["op"] == "fork" else 5)


# ---------------------------------------------------------------- inputs


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _values(shape, g, t, spread):
    """Rows of a type as a projection gives them; keys have columns of very different size."""
    x = torch.randn(shape, device="cuda", generator=g)
    if spread:
        x *= torch.randn(shape[-1], device="cuda", generator=g).mul_(0.7).exp_()
    return x.to(t)


def _quantise(x, dtype):
    """Bytes of two values and of the groups' exponents for rows x."""
    D = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, -D % 32)).unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    part, power = torch.frexp(most)
    # the least e with most <= 7 * 2^e: nothing is further off than half a step of the grid
    e = torch.where(most > 0, power - 3 + (part > 0.875), LEAST[dtype]).clamp(LEAST[dtype], MOST[dtype])
    y = x.abs() * torch.exp2(-e.float())
    code = (y > 0.25).to(torch.uint8)
    code += y >= 0.75
    code += y > 1.25
    code += y >= 1.75
    code += y > 2.5
    code += y >= 3.5
    code += y > 5
    code += 8 * torch.signbit(x).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, torch.where(torch.isfinite(most), e + 127, 255).to(torch.uint8)[..., 0]


def _values_of(byte, scale, D):
    """What bytes and exponents stand for, in fp32."""
    grid = torch.tensor(GRID, device="cuda")
    code = torch.stack([byte & 15, byte >> 4], -1).flatten(-2)
    x = grid[(code & 7).int()]
    x = torch.where(code > 7, -x, x).unflatten(-1, (-1, 32))
    power = torch.where(scale < 255, torch.exp2(scale.float() - 127), math.nan)
    return (x * power[..., None]).flatten(-2)[..., :D]


def _cache4(c, pages, g, fill):
    """Bytes and exponents of a cache, in the order of its case: heads or positions of a page first."""
    P, H, D = c["P"], c["Hkv"], c["D"]
    shape = (pages, H, P) if c["by_head"] else (pages, P, H)
    if fill:
        x, e = _quantise(_values((*shape, D), g, TYPES[c["dtype"]], fill == "k"), c["dtype"])
    else:
        x = torch.randint(0, 256, (*shape, -(-D // 32) * 16), device="cuda", generator=g, dtype=torch.uint8)
        e = torch.randint(120, 130, (*shape, -(-D // 32)), device="cuda", generator=g, dtype=torch.uint8)
    return (x.transpose(1, 2), e.transpose(1, 2)) if c["by_head"] else (x, e)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_rows if case["op"] in ("append", "attend") else _prepare_tables)(case, g)


def _prepare_rows(case, g):
    ctx, new = _lengths(case)
    R, P, op = case["R"], case["P"], case["op"]
    have = [-(-(c + n) // P) for c, n in zip(ctx, new)]
    T, W, pages = sum(new), max(have) + 3, sum(have) + 5
    order = torch.randperm(pages, device="cuda", generator=g, dtype=torch.int32)
    col = torch.arange(W, device="cuda")
    begin = _ints(have).cumsum(0) - _ints(have)
    table = torch.where(col < _ints(have)[:, None], order[(begin[:, None] + col).clamp(max=pages - 1)], -1).contiguous()
    n = _ints(new)
    s = dict(case=case, T=T, table=table, seq=_ints([c + k for c, k in zip(ctx, new)]))
    s["qptr"] = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), n.cumsum(0).to(torch.int32)])
    Hq, Hkv, D, t = case["Hq"], case["Hkv"], case["D"], TYPES[case["dtype"]]
    if op == "append":
        # one projection gives q, k and v side by side
        qkv = _values((T, Hq + 2 * Hkv, D), g, t, True)
        s["k"], s["v"] = qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["kc"], s["ks"] = _cache4(case, pages, g, "")
        s["vc"], s["vs"] = _cache4(case, pages, g, "")
        r = torch.repeat_interleave(torch.arange(R, device="cuda"), n)
        pos = _ints(ctx)[r] + torch.arange(T, device="cuda") - s["qptr"][r]
        s["slots"] = table[r, pos // P].long() * P + pos % P
        return s
    s["q"] = torch.randn(T, Hq + 2 * Hkv, D, device="cuda", generator=g).to(t)[:, :Hq]
    s["kc"], s["ks"] = _cache4(case, pages, g, "k")
    s["vc"], s["vs"] = _cache4(case, pages, g, "v")
    # rows past a request's end hold whatever was there before
    last = (s["seq"] - 1).clamp(min=0)
    page = table[torch.arange(R, device="cuda"), last // P].long()
    stale = (torch.arange(P, device="cuda") > (last % P)[:, None]) & (s["seq"] > 0)[:, None]
    for x in (s["ks"], s["vs"]):
        x[page] = torch.where(stale[:, :, None, None], 255, x[page])
    if case["window"]:
        behind = (_ints(ctx) - case["window"] + 1).clamp(min=0) // P  # pages that no new token sees
        s["table"] = torch.where(col < behind[:, None], -1, table).contiguous()
    return s


def _prepare_tables(case, g):
    ctx, have, same = _ends(case)
    R, P, op = case["R"], case["P"], case["op"]
    used, pages = _pages(case)
    W = max(have) + 2
    order = torch.randperm(pages, device="cuda", generator=g, dtype=torch.int32)
    kept = torch.zeros(R * W + R + pages, dtype=torch.int32, device="cuda")
    table, seq, shares = kept[:R * W].view(R, W), kept[R * W:R * W + R], kept[R * W + R:]
    col = torch.arange(W, device="cuda")
    mine = _ints(have) - _ints(same)
    at = (mine.cumsum(0) - mine - _ints(same))[:, None] + col
    table.copy_(torch.where(col < _ints(have)[:, None], order[at.clamp(0, pages - 1)], -1))
    if "group" in case:
        first = torch.arange(R, device="cuda")
        table.copy_(torch.where(col < _ints(same)[:, None], table[first - first % case["group"]], table))
    seq.copy_(_ints(ctx))
    held = torch.bincount(table[table >= 0].long(), minlength=pages)
    shares.copy_((held - 1).clamp(min=0))
    now = kept.clone()
    s = dict(case=case, kept=kept, now=now, table=now[:R * W].view(R, W), seq=now[R * W:R * W + R], shares=now[R * W + R:])
    if op == "free":
        rows = list(range(R))
        random.Random(case["mix"] + 3).shuffle(rows)
        s["rows"] = _ints(rows[:case["n"]])
        return s
    if op == "fork":
        parents, children = _family(case)
        s["parents"], s["children"], s["free"] = _ints(parents), _ints(children), order[used:].contiguous()
    shape = (pages, P, case["Hkv"], case["D"])
    s["kc"] = torch.randn(shape, device="cuda", generator=g, dtype=TYPES[case["dtype"]])
    s["vc"] = torch.randn(shape, device="cuda", generator=g, dtype=TYPES[case["dtype"]])
    return s


# ---------------------------------------------------------------- the calls


def run(s):
    if "kept" in s:
        s["now"].copy_(s["kept"])
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2205_11622_amd as slnr

    c = s["case"]
    if c["op"] == "append":
        cache = s["kc"], s["vc"], s["ks"], s["vs"]
        slnr.sparselnr_cache_append_fp4(s["k"], s["v"], s["slots"], *cache)
        return slnr.sparselnr_cache_read_fp4(s["slots"], *cache, c["D"], s["k"].dtype)
    if c["op"] == "attend":
        lse = torch.empty(s["T"], c["Hq"], device="cuda") if c["lse"] else None
        out = slnr.sparselnr_paged_attention_fp4(s["q"], s["kc"], s["vc"], s["ks"], s["vs"], s["table"], s["seq"], s["qptr"], window=c["window"], max_new=c["new_hi"], lse=lse)
        return (out, lse) if c["lse"] else out
    if c["op"] == "fork":
        pairs, counts = slnr.sparselnr_page_fork(s["parents"], s["children"], s["table"], s["seq"], s["shares"], s["free"], c["P"])
        slnr.sparselnr_page_copy(pairs, (s["kc"], s["vc"]))
        return s["table"], s["seq"], s["shares"], pairs, counts, s["kc"], s["vc"]
    if c["op"] == "free":
        freed, counts = slnr.sparselnr_page_free(s["rows"], s["table"], s["seq"], s["shares"], c["P"])
        return s["table"], s["seq"], s["shares"], freed, counts
    pairs, counts = slnr.sparselnr_page_compact(s["table"], s["seq"], s["shares"], c["P"])
    slnr.sparselnr_page_copy(pairs, (s["kc"], s["vc"]))
    return s["table"], s["shares"], pairs, counts, s["kc"], s["vc"]


def _run_plain(s):
    return {"append": _append, "attend": _attend, "fork": _fork, "free": _free, "compact": _compact}[s["case"]["op"]](s)


# ---------------------------------------------------------------- plain forms


def _append(s):
    c = s["case"]
    page, row = s["slots"] // c["P"], s["slots"] % c["P"]
    s["kc"][page, row], s["ks"][page, row] = _quantise(s["k"], c["dtype"])
    s["vc"][page, row], s["vs"][page, row] = _quantise(s["v"], c["dtype"])
    t = TYPES[c["dtype"]]
    return _values_of(s["kc"][page, row], s["ks"][page, row], c["D"]).to(t), _values_of(s["vc"][page, row], s["vs"][page, row], c["D"]).to(t)


def _attend(s):
    c, q, table = s["case"], s["q"], s["table"]
    P, Hq, Hkv, D, window = c["P"], c["Hq"], c["Hkv"], c["D"], c["window"]
    n = s["qptr"][1:] - s["qptr"][:-1]
    ctx, new = _lengths(c)
    at = torch.arange(max(new), device="cuda")
    there = at < n[:, None]
    token = torch.where(there, s["qptr"][:-1, None] + at, 0)
    pos = (s["seq"] - n)[:, None] + at
    R, N = token.shape
    longest = max(a + b for a, b in zip(ctx, new))
    j = torch.arange(longest, device="cuda")
    page = table[:, j // P].long()
    live = (page >= 0) & (j < s["seq"][:, None])  # R, S
    rows = page.clamp(min=0), (j % P).expand_as(page)
    K = torch.where(live[:, :, None, None], _values_of(s["kc"][rows], s["ks"][rows], D), 0.0)  # R, S, Hkv, D
    V = torch.where(live[:, :, None, None], _values_of(s["vc"][rows], s["vs"][rows], D), 0.0)
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


def _copy(s, pairs):
    src, dst = pairs[pairs[:, 0] >= 0].long().unbind(1)
    s["kc"][dst] = s["kc"][src]
    s["vc"][dst] = s["vc"][src]


def _fork(s):
    table, seq, shares, free, P = s["table"], s["seq"], s["shares"], s["free"], s["case"]["P"]
    parents, children, W = s["parents"].long(), s["children"].long(), s["table"].shape[1]
    length = seq[parents]
    full = (length // P)[:, None]
    rows, col = table[parents], torch.arange(W, device="cuda")
    last = torch.where((length % P > 0)[:, None] & (col == full), rows, -1).amax(1)  # the page that is not full
    need = last >= 0
    k = need.cumsum(0) - 1
    fresh = torch.where(need & (k < free.numel()), free[k.clamp(0, free.numel() - 1)], -1)
    held = torch.where(col < full, rows, -1)
    shares.index_add_(0, held[held >= 0].long(), torch.ones_like(held[held >= 0]))
    table[children] = torch.where(col == full, fresh[:, None], held)
    seq[children] = length
    pairs = torch.where((fresh >= 0)[:, None], torch.stack([last, fresh], 1), -1)
    _copy(s, pairs)
    return table, seq, shares, pairs, torch.stack([need.sum(), (need & (fresh < 0)).sum()]).to(torch.int32), s["kc"], s["vc"]


def _compacted(mask, size):
    """The places where mask is set, ascending, in an array of `size` with -1 behind them."""
    rank = torch.where(mask, mask.cumsum(0) - 1, size)
    out = torch.full((size + 1,), -1, dtype=torch.int32, device="cuda")
    out[rank] = torch.arange(mask.numel(), dtype=torch.int32, device="cuda")
    return out[:size]


def _free(s):
    table, seq, shares, rows, P = s["table"], s["seq"], s["shares"], s["rows"].long(), s["case"]["P"]
    W, pages = table.shape[1], shares.numel()
    col = torch.arange(W, device="cuda")
    held = torch.where(col < ((seq[rows] + P - 1) // P)[:, None], table[rows], -1)
    held = held[held >= 0].long()
    drop = torch.zeros_like(shares).index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
    gone = drop > shares
    shares.copy_((shares - drop).clamp(min=0))
    given = torch.where(col < ((seq[rows] + P - 1) // P)[:, None], -1, table[rows])
    table[rows] = given
    seq[rows] = 0
    counts = torch.stack([gone.sum(), drop.sum()]).to(torch.int32)
    return table, seq, shares, _compacted(gone, min(pages, rows.numel() * W)), counts


def _compact(s):
    table, seq, shares, P = s["table"], s["seq"], s["shares"], s["case"]["P"]
    pages = shares.numel()
    held = torch.where(torch.arange(table.shape[1], device="cuda") < ((seq + P - 1) // P)[:, None], table, -1)
    used = torch.zeros(pages, dtype=torch.bool, device="cuda")
    used[held[held >= 0].long()] = True
    page = torch.arange(pages, device="cuda")
    total = used.sum()
    hole, mover = ~used & (page < total), used & (page >= total)
    pairs = torch.stack([_compacted(mover, pages // 2), _compacted(hole, pages // 2)], 1)
    to = page.clone()
    src, dst = pairs[pairs[:, 0] >= 0].long().unbind(1)
    to[src] = dst
    table.copy_(torch.where(held >= 0, to[held.clamp(min=0).long()].to(torch.int32), table))
    shares[dst] = shares[src]
    shares[src] = 0
    _copy(s, pairs)
    return table, shares, pairs, torch.stack([total, mover.sum()]).to(torch.int32), s["kc"], s["vc"]


# ---------------------------------------------------------------- work and reference


def _seen(c, ctx, new):
    """Pairs of query and key, and keys that some query sees, of one request."""
    w = c["window"] or ctx + new
    if ctx + 1 >= w:
        return new * w, min(ctx + new, new + w - 1)
    grow = min(new, w - ctx)  # queries that still see every key
    return grow * ctx + grow * (grow + 1) // 2 + (new - grow) * w, ctx + new


def work(case):
    """Every input that the results depend on read once, every output written once; the multiplications and additions of the definition."""
    ctx, new = _lengths(case)
    op, P, R, T = case["op"], case["P"], case["R"], sum(_lengths(case)[1])
    if op in ("append", "attend"):
        e, D, Hkv = 4 if case["dtype"] == "fp32" else 2, case["D"], case["Hkv"]
        row4 = Hkv * -(-D // 32) * 17
        if op == "append":  # K and V in, their 4 bits out, and back
            return {"bytes": 4 * T * Hkv * D * e + 4 * T * row4 + 16 * T, "flops": 6 * T * Hkv * D}
        pages = sum(-(-(c + n) // P) for c, n in zip(ctx, new))
        pairs, keys = (sum(x) for x in zip(*(_seen(case, c, n) for c, n in zip(ctx, new))))
        return {"bytes": 4 * (2 * R + 1) + 4 * pages + 2 * T * case["Hq"] * D * e + 2 * keys * row4 + (4 * T * case["Hq"] if case["lse"] else 0), "flops": 4 * pairs * case["Hq"] * D}
    ctx, have, same = _ends(case)
    W, (used, pages) = max(have) + 2, _pages(case)
    back = 8 * (R * W + R + pages)  # what a pass begins with: the tables as they were
    if op == "free":
        rows = list(range(R))
        random.Random(case["mix"] + 3).shuffle(rows)
        held = sum(have[r] for r in rows[:case["n"]])
        return {"bytes": back + 8 * case["n"] + 16 * held + 4 * min(pages, case["n"] * W) + 8, "flops": 2 * held}
    page = 2 * P * case["Hkv"] * case["D"] * (4 if case["dtype"] == "fp32" else 2)
    if op == "fork":
        parents, _ = _family(case)
        full = sum(ctx[p] // P for p in parents)
        copies = sum(ctx[p] % P > 0 for p in parents)
        some = set(parents)
        return {"bytes": back + 4 * sum(have[p] for p in some) + 4 * case["n"] * W + 8 * sum(ctx[p] // P for p in some) + 20 * case["n"] + 2 * copies * page, "flops": 2 * full}
    # about used * (1 - used / pages) pages in use lie behind the first `used`
    moves = used * (pages - used) // pages
    return {"bytes": back + 4 * sum(have) + 8 * moves + 4 * moves + 8 * (pages // 2) + 2 * moves * page, "flops": 2 * sum(have)}


def _standing(byte, scale, D):
    """Values of 4-bit rows in fp64, by sign, exponent and last bit of each code."""
    code = torch.stack([byte.long() % 16, byte.long() // 16], -1).reshape(*byte.shape[:-1], -1)
    sign, power, half = 1 - 2 * (code // 8), code // 2 % 4, code % 2
    x = torch.where(power > 0, 2.0 ** (power - 1).double() * (1 + 0.5 * half), 0.5 * half) * sign
    e = scale.long().repeat_interleave(32, -1)
    return (x * torch.where(e == 255, math.nan, 2.0 ** (e - 127).double()))[..., :D]


def _nearest(x, dtype):
    """The values that 4 bits hold for rows x, in fp64: the nearest of the 15, the one with an even last bit of two equally near."""
    D = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -D % 32)).view(*x.shape[:-1], -1, 32)
    most = x.abs().max(-1, keepdim=True).values
    e = torch.full_like(most, LEAST[dtype])
    for k in range(LEAST[dtype], MOST[dtype]):
        e += most > 7 * 2.0 ** k
    grid = torch.tensor([-v for v in GRID[:0:-1]] + list(GRID), dtype=torch.float64, device=x.device)
    odd = torch.tensor([i % 2 for i in range(7, 0, -1)] + [i % 2 for i in range(8)], dtype=torch.float64, device=x.device)
    off = ((x * 2.0 ** -e)[..., None] - grid).abs()
    near = off.amin(-1, keepdim=True)
    pick = torch.where(off == near, odd, 2.0).argmin(-1)
    return (grid[pick] * 2.0 ** e).view(*x.shape[:-2], -1)[..., :D]


def exact(case, seed):
    """fp64, one request and one head after the other; whole numbers have no such value."""
    op, P = case["op"], case["P"]
    if op == "free":
        return None
    s = prepare(case, seed)
    if op == "append":
        return _nearest(s["k"], case["dtype"]), _nearest(s["v"], case["dtype"])
    if op == "attend":
        return _exact_attend(case, s)
    table, seq = s["table"].tolist(), s["seq"].tolist()
    src, dst = [], []
    if op == "fork":
        free = iter(s["free"].tolist())
        for p in s["parents"].tolist():
            if seq[p] % P:
                src.append(table[p][seq[p] // P])
                dst.append(next(free))
    else:
        used = sorted({p for row, n in zip(table, seq) for p in row[:-(-n // P)] if p >= 0})
        src = [p for p in used if p >= len(used)]
        dst = sorted(set(range(len(used))) - set(used))
    kc, vc = s["kc"].double(), s["vc"].double()
    kc[dst], vc[dst] = kc[src], vc[src]
    return (None,) * (5 if op == "fork" else 4) + (kc, vc)


def _exact_attend(case, s):
    P, Hq, Hkv, D, T = case["P"], case["Hq"], case["Hkv"], case["D"], s["T"]
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    qptr, seq, G = s["qptr"].tolist(), s["seq"].tolist(), Hq // Hkv
    for r in range(case["R"]):
        a, b, S = qptr[r], qptr[r + 1], seq[r]
        p = torch.arange(S - (b - a), S, device="cuda")[:, None]
        j = torch.arange(S, device="cuda")
        page = s["table"][r].long().repeat_interleave(P)[:S]
        ok = (page >= 0) & (j <= p)
        if case["window"]:
            ok = ok & (p - j < case["window"])
        at = page.clamp(min=0), j % P
        for h in range(Hkv):
            k, v = (torch.where((page >= 0)[:, None], _standing(x[(*at, h)], e[(*at, h)], D), 0.0) for x, e in ((s["kc"], s["ks"]), (s["vc"], s["vs"])))
            for i in range(h * G, (h + 1) * G):
                x = (s["q"][a:b, i].double() @ k.t().contiguous() / D ** 0.5).masked_fill(~ok, -math.inf)
                lse[a:b, i] = torch.logsumexp(x, 1)
                out[a:b, i] = (x - lse[a:b, i, None]).exp().nan_to_num(0.0) @ v
    return (out, lse) if case["lse"] else out
