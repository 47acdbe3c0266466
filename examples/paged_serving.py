"""A small serving loop on a paged cache: requests come, their prompts are read in
chunks beside the running ones' single tokens, and leave when they are done.

    python examples/paged_serving.py [--requests 12] [--layers 2] [--sparse 0] [--answers 1] [--four-bits] [--check]

Every step is one batch: block tables and slots from the lengths, then per layer the new
tokens' K and V into the cache and attention over it; with --sparse N each token
attends the N pages that the 8-bit score selects.  With --answers N a prompt that has been read
is gone on from N times: the rows of its answers share its full pages, rows that are done are given up
by the device, and now and then the pages in use move to the front.  --four-bits keeps the cache in
4 bits a value.  The model is a stack of random
projections with residuals (there is nothing to say, only to compute).  --check
compares each request's last hidden state with the same model run over its whole
sequence at once, in fp32 on torch (dense attention over a cache of the model's type only).
"""
import argparse
import os
import random
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2205_11622_amd as slnr  # noqa: E402


class Cache:
    """Pages of every layer, the free list, and the requests' rows of the block table."""

    def __init__(self, layers, pages, page_size, heads, dim, slots, width, device, dtype, four_bits=False):
        self.page_size, self.pages, self.four_bits = page_size, pages, four_bits

        def rows(size, dtype):  # a head's rows of a page adjacent
            return [torch.zeros(pages, heads, page_size, size, dtype=dtype, device=device).transpose(1, 2) for _ in range(layers)]

        groups = -(-dim // 32)
        self.k, self.v = (rows(16 * groups, torch.uint8) if four_bits else rows(dim, dtype) for _ in "kv")
        self.k_scale, self.v_scale = (rows(groups, torch.uint8) if four_bits else [] for _ in "kv")
        self.kq = [torch.zeros(pages, heads, dim, dtype=torch.int8, device=device) for _ in range(layers)]
        self.ks = [torch.zeros(pages, heads, device=device) for _ in range(layers)]
        self.table = torch.full((slots, width), -1, dtype=torch.int32, device=device)
        self.shares = torch.zeros(pages, dtype=torch.int32, device=device)
        self.free = list(range(pages))
        self.held = [[] for _ in range(slots)]

    def wanted(self, ctx, new):
        return -(-(ctx + new) // self.page_size) - -(-ctx // self.page_size)

    def release(self, slot):
        self.free.extend(self.held[slot])
        self.held[slot] = []
        self.table[slot] = -1

    # The same where rows share pages: what is free is what the calls say.

    def copy(self, pairs):
        """Pages of every layer, a few arrays a call."""
        arrays = self.k + self.v + self.k_scale + self.v_scale + self.kq + self.ks
        for i in range(0, len(arrays), 8):
            slnr.sparselnr_page_copy(pairs, arrays[i:i + 8])

    def fork(self, parents, children, seq):
        pairs, counts = slnr.sparselnr_page_fork(*(torch.tensor(x, dtype=torch.int32, device=seq.device)
                                                   for x in (parents, children)), self.table, seq, self.shares,
                                                 torch.tensor(self.free, dtype=torch.int32, device=seq.device), self.page_size)
        self.copy(pairs)
        del self.free[:int(counts[0])]

    def give_up(self, rows, seq):
        freed, counts = slnr.sparselnr_page_free(torch.tensor(rows, dtype=torch.int32, device=seq.device), self.table, seq,
                                                 self.shares, self.page_size)
        self.free += freed[:int(counts[0])].tolist()

    def tidy(self, seq):
        pairs, counts = slnr.sparselnr_page_compact(self.table, seq, self.shares, self.page_size)
        used, moved = counts.tolist()
        self.copy(pairs[:moved])
        self.free = list(range(used, self.pages))


class Model:
    def __init__(self, layers, width, Hq, Hkv, dim, device, dtype, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        init = lambda *s: (torch.randn(*s, device=device, generator=g) * s[0] ** -0.5).to(dtype)  # noqa: E731
        self.Hq, self.Hkv, self.dim = Hq, Hkv, dim
        self.qkv = [init(width, (Hq + 2 * Hkv) * dim) for _ in range(layers)]
        self.out = [init(Hq * dim, width) for _ in range(layers)]

    def step(self, x, cache, qptr, seq, slots, table, max_new, sparse):
        Hq, Hkv = self.Hq, self.Hkv
        for i, (w, o) in enumerate(zip(self.qkv, self.out)):
            qkv = (x @ w).view(x.shape[0], Hq + 2 * Hkv, self.dim)
            q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
            summaries = (cache.kq[i], cache.ks[i]) if sparse else (None, None)
            if cache.four_bits:
                four = (cache.k[i], cache.v[i], cache.k_scale[i], cache.v_scale[i])
                slnr.sparselnr_cache_append_fp4(k, v, slots, *four)
            else:
                slnr.sparselnr_cache_append(k, v, slots, cache.k[i], cache.v[i], *summaries)
            if cache.four_bits:
                a = slnr.sparselnr_paged_attention_fp4(q, *four, table, seq, qptr, max_new=max_new)
            elif sparse:
                sel = slnr.sparselnr_block_select(q, *summaries, table, seq, qptr, cache.page_size, sparse,
                                                  first=1, local=min(2, sparse - 1))
                a = slnr.sparselnr_block_attention(q, cache.k[i], cache.v[i], table, seq, qptr, sel)
            else:
                a = slnr.sparselnr_paged_attention(q, cache.k[i], cache.v[i], table, seq, qptr, max_new=max_new)
            x = x + a.reshape(x.shape[0], -1) @ o
        return x

    def whole(self, x):
        """The same over one whole sequence in fp32, without a cache."""
        n, G = x.shape[0], self.Hq // self.Hkv
        x = x.float()
        seen = torch.ones(n, n, dtype=torch.bool, device=x.device).tril()
        for w, o in zip(self.qkv, self.out):
            qkv = (x @ w.float()).view(n, -1, self.dim).transpose(0, 1)
            q, k, v = qkv[:self.Hq], qkv[self.Hq:self.Hq + self.Hkv], qkv[self.Hq + self.Hkv:]
            k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
            s = (q @ k.transpose(1, 2).contiguous()) * self.dim ** -0.5
            p = s.masked_fill(~seen, float("-inf")).softmax(2)
            x = x + (p @ v).transpose(0, 1).reshape(n, -1) @ o.float()
        return x


def serve(requests=12, layers=2, width=256, Hq=8, Hkv=2, dim=64, page_size=16, batch=4, chunk=64, sparse=0, check=False,
          dtype=torch.float32, device="cuda:0", seed=0, answers=1, four_bits=False):
    """Runs the loop; returns (tokens, steps, worst relative error or None)."""
    if sparse and four_bits:
        raise ValueError("pages are selected in a cache of the model's type")
    rng = random.Random(seed)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    model = Model(layers, width, Hq, Hkv, dim, device, dtype)
    waiting = [(rng.randrange(1, 4 * chunk), rng.randrange(1, 24)) for _ in range(requests)]  # prompt, answer
    longest = max(p + a for p, a in waiting)
    rows = batch * answers  # of the table; a request's answers have adjacent ones, and the first reads the prompt
    cache = Cache(layers, rows * -(-longest // page_size), page_size, Hkv, dim, rows, -(-longest // page_size), device,
                  dtype, four_bits)
    running = [None] * rows
    tokens = steps = 0
    worst = 0.0 if check else None
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=device)  # noqa: E731
    while waiting or any(running):
        for s in range(0, rows, answers):
            if not any(running[s:s + answers]) and waiting:
                p, a = waiting.pop(0)
                running[s] = dict(ctx=0, x=torch.randn(p + a, width, device=device, generator=g).to(dtype), prompt=p)
        ctx = [r["ctx"] if r else 0 for r in running]
        new = [(min(chunk, r["prompt"] - r["ctx"]) if r["ctx"] < r["prompt"] else 1) if r else 0 for r in running]
        T = sum(new)
        qptr, seq, slots, counts = slnr.sparselnr_page_tables(ints(ctx), ints(new), cache.table, ints(cache.free), T,
                                                              page_size)
        for s in range(rows):  # the host's own books: what the call handed out, in its order
            n = cache.wanted(ctx[s], new[s])
            if answers == 1:
                cache.held[s] += cache.free[:n]
            del cache.free[:n]
        x = torch.cat([r["x"][r["ctx"]:r["ctx"] + n] for r, n in zip(running, new) if r])
        y = model.step(x, cache, qptr, seq, slots, cache.table, max(new), sparse)
        at = 0
        done, parents, children = [], [], []
        for s, r in enumerate(running):
            if r is None or new[s] == 0:
                continue
            at += new[s]
            r["ctx"] += new[s]
            if answers > 1 and r["ctx"] == r["prompt"] and s % answers == 0:
                for c in range(s + 1, s + answers):
                    x = torch.randn(len(r["x"]) - r["prompt"], width, device=device, generator=g).to(dtype)
                    running[c] = dict(ctx=r["ctx"], x=torch.cat([r["x"][:r["prompt"]], x]), prompt=r["prompt"])
                    parents.append(s)
                    children.append(c)
            if r["ctx"] == r["x"].shape[0]:
                if check:
                    want = model.whole(r["x"])[-1]
                    worst = max(worst, float((y[at - 1].float() - want).norm() / want.norm()))
                if answers == 1:
                    cache.release(s)
                done.append(s)
        if answers > 1:
            lengths = [r["ctx"] if r else 0 for r in running]
            for c in children:
                lengths[c] = 0  # until the fork
            lengths = ints(lengths)
            if children:
                cache.fork(parents, children, lengths)
            if done:
                cache.give_up(done, lengths)
            if steps % 8 == 7:
                cache.tidy(lengths)
        for s in done:
            running[s] = None
        tokens += T
        steps += 1
    return tokens, steps, worst


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--requests", type=int, default=12)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--sparse", type=int, default=0, help="pages that a token attends (0: all)")
    ap.add_argument("--answers", type=int, default=1, help="of each request, over the same pages of its prompt")
    ap.add_argument("--four-bits", action="store_true", help="the cache in 4 bits a value")
    ap.add_argument("--dtype", choices=["bf16", "fp16", "fp32"], default="bf16")
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    dtype = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[a.dtype]
    t = time.perf_counter()
    tokens, steps, worst = serve(a.requests, a.layers, sparse=a.sparse, check=a.check and not a.sparse and not a.four_bits,
                                 dtype=dtype, answers=a.answers, four_bits=a.four_bits)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print("%d tokens in %d steps, %.2f s%s" % (tokens, steps, t, "" if worst is None else
                                               ", worst last state %.2e off the whole-sequence run" % worst))


if __name__ == "__main__":
    main()
