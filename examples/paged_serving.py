"""A small serving loop on a paged cache: requests come, their prompts are read in
chunks beside the running ones' single tokens, and leave when they are done.

    python examples/paged_serving.py [--requests 12] [--layers 2] [--sparse 0] [--check]

Every step is one batch: block tables and slots from the lengths, then per layer the new
tokens' K and V into the cache and attention over it; with --sparse N each token
attends the N pages that the 8-bit score selects.  The model is a stack of random
projections with residuals (there is nothing to say, only to compute).  --check
compares each request's last hidden state with the same model run over its whole
sequence at once, in fp32 on torch (dense attention only).
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

    def __init__(self, layers, pages, page_size, heads, dim, slots, width, device, dtype):
        shape = (pages, page_size, heads, dim)
        self.page_size = page_size
        self.k = [torch.zeros(shape, dtype=dtype, device=device) for _ in range(layers)]
        self.v = [torch.zeros(shape, dtype=dtype, device=device) for _ in range(layers)]
        self.kq = [torch.zeros(pages, heads, dim, dtype=torch.int8, device=device) for _ in range(layers)]
        self.ks = [torch.zeros(pages, heads, device=device) for _ in range(layers)]
        self.table = torch.full((slots, width), -1, dtype=torch.int32, device=device)
        self.free = list(range(pages))
        self.held = [[] for _ in range(slots)]

    def wanted(self, ctx, new):
        return -(-(ctx + new) // self.page_size) - -(-ctx // self.page_size)

    def release(self, slot):
        self.free.extend(self.held[slot])
        self.held[slot] = []
        self.table[slot] = -1


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
            slnr.sparselnr_cache_append(k, v, slots, cache.k[i], cache.v[i], *summaries)
            if sparse:
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
          dtype=torch.float32, device="cuda:0", seed=0):
    """Runs the loop; returns (tokens, steps, worst relative error or None)."""
    rng = random.Random(seed)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    model = Model(layers, width, Hq, Hkv, dim, device, dtype)
    waiting = [(rng.randrange(1, 4 * chunk), rng.randrange(1, 24)) for _ in range(requests)]  # prompt, answer
    longest = max(p + a for p, a in waiting)
    cache = Cache(layers, batch * -(-longest // page_size), page_size, Hkv, dim, batch, -(-longest // page_size), device,
                  dtype)
    running = [None] * batch
    tokens = steps = 0
    worst = 0.0 if check else None
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=device)  # noqa: E731
    while waiting or any(running):
        for s in range(batch):
            if running[s] is None and waiting:
                p, a = waiting.pop(0)
                running[s] = dict(ctx=0, x=torch.randn(p + a, width, device=device, generator=g).to(dtype), prompt=p)
        ctx = [r["ctx"] if r else 0 for r in running]
        new = [(min(chunk, r["prompt"] - r["ctx"]) if r["ctx"] < r["prompt"] else 1) if r else 0 for r in running]
        T = sum(new)
        qptr, seq, slots, counts = slnr.sparselnr_page_tables(ints(ctx), ints(new), cache.table, ints(cache.free), T,
                                                              page_size)
        for s in range(batch):  # the host's own books: what the call handed out, in its order
            n = cache.wanted(ctx[s], new[s])
            cache.held[s] += cache.free[:n]
            del cache.free[:n]
        x = torch.cat([r["x"][r["ctx"]:r["ctx"] + n] for r, n in zip(running, new) if r])
        y = model.step(x, cache, qptr, seq, slots, cache.table, max(new), sparse)
        at = 0
        for s, r in enumerate(running):
            if r is None:
                continue
            at += new[s]
            r["ctx"] += new[s]
            if r["ctx"] == r["x"].shape[0]:
                if check:
                    want = model.whole(r["x"])[-1]
                    worst = max(worst, float((y[at - 1].float() - want).norm() / want.norm()))
                cache.release(s)
                running[s] = None
        tokens += T
        steps += 1
    return tokens, steps, worst


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--requests", type=int, default=12)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--sparse", type=int, default=0, help="pages that a token attends (0: all)")
    ap.add_argument("--dtype", choices=["bf16", "fp16", "fp32"], default="bf16")
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    dtype = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[a.dtype]
    t = time.perf_counter()
    tokens, steps, worst = serve(a.requests, a.layers, sparse=a.sparse, check=a.check and not a.sparse, dtype=dtype)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print("%d tokens in %d steps, %.2f s%s" % (tokens, steps, t, "" if worst is None else
                                               ", worst last state %.2e off the whole-sequence run" % worst))


if __name__ == "__main__":
    main()
