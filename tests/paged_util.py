"""Plain forms of the paged-cache operators in 64 bits on the CPU, and inputs for
them.  Nothing here uses the library."""
from __future__ import annotations

import math

import torch

EPS = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}  # half a unit: 2^-8, 2^-11, 2^-24


def page_tables(ctx, new, table, free, tokens, P):
    """(qptr, seq, slots, counts, table) by a loop over requests and tokens."""
    table = [list(row) for row in table]
    R, W = len(ctx), len(table[0]) if table else 0
    slots, qptr, seq, taken, lost, t = [-1] * tokens, [0], [], 0, 0, 0
    for r in range(R):
        c, n = max(ctx[r], 0), max(new[r], 0)
        have, want = -(-c // P), -(-(c + n) // P)
        for i in range(n):
            pos = c + i
            j = pos // P
            if j >= W:
                page = -1
            elif j < have:
                page = table[r][j]
            else:
                k = taken + j - have
                page = free[k] if k < len(free) else -1
                if t < tokens and pos % P == 0:
                    table[r][j] = page
            if page < 0:
                lost += 1
            elif t < tokens:
                slots[t] = page * P + pos % P
            t += 1
        taken += want - have
        qptr.append(t)
        seq.append(c + n)
    return qptr, seq, slots, [t, taken, lost], table


def summary(rows):
    """8-bit mean of K rows (n x D fp64): (kq, kscale) as the interface defines them."""
    mean = (rows.sum(0) / rows.shape[0]).float()
    top = mean.abs().max()
    if not torch.isfinite(mean).all():
        return torch.zeros_like(mean).to(torch.int8), math.inf
    step = top * torch.tensor(1.0 / 127.0, dtype=torch.float32)
    if step == 0:
        return torch.zeros_like(mean).to(torch.int8), 0.0
    return (mean / step).round().clamp(-127, 127).to(torch.int8), float(step)


def gather(kcache, vcache, row, keys):
    """fp64 K and V rows (n x Hkv x D) of the positions `keys`, and which are there."""
    pages, P = kcache.shape[:2]
    at = torch.tensor([row[j // P] if j // P < len(row) else -1 for j in keys], dtype=torch.long)
    there = (at >= 0) & (at < pages)
    place = torch.tensor([j % P for j in keys], dtype=torch.long)
    k = kcache[at.clamp(0, pages - 1), place].double()
    v = vcache[at.clamp(0, pages - 1), place].double()
    k[~there] = 0.0
    v[~there] = 0.0
    return k, v, there


def softmax_rows(q, k, v, seen, scale):
    """One head: q (n x D), k, v (S x D), seen (n x S), all fp64.  (out, lse, sum p|v|)."""
    n, D = q.shape
    out, lse = torch.zeros(n, D, dtype=torch.float64), torch.full((n,), -math.inf, dtype=torch.float64)
    weight = torch.zeros(n, D, dtype=torch.float64)
    for i in range(n):
        idx = seen[i].nonzero()[:, 0]
        if not idx.numel():
            continue
        s = (k[idx] @ q[i]) * scale
        lse[i] = torch.logsumexp(s, 0)
        p = (s - lse[i]).exp()
        out[i] = p @ v[idx]
        weight[i] = p @ v[idx].abs()
    return out, lse, weight


def attention(q, kcache, vcache, table, seq, qptr, scale, window=0, sel=None):
    """(out, lse, weight) fp64 of the attention calls; sel for the sparse one.  CPU tensors and lists."""
    T, Hq, D = q.shape
    P, Hkv = kcache.shape[1], kcache.shape[2]
    G = Hq // Hkv
    out = torch.zeros(T, Hq, D, dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    weight = torch.zeros(T, Hq, D, dtype=torch.float64)
    for r in range(len(seq)):
        a, b, S = qptr[r], qptr[r + 1], min(seq[r], len(table[r]) * P)
        if b == a:
            continue
        pos = torch.arange(S - (b - a), S)[:, None]
        keys = list(range(S))
        k, v, there = gather(kcache, vcache, table[r], keys)
        j = torch.arange(S)
        ok = there & (j <= pos)
        if window:
            ok &= j > pos - window
        for h in range(Hkv):
            see = ok
            if sel is not None:
                mine = torch.zeros(b - a, S, dtype=torch.bool)
                for t in range(a, b):
                    for blk in sel[t][h]:
                        if 0 <= blk < len(table[r]):
                            mine[t - a, blk * P:(blk + 1) * P] = True
                see = ok & mine
            for g in range(h * G, (h + 1) * G):
                out[a:b, g], lse[a:b, g], weight[a:b, g] = softmax_rows(q[a:b, g].double(), k[:, h], v[:, h], see, scale)
    return out, lse, weight


def tolerance(dtype, weight, S, D, vmax, logits=8.0):
    """Bound on |out - fp64| per element.

    Scores: fp32 sums of D products, off by up to D 2^-24 of the sum of magnitudes
    (about `logits` after scaling), plus 2^-22 of exp2 and of its argument: a weight is off by
    (D + 32) 2^-24 logits relative, twice (weight and sum).  Weights are rounded to the
    type once (2^-8 or 2^-11; fp16 also loses 2^-25 absolute below 2^-14), the fp32 sums over S
    keys add S 2^-24, the result is rounded once."""
    e = EPS[dtype]
    rel = 2 * (D + 32) * logits * 2.0 ** -24 + 2 * S * 2.0 ** -24
    if dtype != torch.float32:
        rel += 2 * e * (1 + e)
    else:
        rel += e
    absolute = (S * 2.0 ** -25 + 2.0 ** -24) * vmax if dtype == torch.float16 else 1e-30
    return rel * weight + absolute


def lse_tolerance(S, D, logits=8.0):
    return (D + 32) * logits * 2.0 ** -24 + (S + 64) * 2.0 ** -24


def check(out, lse, ref, dtype, S, D, vmax, logits=8.0):
    """Every element of out (and lse) within the bounds of the fp64 reference."""
    want, want_lse, weight = ref
    assert out.dtype == dtype
    err = (out.double().cpu() - want).abs()
    tol = tolerance(dtype, weight, S, D, vmax, logits)
    bad = ~(err <= tol)
    assert not bad.any(), "out: %d of %d off, worst %.3g of its bound at %s" % (
        int(bad.sum()), bad.numel(), float((err / tol)[bad].max()), bad.nonzero()[0].tolist())
    if lse is not None:
        got = lse.double().cpu()
        empty = want_lse == -math.inf
        assert (got[empty] == -math.inf).all()
        off = (got - want_lse)[~empty].abs()
        assert (off <= lse_tolerance(S, D, logits) + 1e-6 * want_lse[~empty].abs()).all(), float(off.max())


def select(q, kq, kscale, table, seq, qptr, P, top, first, local):
    """Lists of chosen pages by the definition, one token and head after the other."""
    T, Hq, D = q.shape
    Hkv = kq.shape[1]
    out = []
    r = 0
    big = torch.finfo(torch.float32).max
    for t in range(T):
        while qptr[r + 1] <= t:
            r += 1
        p = seq[r] - qptr[r + 1] + t
        near = p // P if p >= 0 else -1
        heads = []
        for h in range(Hkv):
            u = q[t].view(Hkv, -1, D)[h].double().sum(0).float()
            top_u = u.abs().max()
            step = top_u * torch.tensor(1.0 / 127.0, dtype=torch.float32)
            if torch.isfinite(u).all() and step > 0:
                q8 = (u / step).round().clamp(-127, 127).to(torch.int64)
            else:
                q8 = torch.zeros(D, dtype=torch.int64)
            cand = [(b, table[r][b]) for b in range(min(near + 1, len(table[r]))) if 0 <= table[r][b] < kq.shape[0]]
            ranked = []
            if cand:
                pages = torch.tensor([c[1] for c in cand])
                score = (kq[pages, h].long() @ q8).float() * kscale[pages, h]
                score = score.nan_to_num(nan=big, posinf=big, neginf=-big).tolist()
                ranked = [(-math.inf if b < first or b > near - local else -s, b) for (b, _), s in zip(cand, score)]
            pick = sorted(b for _, b in sorted(ranked)[:top])
            heads.append(pick + [-1] * (top - len(pick)))
        out.append(heads)
    return torch.tensor(out, dtype=torch.int32).view(T, Hkv, top)


class Batch:
    """A seeded batch in a shuffled paged cache.  Places past a request's end, and pages
    of nobody, hold NaN.  order: 'slots' (pages, P, Hkv, D in memory), 'heads' (Hkv before
    P), 'pairs' (K and V of a page side by side)."""

    def __init__(self, ctx, new, Hq, Hkv, D, P, dtype, seed=0, order="slots", spare=3, extra_w=2, amp=1.0):
        g = torch.Generator().manual_seed(seed)
        self.ctx, self.new, self.P, self.dtype = list(ctx), list(new), P, dtype
        self.seq = [c + n for c, n in zip(ctx, new)]
        self.qptr = [0]
        for n in new:
            self.qptr.append(self.qptr[-1] + n)
        T = self.qptr[-1]
        need = [-(-s // P) for s in self.seq]
        pages = sum(need) + spare
        perm = torch.randperm(pages, generator=g).tolist()
        W = max(need + [0]) + extra_w
        self.table, at = [], 0
        for n in need:
            self.table.append(perm[at:at + n] + [-1] * (W - n))
            at += n
        if order == "slots":
            kc = torch.full((pages, P, Hkv, D), math.nan).to(dtype)
            vc = torch.full((pages, P, Hkv, D), math.nan).to(dtype)
        elif order == "heads":
            kc = torch.full((pages, Hkv, P, D), math.nan).to(dtype).transpose(1, 2)
            vc = torch.full((pages, Hkv, P, D), math.nan).to(dtype).transpose(1, 2)
        else:
            both = torch.full((pages, 2, P, Hkv, D), math.nan).to(dtype)
            kc, vc = both[:, 0], both[:, 1]
        for r, s in enumerate(self.seq):
            for b in range(need[r]):
                n = min(P, s - b * P)
                kc[self.table[r][b], :n] = (amp * torch.randn(n, Hkv, D, generator=g)).to(dtype)
                vc[self.table[r][b], :n] = torch.randn(n, Hkv, D, generator=g).to(dtype)
        self.kc, self.vc = kc, vc
        # q as a slice of one projection: its rows are not adjacent
        self.qkv = torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(dtype)
        self.q = self.qkv[:, :Hq]

    def ints(self, v, device):
        return torch.tensor(v, dtype=torch.int32, device=device)

    def upload(self, device="cuda:0"):
        """(q, kcache, vcache, table, seq, qptr) on the device, with the strides that they have here."""
        def put(t):
            base = t._base if t._base is not None else t
            while base._base is not None:
                base = base._base
            flat = base.to(device)
            return flat.as_strided(t.shape, t.stride(), t.storage_offset())
        return (put(self.q), put(self.kc), put(self.vc), self.ints(self.table, device).view(len(self.seq), -1),
                self.ints(self.seq, device), self.ints(self.qptr, device))

    def reference(self, scale=None, window=0, sel=None):
        scale = self.q.shape[2] ** -0.5 if scale is None else scale
        return attention(self.q, self.kc, self.vc, self.table, self.seq, self.qptr, scale, window, sel)
