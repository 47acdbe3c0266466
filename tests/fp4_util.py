"""Plain forms of the 4-bit cache and of the pages' life in 64 bits on the CPU, and inputs for
them.  Nothing here uses the library."""
from __future__ import annotations

import math

import torch

from tests import paged_util as pu

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
LIMITS = {torch.bfloat16: (-125, 125), torch.float16: (-23, 13), torch.float32: (-125, 125)}


def exponent(top, dtype):
    """The least e with top <= 7 * 2^e, within the type's limits."""
    lo, hi = LIMITS[dtype]
    if top == 0:
        return lo
    e = math.frexp(top / 7.0)[1] - 2  # below it or equal
    while top > 7.0 * 2.0 ** e:
        e += 1
    while e > lo and top <= 7.0 * 2.0 ** (e - 1):
        e -= 1
    return min(max(e, lo), hi)


def code_of(x, e):
    """Code of the grid value nearest to x / 2^e, the even code of two equally near."""
    y = abs(x) / 2.0 ** e
    best = min(range(8), key=lambda c: (abs(GRID[c] - y), c & 1))
    return best | (8 if math.copysign(1.0, x) < 0 else 0)


def quantise_row(row, dtype):
    """(bytes, exponents) of one row, a list of floats."""
    row = list(row) + [0.0] * (-len(row) % 32)
    codes, scales = [], []
    for g in range(0, len(row), 32):
        part = row[g:g + 32]
        if not all(math.isfinite(x) for x in part):
            codes += [0] * 32
            scales.append(255)
            continue
        e = exponent(max(abs(x) for x in part), dtype)
        codes += [code_of(x, e) for x in part]
        scales.append(e + 127)
    return [codes[i] | codes[i + 1] << 4 for i in range(0, len(codes), 2)], scales


def quantise(x):
    """(bytes, exponents) of the rows of x, which decides the type: the definition above, on tensors."""
    lo, hi = LIMITS[x.dtype]
    D = x.shape[-1]
    y = torch.nn.functional.pad(x.double(), (0, -D % 32))
    y = y.unflatten(-1, (-(-D // 32), 32))
    top = y.abs().amax(-1)
    fine = torch.isfinite(top)
    y = torch.where(fine[..., None], y, 0.0)
    top = torch.where(fine, top, 0.0)
    part, power = torch.frexp(top / 7.0)
    e = torch.where(part == 0.5, power - 1, power)  # top / 7 <= 2^e, up to the division's rounding
    e = torch.where(top > 7.0 * torch.ldexp(torch.ones_like(top), e), e + 1, e)
    e = torch.where(top <= 7.0 * torch.ldexp(torch.ones_like(top), e - 1), e - 1, e)
    e = torch.where(top == 0, lo, e).clamp(lo, hi)
    grid = torch.tensor(GRID, dtype=torch.float64)
    off = (torch.ldexp(y.abs(), -e[..., None])[..., None] - grid).abs()
    near = off.amin(-1, keepdim=True)
    code = torch.where(off == near, torch.arange(8) % 2, 2).argmin(-1)
    code = (code | (torch.signbit(y).long() * 8)).flatten(-2)
    scale = torch.where(fine, e + 127, 255)
    code = torch.where(fine.repeat_interleave(32, -1), code, 0)
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), scale.to(torch.uint8)


def stand_for(codes, scales, D):
    """fp64 values of the rows' bytes and exponents."""
    c = torch.stack([codes.long() & 15, codes.long() >> 4], -1).flatten(-2)
    x = torch.tensor(GRID, dtype=torch.float64)[c & 7] * (1 - 2 * (c >> 3))
    e = scales.long().repeat_interleave(32, -1)
    return torch.where(e == 255, math.nan, torch.ldexp(x, e - 127))[..., :D]


class Batch4(pu.Batch):
    """A seeded batch whose cache is in 4 bits: places past a request's end, and pages of nobody, are
    NaN groups over any codes.  kc and vc are what the bytes stand for, in fp64."""

    def __init__(self, *args, order="slots", scale_order=None, **kw):
        super().__init__(*args, **kw)
        self.order, self.scale_order = order, scale_order or order
        self.D = self.q.shape[2]
        self.requantise()

    def requantise(self):
        g = torch.Generator().manual_seed(5)
        self.bytes = {}
        for name in "kv":
            x = getattr(self, name + "c").to(self.dtype)
            codes, scales = quantise(x)
            junk = torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8)
            codes = torch.where((scales == 255).repeat_interleave(16, -1), junk, codes)
            self.bytes[name], self.bytes[name + "s"] = self.ordered(codes, self.order), self.ordered(scales, self.scale_order)
        self.refresh()

    def refresh(self):
        """kc and vc out of the bytes."""
        self.kc = stand_for(self.bytes["k"], self.bytes["ks"], self.D)
        self.vc = stand_for(self.bytes["v"], self.bytes["vs"], self.D)

    @staticmethod
    def ordered(x, order):
        pages, P, H, n = x.shape
        if order == "slots":
            return x.clone()
        if order == "heads":
            return x.transpose(1, 2).contiguous().transpose(1, 2)
        if order == "padded":  # rows, heads, places and pages with room between them
            base = torch.full((pages, P + 1, H + 2, n + 16), 7, dtype=torch.uint8)
            base[:, :P, :H, :n] = x
            return base[:, :P, :H, :n]
        both = torch.stack([x, x], 1)  # "pairs": every page twice, one behind the other
        return both[:, 1]

    def cache(self, device):
        """(kcache, vcache, kscale, vscale) on the device, with the strides that they have here."""
        return tuple(self._put(self.bytes[n], device) for n in ("k", "v", "ks", "vs"))

    @staticmethod
    def _put(t, device):
        base = t
        while base._base is not None:
            base = base._base
        return base.to(device).as_strided(t.shape, t.stride(), t.storage_offset())

    def upload(self, device="cuda:0"):
        return (self._put(self.q, device), *self.cache(device), self.ints(self.table, device).view(len(self.seq), -1),
                self.ints(self.seq, device), self.ints(self.qptr, device))


def query_error(b, scale, pieces):
    """Bound on a score's error by the query's pieces, T x Hq: a group's rest is at most 2^-12 (three), 2^-17 or
    2^-22 of a unit, which is at most the group's largest value / 3.75; the keys' values multiply it."""
    unit = 2.0 ** (3 - 5 * pieces) / 3.75
    T, Hq, D = b.q.shape
    G = Hq // b.kc.shape[2]
    pad = (0, -D % 32)
    top = torch.nn.functional.pad(b.q.double(), pad).unflatten(-1, (-1, 32)).abs().nan_to_num(0.0, 0.0, 0.0).amax(-1)
    k = torch.nn.functional.pad(b.kc.abs().nan_to_num(0.0, 0.0, 0.0), pad)
    k = k.unflatten(-1, (-1, 32)).sum(-1).amax((0, 1))  # Hkv x groups: no key has more
    return unit * scale * (top * k.repeat_interleave(G, 0)).sum(-1)


def check(b, out, lse, ref, scale=None, logits=8.0):
    """Every element of out (and lse) within the bounds of the fp64 reference: paged_util's, and what the query's
    pieces and, in fp32, the weights' three pieces (2^-26 of each) leave."""
    D = b.q.shape[2]
    scale = D ** -0.5 if scale is None else scale
    want, want_lse, weight = ref
    assert out.dtype == b.dtype
    S = max(b.seq + [1])
    vmax = float(b.vc.nan_to_num(0.0, 0.0, 0.0).abs().max()) if b.vc.numel() else 0.0
    extra = query_error(b, scale, 5 if b.dtype == torch.float32 else 3 if lse is None else 4)
    tol = pu.tolerance(b.dtype, weight, S, D, vmax, logits) + 2 * extra[..., None] * (1 + extra[..., None]) * weight
    tol = tol + 2.0 ** -25 * weight
    err = (out.double().cpu() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), "out: %d of %d off, worst %.3g of its bound at %s" % (
        int(bad.sum()), bad.numel(), float((err / tol)[bad].max()), bad.nonzero()[0].tolist())
    if lse is not None:
        got = lse.double().cpu()
        empty = want_lse == -math.inf
        assert (got[empty] == -math.inf).all()
        off = (got - want_lse)[~empty].abs()
        assert (off <= (pu.lse_tolerance(S, D, logits) + extra)[~empty] + 1e-6 * want_lse[~empty].abs()).all(), float(off.max())


# ------------------------------------------------------------ the pages' life


class Books:
    """Tables, lengths and shares as lists, and what the calls make of them, one page after the other."""

    def __init__(self, table, seq, shares, P):
        self.table, self.seq, self.shares, self.P = [list(r) for r in table], list(seq), list(shares), P
        self.pages, self.W = len(shares), len(table[0]) if table else 0

    def length(self, r):
        return min(max(self.seq[r], 0), self.W * self.P)

    def held(self, r):
        return -(-self.length(r) // self.P)

    def is_page(self, p):
        return 0 <= p < self.pages

    def fork(self, parents, children, free):
        R, pairs, taken, lost = len(self.seq), [], 0, 0
        for p, c in zip(parents, children):
            pair = [-1, -1]
            if 0 <= p < R and 0 <= c < R and p != c:
                S = self.length(p)
                full = S // self.P
                row = [-1] * self.W
                for j in range(full):
                    if self.is_page(self.table[p][j]):
                        row[j] = self.table[p][j]
                        self.shares[row[j]] += 1
                if S % self.P and self.is_page(self.table[p][full]):
                    f = free[taken] if taken < len(free) else -1
                    taken += 1
                    if self.is_page(f):
                        row[full] = f
                        pair = [self.table[p][full], f]
                    else:
                        lost += 1
                self.table[c], self.seq[c] = row, S
            pairs.append(pair)
        return pairs, [taken, lost]

    def free(self, rows):
        freed, given = [], 0
        for r in rows:
            if not 0 <= r < len(self.seq):
                continue
            for j in range(self.held(r)):
                p = self.table[r][j]
                self.table[r][j] = -1
                if not self.is_page(p):
                    continue
                given += 1
                if self.shares[p] > 0:
                    self.shares[p] -= 1
                elif p not in freed:
                    freed.append(p)
            self.seq[r] = 0
        return sorted(freed), [len(freed), given]

    def compact(self):
        used = sorted({self.table[r][j] for r in range(len(self.seq)) for j in range(self.held(r))
                       if self.is_page(self.table[r][j])})
        n = len(used)
        movers = [p for p in used if p >= n]
        holes = sorted(set(range(n)) - set(used))
        to = dict(zip(movers, holes))
        for r in range(len(self.seq)):
            for j in range(self.held(r)):
                self.table[r][j] = to.get(self.table[r][j], self.table[r][j])
        for a, b in to.items():
            self.shares[b], self.shares[a] = self.shares[a], 0
        return [[a, to[a]] for a in movers], [n, len(movers)]
