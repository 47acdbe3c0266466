"""Variants of the paged-cache kernels that the sizes of a call choose, each against the
definitions in 64 bits: pages that hold whole tiles of keys, large groups of heads, calls by
pages."""
import math
import random

import pytest
import torch

import paper_2205_11622_amd as slnr
from tests import paged_util as pu
from tests.test_gpu_paged import BF16, FP16, FP32, compare, compare_sparse, random_selection, run_attention, vmax

pytestmark = pytest.mark.gpu


# A chunk of more than 64 rows whose pages hold 64 positions and more has a kernel of its own.


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("D,P", [(8, 64), (64, 128), (72, 64), (128, 64), (128, 1024), (136, 64), (256, 64), (256, 128)])
def test_chunks_in_pages_of_whole_tiles(gpu, dtype, D, P):
    """One is cut and joined, one begins in the middle of a page, one has no context."""
    b = pu.Batch([1500, 130, 0], [67, 40, 150], 4, 2, D, P, dtype, seed=D + P)
    print(dtype, D, P, flush=True)
    compare(b, gpu)


@pytest.mark.parametrize("D,P,order", [(128, 64, "heads"), (128, 128, "pairs"), (64, 256, "heads"), (256, 64, "pairs")])
def test_chunks_in_pages_of_whole_tiles_in_other_orders(gpu, D, P, order):
    b = pu.Batch([700, 3], [60, 90], 6, 2, D, P, BF16, seed=D, order=order)
    compare(b, gpu)


@pytest.mark.parametrize("dtype,D,P", [(BF16, 128, 64), (FP16, 64, 128), (FP32, 128, 64), (BF16, 200, 256)])
@pytest.mark.parametrize("window", [1, 63, 64, 65, 500])
def test_windows_in_pages_of_whole_tiles(gpu, dtype, D, P, window):
    b = pu.Batch([0, 3, 900], [150, 70, 80], 4, 2, D, P, dtype, seed=window)
    for r in range(3):  # pages behind the window are given back
        for j in range(max(0, b.ctx[r] - window + 1) // P):
            b.table[r][j] = -1
    print(dtype, D, P, window, flush=True)
    compare(b, gpu, window=window)


@pytest.mark.parametrize("dtype,D,P", [(BF16, 128, 64), (FP16, 72, 64), (FP32, 64, 128), (BF16, 256, 64)])
def test_absent_pages_of_whole_tiles(gpu, dtype, D, P):
    b = pu.Batch([9 * P + 5, P, 10], [90] * 3, 8, 2, D, P, dtype, seed=5)
    for j in (0, 3, 4, 9):
        b.table[0][j] = -1
    b.table[1] = [-1] * len(b.table[1])  # nothing left: empty rows
    b.table[2][0] = b.kc.shape[0]        # past the cache
    out, lse = compare(b, gpu)
    a, e = b.qptr[1], b.qptr[2]
    assert (out[a:e] == 0).all() and (lse[a:e] == -math.inf).all()


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (FP16, 64), (FP32, 72), (BF16, 256)])
@pytest.mark.parametrize("P", [64, 128])
@pytest.mark.parametrize("window", [0, 100])
def test_infinities_and_nan_in_pages_of_whole_tiles(gpu, dtype, D, P, window):
    """Rows that hold inf and NaN reach the tokens that see them, in the columns that have them, and no other."""
    new, ctx = 130, 61
    b = pu.Batch([ctx, 0], [new, 70], 4, 2, D, P, dtype, seed=9)
    ref, _, _ = b.reference(window=window)
    S = b.seq[0]
    for j, d, x in ((S - 1, 3, math.nan), (S - 2, 5, math.inf), (S - 70, 6, -math.inf), (4, 7, math.inf)):
        if j != 4 or window:  # one that only the first tokens still see
            b.vc[b.table[0][j // P], j % P, :, d] = x
    b.kc[b.table[0][(S - 1) // P], (S - 1) % P, 1, :] = math.nan  # key of the last token, second head
    out, _ = run_attention(b, gpu, window=window)
    tol = pu.tolerance(dtype, b.reference(window=window)[2], S, D, vmax(b)).nan_to_num(math.inf, math.inf)
    fine = [d for d in range(D) if d not in (3, 5, 6, 7)]
    for i in range(new):
        p = ctx + i
        o = out[i].float()
        nan_head = p == S - 1
        assert torch.isnan(o[2:]).all() == nan_head
        for h in range(2 if nan_head else 4):
            assert bool(torch.isnan(o[h, 3])) == (p >= S - 1), (i, h)
            assert bool(o[h, 5] == math.inf) == (p >= S - 2), (i, h)
            assert bool(o[h, 6] == -math.inf) == (p >= S - 70 and (not window or p - (S - 70) < window)), (i, h)
            if window:
                assert bool(o[h, 7] == math.inf) == (p - 4 < window), (i, h)
            assert ((out[i, h, fine].double() - ref[i, h, fine]).abs() <= tol[i, h, fine]).all(), (i, h)
    assert ((out[new:].double() - ref[new:]).abs() <= tol[new:]).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("new", [1, 3])
def test_groups_of_128_heads(gpu, dtype, new):
    b = pu.Batch([200, 17], [new, new], 128, 1, 64, 64, dtype, seed=90)
    compare(b, gpu)
    compare_sparse(b, random_selection(b, 1, 3, 91), gpu)


# Selections that are gone through by pages.


def sampled(b, sel, out, lse, tokens, dtype):
    """Some tokens of a sparse call against the definition; a page that is named twice counts twice."""
    T, Hq, D = b.q.shape
    Hkv, P = b.kc.shape[2], b.P
    G = Hq // Hkv
    for t in tokens:
        r = max(i for i in range(len(b.seq)) if b.qptr[i] <= t)
        pos = b.ctx[r] + t - b.qptr[r]
        for h in range(Hkv):
            keys = [blk * P + i for blk in sel[t][h] if 0 <= blk < len(b.table[r]) for i in range(P) if blk * P + i <= pos]
            k, v, there = pu.gather(b.kc, b.vc, b.table[r], keys)
            see = there[None].expand(G, -1)
            ref, want, weight = pu.softmax_rows(b.q[t, h * G:(h + 1) * G].double(), k[:, h], v[:, h], see, D ** -0.5)
            tol = pu.tolerance(dtype, weight, len(keys) + 1, D, vmax(b))
            assert ((out[t, h * G:(h + 1) * G].double().cpu() - ref).abs() <= tol).all(), (t, h)
            got = lse[t, h * G:(h + 1) * G].double().cpu()
            some = want > -math.inf
            assert (got[~some] == -math.inf).all()
            assert ((got - want).abs()[some] <= pu.lse_tolerance(len(keys) + 1, D) + 1e-6 * want[some].abs()).all(), (t, h)


def run_sparse(b, sel, gpu):
    q, kc, vc, table, seq, qptr = b.upload(gpu)
    lse = torch.full(q.shape[:2], math.nan, device=gpu)
    return slnr.sparselnr_block_attention(q, kc, vc, table, seq, qptr, b.ints(sel, gpu), lse=lse), lse


@pytest.mark.parametrize("dtype,T,P,D", [(BF16, 3, 16, 64), (BF16, 900, 64, 128), (FP32, 700, 64, 64)])
def test_a_page_that_is_named_twice_counts_twice(gpu, dtype, T, P, D):
    """Few tokens go by queries, many by pages."""
    b = pu.Batch([12 * P + 3], [T], 8, 8, D, P, dtype, seed=92)
    sel = random_selection(b, 8, 12, 93)
    for t in range(T):
        for h in range(0, 8, 2):
            sel[t][h][8:] = [2, 2, 5, 5]
    out, lse = run_sparse(b, sel, gpu)
    sampled(b, sel, out, lse, sorted({0, 1, T // 2, T - 1}), dtype)


@pytest.mark.parametrize("G,P,D,T", [(128, 512, 64, 900), (40, 256, 128, 900), (1, 64, 64, 3000), (3, 4096, 72, 200)])
def test_by_pages_groups_of_heads(gpu, G, P, D, T):
    """Tiles of one query of 128 heads to 128 of one; pages of many tiles of keys."""
    Hkv = 1 if G > 1 else 8
    b = pu.Batch([2 * P + 9], [T], G * Hkv, Hkv, D, P, BF16, seed=94)
    top = 3 if P > 64 else 16
    sel = random_selection(b, Hkv, top, 95)
    out, lse = run_sparse(b, sel, gpu)
    sampled(b, sel, out, lse, sorted({0, 1, 130, T - 1}), BF16)


# Offsets that do not fit.


@pytest.mark.parametrize("what", ["tokens past T", "backwards", "negative"])
@pytest.mark.parametrize("new,P", [(3, 16), (70, 64)])
def test_offsets_that_do_not_fit_leave_guards_and_other_rows(gpu, what, new, P):
    """Offsets outside [0, T] end there; queries are read and results written inside their tensors only (NaN and a
    mark lie around them), and the tokens that a request is left with are right."""
    b = pu.Batch([3 * P + 5, 30], [new, new], 4, 2, 64, P, BF16, seed=7)
    _, kc, vc, table, seq, _ = b.upload(gpu)
    T = 2 * new
    qptr = {"tokens past T": [0, new, 3 * T + 100], "backwards": [0, T, new], "negative": [-5, new, T]}[what]
    ends = {"tokens past T": [0, new, T], "backwards": [0, T, T], "negative": [0, new, T]}[what]
    ptr = b.ints(qptr, gpu)
    around = torch.full((T + 16, 4, 64), math.nan, dtype=BF16, device=gpu)
    around[8:8 + T] = b.q.to(gpu)
    q = around[8:8 + T]
    kq = torch.zeros(kc.shape[0], 2, 64, dtype=torch.int8, device=gpu)
    marks = torch.full((T + 16, 2, 4), 77, dtype=torch.int32, device=gpu)
    slnr.sparselnr_block_select(q, kq, torch.ones(kc.shape[0], 2, device=gpu), table, seq, ptr, P, 4, sel=marks[8:8 + T])
    want = pu.select(b.q, kq.cpu(), torch.ones(kc.shape[0], 2), b.table, b.seq, ends, P, 4, 1, 1)
    assert torch.equal(marks[8:8 + T].cpu(), want)
    assert (marks[:8] == 77).all() and (marks[8 + T:] == 77).all()
    for sel in (None, marks[8:8 + T]):
        out = torch.full((T + 16, 4, 64), 7.0, dtype=BF16, device=gpu)
        lse = torch.full((T + 16, 4), 7.0, device=gpu)
        if sel is None:
            slnr.sparselnr_paged_attention(q, kc, vc, table, seq, ptr, out=out[8:8 + T], lse=lse[8:8 + T])
        else:
            slnr.sparselnr_block_attention(q, kc, vc, table, seq, ptr, sel, out=out[8:8 + T], lse=lse[8:8 + T])
        for x in (out, lse):
            assert (x[:8] == 7).all() and (x[8 + T:] == 7).all()
        ref = pu.attention(b.q, b.kc, b.vc, b.table, b.seq, ends, 0.125, sel=None if sel is None else sel.tolist())
        pu.check(out[8:8 + T].cpu(), lse[8:8 + T], ref, BF16, max(b.seq), 64, vmax(b))


# Selections whose number is no multiple of four (queries in LDS behind rows of any length).


@pytest.mark.parametrize("top", [1, 2, 3, 5, 6, 7, 255])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_select_any_number_of_pages(gpu, top, D):
    rng = random.Random(top)
    b = pu.Batch([rng.randrange(100, 700), 90], [1, 1], 4, 2, D, 4, BF16, seed=top)
    g = torch.Generator().manual_seed(D)
    kq = torch.randint(-127, 128, (b.kc.shape[0], 2, D), generator=g).to(torch.int8)
    ks = torch.rand(b.kc.shape[0], 2, generator=g)
    q, _, _, table, seq, qptr = b.upload(gpu)
    got = slnr.sparselnr_block_select(q, kq.to(gpu), ks.to(gpu), table, seq, qptr, 4, top, first=0, local=1).cpu()
    assert torch.equal(got, pu.select(b.q, kq, ks, b.table, b.seq, b.qptr, 4, top, 0, 1))


@pytest.mark.parametrize("dtype,D,P", [(BF16, 64, 64), (FP16, 128, 32), (FP32, 64, 64), (BF16, 256, 128)])
def test_chunks_whose_last_tiles_are_cut_finer(gpu, dtype, D, P):
    """Eight tiles more than the GPU has units, 42 steps of 64 keys and more each."""
    units = torch.cuda.get_device_properties(0).multi_processor_count
    rows = 128 if dtype == FP32 or D > 128 else 256  # of a tile; 8 KV heads of 32 heads each
    T = (units + 8) * rows // 256
    b = pu.Batch([2700], [T], 256, 8, D, P, dtype, seed=96)
    q, kc, vc, table, seq, qptr = b.upload(gpu)
    lse = torch.full(q.shape[:2], math.nan, device=gpu)
    out = slnr.sparselnr_paged_attention(q, kc, vc, table, seq, qptr, lse=lse)
    again = slnr.sparselnr_paged_attention(q, kc, vc, table, seq, qptr)
    assert torch.equal(out, again) and torch.isfinite(lse).all()
    every = list(range(len(b.table[0])))
    sampled(b, [[every] * 8] * T, out, lse, sorted({0, 1, 5, T // 3, T // 2, 3 * T // 4, T - 9, T - 1}), dtype)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("P", [16, 64])
def test_the_largest_weight_is_not_rounded_at_64_columns(gpu, dtype, P):
    """Two keys matter, the second, of the larger score, in a later tile and alone with a value: the result is its weight
    over the sum, which is rounded once only if the weight is exactly one."""
    T, ctx = 60, 200
    b = pu.Batch([ctx], [T], 2, 1, 64, P, dtype, seed=97)
    b.q.zero_()
    b.q[:, :, 0] = torch.linspace(0.5, 5.5, 2 * T).view(T, 2).to(dtype)
    k = torch.zeros(ctx + T, 64)
    k[:, 0] = -64.0
    k[3, 0], k[130, 0] = 0.0, 1.0
    v = torch.zeros(ctx + T, 64)
    v[130] = 1.0
    for j in range(ctx + T):
        b.kc[b.table[0][j // P], j % P, 0], b.vc[b.table[0][j // P], j % P, 0] = k[j].to(dtype), v[j].to(dtype)
    out, _ = run_attention(b, gpu, scale=1.0)
    x = b.q[:, :, :1].double()
    want = (1 / (1 + (-x).exp())).expand(-1, -1, 64)  # the others weigh below e^-32
    # one rounding of a number of [1/2, 1): half a unit, which is EPS / 2; the rest in 32 bits
    assert ((out.double() - want).abs() <= pu.EPS[dtype] / 2 + 2.0 ** -20).all()
