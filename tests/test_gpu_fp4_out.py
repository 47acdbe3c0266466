"""Attention over the 4-bit cache where lse is not asked for, on the GPU against its definition in 64 bits: the
many-row kernel with as few pieces of the query as out needs, and rows beside those of the call."""
import math

import pytest
import torch

import paper_2205_11622_amd as slnr
from tests import fp4_util as fu
from tests import paged_util as pu

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
PIECES = {BF16: 3, FP16: 4, FP32: 5}


def attend(b, gpu, window=0, max_new=0, qptr=None, lse=None):
    """out, with 8 rows of sevens before and behind it that have to stay."""
    up = b.upload(gpu)
    q = up[0]
    T = q.shape[0]
    base = torch.full((T + 16, *q.shape[1:]), 7.0, dtype=q.dtype, device=gpu)
    at = up[-1] if qptr is None else b.ints(qptr, gpu)
    slnr.sparselnr_paged_attention_fp4(*up[:-1], at, window=window, max_new=max_new, out=base[8:8 + T], lse=lse)
    torch.cuda.synchronize()
    assert (base[:8] == 7).all() and (base[8 + T:] == 7).all()
    return base[8:8 + T].cpu()


def check(b, out, ref, extra, logits=8.0, nan=False):
    """out within paged_util's bound for its type, what the query's pieces leave (`extra`), and 2^-25 of fp32's
    weights in three pieces; NaN (nan: there may be any) where the definition has it."""
    want, _, weight = ref
    D = b.q.shape[2]
    vmax = float(b.vc.nan_to_num(0.0, 0.0, 0.0).abs().max())
    tol = pu.tolerance(b.dtype, weight, max(b.seq + [1]), D, vmax, logits) + extra + 2.0 ** -25 * weight
    assert out.dtype == b.dtype and (nan or not want.isnan().any())
    assert torch.equal(out.isnan(), want.isnan())
    fine = ~want.isnan()
    err = (out.double() - want).abs()
    bad = fine & ~(err <= tol)
    assert not bad.any(), "%d of %d off, worst %.3g of its bound at %s" % (
        int(bad.sum()), bad.numel(), float((err / tol)[bad].max()), bad.nonzero()[0].tolist())


def pieces_bound(b, weight):
    """What a type's pieces may do to out: a score off by x makes its weight, and the sum, off by x relative."""
    x = fu.query_error(b, b.q.shape[2] ** -0.5, PIECES[b.dtype])[..., None]
    return 2 * x * (1 + x) * weight


def compare(b, gpu, window=0, max_new=0, nan=False):
    ref = b.reference(window=window)
    out = attend(b, gpu, window, max_new)
    check(b, out, ref, pieces_bound(b, ref[2]), nan=nan)
    return out


# ------------------------------------------------------------ the default call of a chunk


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("D", [8, 64, 96, 128, 200, 256])
@pytest.mark.parametrize("P", [16, 64])
def test_widths_and_pages(gpu, dtype, D, P):
    compare(fu.Batch4([0, 5, 130], [70, 1, 301], 4, 2, D, P, dtype, seed=D + 3), gpu)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("window", [1, 31, 64, 100])
@pytest.mark.parametrize("D,P", [(64, 64), (128, 16), (256, 64)])
def test_windows(gpu, dtype, window, D, P):
    compare(fu.Batch4([0, 3, 400], [90, 90, 90], 4, 2, D, P, dtype, seed=window), gpu, window=window)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("D,P", [(64, 16), (64, 64), (128, 16), (128, 64), (256, 16), (256, 64)])
def test_pages_that_are_not_there(gpu, dtype, D, P):
    b = fu.Batch4([300, 64, 10], [90] * 3, 8, 2, D, P, dtype, seed=5)
    for j in (0, 3, 4):
        b.table[0][j] = -1
    b.table[1] = [-1] * len(b.table[1])  # nothing left: empty rows
    b.table[2][0] = b.kc.shape[0]        # past the cache
    out = compare(b, gpu)
    assert (out[b.qptr[1]:b.qptr[2]] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("D,P", [(64, 16), (64, 64), (128, 16), (128, 64), (256, 16), (256, 64)])
def test_nan_groups(gpu, dtype, window, D, P):
    """NaN in V and K of the newest tokens, and of one that only the first tokens still see."""
    b = fu.Batch4([61, 0], [130, 80], 4, 2, D, P, dtype, seed=9)
    S, n = b.seq[0], b.bytes["vs"].shape[3]

    def at(j, *rest):
        return (b.table[0][j // P], j % P, *rest)
    b.bytes["vs"][at(S - 1, slice(None), n - 1)] = 255
    b.bytes["vs"][at(S - 2, 0, 0)] = 255
    if window:
        b.bytes["vs"][at(30, slice(None), 0)] = 255
    b.bytes["ks"][at(S - 1, 1, 0)] = 255
    b.refresh()
    compare(b, gpu, window=window, nan=True)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("P", [32, 64])
def test_long_contexts_are_cut_and_joined(gpu, dtype, D, P):
    compare(fu.Batch4([4000], [170], 4, 2, D, P, dtype, seed=11), gpu, max_new=170)


@pytest.mark.parametrize("Hq,Hkv", [(3, 3), (7, 1), (12, 4), (128, 1)])
def test_head_layouts(gpu, Hq, Hkv):
    compare(fu.Batch4([100, 0, 37], [40, 1, 90], Hq, Hkv, 128, 16, BF16, seed=Hq), gpu)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("new", [1, 20, 130])
@pytest.mark.parametrize("D,P", [(64, 64), (128, 16), (128, 64), (256, 64)])
def test_nan_groups_that_all_tokens_see(gpu, dtype, new, D, P):
    """In tiles that are whole: columns of V's group are NaN, and of a head whose K is, all."""
    b = fu.Batch4([300, 70], [new, new], 4, 2, D, P, dtype, seed=19)
    b.bytes["vs"][b.table[0][5 // P], 5 % P, 0, 1] = 255
    b.bytes["vs"][b.table[0][130 // P], 130 % P, :, 0] = 255
    b.bytes["ks"][b.table[1][40 // P], 40 % P, 1, 1] = 255
    b.refresh()
    out = compare(b, gpu, nan=True)
    assert out[:new, :2, :64].isnan().all() and not out[:new, :2, 64:].isnan().any() and not out[:new, 2:, 32:].isnan().any()
    assert out[new:, 2:].isnan().all() and not out[new:, :2].isnan().any()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("D,P", [(64, 64), (128, 16), (256, 64)])
def test_values_at_the_ends_of_the_type(gpu, dtype, new, D, P):
    """A page a token of which nothing but one key is there: out is its value, from subnormals of fp16 to 6 * 2^125."""
    lo, hi = fu.LIMITS[dtype]
    b = fu.Batch4([0, 0], [new, new], 4, 2, D, P, dtype, seed=20)
    g = torch.Generator().manual_seed(3)
    for r in range(2):
        for x in ("v", "vs", "k", "ks"):
            page = b.bytes[x][b.table[r][0]]
            page[0] = torch.randint(0, 256, page[0].shape, generator=g, dtype=torch.uint8)
        b.bytes["ks"][b.table[r][0], 0] = 120
        b.bytes["vs"][b.table[r][0], 0] = torch.tensor([lo + 127, hi + 127][r], dtype=torch.uint8)
    b.seq = [1, 1]  # more tokens than positions: the last one sees the key, those before it nothing
    b.refresh()
    out = attend(b, gpu)
    for r in range(2):
        want = b.vc[b.table[r][0], 0].repeat_interleave(2, 0)
        assert want.abs().max() == 6 * 2.0 ** [lo, hi][r]
        assert torch.equal(out[b.qptr[r + 1] - 1].double(), want) and (out[b.qptr[r]:b.qptr[r + 1] - 1] == 0).all()


# ------------------------------------------------------------ channels of very different size


def with_outliers(b, by):
    """A channel of each group `by` times the others in q, and the others `by` times it in K: all count alike."""
    b.q = b.q.clone()
    b.q[..., 5::32] *= by
    b.kc = b.kc.to(b.dtype)
    b.kc[..., 5::32] /= by
    b.vc = b.vc.to(b.dtype)
    b.requantise()
    return b


def first_order(b, window=0):
    """Bound on what the query's pieces do to out, T x Hq x D.  With q off by r, scores are off by s = scale r.k and
    out by sum_j p_j (v_j - out) s_j = scale sum_d r_d C_d, C_d = sum_j p_j (v_j - out) k_jd, and by less than 2 x^2
    of the weighted |v| beyond that, x the largest |s_j|.  |r_d| is at most 2^(3 - 5 pieces) / 3.75 of its group's largest value."""
    T, Hq, D = b.q.shape
    G, P, scale = Hq // b.kc.shape[2], b.P, D ** -0.5
    unit = 2.0 ** (3 - 5 * PIECES[b.dtype]) / 3.75
    top = torch.nn.functional.pad(b.q.double(), (0, -D % 32)).unflatten(-1, (-1, 32)).abs().amax(-1)
    rest = unit * top.repeat_interleave(32, -1)[..., :D]
    bound = torch.zeros(T, Hq, D, dtype=torch.float64)
    for r, S in enumerate(b.seq):
        k, v, there = pu.gather(b.kc, b.vc, b.table[r], list(range(S)))
        for t in range(b.qptr[r], b.qptr[r + 1]):
            n = S - b.qptr[r + 1] + t + 1
            seen = there[:n] & (torch.arange(n) >= n - window if window else True)
            for h in range(Hq):
                kk, vv = k[:n][seen, h // G], v[:n][seen, h // G]
                p = torch.softmax(kk @ b.q[t, h].double() * scale, 0)
                c = (p[:, None] * kk).t() @ (vv - p @ vv)
                x = scale * (rest[t, h] * kk.abs()).sum(1).max()
                bound[t, h] = scale * (rest[t, h] @ c.abs()) + 2 * x * x * (p @ vv.abs())
    return bound


@pytest.mark.parametrize("dtype,D,P,by", [(FP16, 64, 64, 100), (FP16, 96, 16, 100), (FP16, 128, 64, 100), (FP16, 128, 32, 200),
                                          (FP16, 256, 64, 100), (BF16, 128, 64, 100), (BF16, 256, 16, 100),
                                          (FP32, 128, 64, 100)])
def test_channels_of_very_different_size(gpu, dtype, D, P, by):
    """What the pieces leave is the type's own bound at most, by their number of pieces."""
    b = with_outliers(fu.Batch4([0, 120], [90, 70], 4, 2, D, P, dtype, seed=31), by)
    ref = b.reference()
    check(b, attend(b, gpu), ref, first_order(b))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("power", [100, 112, 120])
@pytest.mark.parametrize("P", [16, 64])
def test_very_small_queries(gpu, dtype, power, P):
    """Queries near the least numbers and keys as large: the last piece's unit is at least 2^-125 and its steps an eighth
    of it, so what is left is 2^-128 at most, of q by few rows and of q * scale * log2(e) by many."""
    b = fu.Batch4([200, 90], [1, 80], 4, 2, 64, P, dtype, seed=10, amp=2.0 ** power)
    b.q = (b.q.double() * 2.0 ** -power).to(dtype)
    ref = b.reference()
    k = b.kc.abs().nan_to_num(0.0, 0.0, 0.0).sum(-1).amax((0, 1)).repeat_interleave(2)  # no key has more
    x = (fu.query_error(b, 0.125, PIECES[dtype]) + 2.0 ** -128 * k)[..., None]
    check(b, attend(b, gpu), ref, 2 * x * (1 + x) * ref[2])


@pytest.mark.parametrize("dtype", [FP16, FP32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("P", [16, 64])
def test_out_does_not_depend_on_lse(gpu, dtype, D, P):
    """Where lse is exact enough with the pieces that out has, both calls are one."""
    b = fu.Batch4([0, 5, 130], [70, 1, 301], 4, 2, D, P, dtype, seed=D + 1)
    lse = torch.full(b.q.shape[:2], math.nan, device=gpu)
    assert torch.equal(attend(b, gpu), attend(b, gpu, lse=lse)) and not lse.isnan().any()


# ------------------------------------------------------------ offsets that do not fit


@pytest.mark.parametrize("what", ["tokens past T", "backwards", "negative"])
@pytest.mark.parametrize("n", [3, 90])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_offsets_that_do_not_fit(gpu, what, n, dtype):
    """Offsets count as the nearest ones in [0, T], and a request that ends before it begins has no tokens: what is
    left is attended, and other rows stay as they were."""
    b = fu.Batch4([200, 200], [n, n], 4, 2, 64, 16, dtype, seed=7)
    b.q = torch.cat([b.q, b.q[:n]])
    T = 3 * n
    qptr, held = {"tokens past T": ([0, n, 100 * n], [0, n, T]), "backwards": ([0, 2 * n, n], [0, 2 * n, 2 * n]),
                  "negative": ([-5, n, 2 * n], [0, n, 2 * n])}[what]
    out = attend(b, gpu, qptr=qptr)
    assert (out[held[-1]:] == 7).all()
    b.qptr = held
    b.q, out = b.q[:held[-1]], out[:held[-1]]
    ref = b.reference()
    check(b, out, ref, pieces_bound(b, ref[2]))
