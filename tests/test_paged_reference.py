"""The 64-bit definitions that the GPU tests compare with, against closed forms (CPU)."""
import math

import pytest
import torch

from tests import paged_util as pu


def batch(ctx, new, Hq=4, Hkv=2, D=8, P=4, **kw):
    return pu.Batch(ctx, new, Hq, Hkv, D, P, torch.float32, **kw)


def rows(b, r, h):
    """K and V rows of request r, KV head h, in the order of positions."""
    at = [(b.table[r][j // b.P], j % b.P) for j in range(b.seq[r])]
    return (torch.stack([c[p, i, h] for p, i in at]).double() for c in (b.kc, b.vc))


def test_one_key_is_its_value():
    b = batch([0], [1])
    out, lse, weight = b.reference(scale=0.5)
    for h in range(4):
        k, v = rows(b, 0, h // 2)
        assert torch.equal(out[0, h], v[0]) and torch.equal(weight[0, h], v[0].abs())
        assert float(lse[0, h]) == pytest.approx(0.5 * float(b.q[0, h].double() @ k[0]), abs=1e-14)


def test_equal_scores_give_the_mean():
    b = batch([9], [2])
    b.q.zero_()
    out, lse, _ = b.reference()
    for h in range(4):
        _, v = rows(b, 0, h // 2)
        for t, n in ((0, 10), (1, 11)):  # causal: the first token does not see the second
            assert torch.allclose(out[t, h], v[:n].mean(0), rtol=0, atol=1e-14)
            assert float(lse[t, h]) == pytest.approx(math.log(n), abs=1e-14)


def test_two_keys_whose_scores_differ_by_log_3():
    b = batch([1], [1], Hq=1, Hkv=1)
    p = b.table[0][0]
    b.q[0, 0] = torch.tensor([1.0] + [0.0] * 7)
    b.kc[p, 0, 0], b.kc[p, 1, 0] = 0.0, 0.0
    b.kc[p, 0, 0, 0] = 1.0
    out, lse, _ = b.reference(scale=math.log(3.0))
    _, v = rows(b, 0, 0)
    assert torch.allclose(out[0, 0], 0.75 * v[0] + 0.25 * v[1], rtol=0, atol=1e-14)
    assert float(lse[0, 0]) == pytest.approx(math.log(4.0), abs=1e-14)


@pytest.mark.parametrize("window", [1, 3])
def test_a_window_holds_the_tokens_own_key_and_those_before(window):
    b = batch([20], [3])
    b.q.zero_()
    out, lse, _ = b.reference(window=window)
    _, v = rows(b, 0, 1)
    for t in range(3):
        p = 20 + t
        assert torch.allclose(out[t, 2], v[p - window + 1:p + 1].mean(0), rtol=0, atol=1e-14)
        assert float(lse[t, 2]) == pytest.approx(math.log(window), abs=1e-14)


def test_rows_that_see_nothing():
    b = batch([5, 6], [2, 1])
    b.table[0] = [-1] * len(b.table[0])
    out, lse, _ = b.reference()
    assert (out[:2] == 0).all() and (lse[:2] == -math.inf).all()
    assert torch.isfinite(lse[2]).all()
    b.table[1][0] = b.kc.shape[0]  # past the cache: the first four keys are not seen
    b.q.zero_()
    _, v = rows(batch([5, 6], [2, 1]), 1, 0)
    out, _, _ = b.reference()
    assert torch.allclose(out[2, 0], v[4:].mean(0), rtol=0, atol=1e-14)


def test_selected_pages_only():
    b = batch([10], [1])
    b.q.zero_()
    out, lse, _ = b.reference(sel=[[[0, 2, -1], [1, 9, -5]]])
    _, v = rows(b, 0, 0)
    assert torch.allclose(out[0, 0], torch.cat([v[:4], v[8:11]]).mean(0), rtol=0, atol=1e-14)
    _, v = rows(b, 0, 1)
    assert torch.allclose(out[0, 3], v[4:8].mean(0), rtol=0, atol=1e-14)
    assert float(lse[0, 3]) == pytest.approx(math.log(4), abs=1e-14)


def test_tables_of_a_batch_done_by_hand():
    got = pu.page_tables([5, 0, 4], [4, 0, 1], [[7, 3, -1], [-1] * 3, [2, -1, -1]], [9, 8], 6, 4)
    assert got[0] == [0, 4, 4, 5] and got[1] == [9, 0, 5]
    assert got[2] == [13, 14, 15, 36, 32, -1]  # places 1 to 3 of page 3, page 9, then page 8
    assert got[3] == [5, 2, 0] and got[4] == [[7, 3, 9], [-1] * 3, [2, 8, -1]]


def test_summary_done_by_hand():
    kq, ks = pu.summary(torch.tensor([[1.0, -2.0, 0.0], [3.0, -6.0, 0.5]], dtype=torch.float64))
    step = float(torch.tensor(4.0) * torch.tensor(1.0 / 127.0))
    assert ks == step and kq.tolist() == [round(2 / step), -127, round(0.25 / step)]
    assert pu.summary(torch.zeros(2, 3, dtype=torch.float64))[1] == 0.0
    assert pu.summary(torch.tensor([[math.inf, 0.0]], dtype=torch.float64))[1] == math.inf


def test_selection_done_by_hand():
    """Scores 3, 1, 3, 2 and the token's own page, which is forced: ties go to the lower page."""
    P, D = 2, 8
    q = torch.zeros(1, 1, D)
    q[0, 0, 0] = 1.0  # 127 in 8 bits
    kq = torch.zeros(6, 1, D, dtype=torch.int8)
    table = [[4, 2, 0, 1, 5, -1]]
    for page, level in zip(table[0], (3, 1, 3, 2, -100)):
        kq[page, 0, 0] = level
    ks = torch.ones(6, 1)
    pick = lambda top, first, local: pu.select(q, kq, ks, table, [9], [0, 1], P, top, first, local)[0, 0].tolist()  # noqa: E731
    assert pick(1, 0, 0) == [0] and pick(2, 0, 0) == [0, 2] and pick(3, 0, 0) == [0, 2, 3]
    assert pick(2, 0, 1) == [0, 4] and pick(3, 1, 1) == [0, 2, 4] and pick(6, 0, 0) == [0, 1, 2, 3, 4, -1]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_tolerances_hold_what_one_rounding_does(dtype):
    """A result rounded once is within the bound, one that is off by four units is not."""
    x = torch.linspace(0.3, 1.9, 1001, dtype=torch.float64)
    tol = pu.tolerance(dtype, x, 1, 8, 2.0)
    assert ((x.to(dtype).double() - x).abs() <= tol).all()
    if dtype != torch.float32:
        assert (8 * pu.EPS[dtype] * x > tol).all()
