"""The plain forms of the 4-bit cache and of the pages' life against closed forms (CPU)."""
import math

import pytest
import torch

from tests import fp4_util as fu


def test_exponents_at_the_borders():
    for e in (-100, -3, 0, 5, 60):
        top = 7.0 * 2.0 ** e
        assert fu.exponent(top, torch.float32) == e
        assert fu.exponent(math.nextafter(top, math.inf), torch.float32) == e + 1
    assert fu.exponent(0.0, torch.float16) == -23 and fu.exponent(65504.0, torch.float16) == 13
    assert fu.exponent(2.0 ** -24, torch.float16) == -23
    assert fu.exponent(3.3e38, torch.bfloat16) == 125 and fu.exponent(1e-45, torch.float32) == -125


@pytest.mark.parametrize("x,code", [(0.25, 0), (0.2500001, 1), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (2.6, 5), (3.5, 6),
                                    (5.0, 6), (5.1, 7), (7.0, 7), (-0.25, 8), (-1.0, 10), (0.0, 0)])
def test_ties_go_to_even_codes(x, code):
    assert fu.code_of(x, 0) == code


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_tensors_and_rows_agree(dtype):
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(40, 72, generator=g) * torch.randn(40, 1, generator=g).mul(4).exp()).to(dtype)
    x[0], x[1, 40], x[2, 3], x[3, 64] = 0.0, math.inf, math.nan, -0.0
    x[4, :32] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0] * 4).to(dtype)
    codes, scales = fu.quantise(x)
    for i in range(40):
        b, e = fu.quantise_row(x[i].double().tolist(), dtype)
        assert codes[i].tolist() == b and scales[i].tolist() == e
    stand = fu.stand_for(codes, scales, 72)
    step = torch.ldexp(torch.ones_like(stand), scales.long().repeat_interleave(32, -1)[:, :72] - 127)
    fine = torch.isfinite(stand)
    whole = torch.nn.functional.pad(x.double(), (0, 24)).view(40, 3, 32).isfinite().all(2).repeat_interleave(32, 1)[:, :72]
    assert torch.equal(fine, whole) and not fine[1, 32:64].any() and not fine[2, :32].any()
    big = x.double().abs() > 7 * step  # above the largest exponent's range
    assert ((stand - x.double()).abs() <= step)[fine & ~big].all()
    assert torch.equal(stand[fine], stand.to(dtype).double()[fine])  # values of the type


def test_books_by_hand():
    b = fu.Books([[3, 5, 7, -1], [-1] * 4, [2, -1, -1, -1]], [10, 0, 4], [0] * 9, 4)
    pairs, counts = b.fork([0, 2], [1, 0][:1] + [9], [8])
    assert pairs == [[7, 8], [-1, -1]] and counts == [1, 0]
    assert b.table[1] == [3, 5, 8, -1] and b.seq == [10, 10, 4] and [b.shares[3], b.shares[5], b.shares[7]] == [1, 1, 0]
    freed, counts = b.free([0, 0, -1])
    assert freed == [7] and counts == [1, 3] and b.shares == [0] * 9 and b.seq[0] == 0
    pairs, counts = b.compact()  # 2, 3, 5, 8 are in use
    assert counts == [4, 2] and pairs == [[5, 0], [8, 1]] and b.table[1] == [3, 0, 1, -1] and b.table[2][0] == 2
