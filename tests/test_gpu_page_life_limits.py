"""The pages' life at the largest tables that it takes, on the GPU."""
import pytest
import torch

import paper_2205_11622_amd as slnr

pytestmark = pytest.mark.gpu

I32 = torch.int32
WIDEST = 2 ** 31 - 4096  # entries of a row, of pages of one position


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def test_the_widest_rows(gpu):
    """Rows of 8 GB: the last step of those who go along them ends past 2^31.  Neighbours stay as they were."""
    table = torch.full((4, WIDEST), -1, dtype=I32, device=gpu)
    table[0, :10] = torch.arange(10, dtype=I32, device=gpu)
    table[0, -3:] = torch.tensor([20, 21, 22], dtype=I32, device=gpu)
    table[1] = 99  # of no page: forgotten
    table[3, 0] = 30
    seq = torch.tensor([WIDEST, 0, WIDEST, 1], dtype=I32, device=gpu)
    shares = torch.zeros(40, dtype=I32, device=gpu)
    ints = lambda *v: torch.tensor(v, dtype=I32, device=gpu)  # noqa: E731
    pairs, counts = slnr.sparselnr_page_fork(ints(0), ints(1), table, seq, shares, ints(), 1)
    assert pairs.tolist() == [[-1, -1]] and counts.tolist() == [0, 0]
    assert seq.tolist() == [WIDEST, WIDEST, WIDEST, 1]
    want = torch.zeros(40, dtype=I32, device=gpu)
    want[:10] = want[20:23] = 1
    assert torch.equal(shares, want) and torch.equal(table[0], table[1])
    assert (table[2] == -1).all() and (table[3, 1:] == -1).all() and table[3, 0] == 30
    # two rows given up, the other two moved
    freed, counts = slnr.sparselnr_page_free(ints(0, 2), table, seq, shares, 1, freed=ints(7, 7))
    assert counts.tolist() == [0, 13] and freed.tolist() == [-1, -1] and (shares == 0).all()
    assert (table[0] == -1).all() and (table[2] == -1).all()
    pairs, counts = slnr.sparselnr_page_compact(table, seq, shares, 1)
    assert counts.tolist() == [14, 4] and pairs[:5].tolist() == [[20, 10], [21, 11], [22, 12], [30, 13], [-1, -1]]
    assert table[1, :10].tolist() == list(range(10)) and table[1, -3:].tolist() == [10, 11, 12] and table[3, 0] == 13
    assert (table[1, 10:-3] == -1).all() and (table[0] == -1).all() and (table[2] == -1).all()


def test_more_entries_than_a_count_holds(gpu):
    """64 rows of 2^25 + 1000 entries, 2^31 + 64000 in all, over a million pages whose shares are too low by far."""
    R, W, pages = 64, 2 ** 25 + 1000, 1 << 20
    table = torch.arange(W, dtype=I32, device=gpu).remainder_(pages).repeat(R, 1)
    seq = torch.full((R,), W, dtype=I32, device=gpu)
    shares = torch.zeros(pages, dtype=I32, device=gpu)
    freed, counts = slnr.sparselnr_page_free(torch.arange(R, dtype=I32, device=gpu), table, seq, shares, 1)
    assert counts.tolist() == [pages, 2 ** 31 - 1]
    assert torch.equal(freed, torch.arange(pages, dtype=I32, device=gpu))
    assert (table == -1).all() and (seq == 0).all() and (shares == 0).all()
