"""Rows that share pages, rows given up, pages moved and copied, on the GPU against the same by lists."""
import random

import pytest
import torch

import paper_2205_11622_amd as slnr
from tests import fp4_util as fu

pytestmark = pytest.mark.gpu

I32 = torch.int32


class Held:
    """Seeded books and their tensors: rows with prefixes in common, entries that are no pages, a table with
    room between its rows."""

    def __init__(self, gpu, R, W, P, pages, seed, extra=0, holes=True, empty=0.2):
        rng = random.Random(seed)
        self.rng = rng
        pool = list(range(pages))
        rng.shuffle(pool)
        table, seq = [], []
        for r in range(R):
            S = 0 if rng.random() < empty else rng.randrange(0, W * P + 1)
            n = -(-S // P)
            row = [-1] * W
            share = 0
            if table and rng.random() < 0.5:
                f = rng.randrange(len(table))
                share = rng.randrange(0, min(seq[f], S) // P + 1)
                row[:share] = table[f][:share]
            for j in range(share, n):
                if not pool:
                    S = j * P
                    break
                row[j] = pool.pop()
            table.append(row)
            seq.append(S)
        if holes:  # given back, or never there
            for r in range(R):
                for j in range(W):
                    if rng.random() < 0.03:
                        table[r][j] = rng.choice([-7, pages, 2 ** 31 - 1])
        n = [0] * pages
        for r in range(R):
            for p in table[r][:-(-seq[r] // P)]:
                if 0 <= p < pages:
                    n[p] += 1
        self.free = [p for p in range(pages) if n[p] == 0]
        rng.shuffle(self.free)
        self.books = fu.Books(table, seq, [max(x - 1, 0) for x in n], P)
        self.gpu = gpu
        base = torch.full((max(R, 1), W + extra), -99, dtype=I32)
        base[:R, :W] = torch.tensor(table, dtype=I32).view(R, W)
        self.base = base.to(gpu)
        self.table = self.base[:R, :W]
        self.seq = self.ints(seq)
        self.shares = self.ints(self.books.shares)
        self.extra, self.P = extra, P

    def ints(self, v):
        return torch.tensor(v, dtype=I32, device=self.gpu)

    def same(self):
        assert self.table.tolist() == self.books.table
        assert self.seq.tolist() == self.books.seq and self.shares.tolist() == self.books.shares
        if self.extra:
            assert (self.base[:, -self.extra:] == -99).all()


SHAPES = [(1, 1, 16, 4), (3, 5, 16, 40), (20, 7, 4, 130), (64, 40, 8, 3000), (300, 9, 1, 1500), (9, 700, 2, 5000), (37, 30, 2, 24001),
          (70, 64, 4, 4500), (6, 11, 16, 40000), (1, 4096, 1, 5), (7, 3001, 2, 16000), (3, 40000, 1, 90001)]


@pytest.mark.parametrize("R,W,P,pages", SHAPES)
@pytest.mark.parametrize("extra", [0, 3])
def test_forks(gpu, R, W, P, pages, extra):
    for seed in range(3):
        h = Held(gpu, R, W, P, pages, seed, extra)
        rows = list(range(R))
        h.rng.shuffle(rows)
        some = rows[:max(1, R // 3)]
        children = rows[len(some):]
        parents = [h.rng.choice(some) for _ in children]
        if len(children) > 3:  # left out: no rows
            parents[1], children[2] = R, -1
        free = h.free[:h.rng.choice([len(h.free), len(children) // 2])]
        if len(free) > 2:
            free[1] = -1
        pairs, counts = slnr.sparselnr_page_fork(h.ints(parents), h.ints(children), h.table, h.seq, h.shares, h.ints(free), P)
        want_pairs, want_counts = h.books.fork(parents, children, free)
        assert pairs.tolist() == want_pairs and counts.tolist() == want_counts
        h.same()


def test_many_forks(gpu):
    """More forks than blocks count alone, of one long row and of short ones."""
    R, W, P = 5000, 12, 8
    h = Held(gpu, R, W, P, 70000, 5, empty=0.0, holes=False)
    parents = [h.rng.randrange(100) for _ in range(R - 100)]
    children = list(range(100, R))
    pairs, counts = slnr.sparselnr_page_fork(h.ints(parents), h.ints(children), h.table, h.seq, h.shares, h.ints(h.free), P)
    want_pairs, want_counts = h.books.fork(parents, children, h.free)
    assert pairs.tolist() == want_pairs and counts.tolist() == want_counts
    h.same()


def test_a_row_may_not_be_its_own_child(gpu):
    h = Held(gpu, 4, 5, 4, 60, 1, empty=0.0, holes=False)
    pairs, counts = slnr.sparselnr_page_fork(h.ints([1, 2]), h.ints([1, 2]), h.table, h.seq, h.shares, h.ints(h.free), 4)
    assert (pairs == -1).all() and counts.tolist() == [0, 0]
    h.same()


@pytest.mark.parametrize("R,W,P,pages", SHAPES)
@pytest.mark.parametrize("extra", [0, 3])
def test_rows_given_up(gpu, R, W, P, pages, extra):
    for seed in range(3):
        h = Held(gpu, R, W, P, pages, seed + 10, extra)
        rows = h.rng.sample(range(R), h.rng.randrange(0, R + 1))
        rows += rows[:2] + [-1, R, 2 ** 31 - 1]  # twice, and no rows
        freed, counts = slnr.sparselnr_page_free(h.ints(rows), h.table, h.seq, h.shares, P)
        want, want_counts = h.books.free(rows)
        assert freed.numel() == min(pages, len(rows) * W) and counts.tolist() == want_counts
        assert freed.tolist() == want + [-1] * (freed.numel() - len(want))
        h.same()


def test_a_list_that_is_too_short(gpu):
    h = Held(gpu, 30, 6, 4, 200, 3, empty=0.0)
    freed = h.ints([7] * 5)
    _, counts = slnr.sparselnr_page_free(h.ints(list(range(30))), h.table, h.seq, h.shares, 4, freed=freed)
    want, want_counts = h.books.free(list(range(30)))
    assert counts.tolist() == want_counts and len(want) > 5 and freed.tolist() == want[:5]
    h.same()


def test_shares_that_are_too_low_free_a_page_once(gpu):
    """Three rows hold a page that is said to be of one: freed by the first, not listed twice, shares 0."""
    table = torch.tensor([[2, 4], [2, -1], [2, 1]], dtype=I32, device=gpu)
    seq, shares = torch.tensor([8, 4, 8], dtype=I32, device=gpu), torch.zeros(6, dtype=I32, device=gpu)
    freed, counts = slnr.sparselnr_page_free(torch.arange(3, dtype=I32, device=gpu), table, seq, shares, 4)
    assert freed.tolist()[:4] == [1, 2, 4, -1] and counts.tolist() == [3, 5] and (shares == 0).all() and (table == -1).all()


@pytest.mark.parametrize("R,W,P,pages", SHAPES)
@pytest.mark.parametrize("extra", [0, 3])
def test_pages_moved_to_the_front(gpu, R, W, P, pages, extra):
    for seed in range(3):
        h = Held(gpu, R, W, P, pages, seed + 20, extra)
        pairs, counts = slnr.sparselnr_page_compact(h.table, h.seq, h.shares, P)
        want, want_counts = h.books.compact()
        assert counts.tolist() == want_counts
        assert pairs.shape == (pages // 2, 2) and pairs.tolist() == want + [[-1, -1]] * (pages // 2 - len(want))
        h.same()
        again, counts = slnr.sparselnr_page_compact(h.table, h.seq, h.shares, P)
        assert (again == -1).all() and counts.tolist() == [want_counts[0], 0]
        h.same()


def test_many_pages(gpu):
    """Bitmaps of many blocks, with borders at and beside multiples of 64."""
    for pages in (64 * 64 * 3, 64 * 64 * 3 + 1, 400003):
        h = Held(gpu, 40, 900, 4, pages, pages, empty=0.0, holes=False)
        pairs, counts = slnr.sparselnr_page_compact(h.table, h.seq, h.shares, 4)
        want, want_counts = h.books.compact()
        assert counts.tolist() == want_counts and pairs[:len(want)].tolist() == want and (pairs[len(want):] == -1).all()
        h.same()
        rows = list(range(0, 40, 2))
        freed, counts = slnr.sparselnr_page_free(h.ints(rows), h.table, h.seq, h.shares, 4)
        want, want_counts = h.books.free(rows)
        assert counts.tolist() == want_counts and freed[:len(want)].tolist() == want and (freed[len(want):] == -1).all()
        h.same()


def test_empty_calls(gpu):
    none, one = torch.zeros(0, dtype=I32, device=gpu), torch.ones(1, dtype=I32, device=gpu)
    for R, W, pages in ((0, 0, 0), (2, 0, 3), (2, 3, 0), (0, 3, 5)):
        table = torch.zeros(R, W, dtype=I32, device=gpu)
        seq, shares = torch.full((R,), 50, dtype=I32, device=gpu), torch.zeros(pages, dtype=I32, device=gpu)
        pairs, counts = slnr.sparselnr_page_fork(none, none, table, seq, shares, none, 16)
        assert pairs.shape == (0, 2) and counts.tolist() == [0, 0]
        freed, counts = slnr.sparselnr_page_free(none, table, seq, shares, 16)
        assert freed.numel() == 0 and counts.tolist() == [0, 0]
        pairs, counts = slnr.sparselnr_page_compact(table, seq, shares, 16)
        # pages 0 of rows of zeros are in use, where there are any
        assert counts.tolist() == [1 if R and W and pages else 0, 0] and (pairs == -1).all()
        slnr.sparselnr_page_free(one, table, seq, shares, 16)
    slnr.sparselnr_page_copy(torch.zeros(0, 2, dtype=I32, device=gpu), (torch.zeros(3, 4, device=gpu),))
    slnr.sparselnr_page_copy(torch.zeros(1, 2, dtype=I32, device=gpu), ())


# -------------------------------------------------------------------- copies


def pages_of(gpu, kind, pages=23):
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randint(0, 256, s, generator=g, dtype=torch.uint8).to(gpu)  # noqa: E731
    if kind == "dense":
        return r(pages, 16, 2, 64)
    if kind == "bytes":
        return r(pages, 7, 3)
    if kind == "one byte off":
        return r(pages * 48 + 1)[1:].view(pages, 16, 3)
    if kind == "words":
        return torch.randn(pages, 5, device=gpu)
    if kind == "heads first":
        return r(pages, 2, 16, 64).transpose(1, 2)
    if kind == "pairs":
        return r(pages, 2, 16, 2, 32)[:, 1]
    if kind == "some heads":
        return r(pages, 16, 5, 64)[:, :, 1:4]
    if kind == "padded":
        return r(pages, 18, 5, 80)[:, 1:17, :4, :48]
    if kind == "pages inside":
        return r(16, pages, 2, 32).transpose(0, 1)
    if kind == "large":
        return r(pages, 64, 8, 256)
    return r(pages, 1, 33, 2)[:, :, ::2, :1]


@pytest.mark.parametrize("kind", ["dense", "bytes", "one byte off", "words", "heads first", "pairs", "some heads", "padded",
                                  "pages inside", "large", "single bytes"])
def test_copies_of_any_order(gpu, kind):
    x = pages_of(gpu, kind)
    base = x._base if x._base is not None else x
    before = base.clone()
    pairs = [[3, 20], [4, 0], [-1, 5], [6, -1], [7, 7], [23, 1], [2, 23], [8, 22], [3, 10], [2 ** 31 - 1, 2]]
    good = [p for p in pairs if 0 <= p[0] < 23 and 0 <= p[1] < 23]
    copy = before.as_strided(x.shape, x.stride(), x.storage_offset())
    for a, b in good:
        copy[b] = copy[a].clone()
    slnr.sparselnr_page_copy(torch.tensor(pairs, dtype=I32, device=gpu), x)
    assert torch.equal(base, before) and not torch.equal(x[20], x[21])  # nothing outside the pages changed


def test_several_arrays_at_once(gpu):
    kinds = ["dense", "bytes", "words", "pairs", "some heads", "large", "padded", "heads first"]
    xs = [pages_of(gpu, k) for k in kinds]
    want = [x.clone() for x in xs]
    pairs = torch.tensor([[i, 22 - i] for i in range(9)] + [[-1, -1]] * 40, dtype=I32, device=gpu)
    for w in want:
        for i in range(9):
            w[22 - i] = w[i]
    slnr.sparselnr_page_copy(pairs, xs)
    for x, w in zip(xs, want):
        assert torch.equal(x.contiguous().view(torch.uint8), w.contiguous().view(torch.uint8))


@pytest.mark.parametrize("n", [70000, 70001, 131072])
def test_long_lists_of_few_pairs(gpu, n):
    """Pairs between many that are left out: each block looks at many steps at once."""
    pages = 3000
    xs = [torch.arange(pages * w, dtype=torch.int32, device=gpu).view(pages, w) for w in (5, 4096, 12)]
    want = [x.clone() for x in xs]
    g = torch.Generator().manual_seed(n)
    at = torch.randperm(n - 2, generator=g)[:200].tolist() + [n - 2, n - 1]
    order = torch.randperm(pages, generator=g)[:2 * len(at)].view(-1, 2)
    pairs = torch.full((n, 2), -1, dtype=I32)
    pairs[::3, 0] = 7  # only half of a pair
    pairs[at] = order.int()
    for w in want:
        w[order[:, 1].to(gpu)] = w[order[:, 0].to(gpu)]
    slnr.sparselnr_page_copy(pairs.to(gpu), xs)
    for x, w in zip(xs, want):
        assert torch.equal(x, w)


def test_pages_past_32_bits(gpu):
    x = torch.empty(700, 1 << 23, dtype=torch.uint8, device=gpu)
    x[3], x[699], x[350] = 1, 2, 3
    slnr.sparselnr_page_copy(torch.tensor([[699, 0], [3, 698], [350, 600]], dtype=I32, device=gpu), (x,))
    assert (x[0] == 2).all() and (x[698] == 1).all() and (x[600] == 3).all() and (x[3] == 1).all()


# --------------------------------------------------------------- in a graph


@pytest.mark.parametrize("R,W,pages", [(24, 20, 900), (60, 40, 40000)])
def test_a_captured_tidying_up(gpu, R, W, pages):
    """Fork, free and compact with their copies, captured, replayed on other tables between eager calls."""
    P = 8
    hs = [Held(gpu, R, W, P, pages, 40 + i, empty=0.0, holes=False) for i in range(4)]
    table, seq, shares = hs[0].table.clone(), hs[0].seq.clone(), hs[0].shares.clone()
    parents, children = hs[0].ints([0, 1, 2]), hs[0].ints([20, 21, 22])
    rows, gone = hs[0].ints([3, 4, 20]), hs[0].ints([20, 21, 22])
    free = torch.zeros(3, dtype=I32, device=gpu)
    x = torch.arange(pages, device=gpu).repeat_interleave(64).view(pages, 64).float()

    def step():
        a = slnr.sparselnr_page_free(gone, table, seq, shares, P)
        free.copy_(a[0][:3])
        b = slnr.sparselnr_page_fork(parents, children, table, seq, shares, free, P)
        slnr.sparselnr_page_copy(b[0], (x,))
        c = slnr.sparselnr_page_free(rows, table, seq, shares, P)
        d = slnr.sparselnr_page_compact(table, seq, shares, P)
        slnr.sparselnr_page_copy(d[0], (x,))
        return [t for pair in (a, b, c, d) for t in pair]

    def put(h):
        table.copy_(h.table), seq.copy_(h.seq), shares.copy_(h.shares)
        x.copy_(torch.arange(pages, device=gpu).repeat_interleave(64).view(pages, 64))
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = step()
    with torch.cuda.stream(stream):
        for i in (1, 2, 3, 1):
            put(hs[i])
            graph.replay()
            got = [t.clone() for t in (*outs, table, seq, shares, x)]
            slnr.sparselnr_page_compact(*(t.clone() for t in (hs[0].table, hs[0].seq, hs[0].shares)), P)
            put(hs[i])
            want = [*step(), table, seq, shares, x]
            stream.synchronize()
            for g, w in zip(got, want):
                assert torch.equal(g, w)
            hs[i].books = fu.Books(hs[i].table.tolist(), hs[i].seq.tolist(), hs[i].shares.tolist(), P)
            freed, _ = hs[i].books.free([20, 21, 22])
            hs[i].books.fork([0, 1, 2], [20, 21, 22], (freed + [-1] * 3)[:3])
            hs[i].books.free([3, 4, 20])
            hs[i].books.compact()
            assert got[-4].tolist() == hs[i].books.table and got[-2].tolist() == hs[i].books.shares
