"""The calls of the 4-bit cache and of the pages' life as a server makes them, one after the other: prompts, forked
answers, single tokens, rows given up, pages moved, over a cache in 4 bits and one in the rows' type with one table."""
import threading
import types

import pytest
import torch

import paper_2205_11622_amd as slnr
from tests import fp4_util as fu
from tests import paged_util as pu

pytestmark = pytest.mark.gpu

I32 = torch.int32


class Server:
    def __init__(self, gpu, dtype, P, D, Hq=6, Hkv=2, rows=8, pages=60, W=12, seed=1):
        self.gpu, self.dtype, self.P, self.D, self.Hq, self.Hkv, self.rows, self.pages = gpu, dtype, P, D, Hq, Hkv, rows, pages
        self.rng = torch.Generator().manual_seed(seed)
        NG = -(-D // 32)
        # bytes of a head adjacent, exponents of a place; nothing is defined before it is written
        self.k4, self.v4 = (torch.full((pages, Hkv, P, 16 * NG), 0x5a, dtype=torch.uint8, device=gpu).transpose(1, 2) for _ in "kv")
        self.ks, self.vs = (torch.full((pages, P, Hkv, NG), 255, dtype=torch.uint8, device=gpu) for _ in "kv")
        self.k, self.v = (torch.full((pages, P, Hkv, D), float("nan"), dtype=dtype, device=gpu) for _ in "kv")
        self.table = torch.full((rows, W), -1, dtype=I32, device=gpu)
        self.seq = torch.zeros(rows, dtype=I32, device=gpu)
        self.shares = torch.zeros(pages, dtype=I32, device=gpu)
        self.free = torch.randperm(pages, generator=self.rng).tolist()
        self.past = {r: (torch.zeros(0, Hkv, D, dtype=dtype), torch.zeros(0, Hkv, D, dtype=dtype)) for r in range(rows)}

    def ints(self, v):
        return torch.tensor(v, dtype=I32, device=self.gpu)

    def random(self, *shape):
        return torch.randn(*shape, generator=self.rng).to(self.dtype)

    def caches(self):
        return self.k4, self.v4, self.ks, self.vs, self.k, self.v

    def attend(self, q, seq, qptr, window=0):
        lse = [torch.empty(q.shape[:2], device=self.gpu) for _ in range(2)]
        out4 = slnr.sparselnr_paged_attention_fp4(q, self.k4, self.v4, self.ks, self.vs, self.table, seq, qptr, window=window, lse=lse[0])
        out = slnr.sparselnr_paged_attention(q, self.k, self.v, self.table, seq, qptr, window=window, lse=lse[1])
        return out4, lse[0], out, lse[1]

    def step(self, new, window=0):
        """new[r] tokens of each row: tables, both caches, both attentions, checked."""
        new = new + [0] * (self.rows - len(new))
        T = sum(new)
        qptr, seq, slots, counts = slnr.sparselnr_page_tables(self.seq, self.ints(new), self.table, self.ints(self.free), T, self.P)
        total, taken, lost = counts.tolist()
        assert total == T and lost == 0
        self.free = self.free[taken:]
        k, v, q = self.random(T, self.Hkv, self.D), self.random(T, self.Hkv, self.D), self.random(T, self.Hq, self.D)
        kd, vd = k.to(self.gpu), v.to(self.gpu)
        slnr.sparselnr_cache_append_fp4(kd, vd, slots, self.k4, self.v4, self.ks, self.vs)
        slnr.sparselnr_cache_append(kd, vd, slots, self.k, self.v)
        self.seq = seq
        at = 0
        for r, n in enumerate(new):
            a, b = self.past[r]
            self.past[r] = torch.cat([a, k[at:at + n]]), torch.cat([b, v[at:at + n]])
            at += n
        self.check(q, self.attend(q.to(self.gpu), seq, qptr, window), new, window)
        # what the slots stand for
        rk, rv = slnr.sparselnr_cache_read_fp4(slots, self.k4, self.v4, self.ks, self.vs, self.D, self.dtype)
        for got, x in ((rk, k), (rv, v)):
            assert torch.equal(got.double().cpu(), fu.stand_for(*fu.quantise(x), self.D))

    def check(self, q, got, new, window):
        """Against the rows' whole pasts, laid out one behind the other."""
        lens = [len(self.past[r][0]) for r in range(self.rows)]
        assert self.seq.tolist() == lens
        n = max(max(lens), 1)
        b = types.SimpleNamespace(q=q, dtype=self.dtype, seq=lens)
        qptr = [0]
        for x in new:
            qptr.append(qptr[-1] + x)
        table = [[r] for r in range(self.rows)]
        for four, out, lse in ((True, *got[:2]), (False, *got[2:])):
            kv = []
            for i in range(2):
                x = torch.zeros(self.rows, n, self.Hkv, self.D, dtype=torch.float64)
                for r in range(self.rows):
                    past = self.past[r][i]
                    x[r, :lens[r]] = fu.stand_for(*fu.quantise(past), self.D) if four else past.double()
                kv.append(x)
            ref = pu.attention(q, *kv, table, lens, qptr, self.D ** -0.5, window)
            b.kc, b.vc = kv
            if four:
                fu.check(b, out, lse, ref)
            else:
                pu.check(out, lse, ref, self.dtype, n, self.D, float(kv[1].abs().max()))

    def fork(self, parents, children):
        pairs, counts = slnr.sparselnr_page_fork(self.ints(parents), self.ints(children), self.table, self.seq, self.shares,
                                                 self.ints(self.free), self.P)
        taken, lost = counts.tolist()
        assert lost == 0
        self.free = self.free[taken:]
        slnr.sparselnr_page_copy(pairs, self.caches())
        for p, c in zip(parents, children):
            self.past[c] = self.past[p]

    def give_up(self, rows):
        freed, counts = slnr.sparselnr_page_free(self.ints(rows), self.table, self.seq, self.shares, self.P)
        n = counts[0].item()
        self.free += freed[:n].tolist()
        for r in rows:
            self.past[r] = tuple(x[:0] for x in self.past[r])

    def tidy(self):
        """Attention gives the same bits wherever the pages lie."""
        live = [r for r in range(self.rows) if len(self.past[r][0])]
        new = [int(r in live) for r in range(self.rows)]
        qptr = self.ints([sum(new[:r]) for r in range(self.rows + 1)])
        q = self.random(len(live), self.Hq, self.D)
        before = self.attend(q.to(self.gpu), self.seq, qptr)
        self.check(q, before, new, 0)
        pairs, counts = slnr.sparselnr_page_compact(self.table, self.seq, self.shares, self.P)
        slnr.sparselnr_page_copy(pairs, self.caches())
        used, moved = counts.tolist()
        assert used + len(self.free) == self.pages and moved > 0
        assert self.table.max().item() == used - 1
        self.free = list(range(used, self.pages))
        for x in self.caches():  # nothing is read from the pages that are free
            x[used:] = 255 if x.dtype == torch.uint8 else float("nan")
        for a, b in zip(before, self.attend(q.to(self.gpu), self.seq, qptr)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("P,D,window", [(16, 64, 0), (64, 72, 0), (8, 128, 11), (1, 32, 0)])
def test_a_server(gpu, dtype, P, D, window):
    pages, W = {1: (700, 150), 8: (150, 30)}.get(P, (60, 12))
    s = Server(gpu, dtype, P, D, pages=pages, W=W)
    s.step([37, 5, P, 0, 0, 0, 0, 90], window)
    s.fork([0, 0, 2, 7], [3, 4, 5, 6])  # in mid-page, at its end, more than one child
    s.step([1] * 8, window)
    s.fork([], [])
    s.step([1, 2, 0, 1, 0, 1, 3, 1], window)
    s.give_up([0, 4, 7])
    s.tidy()
    s.step([50, 1, 1, 1, 0, 1, 1, 0], window)
    s.give_up([1, 1, 2, 3, 5, 6])
    s.tidy() if P < 64 else None
    s.give_up([0])
    assert sorted(s.free) == list(range(pages)) and (s.shares == 0).all() and (s.table == -1).all()


def test_two_streams_and_two_threads(gpu):
    """Each thread serves on a stream of its own, and then both on one: every step is checked."""
    failed = []

    def serve(stream, seed):
        try:
            with torch.cuda.device(gpu), torch.cuda.stream(stream):
                s = Server(gpu, torch.bfloat16, 16, 64, seed=seed)
                s.step([20, 0, 30])
                s.fork([0, 2], [1, 3])
                s.step([1] * 5)
                s.give_up([0, 2])
                s.tidy()
                stream.synchronize()
        except BaseException as e:  # noqa: B036 - a thread's failure is the test's
            failed.append(e)

    one = torch.cuda.Stream()
    for streams in ((torch.cuda.Stream(), torch.cuda.Stream()), (one, one)):
        threads = [threading.Thread(target=serve, args=(x, i)) for i, x in enumerate(streams)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    assert not failed, failed


def test_many_forks_of_a_long_row_share_its_pages(gpu):
    """40 answers to one prompt: the prompt's pages once in the cache, and each answer its own last page."""
    s = Server(gpu, torch.float16, 32, 64, rows=41, pages=100, W=20)
    s.step([500])
    held = s.pages - len(s.free)
    assert held == 16
    s.fork([0] * 40, list(range(1, 41)))
    assert s.pages - len(s.free) == held + 40 and s.shares.max().item() == 40 and int(s.shares.sum()) == 40 * 15
    s.step([1] * 41)
    s.give_up(list(range(0, 41, 2)))
    s.step([int(r % 2 == 1) for r in range(41)])
    s.tidy()
