"""Whose memory a result is that a call allocates (no GPU is needed: tensors that say they are on GPU 1, streams that
are numbers, and an allocator that notes the current one)."""
import contextlib
import ctypes

import pytest

import paper_2205_11622_amd as slnr
from tests import test_binding_device as d

torch = pytest.importorskip("torch")

I32, I64, U8, BF = torch.int32, torch.int64, torch.uint8, torch.bfloat16


class Stream:
    def __init__(self, cuda_stream, device=None):
        self.cuda_stream = cuda_stream


class Result(d.OnGpu1):
    """What the allocator gave out: the stream that it is of, and those that use it."""

    def record_stream(self, stream):
        self.used.append(stream.cuda_stream)

    def split_with_sizes(self, sizes):
        parts = [torch.Tensor._make_subclass(Result, x) for x in self.as_subclass(torch.Tensor).split_with_sizes(sizes)]
        for p in parts:
            p.of, p.used = self.of, self.used
        return parts


@pytest.fixture
def streams(monkeypatch):
    """now: the current stream; made: all results."""
    class Now:
        def __init__(self):
            self.stream, self.made = Stream(5), []
    now = Now()
    real = torch.empty

    def empty(*shape, dtype=None, device=None):
        t = torch.Tensor._make_subclass(Result, real(*shape, dtype=dtype))
        t.of, t.used = now.stream.cuda_stream, []
        now.made.append(t)
        return t

    @contextlib.contextmanager
    def stream(s):
        before, now.stream = now.stream, s
        yield
        now.stream = before

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now.stream)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0))
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: now.stream.cuda_stream, raising=False)
    monkeypatch.setattr(slnr, "_raw_stream", None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(slnr, "_get_device", None)
    library = d.Library(lambda: 1)
    monkeypatch.setattr(slnr, "lib", lambda: library)
    return now


def calls():
    """(name, call, how many results it allocates)."""
    g = d.gpu1
    rowptr, colidx, vals = g(5, dtype=I32), g(7, dtype=I32), g(7)
    C, D, E, W = g(4, 16), g(6, 16), g(6, 16), g(16, 3)
    yield "fused", lambda **k: slnr.sparselnr_fused_sddmm_spmm(rowptr, colidx, vals, C, D, E, **k), 1
    yield "sddmm", lambda **k: slnr.sparselnr_sddmm(rowptr, colidx, vals, C, D, **k), 1
    yield "spmm", lambda **k: slnr.sparselnr_spmm(rowptr, colidx, vals, E, **k), 1
    yield "unfused", lambda **k: slnr.sparselnr_unfused_sddmm_spmm(rowptr, colidx, vals, C, D, E, **k), 2
    yield "fused_gemm", lambda **k: slnr.sparselnr_fused_sddmm_spmm_gemm(rowptr, colidx, vals, C, D, E, W, **k), 1
    yield "spmm_gemm", lambda **k: slnr.sparselnr_spmm_gemm(rowptr, colidx, vals, D, W, **k), 1
    yield "spmmh_gemm", lambda **k: slnr.sparselnr_spmmh_gemm(rowptr, colidx, vals, D, E, W, **k), 1
    yield "fused_dt", lambda **k: slnr.sparselnr_fused_sddmm_spmm_dt(rowptr, colidx, vals, C, g(16, 6), E, **k), 1
    q, cache = g(3, 4, 64, dtype=BF), g(5, 16, 2, 64, dtype=BF)
    table, seq, qptr, slots = g(2, 4, dtype=I32), g(2, dtype=I32), g(3, dtype=I32), g(3, dtype=I64)
    kq, ks, sel = g(5, 2, 64, dtype=torch.int8), g(5, 2), g(3, 2, 4, dtype=I32)
    yield "page_tables", lambda **k: slnr.sparselnr_page_tables(seq, seq, table, seq, 3, 16, **k), 2
    yield "page_tables, lengths given", lambda **k: slnr.sparselnr_page_tables(seq, seq, table, seq, 3, 16, seq_len=seq, **k), 3
    yield "paged_attention", lambda **k: slnr.sparselnr_paged_attention(q, cache, cache, table, seq, qptr, **k), 1
    yield "block_select", lambda **k: slnr.sparselnr_block_select(q, kq, ks, table, seq, qptr, 16, 4, **k), 1
    yield "block_attention", lambda **k: slnr.sparselnr_block_attention(q, cache, cache, table, seq, qptr, sel, **k), 1
    four, exps, shares = g(5, 16, 2, 32, dtype=U8), g(5, 16, 2, 2, dtype=U8), g(9, dtype=I32)
    yield "cache_read_fp4", lambda **k: slnr.sparselnr_cache_read_fp4(slots, four, four, exps, exps, 64, BF, **k), 2
    yield "paged_attention_fp4", lambda **k: slnr.sparselnr_paged_attention_fp4(q, four, four, exps, exps, table, seq, qptr, **k), 1
    yield "page_fork", lambda **k: slnr.sparselnr_page_fork(seq, seq, table, seq, shares, shares, 16, **k), 2
    yield "page_free", lambda **k: slnr.sparselnr_page_free(seq, table, seq, shares, 16, **k), 2
    yield "page_compact", lambda **k: slnr.sparselnr_page_compact(table, seq, shares, 16, **k), 2


@pytest.mark.parametrize("which", range(18), ids=[name for name, _, _ in calls()])
def test_results_are_of_the_stream_that_writes_them(streams, which):
    """Memory of the current stream may be in use there, and another stream does not wait for that."""
    _, call, n = list(calls())[which]
    for given, of, used in ((None, 5, []), (5, 5, []), (Stream(5), 5, []), (7, 7, [5]), (Stream(7), 7, [5]), (0, 0, [5]),
                            (ctypes.c_void_p(7), 7, [5]), (ctypes.c_void_p(5), 5, []), (ctypes.c_void_p(), 0, [5])):
        streams.made.clear()
        call(stream=given)
        assert len(streams.made) == n and streams.stream.cuda_stream == 5
        assert all(t.of == of and t.used == used for t in streams.made), (given, [(t.of, t.used) for t in streams.made])
