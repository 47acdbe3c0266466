"""The binding makes its calls with the inputs' GPU current (no GPU is needed: tensors that say they
are on GPU 1, and a library that notes which GPU is current)."""
import pytest

import paper_2205_11622_amd as slnr

torch = pytest.importorskip("torch")


class OnGpu1(torch.Tensor):
    """A CPU tensor that says it is on GPU 1."""
    is_cuda = True
    device = torch.device("cuda:1")

    def get_device(self):
        return 1


def gpu1(*shape, dtype=torch.float32):
    return torch.Tensor._make_subclass(OnGpu1, torch.zeros(*shape, dtype=dtype))


class Library:
    def __init__(self, current):
        self.seen = {}
        self.current = current

    def __getattr__(self, name):
        def entry(*args):
            self.seen[name] = self.current()
            return slnr.OK
        return entry


def calls():
    i32, bf = torch.int32, torch.bfloat16
    rowptr, colidx, vals = gpu1(5, dtype=i32), gpu1(7, dtype=i32), gpu1(7)
    C, D, E, W, A = gpu1(4, 16), gpu1(6, 16), gpu1(6, 16), gpu1(16, 3), gpu1(4, 16)
    k = dict(stream=1)
    yield lambda: slnr.sparselnr_fused_sddmm_spmm(rowptr, colidx, vals, C, D, E, A=A, **k)
    yield lambda: slnr.sparselnr_fused_sddmm_spmm_noalloc(rowptr, colidx, vals, C, D, E, A, **k)
    yield lambda: slnr.sparselnr_sddmm(rowptr, colidx, vals, C, D, Y=vals, **k)
    yield lambda: slnr.sparselnr_spmm(rowptr, colidx, vals, E, A=A, **k)
    yield lambda: slnr.sparselnr_unfused_sddmm_spmm(rowptr, colidx, vals, C, D, E, Y=vals, A=A, **k)
    yield lambda: slnr.sparselnr_fused_sddmm_spmm_gemm(rowptr, colidx, vals, C, D, E, W, A=gpu1(4, 3), **k)
    yield lambda: slnr.sparselnr_spmm_gemm(rowptr, colidx, vals, D, W, A=gpu1(4, 3), **k)
    yield lambda: slnr.sparselnr_spmmh_gemm(rowptr, colidx, vals, D, E, W, A=gpu1(4, 3), **k)
    yield lambda: slnr.sparselnr_fused_sddmm_spmm_dt(rowptr, colidx, vals, C, gpu1(16, 6), E, A=A, **k)
    yield lambda: slnr.sparselnr_validate_csr(rowptr, colidx, 6, **k)
    q, new, cache = gpu1(3, 4, 64, dtype=bf), gpu1(3, 2, 64, dtype=bf), gpu1(5, 16, 2, 64, dtype=bf)
    table, seq, qptr, slots = gpu1(2, 4, dtype=i32), gpu1(2, dtype=i32), gpu1(3, dtype=i32), gpu1(3, dtype=torch.int64)
    kq, ks, sel = gpu1(5, 2, 64, dtype=torch.int8), gpu1(5, 2), gpu1(3, 2, 4, dtype=i32)
    yield lambda: slnr.sparselnr_page_tables(seq, seq, table, seq, 3, 16, qptr=qptr, seq_len=seq, slots=slots,
                                             counts=gpu1(3, dtype=i32), **k)
    yield lambda: slnr.sparselnr_cache_append(new, new, slots, cache, cache, kq, ks, **k)
    yield lambda: slnr.sparselnr_paged_attention(q, cache, cache, table, seq, qptr, out=gpu1(3, 4, 64, dtype=bf), **k)
    yield lambda: slnr.sparselnr_block_select(q, kq, ks, table, seq, qptr, 16, 4, sel=sel, **k)
    yield lambda: slnr.sparselnr_block_attention(q, cache, cache, table, seq, qptr, sel, out=gpu1(3, 4, 64, dtype=bf), **k)


@pytest.mark.parametrize("current", [0, 1])
def test_calls_run_on_their_inputs_gpu(monkeypatch, current):
    now = [current]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, now[0] = now[0], self.index

        def __exit__(self, *e):
            now[0] = self.before

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    library = Library(lambda: now[0])
    monkeypatch.setattr(slnr, "lib", lambda: library)
    for call in calls():
        call()
        assert now[0] == current
    assert len(library.seen) == 15
    assert all(index == 1 for index in library.seen.values()), library.seen
