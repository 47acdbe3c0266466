"""The 4-bit cache and the pages' life without a GPU: refusals before any HIP call, and the binding's checks."""
import ctypes
import math

import pytest

import paper_2205_11622_amd as slnr
from tests.test_paged import FAKE, requests

INVALID, UNSUPPORTED, OK = slnr.ERR_INVALID_ARG, slnr.ERR_UNSUPPORTED, slnr.OK


def cache(**kw):
    c = dict(k=FAKE, v=FAKE, k_scale=FAKE + 3, v_scale=FAKE + 5, pages=4, page_size=16, heads=2, dim=64, k_page=1024,
             k_slot=64, k_head=32, v_page=1024, v_slot=64, v_head=32, ks_page=64, ks_slot=4, ks_head=2, vs_page=64,
             vs_slot=4, vs_head=2, dtype=0)
    c.update(kw)
    return slnr._Fp4Cache(**c)


def attend(c=None, r=None, q=FAKE, qt=512, qh=64, Hq=8, scale=0.1, window=0, max_new=0, out=FAKE):
    return slnr.lib().sparselnr_paged_attention_fp4(q, qt, qh, Hq, c or cache(), r or requests(T=3), scale, window, max_new,
                                                    out, None, None)


def append(c=None, k=FAKE, v=FAKE, slots=FAKE, T=3, kt=128, kh=64):
    return slnr.lib().sparselnr_cache_append_fp4(k, kt, kh, v, 128, 64, slots, c or cache(), T, None)


def read(c=None, k=FAKE, v=FAKE, slots=FAKE, T=3):
    return slnr.lib().sparselnr_cache_read_fp4(slots, c or cache(), k, v, T, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(pages=-1), INVALID), (dict(heads=0), INVALID),
    (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(k_scale=0), INVALID), (dict(v_scale=0), INVALID),
    (dict(k_page=-16), INVALID), (dict(vs_head=-1), INVALID), (dict(ks_slot=-1), INVALID), (dict(dim=-8), INVALID),
    (dict(dim=0), UNSUPPORTED), (dict(dim=4), UNSUPPORTED), (dict(dim=100), UNSUPPORTED), (dict(dim=264), UNSUPPORTED),
    (dict(page_size=0), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=8192), UNSUPPORTED),
    (dict(k=FAKE + 8), UNSUPPORTED), (dict(v=FAKE + 4), UNSUPPORTED), (dict(k_slot=72), UNSUPPORTED),
    (dict(v_page=1025), UNSUPPORTED), (dict(k_head=8), UNSUPPORTED), (dict(pages=1 << 31), UNSUPPORTED),
    (dict(heads=65536), UNSUPPORTED)])
def test_cache_refusals(kw, code):
    assert attend(cache(**kw), Hq=8 if kw.get("heads") != 65536 else 65536) == code
    assert append(cache(**kw)) == code
    assert read(cache(**kw)) == code


def test_nothing_to_do():
    assert attend(r=requests(T=0)) == OK and attend(r=requests(R=0, T=0)) == OK
    assert append(T=0) == OK and append(cache(pages=0, k=0, v=0, k_scale=0, v_scale=0)) == OK and read(T=0) == OK
    # strides of extents of one do not count
    assert append(cache(pages=1, k_page=5, ks_page=1, heads=1, k_head=3, v_head=3), T=0) == OK


@pytest.mark.parametrize("kw,code", [
    (dict(q=0), INVALID), (dict(out=0), INVALID), (dict(scale=0.0), INVALID), (dict(scale=math.nan), INVALID),
    (dict(scale=math.inf), INVALID), (dict(scale=1e-46), INVALID), (dict(window=-1), INVALID), (dict(max_new=-1), INVALID),
    (dict(Hq=0), INVALID), (dict(Hq=3), INVALID), (dict(Hq=65538), UNSUPPORTED), (dict(qt=-1), INVALID),
    (dict(qt=12), UNSUPPORTED), (dict(qh=4), UNSUPPORTED), (dict(q=FAKE + 2), UNSUPPORTED), (dict(out=FAKE + 8), UNSUPPORTED),
    (dict(r=requests(T=-1)), INVALID), (dict(r=requests(T=3, table=0)), INVALID), (dict(r=requests(T=3, table_stride=7)), INVALID),
    (dict(r=requests(T=3, R=1 << 24)), UNSUPPORTED), (dict(r=requests(T=1 << 28)), UNSUPPORTED),
    (dict(r=requests(T=3, W=1 << 27, table_stride=1 << 27)), UNSUPPORTED)])
def test_attention_refusals(kw, code):
    assert attend(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), INVALID), (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(slots=0), INVALID), (dict(kt=-8), INVALID),
    (dict(kt=12), UNSUPPORTED), (dict(kh=4), UNSUPPORTED), (dict(k=FAKE + 8), UNSUPPORTED), (dict(T=1 << 28), UNSUPPORTED)])
def test_append_and_read_refusals(kw, code):
    assert append(**kw) == code
    if not {"kt", "kh"} & kw.keys():
        assert read(**kw) == code


def test_null_structures():
    L = slnr.lib()
    assert L.sparselnr_paged_attention_fp4(FAKE, 512, 64, 8, None, requests(T=3), 0.1, 0, 0, FAKE, None, None) == INVALID
    assert L.sparselnr_paged_attention_fp4(FAKE, 512, 64, 8, cache(), None, 0.1, 0, 0, FAKE, None, None) == INVALID
    assert L.sparselnr_cache_append_fp4(FAKE, 128, 64, FAKE, 128, 64, FAKE, None, 3, None) == INVALID
    assert L.sparselnr_cache_read_fp4(FAKE, None, FAKE, FAKE, 3, None) == INVALID
    assert L.sparselnr_page_copy(FAKE, 1, None, 1, 4, None) == INVALID


# ------------------------------------------------------------ the pages' life


def fork(parents=FAKE, children=FAKE, table=FAKE, stride=8, seq=FAKE, shares=FAKE, free=FAKE, pairs=FAKE, counts=FAKE,
         n=2, R=3, W=8, F=4, pages=9, P=16):
    return slnr.lib().sparselnr_page_fork(parents, children, table, stride, seq, shares, free, pairs, counts, n, R, W, F,
                                          pages, P, None)


def free(rows=FAKE, table=FAKE, stride=8, seq=FAKE, shares=FAKE, freed=FAKE, counts=FAKE, n=2, R=3, W=8, most=9, pages=9,
         P=16):
    return slnr.lib().sparselnr_page_free(rows, table, stride, seq, shares, freed, counts, n, R, W, most, pages, P, None)


def compact(table=FAKE, stride=8, seq=FAKE, shares=FAKE, pairs=FAKE, counts=FAKE, R=3, W=8, pages=9, P=16):
    return slnr.lib().sparselnr_page_compact(table, stride, seq, shares, pairs, counts, R, W, pages, P, None)


@pytest.mark.parametrize("call", [fork, free, compact])
@pytest.mark.parametrize("kw,code", [
    (dict(table=0), INVALID), (dict(seq=0), INVALID), (dict(shares=0), INVALID), (dict(counts=0), INVALID),
    (dict(stride=7), INVALID), (dict(stride=-1), INVALID), (dict(R=-1), INVALID), (dict(W=-1), INVALID),
    (dict(pages=-1), INVALID), (dict(P=0), UNSUPPORTED), (dict(P=24), UNSUPPORTED), (dict(P=8192), UNSUPPORTED),
    (dict(R=1 << 24), UNSUPPORTED), (dict(pages=1 << 31), UNSUPPORTED), (dict(W=1 << 27, stride=1 << 27), UNSUPPORTED)])
def test_life_refusals(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("call,kw,code", [
    (fork, dict(parents=0), INVALID), (fork, dict(children=0), INVALID), (fork, dict(pairs=0), INVALID),
    (fork, dict(free=0), INVALID), (fork, dict(n=-1), INVALID), (fork, dict(F=-1), INVALID),
    (fork, dict(n=1 << 24), UNSUPPORTED), (fork, dict(F=1 << 31), UNSUPPORTED), (free, dict(rows=0), INVALID),
    (free, dict(freed=0), INVALID), (free, dict(n=-1), INVALID), (free, dict(most=-1), INVALID),
    (free, dict(n=1 << 24), UNSUPPORTED), (free, dict(most=1 << 31), UNSUPPORTED), (compact, dict(pairs=0), INVALID)])
def test_life_refusals_of_one(call, kw, code):
    assert call(**kw) == code


def copy(pairs=FAKE, n=2, count=1, pages=4, **kw):
    a = dict(data=FAKE, page=1024, outer=1, outer_stride=0, inner=1, inner_stride=0, row=1024)
    a.update(kw)
    return slnr.lib().sparselnr_page_copy(pairs, n, (slnr._PageArray * max(count, 1))(*[slnr._PageArray(**a)] * max(count, 1)),
                                          count, pages, None)


@pytest.mark.parametrize("kw,code", [
    (dict(pairs=0), INVALID), (dict(n=-1), INVALID), (dict(count=-1), INVALID), (dict(count=9), UNSUPPORTED),
    (dict(pages=-1), INVALID), (dict(pages=1 << 31), UNSUPPORTED), (dict(n=1 << 31), UNSUPPORTED), (dict(data=0), INVALID),
    (dict(page=-1), INVALID), (dict(outer=-1), INVALID), (dict(inner=-1), INVALID), (dict(row=-1), INVALID),
    (dict(outer_stride=-1), INVALID), (dict(inner_stride=-4), INVALID), (dict(row=1 << 31), UNSUPPORTED),
    (dict(inner=1 << 31), UNSUPPORTED), (dict(outer=1 << 30, inner=1 << 30), UNSUPPORTED),
    (dict(n=0), OK), (dict(count=0), OK), (dict(row=0), OK), (dict(outer=0, data=0), OK), (dict(pages=0, data=0), OK)])
def test_copy_refusals(kw, code):
    assert copy(**kw) == code


# ------------------------------------------------------------ the binding

torch = pytest.importorskip("torch")


def test_binding_refuses_cpu_tensors():
    c = torch.zeros(4, 16, 2, 32, dtype=torch.uint8)
    s = torch.zeros(4, 16, 2, 2, dtype=torch.uint8)
    k, i = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    table, slots = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: slnr.sparselnr_cache_append_fp4(k, k, slots, c, c, s, s),
                 lambda: slnr.sparselnr_cache_read_fp4(slots, c, c, s, s, 64, torch.bfloat16),
                 lambda: slnr.sparselnr_paged_attention_fp4(k, c, c, s, s, table, i, i),
                 lambda: slnr.sparselnr_page_fork(i, i, table, i, i, i, 16),
                 lambda: slnr.sparselnr_page_free(i, table, i, i, 16),
                 lambda: slnr.sparselnr_page_compact(table, i, i, 16),
                 lambda: slnr.sparselnr_page_copy(torch.zeros(1, 2, dtype=torch.int32), (c,))):
        with pytest.raises(ValueError, match="GPU"):
            call()


class Fake(torch.Tensor):
    """A CPU tensor that says it is on GPU 0."""
    is_cuda = True

    def get_device(self):
        return 0


def gpu0(*shape, dtype=torch.float32):
    return torch.Tensor._make_subclass(Fake, torch.zeros(*shape, dtype=dtype))


@pytest.fixture
def library(monkeypatch):
    class Library:
        def __init__(self):
            self.calls = []

        def __getattr__(self, name):
            return lambda *a: self.calls.append((name, a)) or slnr.OK
    seen = Library()
    monkeypatch.setattr(slnr, "lib", lambda: seen)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return seen


U8, I32, I64, BF = torch.uint8, torch.int32, torch.int64, torch.bfloat16


@pytest.mark.parametrize("what,change,error", [
    ("kc", gpu0(4, 16, 2, 48, dtype=U8), ValueError), ("kc", gpu0(4, 16, 2, 32, dtype=torch.int8), TypeError),
    ("vc", gpu0(4, 16, 3, 32, dtype=U8), ValueError), ("ks", gpu0(4, 16, 2, 3, dtype=U8), ValueError),
    ("ks", gpu0(4, 16, 2, 4, dtype=U8)[..., ::2], ValueError), ("vs", gpu0(4, 16, 2, dtype=U8), ValueError),
    ("vs", None, TypeError), ("q", gpu0(3, 4, 64, dtype=torch.float64), TypeError), ("q", gpu0(3, 5, 64, dtype=BF), ValueError),
    ("q", gpu0(3, 256, dtype=BF), ValueError), ("q", gpu0(3, 4, 96, dtype=BF), ValueError),
    ("table", gpu0(2, 4, dtype=I64), TypeError), ("seq", gpu0(3, dtype=I32), ValueError), ("lse", gpu0(3, 5), ValueError),
    ("out", gpu0(3, 4, 64), TypeError)])
def test_binding_checks_of_attention(library, what, change, error):
    a = dict(q=gpu0(3, 4, 64, dtype=BF), kc=gpu0(4, 16, 2, 32, dtype=U8), vc=gpu0(4, 16, 2, 32, dtype=U8),
             ks=gpu0(4, 16, 2, 2, dtype=U8), vs=gpu0(4, 16, 2, 2, dtype=U8), table=gpu0(2, 4, dtype=I32),
             seq=gpu0(2, dtype=I32), qptr=gpu0(3, dtype=I32), out=gpu0(3, 4, 64, dtype=BF), lse=gpu0(3, 4))

    def call():
        return slnr.sparselnr_paged_attention_fp4(a["q"], a["kc"], a["vc"], a["ks"], a["vs"], a["table"], a["seq"], a["qptr"],
                                                  out=a["out"], lse=a["lse"], stream=1)
    call()
    assert [n for n, _ in library.calls] == ["sparselnr_paged_attention_fp4"]
    a[what] = change
    with pytest.raises(error):
        call()
    assert len(library.calls) == 1


def test_binding_checks_of_the_others(library):
    kc, ks = gpu0(4, 16, 2, 48, dtype=U8), gpu0(4, 16, 2, 3, dtype=U8)
    k, slots = gpu0(3, 2, 80, dtype=BF), gpu0(3, dtype=I64)
    slnr.sparselnr_cache_append_fp4(k, k, slots, kc, kc, ks, ks, stream=1)
    slnr.sparselnr_cache_read_fp4(slots, kc, kc, ks, ks, 80, BF, k=k, v=k, stream=1)
    i, t, s = gpu0(2, dtype=I32), gpu0(3, 8, dtype=I32), gpu0(9, dtype=I32)
    seq, pairs = gpu0(3, dtype=I32), gpu0(2, 2, dtype=I32)
    slnr.sparselnr_page_fork(i, i, t, seq, s, s, 16, pairs=pairs, counts=i, stream=1)
    slnr.sparselnr_page_free(i, t, seq, s, 16, freed=s, counts=i, stream=1)
    slnr.sparselnr_page_compact(t, seq, s, 16, pairs=gpu0(4, 2, dtype=I32), counts=i, stream=1)
    slnr.sparselnr_page_copy(pairs, (kc, ks), stream=1)
    assert len(library.calls) == 6
    for bad in (lambda: slnr.sparselnr_cache_append_fp4(k, gpu0(3, 3, 80, dtype=BF), slots, kc, kc, ks, ks),
                lambda: slnr.sparselnr_cache_append_fp4(gpu0(3, 2, 80, dtype=U8), k, slots, kc, kc, ks, ks),
                lambda: slnr.sparselnr_cache_append_fp4(k, k, gpu0(4, dtype=I64), kc, kc, ks, ks),
                lambda: slnr.sparselnr_cache_append_fp4(k, k, gpu0(3, dtype=I32), kc, kc, ks, ks),
                lambda: slnr.sparselnr_cache_read_fp4(slots, kc, kc, ks, ks, 104, BF, k=k, v=k),
                lambda: slnr.sparselnr_cache_read_fp4(slots, kc, kc, ks, ks, 80, BF, k=gpu0(3, 2, 80), v=k),
                lambda: slnr.sparselnr_page_fork(i, s, t, seq, s, s, 16, pairs=pairs, counts=i),
                lambda: slnr.sparselnr_page_fork(i, i, t, i, s, s, 16, pairs=pairs, counts=i),
                lambda: slnr.sparselnr_page_fork(i, i, t, seq, s, s, 16, pairs=gpu0(3, 2, dtype=I32), counts=i),
                lambda: slnr.sparselnr_page_free(slots, t, seq, s, 16, freed=s, counts=i),
                lambda: slnr.sparselnr_page_free(i, t, seq, s, 16, freed=s, counts=seq),
                lambda: slnr.sparselnr_page_compact(t, seq, s, 16, pairs=pairs, counts=i),
                lambda: slnr.sparselnr_page_compact(gpu0(3, 8, dtype=I64), seq, s, 16, pairs=pairs, counts=i),
                lambda: slnr.sparselnr_page_copy(gpu0(2, 3, dtype=I32), (kc,)),
                lambda: slnr.sparselnr_page_copy(gpu0(4, dtype=I32), (kc,)),
                lambda: slnr.sparselnr_page_copy(pairs, (kc, gpu0(5, 3))),
                lambda: slnr.sparselnr_page_copy(pairs, (kc, None)),
                lambda: slnr.sparselnr_page_copy(pairs, (gpu0(4, 1, 3).expand(4, 5, 3),)),
                lambda: slnr.sparselnr_page_copy(pairs, (gpu0(4, 6, 6, 6, 6)[:, ::2, ::2, ::2],))):
        with pytest.raises((ValueError, TypeError)):
            bad()
    assert len(library.calls) == 6


@pytest.mark.parametrize("make,want", [
    (lambda: gpu0(5, 16, 2, 64, dtype=BF), (4096, 1, 0, 1, 0, 4096)),
    (lambda: gpu0(5, 2, 16, 64, dtype=BF).transpose(1, 2), (4096, 1, 0, 1, 0, 4096)),
    (lambda: gpu0(5, 2, 16, 2, 64, dtype=BF)[:, 1], (8192, 1, 0, 1, 0, 4096)),
    (lambda: gpu0(5, 16, 3, 64, dtype=BF)[:, :, :2], (6144, 1, 0, 16, 384, 256)),
    (lambda: gpu0(16, 5, 2, 64, dtype=BF).transpose(0, 1), (256, 1, 0, 16, 1280, 256)),
    (lambda: gpu0(5, 9, 4, 80, dtype=U8)[:, :8, :2, :48], (2880, 8, 320, 2, 80, 48)),
    (lambda: gpu0(5), (4, 1, 0, 1, 0, 4)), (lambda: gpu0(5, 0, 3), (0, 1, 0, 0, 12, 12))])
def test_pages_as_rows(make, want):
    a = slnr._page_array(make(), "x", 0, 5)
    got = (a.page, a.outer, a.outer_stride, a.inner, a.inner_stride, a.row)
    if 0 in make().shape:
        assert a.outer * a.inner * a.row == 0
    else:
        assert got == want


def test_calls_run_on_their_inputs_gpu(monkeypatch):
    """As test_binding_device, for these calls: GPU 1 is current while the library is called."""
    from tests import test_binding_device as d
    now = [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, now[0] = now[0], self.index

        def __exit__(self, *e):
            now[0] = self.before
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    library = d.Library(lambda: now[0])
    monkeypatch.setattr(slnr, "lib", lambda: library)
    g = d.gpu1
    kc, ks, k, slots = g(4, 16, 2, 32, dtype=U8), g(4, 16, 2, 2, dtype=U8), g(3, 2, 64, dtype=BF), g(3, dtype=I64)
    i, t, s, seq = g(2, dtype=I32), g(3, 8, dtype=I32), g(9, dtype=I32), g(3, dtype=I32)
    pairs = g(2, 2, dtype=I32)
    slnr.sparselnr_cache_append_fp4(k, k, slots, kc, kc, ks, ks, stream=1)
    slnr.sparselnr_cache_read_fp4(slots, kc, kc, ks, ks, 64, BF, k=k, v=k, stream=1)
    slnr.sparselnr_paged_attention_fp4(k, kc, kc, ks, ks, t, seq, g(4, dtype=I32), out=k, stream=1)
    slnr.sparselnr_page_fork(i, i, t, seq, s, s, 16, pairs=pairs, counts=i, stream=1)
    slnr.sparselnr_page_free(i, t, seq, s, 16, freed=s, counts=i, stream=1)
    slnr.sparselnr_page_compact(t, seq, s, 16, pairs=g(4, 2, dtype=I32), counts=i, stream=1)
    slnr.sparselnr_page_copy(pairs, (kc,), stream=1)
    assert len(library.seen) == 7 and all(v == 1 for v in library.seen.values())
