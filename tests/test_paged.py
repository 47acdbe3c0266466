"""The paged-cache entry points without a GPU: exports, refusals before any HIP
call, and the binding's checks."""
import ctypes
import math

import pytest

import paper_2205_11622_amd as slnr

FAKE = 0x1000  # never dereferenced: every case fails validation first, or has nothing to do
ENTRIES = ["sparselnr_page_tables", "sparselnr_cache_append", "sparselnr_paged_attention",
           "sparselnr_block_select", "sparselnr_block_attention"]


def cache(**kw):
    c = dict(k=FAKE, v=FAKE, pages=4, page_size=16, heads=2, dim=64, k_page=2048, k_slot=128, k_head=64,
             v_page=2048, v_slot=128, v_head=64, dtype=0)
    c.update(kw)
    return slnr._KvCache(**c)


def requests(**kw):
    r = dict(table=FAKE, table_stride=8, seq_len=FAKE, qptr=FAKE, R=2, W=8, T=0)
    r.update(kw)
    return slnr._Requests(**r)


def attend(c=None, r=None, q=FAKE, qt=512, qh=64, Hq=8, scale=0.1, window=0, max_new=0, out=FAKE):
    return slnr.lib().sparselnr_paged_attention(q, qt, qh, Hq, c or cache(), r or requests(T=3), scale, window,
                                                max_new, out, None, None)


def sparse(c=None, r=None, q=FAKE, sel=FAKE, top=4, scale=0.1, Hq=8):
    return slnr.lib().sparselnr_block_attention(q, 512, 64, Hq, c or cache(), r or requests(T=3), sel, top, scale,
                                                FAKE, None, None)


def select(r=None, q=FAKE, dtype=0, kq=FAKE, ks=FAKE, pages=4, P=16, Hkv=2, dim=64, top=4, first=1, local=1, Hq=8):
    return slnr.lib().sparselnr_block_select(q, 512, 64, Hq, dtype, kq, ks, pages, P, Hkv, dim, r or requests(T=3),
                                             top, first, local, FAKE, None)


def append(c=None, k=FAKE, v=FAKE, slots=FAKE, kq=FAKE, ks=FAKE, T=3, kt=128, kh=64):
    return slnr.lib().sparselnr_cache_append(k, kt, kh, v, 128, 64, slots, c or cache(), kq, ks, T, None)


def tables(ctx=FAKE, new=FAKE, table=FAKE, stride=8, free=FAKE, qptr=FAKE, seq=FAKE, slots=FAKE, counts=FAKE,
           R=2, W=8, F=4, T=3, P=16):
    return slnr.lib().sparselnr_page_tables(ctx, new, table, stride, free, qptr, seq, slots, counts, R, W, F, T, P,
                                            None)


def test_exports():
    for name in ENTRIES:
        assert hasattr(slnr.lib(), name) and name in slnr.__all__


INVALID, UNSUPPORTED, OK = slnr.ERR_INVALID_ARG, slnr.ERR_UNSUPPORTED, slnr.OK


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(pages=-1), INVALID), (dict(heads=0), INVALID),
    (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(k_page=-8), INVALID), (dict(v_head=-8), INVALID),
    (dict(dim=-8), INVALID), (dict(dim=0), UNSUPPORTED), (dict(dim=4), UNSUPPORTED), (dict(dim=100), UNSUPPORTED),
    (dict(dim=264), UNSUPPORTED), (dict(page_size=0), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED),
    (dict(page_size=8192), UNSUPPORTED), (dict(page_size=-16), UNSUPPORTED), (dict(k=FAKE + 8), UNSUPPORTED),
    (dict(v=FAKE + 4), UNSUPPORTED), (dict(k_slot=132), UNSUPPORTED), (dict(v_page=2049), UNSUPPORTED),
    (dict(k_head=4, dtype=2), OK), (dict(pages=1 << 31), UNSUPPORTED)])
def test_cache_refusals(kw, code):
    if code == OK:  # admitted: with no tokens the call returns at once
        assert attend(cache(**kw), requests(T=0), Hq=8) == OK
        return
    assert attend(cache(**kw)) == code
    assert sparse(cache(**kw)) == code
    assert append(cache(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(R=-1), INVALID), (dict(W=-1), INVALID), (dict(T=-1), INVALID), (dict(table=0), INVALID),
    (dict(seq_len=0), INVALID), (dict(qptr=0), INVALID), (dict(table_stride=7), INVALID),
    (dict(table_stride=-1), INVALID), (dict(R=1 << 24), UNSUPPORTED), (dict(T=1 << 28), UNSUPPORTED),
    (dict(W=1 << 27, table_stride=1 << 27), UNSUPPORTED)])
def test_request_refusals(kw, code):
    r = dict(T=3)
    r.update(kw)
    assert attend(r=requests(**r)) == code
    assert sparse(r=requests(**r)) == code
    assert select(r=requests(**r)) == code


def test_attention_refusals():
    for kw in (dict(q=0), dict(out=0), dict(qt=-512), dict(qh=-64), dict(Hq=7), dict(Hq=0), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e300), dict(window=-1),
               dict(max_new=-1)):
        assert attend(**kw) == INVALID, kw
    for kw in (dict(q=FAKE + 2), dict(out=FAKE + 8), dict(qt=513), dict(qh=4), dict(Hq=1 << 20)):
        assert attend(**kw) == UNSUPPORTED, kw
    assert slnr.lib().sparselnr_paged_attention(FAKE, 512, 64, 8, None, requests(), 0.1, 0, 0, FAKE, None, None) == INVALID
    assert slnr.lib().sparselnr_paged_attention(FAKE, 512, 64, 8, cache(), None, 0.1, 0, 0, FAKE, None, None) == INVALID
    # nothing to do: no HIP call
    assert attend(r=requests(T=0), q=0, out=0) == OK
    assert attend(r=requests(R=0, T=0, table=0, seq_len=0, qptr=0), q=0, out=0) == OK
    assert sparse(sel=0) == INVALID
    assert sparse(top=0) == INVALID
    assert sparse(top=1 << 26) == UNSUPPORTED
    assert sparse(r=requests(T=0), sel=0) == OK


def test_select_refusals():
    for kw in (dict(q=0), dict(dtype=7), dict(kq=0), dict(ks=0), dict(pages=-1), dict(Hkv=0), dict(Hkv=3),
               dict(top=0), dict(first=-1), dict(local=-1), dict(first=3, local=2), dict(local=5)):
        assert select(**kw) == INVALID, kw
    for kw in (dict(top=257), dict(dim=60), dict(P=24), dict(kq=FAKE + 4), dict(pages=1 << 31)):
        assert select(**kw) == UNSUPPORTED, kw
    assert select(r=requests(T=0)) == OK


def test_append_refusals():
    for kw in (dict(k=0), dict(v=0), dict(slots=0), dict(T=-1), dict(kq=0), dict(ks=0), dict(kt=-128)):
        assert append(**kw) == INVALID, kw
    for kw in (dict(k=FAKE + 8), dict(kt=129), dict(kq=FAKE + 4), dict(kh=60)):
        assert append(**kw) == UNSUPPORTED, kw
    assert append(T=0, k=0, v=0, slots=0) == OK


def test_tables_refusals():
    for kw in (dict(R=-1), dict(W=-1), dict(F=-1), dict(T=-1), dict(stride=7), dict(ctx=0), dict(new=0), dict(table=0),
               dict(free=0), dict(qptr=0), dict(seq=0), dict(slots=0), dict(counts=0)):
        assert tables(**kw) == INVALID, kw
    for kw in (dict(P=0), dict(P=24), dict(P=8192), dict(R=1 << 24), dict(T=1 << 28), dict(W=1 << 28, stride=1 << 28)):
        assert tables(**kw) == UNSUPPORTED, kw


def test_refusals_leave_no_hip_error():
    before = slnr.sparselnr_last_hip_error()  # what other tests of this thread left
    attend(cache(dim=100))
    tables(P=24)
    assert slnr.sparselnr_last_hip_error() == before


def test_binding_checks():
    torch = pytest.importorskip("torch")
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    kc = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    table = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError):  # CPU tensors
        slnr.sparselnr_paged_attention(q, kc, kc, table, i, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        slnr.sparselnr_page_tables(i, i, table, i, 4, 16)
    with pytest.raises(TypeError):
        slnr.sparselnr_block_select([1], None, None, table, i, i, 16, 4)
    with pytest.raises(ValueError):
        slnr.sparselnr_cache_append(q, q, i, kc, kc)


def test_structs_have_the_layout_of_the_header(tmp_path):
    """The binding's structs against a C program that includes the header."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = []
    for st, name in ((slnr._KvCache, "sparselnr_kv_cache"), (slnr._Requests, "sparselnr_requests")):
        lines += ['printf("%%zu ", offsetof(%s, %s));' % (name, f) for f, _ in st._fields_]
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "sparselnr.h"\nint main(void) { %s return 0; }\n' % "\n".join(lines))
    exe = str(tmp_path / "layout")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I" + os.path.join(root, "include"), str(src), "-o", exe])
    got = subprocess.check_output([exe], text=True).split("\n")
    for line, st in zip(got, (slnr._KvCache, slnr._Requests)):
        assert [int(x) for x in line.split()] == [getattr(st, f).offset for f, _ in st._fields_] + [ctypes.sizeof(st)]


def test_strides_of_extents_of_one_do_not_count():
    """One token, page, place or head has no next one: torch gives such a dimension any stride."""
    one = dict(pages=1, k_page=1, v_page=3)
    r = requests(T=0)
    assert attend(cache(**one), r) == OK and attend(cache(**dict(one, pages=2))) == UNSUPPORTED
    assert attend(cache(page_size=1, k_slot=1, v_slot=5), r) == OK
    assert attend(cache(heads=1, k_head=1, v_head=7), r) == OK
    assert attend(cache(page_size=1, k_slot=-1), r) == INVALID
    assert attend(r=requests(T=1, R=0), qt=1) == OK and attend(r=requests(T=2, R=0), qt=1) == UNSUPPORTED
    assert attend(cache(heads=1), requests(T=1, R=0), Hq=1, qh=1) == OK
    assert append(cache(pages=0, heads=1), T=1, kt=1, kh=1) == OK  # no pages: nothing to do
    assert append(cache(pages=0), T=2, kt=1) == UNSUPPORTED
