"""What the paged-cache entry points allocate and launch, on a recording stand-in for the HIP
runtime: no GPU is needed."""
import pytest

from tests import host_record as hr


# ------------------------------------------------------------- workspaces


def workspace_scenario(rec):
    """Dense and sparse calls of every kind on one stream, a few tokens first."""
    out = []

    def look(what, call):
        events = rec.events(call)
        out.append([what, [e.bytes for e in events if e.kind == hr.MALLOC], len([e for e in events if e.kind == hr.FREE])])

    look("4 tokens", lambda: rec.attend(4))
    look("64 tokens", lambda: rec.attend(64))
    look("64 tokens, hint 1", lambda: rec.attend(64, max_new=1))
    look("64 heads a group", lambda: rec.attend(4, Hq=64, heads=1))
    look("4096 tokens of 64 requests", lambda: rec.attend(4096, requests=rec.requests(4096, 64)))
    look("selection of 4", lambda: rec.sparse(4, 16))
    for dtype in (0, 1, 2):
        for dim in (64, 128, 256):
            look("dim %d, dtype %d" % (dim, dtype), lambda: rec.attend(600, dim=dim, dtype=dtype))
    pages = rec.events(lambda: rec.sparse(2000, 16))
    out.append(["by pages", [e.bytes for e in pages if e.kind == hr.MALLOC], len([e for e in pages if e.kind == hr.FREE])])
    assert any("attend_pages" in e.name for e in pages)
    look("more by pages", lambda: rec.sparse(4000, 32))
    look("4 tokens again", lambda: rec.attend(4))
    return out


def test_a_streams_attention_workspace_is_allocated_once(tmp_path):
    """The first call allocates it and no later one frees or grows it, whatever its tokens, heads, hint,
    type and dim are: a captured graph that holds its address stays right.  Attention by pages has one of its own."""
    seen = hr.run(workspace_scenario, tmp_path)
    what, allocated, freed = seen[0]
    assert len(allocated) == 1 and freed == 0 and allocated[0] <= 140e6
    for what, allocated, freed in seen[1:]:
        if what == "by pages":
            assert len(allocated) == 1 and freed == 0
        elif what == "more by pages":
            assert freed <= 1  # of its own
        else:
            assert allocated == [] and freed == 0, what


# ------------------------------------------------------------- host threads


def thread_scenario(rec):
    """Two threads call on one stream, every launch waiting for the other thread's next one."""
    import threading
    out = []
    for kind in ("decode", "chunk", "selection", "by pages"):
        call = {"decode": lambda: rec.attend(4), "chunk": lambda: rec.attend(600), "selection": lambda: rec.sparse(4, 16),
                "by pages": lambda: rec.sparse(2000, 16)}[kind]
        call()  # workspaces
        rec.events()
        rec.wait(150)
        threads = [threading.Thread(target=call) for _ in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        rec.wait(0)
        out.append([kind, [[e.thread, e.name] for e in rec.events() if e.kind == hr.LAUNCH]])
    # a larger call by pages and one that is under way
    rec.wait(150)
    threads = [threading.Thread(target=lambda n=n: rec.sparse(n, 32)) for n in (2000, 4000)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    rec.wait(0)
    out.append(["growth", [[e.thread, e.name or "malloc"] for e in rec.events()]])
    return out


def test_calls_of_two_threads_on_one_stream_do_not_mix(tmp_path):
    """A call's launches share partial results in the stream's workspace: the other thread's come before
    or after all of them, and so does an allocation that frees the workspace."""
    for kind, events in hr.run(thread_scenario, tmp_path):
        who = [t for t, _ in events]
        runs = 1 + sum(a != b for a, b in zip(who, who[1:]))
        names = [n for _, n in events]
        assert len(set(who)) == 2, kind
        if kind in ("decode", "chunk", "selection"):  # a walk and its join at a time
            assert len(names) % 2 == 0
            for i in range(0, len(names), 2):
                assert who[i] == who[i + 1] and "attend" in names[i] and "join" in names[i + 1], (kind, names)
        else:
            assert runs == 2, (kind, names)


# ------------------------------------------------------------- limits


def huge_selection_scenario(rec):
    """Selections of so many pages a token that one token's entries pass 2^30."""
    out = []
    for top, heads in ((1 << 26, 16), (1 << 26, 64), ((1 << 27) - 1, 8), (1 << 26, 15)):
        c = dict(page_size=4, heads=heads, dim=64)
        out.append(rec.sparse(2, top, Hq=heads, requests=rec.requests(2, 1, 1 << 24), **c))
    return out


def test_selections_past_the_lists_do_not_divide_by_nothing(tmp_path):
    """They go by queries, whose walk has no lists."""
    assert hr.run(huge_selection_scenario, tmp_path) == [0, 0, 0, 0]


def select_shapes_scenario(rec):
    out = []
    for T in (1, 3, 700):
        for W in (1, 20, 100, 511, 5000):
            for top in (1, 2, 3, 4, 5, 6, 7, 64, 101, 254, 255, 256):
                for dim in (8, 72, 256):
                    def call():
                        rc = rec.lib.sparselnr_block_select(1 << 37, 8 * dim, dim, 8, 0, 1 << 32, 1 << 33, 1 << 20, 16, 2, dim,
                                                            rec.requests(T, 1, W), top, 0, 1, 1 << 38, 1)
                        assert rc == 0
                    e, = rec.events(call)
                    assert "block_select" in e.name
                    out.append([T, W, top, dim, e.lds])
    return out


def test_selection_lays_its_lds_out_in_16_bytes(tmp_path):
    """Its parts (keys, indices, 8-bit queries, which are read 16 bytes at a time, counts) follow one another, and the
    last ones are multiples of 16 bytes: so is the whole, if the queries begin at one."""
    for T, W, top, dim, lds in hr.run(select_shapes_scenario, tmp_path):
        assert lds % 16 == 0 and lds <= 160 * 1024, (T, W, top, dim, lds)


def huge_batches_scenario(rec):
    """The largest numbers of requests and tokens that the interface admits."""
    out = []

    def look(what, call):
        rc = []
        events = rec.events(lambda: rc.append(call()))
        out.append([what, rc[0], [[e.name, list(e.grid), list(e.block)] for e in events if e.kind == hr.LAUNCH]])

    R, T = (1 << 24) - 1, (1 << 28) - 1
    for heads, Hq in ((1, 1), (4, 4), (2, 6), (8, 8), (128, 128)):
        T = min((1 << 28) - 1, ((1 << 31) - 1) // Hq)
        c = dict(heads=heads, dim=64)
        look("attend", lambda: rec.attend(T, Hq=Hq, requests=rec.requests(T, R, 4), **c))
        look("sparse", lambda: rec.sparse(T, 2, Hq=Hq, requests=rec.requests(T, R, 4), **c))
        look("sparse", lambda: rec.sparse(T, 4, Hq=Hq, requests=rec.requests(T, 3, 4), **c))
        for r in (R, 16, 1 << 23):
            look("select", lambda: rec.lib.sparselnr_block_select(1 << 37, 64 * Hq, 64, Hq, 0, 1 << 32, 1 << 33, 1 << 20, 16, heads, 64,
                                                                  rec.requests(T, r, 4), 2, 1, 1, 1 << 38, 1))
    T = (1 << 28) - 1
    k = rec.cache(heads=2, dim=64)
    look("append", lambda: rec.lib.sparselnr_cache_append(1 << 32, 128, 64, 1 << 33, 128, 64, 1 << 34, k, 1 << 35, 1 << 36, T, 1))
    look("append too many", lambda: rec.lib.sparselnr_cache_append(1 << 32, 128, 64, 1 << 33, 128, 64, 1 << 34, k, 1 << 35, 1 << 36,
                                                                   T + 1, 1))
    look("tables", lambda: rec.lib.sparselnr_page_tables(1 << 32, 1 << 33, 1 << 34, 4, 1 << 35, 1 << 36, 1 << 37, 1 << 38, 1 << 39, R, 4,
                                                         1 << 30, T, 16, 1))
    return out


def test_launches_of_the_largest_batches_fit(tmp_path):
    """A launch has fewer than 2^32 threads a dimension, whatever sizes are admitted."""
    for what, rc, launches in hr.run(huge_batches_scenario, tmp_path):
        assert rc == (2 if what == "append too many" else 0), what
        assert bool(launches) == (rc == 0)
        for name, grid, block in launches:
            for g, b in zip(grid, block):
                assert 0 < g * b < 1 << 32, (what, name, grid, block)


# ------------------------------------------------------------- memory of the host


def no_memory_scenario(rec):
    """Calls whose records cannot be allocated: the device's facts first, then a stream's workspace."""
    out = []
    for _ in range(2):
        rec.fake.record_no_memory(1)
        out.append([rec.attend(4, stream=7), rec.sparse(2000, 16, stream=7)])
        rec.fake.record_no_memory(0)
        assert rec.attend(4) == 0 and rec.sparse(2000, 16) == 0  # the device is known from here on
    return out


def test_no_memory_is_a_status(tmp_path):
    """No exception crosses the interface."""
    assert hr.run(no_memory_scenario, tmp_path) == [[4, 4], [4, 4]]


def by_pages_scenario(rec):
    out = []
    for G, P, D, T, Hkv, top in ((128, 512, 64, 900, 1, 3), (40, 256, 128, 900, 1, 3), (1, 64, 64, 3000, 8, 16), (3, 4096, 72, 200, 1, 3),
                                 (1, 64, 128, 900, 8, 12), (129, 1024, 64, 900, 1, 3), (16, 32, 64, 900, 1, 3)):
        events = rec.events(lambda: rec.sparse(T, top, Hq=G * Hkv, requests=rec.requests(T, 1, 40), heads=Hkv, dim=D, page_size=P))
        out.append(any("attend_pages" in e.name for e in events))
    return out


def test_which_selections_go_by_pages(tmp_path):
    """The shapes that the GPU tests mean to; not groups past a tile's rows, nor pages of less than four keys a head."""
    assert hr.run(by_pages_scenario, tmp_path) == [True] * 5 + [False] * 2
