"""What the calls of the 4-bit cache and of the pages' life allocate and launch, on a recording stand-in for
the HIP runtime: no GPU is needed."""
from tests import host_record as hr


def fp4_cache(rec, pages=1 << 20, page_size=64, heads=8, dim=128, dtype=0):
    row, exps = 16 * (-(-dim // 32)), -(-dim // 32)
    c = dict(k=1 << 32, v=1 << 33, k_scale=1 << 40, v_scale=1 << 41, pages=pages, page_size=page_size, heads=heads, dim=dim,
             dtype=dtype)
    for x, size in (("k", row), ("v", row), ("ks", exps), ("vs", exps)):
        c.update({x + "_page": heads * page_size * size, x + "_head": page_size * size, x + "_slot": size})
    return rec.slnr._Fp4Cache(**c)


def attend4(rec, T, Hq=8, max_new=0, stream=1, requests=None, **cache):
    c = fp4_cache(rec, **cache)
    return rec.lib.sparselnr_paged_attention_fp4(1 << 37, Hq * c.dim, c.dim, Hq, c, requests or rec.requests(T), 0.1, 0, max_new,
                                                 1 << 38, None, stream)


def free(rec, n, R=1000, W=64, pages=100000, P=16, most=1000, stream=1):
    return rec.lib.sparselnr_page_free(1 << 32, 1 << 33, W, 1 << 34, 1 << 35, 1 << 36, 1 << 37, n, R, W, most, pages, P, stream)


def compact(rec, R=1000, W=64, pages=100000, P=16, stream=1):
    return rec.lib.sparselnr_page_compact(1 << 33, W, 1 << 34, 1 << 35, 1 << 36, 1 << 37, R, W, pages, P, stream)


def fork(rec, n, R=1000, W=64, F=100, pages=100000, P=16, stream=1):
    return rec.lib.sparselnr_page_fork(1 << 31, 1 << 32, 1 << 33, W, 1 << 34, 1 << 35, 1 << 36, 1 << 37, 1 << 38, n, R, W, F, pages, P,
                                       stream)


def copy(rec, n, rows, pages=1000, stream=1):
    a = rec.slnr._PageArray
    arrays = (a * len(rows))(*(a((i + 1) << 44, outer * inner * row, outer, inner * row, inner, row, row)
                               for i, (outer, inner, row) in enumerate(rows)))
    return rec.lib.sparselnr_page_copy(1 << 32, n, arrays, len(rows), pages, stream)


# ------------------------------------------------------------- workspaces


def workspace_scenario(rec):
    out = []

    def look(what, call):
        rc = []
        events = rec.events(lambda: rc.append(call()))
        out.append([what, rc[0], [e.bytes for e in events if e.kind == hr.MALLOC], len([e for e in events if e.kind == hr.FREE])])

    look("first attend", lambda: attend4(rec, 4))
    for dtype in (0, 1, 2):
        for dim in (8, 64, 72, 128, 256):
            for T, Hq, heads, hint in ((4, 8, 8, 0), (64, 8, 8, 1), (700, 8, 2, 0), (4096, 64, 1, 0), (1, 4096, 4096, 0)):
                look("attend", lambda: attend4(rec, T, Hq=Hq, heads=heads, dim=dim, dtype=dtype, max_new=hint))
    look("attend", lambda: rec.attend(600))  # over the other cache: the same one
    look("few", lambda: free(rec, 5, W=16, pages=3000))
    look("few", lambda: compact(rec, R=5, W=16, pages=3000))
    look("first life", lambda: compact(rec))
    for n, W, pages in ((900, 64, 100000), (1 << 20, 4000, 99999), (1 << 20, 4000, 64), (3, 64, 100000), (70000, 1, 5)):
        look("life", lambda: free(rec, n, R=n, W=W, pages=pages))
        look("life", lambda: compact(rec, R=n, W=W, pages=pages))
    look("more pages", lambda: compact(rec, pages=50 * 1000 * 1000))
    look("life", lambda: free(rec, 900))
    return out


def test_workspaces_do_not_grow(tmp_path):
    """Attention over both caches has one of one size; the pages' sets have one that goes by the pages, and none where
    one block does it all.  A captured graph that holds an address stays right."""
    for what, rc, allocated, freed in hr.run(workspace_scenario, tmp_path):
        assert rc == 0
        if what in ("first attend", "first life"):
            assert len(allocated) == 1 and freed == 0, what
            assert allocated[0] <= (140e6 if what == "first attend" else 512 * 1024)
        elif what == "more pages":
            assert len(allocated) == 1 and freed <= 1 and allocated[0] <= 11e6
        else:
            assert allocated == [] and freed == 0, what


# ------------------------------------------------------------- host threads


def thread_scenario(rec):
    """Two threads call on one stream, every launch waiting for the other thread's next one."""
    import threading
    out = []
    for kind, call in (("decode", lambda: attend4(rec, 4)), ("chunk", lambda: attend4(rec, 600)),
                       ("free", lambda: free(rec, 900)), ("compact", lambda: compact(rec))):
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
    return out


def test_calls_of_two_threads_on_one_stream_do_not_mix(tmp_path):
    """The launches that share a workspace follow one another: a walk and its join, or a whole call."""
    for kind, events in hr.run(thread_scenario, tmp_path):
        who, names = [t for t, _ in events], [n for _, n in events]
        assert len(set(who)) == 2, kind
        if kind in ("decode", "chunk"):
            assert len(names) % 2 == 0
            for i in range(0, len(names), 2):
                assert who[i] == who[i + 1] and "attend" in names[i] and "join" in names[i + 1], (kind, names)
        else:
            assert 1 + sum(a != b for a, b in zip(who, who[1:])) == 2, (kind, names)


# ------------------------------------------------------------- limits


def largest_scenario(rec):
    out = []

    def look(what, call):
        rc = []
        events = rec.events(lambda: rc.append(call()))
        out.append([what, rc[0], [[e.name, list(e.grid), list(e.block), e.lds] for e in events if e.kind == hr.LAUNCH]])

    R = (1 << 24) - 1
    for heads, Hq in ((1, 1), (4, 4), (2, 6), (8, 8), (128, 128)):
        T = min((1 << 28) - 1, ((1 << 31) - 1) // Hq)
        for dtype in (0, 2):
            look("attend", lambda: attend4(rec, T, Hq=Hq, requests=rec.requests(T, R, 4), heads=heads, dim=64, dtype=dtype))
        look("attend", lambda: attend4(rec, T, Hq=Hq, requests=rec.requests(T, R, 4), heads=heads, dim=64, max_new=1))
    for dim in (8, 128, 256):
        look("attend", lambda: attend4(rec, 5000, requests=rec.requests(5000, 3, 4), dim=dim, dtype=1))
    T = (1 << 28) - 1
    c = fp4_cache(rec, heads=2, dim=64)
    for dim, heads in ((64, 2), (256, 8)):
        c = fp4_cache(rec, heads=heads, dim=dim)
        look("append", lambda: rec.lib.sparselnr_cache_append_fp4(1 << 32, dim * heads, dim, 1 << 33, dim * heads, dim, 1 << 34, c, T, 1))
        look("read", lambda: rec.lib.sparselnr_cache_read_fp4(1 << 34, c, 1 << 35, 1 << 36, T, 1))
    pages = (1 << 31) - 1
    for n, W in ((R, 4), (1, 1 << 24), (R, 1 << 24)):
        look("free", lambda: free(rec, n, R=R, W=W, pages=pages, most=pages))
        look("compact", lambda: compact(rec, R=n, W=W, pages=pages))
        look("fork", lambda: fork(rec, n, R=R, W=W, F=pages, pages=pages))
    look("copy", lambda: copy(rec, (1 << 31) - 1, [(1, 1, 1 << 20)], pages=pages))
    look("copy", lambda: copy(rec, 1, [(1 << 10, 1 << 10, 16)] * 8, pages=5))
    return out


def test_launches_of_the_largest_sizes_fit(tmp_path):
    """A launch has fewer than 2^32 threads a dimension and 65536 blocks in the second, and no more LDS than there is."""
    for what, rc, launches in hr.run(largest_scenario, tmp_path):
        assert rc == 0 and launches, what
        for name, grid, block, lds in launches:
            assert lds <= 160 * 1024 and grid[1] < 65536 and grid[2] == 1
            for g, b in zip(grid, block):
                assert 0 < g * b < 1 << 32, (what, name, grid, block)


def no_memory_scenario(rec):
    out = []
    for _ in range(2):
        rec.fake.record_no_memory(1)
        out.append([attend4(rec, 4, stream=7), attend4(rec, 4000, stream=7), free(rec, 900, stream=7), compact(rec, stream=7)])
        rec.fake.record_no_memory(0)
        assert attend4(rec, 4) == 0 and free(rec, 900) == 0
    return out


def test_no_memory_is_a_status(tmp_path):
    """No exception crosses the interface."""
    assert hr.run(no_memory_scenario, tmp_path) == [[4] * 4] * 2


# ------------------------------------------------------------- which way a call goes


def ways_scenario(rec):
    out = []
    for n, W, pages in ((4, 64, 2048), (32, 64, 4096), (32, 64, 16384), (64, 64, 0), (65, 64, 8), (1, 4, 32768), (0, 5, 10),
                        (1, 4, 65536)):
        names = []
        for call in (lambda: free(rec, n, R=max(n, 1), W=W, pages=pages), lambda: compact(rec, R=n, W=W, pages=pages)):
            names.append([e.name for e in rec.events(call) if e.kind == hr.LAUNCH])
        out.append([len(names[0]), len(names[1]), "one" in names[0][-1]])
    for Hq, heads, T, hint in ((8, 8, 64, 0), (8, 8, 65, 0), (64, 8, 8, 0), (64, 8, 9, 0), (64, 8, 900, 8), (64, 8, 900, 9)):
        names = [e.name for e in rec.events(lambda: attend4(rec, T, Hq=Hq, heads=heads, max_new=hint)) if e.kind == hr.LAUNCH]
        out.append([len(names), any("attend_many" in n for n in names)])
    return out


def test_which_calls_go_which_way(tmp_path):
    """One block where entries and an eighth of the pages are at most 4096; rows of many only past 64."""
    one, several = [1, 1, True], [3, 4, False]
    assert hr.run(ways_scenario, tmp_path) == [one, one, one, one, several, several, one, several] + [
        [2, False], [4, True], [2, False], [4, True], [2, False], [4, True]]
