"""Calls of the library on a recording stand-in for the HIP runtime (tests/host_runtime):
which kernels it launches, in which shapes, and what it allocates, without a GPU.

A scenario is a function of a test module that takes a Recorder and returns plain values;
`run` executes it in a process of its own, where the stand-in is loaded first."""
import ctypes
import json
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = os.path.join(ROOT, "tests", "host_runtime", "record_hip.cpp")
LAUNCH, MALLOC, FREE = 0, 1, 2


class Event(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("device", ctypes.c_int32), ("thread", ctypes.c_uint64),
                ("grid", ctypes.c_uint32 * 3), ("block", ctypes.c_uint32 * 3), ("lds", ctypes.c_uint64),
                ("stream", ctypes.c_uint64), ("ptr", ctypes.c_uint64), ("bytes", ctypes.c_uint64),
                ("raw_name", ctypes.c_char * 256)]

    @property
    def name(self):
        return self.raw_name.decode()


class Recorder:
    def __init__(self, path):
        self.fake = ctypes.CDLL(path, mode=ctypes.RTLD_GLOBAL)
        self.fake.record_get.restype = ctypes.POINTER(Event)
        import paper_2205_11622_amd as slnr
        self.slnr = slnr
        self.lib = slnr.lib()

    def events(self, call=None):
        """What was recorded since the last look, by `call` if there is one."""
        if call is not None:
            self.fake.record_reset()
            call()
        out = []
        for i in range(self.fake.record_count()):
            e = Event()
            ctypes.pointer(e)[0] = self.fake.record_get(i)[0]
            out.append(e)
        self.fake.record_reset()
        return out

    def wait(self, ms):
        self.fake.record_wait(ms)

    def cache(self, **kw):
        c = dict(k=1 << 32, v=1 << 33, pages=1 << 20, page_size=64, heads=8, dim=128, dtype=0)
        c.update(kw)
        D, H, P = c["dim"], c["heads"], c["page_size"]
        for x in "kv":
            c.setdefault(x + "_page", P * H * D)
            c.setdefault(x + "_slot", H * D)
            c.setdefault(x + "_head", D)
        return self.slnr._KvCache(**c)

    def requests(self, T, R=1, W=64):
        return self.slnr._Requests(table=1 << 34, table_stride=W, seq_len=1 << 35, qptr=1 << 36, R=R, W=W, T=T)

    def attend(self, T, Hq=8, max_new=0, stream=1, requests=None, **cache):
        c = self.cache(**cache)
        return self.lib.sparselnr_paged_attention(1 << 37, Hq * c.dim, c.dim, Hq, c, requests or self.requests(T), 0.1, 0,
                                                  max_new, 1 << 38, None, stream)

    def sparse(self, T, top, Hq=8, stream=1, requests=None, **cache):
        c = self.cache(**cache)
        return self.lib.sparselnr_block_attention(1 << 37, Hq * c.dim, c.dim, Hq, c, requests or self.requests(T), 1 << 39,
                                                  top, 0.1, 1 << 38, None, stream)


def run(scenario, folder, timeout=100):
    """The value that scenario(recorder) returns, in a process of its own."""
    lib = os.path.join(str(folder), "librecord_hip.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-fvisibility=hidden",
                           "-I/opt/rocm/include", SOURCE, "-o", lib, "-lpthread"])
    code = ("import importlib, json, sys; sys.path.insert(0, %r); from tests import host_record as h; "
            "print(json.dumps(getattr(importlib.import_module(%r), %r)(h.Recorder(%r))))"
            % (ROOT, "tests." + scenario.__module__.split(".")[-1], scenario.__name__, lib))
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=timeout)
    assert r.returncode == 0, "status %d\n%s%s" % (r.returncode, r.stdout, r.stderr)
    return json.loads(r.stdout.splitlines()[-1])
