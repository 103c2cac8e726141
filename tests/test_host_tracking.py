"""What the library's host code tells its kernels, checked without a GPU: razor_api.cu compiled against a fake CUDA runtime
(fake_device.cpp), on which nothing runs and launches, copies and what they were told are counted.

A kernel may start while the one before it on the stream is still running.  Whether it may then read the cache ahead of its
wait is the host's decision, from the kernels that can be in flight: a kernel that was only captured is not one of them."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2407_15891_b200 import binding as rz

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2407_15891_b200", "csrc")
A, B = 0x1000, 0x2000        # streams
PTR = 1 << 20                # an aligned address that nothing reads
SEEN = ("append_early", "decode_stable", "decode_early", "uploads", "captured_uploads", "launches", "records", "captured_records")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    so = str(tmp_path_factory.mktemp("fake") / "host_only.so")
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    cmd = [gxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-fvisibility=hidden", "-Wl,-z,defs", "-I", os.path.join(ROOT, "include"),
           "-I", CSRC, "-I", cuda, "-x", "c++", os.path.join(CSRC, "razor_api.cu"), os.path.join(CSRC, "razor_schedule.cpp"),
           os.path.join(ROOT, "tests", "fake_device.cpp"), "-o", so]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lib = C.CDLL(so)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    lib.fake_capture.argtypes = [vp, C.c_ulonglong]
    lib.fake_seen.argtypes = [vp]
    lib.razor_cache_create.argtypes = [C.POINTER(vp), C.POINTER(rz.RazorConfig), vp, sz, vp, sz, vp]
    lib.razor_cache_destroy.argtypes = [vp]
    lib.razor_query_bytes.argtypes = [C.POINTER(rz.RazorConfig), vp, vp, vp, C.POINTER(sz), C.POINTER(sz)]
    lib.razor_compress.argtypes = [vp, i32, vp, vp, i64, i64, i64, vp, vp, i32, vp, vp]
    lib.razor_compress_seq.argtypes = [vp, i32, i32, vp, vp, i64, i64, i32, vp, i32, i32, vp]
    lib.razor_append.argtypes = [vp, i32, vp, vp, vp]
    lib.razor_append_many.argtypes = [vp, i32, vp, vp, i32, vp]
    lib.razor_append_tree.argtypes = [vp, i32, vp, vp, i64, i64, vp, i32, vp, vp]
    lib.razor_decode_attention.argtypes = [vp, i32, vp, vp, vp]
    lib.razor_decode_attention_multi.argtypes = [vp, i32, vp, vp, i32, vp]
    lib.razor_decode_step.argtypes = [vp, i32, vp, vp, vp, vp, vp]
    lib.razor_decode_attention_tree.argtypes = [vp, i32, vp, i64, i64, vp, vp, i64, i64, vp, i32, vp, vp]
    lib.razor_schedule_query.argtypes = [vp, i32, vp, i32, C.POINTER(i32)]
    return lib


class Host:
    """A cache of two layers (batch 2, 4 KV heads of 2 queries) whose device is not there; calls return the status."""

    def __init__(self, lib, n_ctx=900, max_new=400, layers=2):
        lib.fake_reset()
        self.lib, self.n_ctx, self.batch = lib, n_ctx, 2
        cfg = rz.make_config(2, layers, 8, 4, 128, "bf16", 4, n_ctx, max_new)
        i32, u8 = C.c_int32 * 2, C.c_uint8 * (4 * layers)
        self.ctx, self.win, self.retr = i32(n_ctx, n_ctx), i32(200, 200), u8(*([1, 0, 0, 0] * layers))
        pool, ws, self.h = C.c_size_t(0), C.c_size_t(0), C.c_void_p()
        assert lib.razor_query_bytes(C.byref(cfg), self.ctx, self.win, self.retr, C.byref(pool), C.byref(ws)) == 0
        assert lib.razor_cache_create(C.byref(self.h), C.byref(cfg), PTR, pool, PTR, ws, None) == 0
        for layer in range(layers):
            assert self.compress(layer) == 0

    def compress(self, layer, stream=A):
        n = self.n_ctx
        return self.lib.razor_compress(self.h, layer, PTR, PTR, 4 * n * 128, n * 128, 128, self.ctx, self.retr, 4, self.win, stream)

    def compress_seq(self, layer, b, stream=A):
        n = self.n_ctx
        return self.lib.razor_compress_seq(self.h, layer, b, PTR, PTR, n * 128, 128, n, self.retr, 4, 200, stream)

    def append(self, layer, stream=A):
        return self.lib.razor_append(self.h, layer, PTR, PTR, stream)

    def append_tree(self, layer, counts=(2, 1), stream=A):
        return self.lib.razor_append_tree(self.h, layer, PTR, PTR, 4 * 512, 512, None, 4, (C.c_int32 * 2)(*counts), stream)

    def decode(self, layer, stream=A):
        return self.lib.razor_decode_attention(self.h, layer, PTR, PTR, stream)

    def step(self, layer, stream=A):
        return self.lib.razor_decode_step(self.h, layer, PTR, PTR, PTR, PTR, stream)

    def round(self, layer, n, stream=A):
        return self.lib.razor_decode_attention_multi(self.h, layer, PTR, PTR, n, stream)

    def tree(self, layer, stream=A):
        return self.lib.razor_decode_attention_tree(self.h, layer, PTR, 4 * 1024, 1024, PTR, PTR, 4 * 512, 512, PTR, 4, PTR, stream)

    @property
    def seen(self):
        out = (C.c_int * len(SEEN))()
        self.lib.fake_seen(out)
        return dict(zip(SEEN, out))

    def close(self):
        self.lib.razor_cache_destroy(self.h)


@pytest.fixture
def host(lib):
    h = Host(lib)
    yield h
    h.close()


WAITS = {"tree": lambda h, s: h.tree(0, s), "decode": lambda h, s: h.decode(0, s), "round": lambda h, s: h.round(0, 20, s),
         "tree of another layer": lambda h, s: h.tree(1, s)}


@pytest.mark.parametrize("call", WAITS)
def test_an_append_reads_early_behind_a_call_that_waits(host, call):
    """An append lets its successor start at once; an attention call between two of them does not."""
    assert host.append(0) == 0 and host.append(0) == 0
    assert host.seen["append_early"] == 0
    assert WAITS[call](host, A) == 0 and host.append(0) == 0
    assert host.seen["append_early"] == 1
    assert host.append(1) == 0 and host.append(0) == 0      # behind an append of another layer the first may still run
    assert host.seen["append_early"] == 0


@pytest.mark.parametrize("call", WAITS)
@pytest.mark.parametrize("stream", [A, B])
def test_a_captured_call_is_nothing_to_wait_behind(host, call, stream):
    """Append, an attention call captured (on another stream, or on the same), append: nothing ran between the two appends."""
    assert host.append(0) == 0
    host.lib.fake_capture(stream, 7)
    before = host.seen["launches"]
    assert WAITS[call](host, stream) == 0 and host.seen["launches"] > before
    host.lib.fake_capture(stream, 0)
    assert host.append(0) == 0
    assert host.seen["append_early"] == 0
    # and a decode may not load the head states ahead either
    host.lib.fake_capture(stream, 8)
    assert WAITS[call](host, stream) == 0
    host.lib.fake_capture(stream, 0)
    assert host.decode(0) == 0
    assert host.seen["decode_stable"] == 0
    assert host.append(0) == 0 and host.seen["append_early"] == 1


def test_a_capture_keeps_its_own_account(host):
    """Inside a capture the calls captured before count, over several streams of it too; the next capture starts afresh from what
    is in flight outside."""
    assert host.decode(0) == 0
    for s in (A, B):
        host.lib.fake_capture(s, 3)
    assert host.append(0, A) == 0 and host.seen["append_early"] == 1
    assert host.append(0, B) == 0 and host.seen["append_early"] == 0
    assert host.decode(0, A) == 0 and host.seen["decode_stable"] == 0
    assert host.append(0, A) == 0 and host.seen["append_early"] == 1
    for s in (A, B):
        host.lib.fake_capture(s, 0)
    assert host.append(0, A) == 0 and host.seen["append_early"] == 1     # eagerly, nothing has been appended since the decode
    host.lib.fake_capture(A, 4)
    assert host.append(0, A) == 0 and host.seen["append_early"] == 0     # the append before the capture
    assert host.tree(1, A) == 0 and host.append(0, A) == 0 and host.seen["append_early"] == 1
    host.lib.fake_capture(A, 0)
    assert host.append(0, A) == 0 and host.seen["append_early"] == 0


def test_steps_and_paths_are_writes(host):
    assert host.tree(0) == 0
    for write in (lambda: host.append_tree(0), lambda: host.step(0), lambda: host.compress(0), lambda: host.append(0)):
        assert write() == 0 and host.append(1) == 0 and host.append(0) == 0
        assert host.seen["append_early"] == 0
        assert host.tree(1) == 0 and host.append(0) == 0
        assert host.seen["append_early"] == 1
        assert host.tree(0) == 0


def test_a_layer_that_started_empty_has_a_schedule(lib):
    """A few tokens after an empty start, a captured decode finds a schedule on the device and uploads none: an upload that is
    only captured would leave the next eager decode without."""
    h = Host(lib, n_ctx=0)
    # the plan that the compression kernel writes for such a layer: an empty item per head, a job each
    items, n = (C.c_int32 * 40)(), C.c_int32(0)
    assert lib.razor_schedule_query(h.h, 0, items, 8, C.byref(n)) == 0 and n.value == 8
    assert list(items) == [x for head in range(8) for x in (head, 0, -1, 1, head)]
    assert h.seen["uploads"] == 2           # one plan of the compression for each layer
    for call in (h.decode, h.step):
        assert h.compress(0) == 0 and h.append(0) == 0 and h.append_tree(0, (4, 0)) == 0
        uploads = h.seen["uploads"]
        lib.fake_capture(B, 5)
        assert call(0, B) == 0
        lib.fake_capture(B, 0)
        assert h.decode(0) == 0
        assert h.seen["captured_uploads"] == h.seen["captured_records"] == 0 and h.seen["uploads"] == uploads
    # one sequence emptied again while the other goes on: the device holds another plan for the rest, all of it is sent
    uploads = h.seen["uploads"]
    assert h.compress_seq(0, 1) == 0
    assert h.seen["uploads"] == uploads + 3     # the compression's plan, items, jobs
    assert h.decode(0) == 0 and h.seen["uploads"] == uploads + 3
    h.close()


def test_a_schedule_that_was_only_captured_has_not_been_sent(lib):
    """A call whose schedule is stale, captured: the copies are in the graph.  The next call that runs sends its own, and the
    event that guards the staging area is not the graph's."""
    for n_ctx in (0, 900):               # (two tokens of two query heads: another schedule than the one-token decode's)
        h = Host(lib, n_ctx=n_ctx)
        lib.fake_reset()
        assert h.lib.razor_append_many(h.h, 0, PTR, PTR, 3, A) == 0
        lib.fake_capture(B, 5)
        assert h.round(0, 2, B) == 0
        lib.fake_capture(B, 0)
        seen = h.seen
        assert seen["captured_uploads"] > 0 and seen["captured_records"] == 0 and seen["uploads"] == 0
        assert h.round(0, 2) == 0
        assert h.seen["uploads"] == seen["captured_uploads"] and h.seen["records"] == 1
        assert h.round(0, 2) == 0 and h.seen["uploads"] == seen["captured_uploads"]
        h.close()


def test_the_tree_calls_refuse_before_anything_is_launched(lib, host):
    """Every argument the header rules out, on a layer that is ready: the status, and no launch."""
    base = dict(layer=0, q=PTR, qb=4 * 1024, qt=1024, k=PTR, v=PTR, kb=4 * 512, kt=512, parent=PTR, n=4, out=PTR)

    def tree(**kw):
        a = dict(base, **kw)
        return lib.razor_decode_attention_tree(host.h, a["layer"], a["q"], a["qb"], a["qt"], a["k"], a["v"], a["kb"], a["kt"],
                                               a["parent"], a["n"], a["out"], A)

    def path(counts=(1, 1), **kw):
        a = dict(base, path=None, **kw)
        return lib.razor_append_tree(host.h, a["layer"], a["k"], a["v"], a["kb"], a["kt"], a["path"], a["n"],
                                     (C.c_int32 * 2)(*counts) if counts else None, A)

    before = host.seen["launches"]
    for kw, status in [(dict(layer=2), -1), (dict(layer=-1), -1), (dict(n=0), -1), (dict(n=rz.TREE_MAX_NODES + 1), -1),
                       *[(dict([(name, None)]), -2) for name in ("q", "k", "v", "parent", "out")],
                       *[(dict([(name, PTR + 8)]), -8) for name in ("q", "k", "v", "out")], (dict(parent=PTR + 2), -8),
                       (dict(qt=1028), -8), (dict(kt=516), -8), (dict(qb=4100), -8), (dict(kb=2052), -8), (dict(qt=1016), -1),
                       (dict(kt=504), -1), (dict(kb=504), -1), (dict(qb=0), -1), (dict(qt=-1024), -1), (dict(kt=1 << 37), -1)]:
        assert tree(**kw) == status, kw
    for counts, kw, status in [((5, 0), {}, -1), ((-1, 0), {}, -1), (None, {}, -2), ((1, 1), dict(k=None), -2), ((1, 1), dict(v=None), -2),
                               ((1, 1), dict(layer=2), -1), ((1, 1), dict(n=0), -1), ((1, 1), dict(n=129), -1), ((1, 1), dict(kt=508), -8),
                               ((1, 1), dict(v=PTR + 8), -8), ((1, 1), dict(kb=8), -1)]:
        assert path(counts, **kw) == status, (counts, kw)
    assert path((0, 0)) == 0 and host.seen["launches"] == before
    lib.fake_capture(A, 9)
    assert path() == -1 and host.seen["launches"] == before
    lib.fake_capture(A, 0)
    for _ in range(99):
        assert path((4, 0)) == 0
    assert path((4, 4)) == 0 and path((1, 0)) == -5 and path((0, 4)) == 0     # 400 to a sequence, each on its own
    assert host.append(0) == -5 and tree() == 0
    # a stride that separates nothing may be anything
    assert tree(n=1, qt=0, kt=3) == 0
