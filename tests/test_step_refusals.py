"""A refused razor_decode_step leaves the cache as it was, whichever way the step would have gone (one launch, or an append and a
decode: 8-bit rows, heads without a window).  The library's host code on a fake CUDA runtime."""
import ctypes as C

import numpy as np
import pytest

from paper_2407_15891_b200 import binding as rz

from test_host_tracking import PTR, SEEN, lib  # noqa: F401


@pytest.mark.parametrize("dtype,window", [("i8", 64), ("i8", 0), ("bf16", 64), ("bf16", 0), ("f32", 0)])
def test_a_refused_step_appends_nothing(lib, dtype, window):  # noqa: F811
    lib.fake_reset()
    cfg = rz.make_config(2, 1, 8, 4, 128, dtype, 4, 900, 2)
    h, pool, ws = C.c_void_p(), C.c_size_t(), C.c_size_t()
    retr, lens, win = np.zeros(4, dtype=np.uint8), np.array([900, 900], dtype=np.int32), np.array([window] * 2, dtype=np.int32)
    assert lib.razor_query_bytes(C.byref(cfg), lens.ctypes.data, win.ctypes.data, retr.ctypes.data, C.byref(pool), C.byref(ws)) == 0
    assert lib.razor_cache_create(C.byref(h), C.byref(cfg), PTR, pool, PTR, ws, None) == 0
    assert lib.razor_compress(h, 0, PTR, PTR, 4 * 900 * 128, 900 * 128, 128, lens.ctypes.data, retr.ctypes.data, 4, win.ctypes.data,
                              None) == 0

    def state():
        seen, sizes = (C.c_int * len(SEEN))(), (C.c_size_t(), C.c_size_t())
        lib.fake_seen(seen)
        assert lib.razor_cache_stats(h, 0, C.byref(sizes[0]), C.byref(sizes[1])) == 0
        return dict(zip(SEEN, seen))["launches"], sizes[0].value, sizes[1].value

    lib.razor_cache_stats.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
    before = state()
    for bad in range(4):
        for off in (2, 8):
            args = [PTR + (off if i == bad else 0) for i in range(4)]
            assert lib.razor_decode_step(h, 0, *args, None) == -8, bad
            assert state() == before, bad
    for bad in range(4):
        assert lib.razor_decode_step(h, 0, *[None if i == bad else PTR for i in range(4)], None) == -2
        assert state() == before
    # both tokens that there is room for still go in
    for _ in range(2):
        assert lib.razor_decode_step(h, 0, PTR, PTR, PTR, PTR, None) == 0
    after = state()
    assert after[0] > before[0] and after[2] > before[2]
    assert lib.razor_decode_step(h, 0, PTR, PTR, PTR, PTR, None) == -5 and state() == after
    lib.razor_cache_destroy(h)
