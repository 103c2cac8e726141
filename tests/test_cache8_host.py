"""CPU tests of the 8-bit cache: the oracle's quantiser pinned by its definition, sizes, refusals, what the host code does."""
import ctypes as C

import numpy as np
import pytest

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import binding as rz
from paper_2407_15891_b200 import build as rz_build

from test_host_tracking import PTR, lib  # noqa: F401  (the library's host code on a fake CUDA runtime)


@pytest.fixture(scope="module", autouse=True)
def _built():
    rz_build.build()


def test_quantised_rows_are_within_half_a_step():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((50, 64)) * 10.0 ** rng.uniform(-20, 20, (50, 1))).astype(np.float32)
    codes, scale, held = orc.quantise_rows(x)
    top = np.abs(x).max(1)
    assert np.abs(codes).max(1).tolist() == [127] * 50                            # the largest magnitude is code 127
    assert (np.abs(held.astype(np.float64) - x) <= top[:, None] / 254 * (1 + 1e-5)).all()
    odd = np.zeros((5, 64), dtype=np.float32)
    odd[1, 3], odd[2, 5], odd[3, 7], odd[4, 9] = 1e-31, np.nan, -np.inf, 8e-31
    codes, scale, held = orc.quantise_rows(odd)
    assert (held[:2] == 0).all() and np.isnan(held[2:4]).all() and held[4, 9] == np.float32(8e-31) / np.float32(127) * 127
    ties = np.zeros((1, 64), dtype=np.float32)
    ties[0, :5] = [254, 1, 3, -1, 5]                                              # steps of 2: halves go to even
    assert orc.quantise_rows(ties)[0][0, :5].tolist() == [127, 0, 2, 0, 2]


def test_sizes():
    retr = np.zeros((1, 4), dtype=np.uint8)
    for D in (64, 128):
        cfg = rz.make_config(1, 1, 8, 4, D, "i8", 4, 1000, 8)
        pool, ws = rz.razor_query_bytes(cfg, [1000], [100], retr)
        pages = 4 * 7                                                             # 104 tokens a head
        assert pool == -(-pages * 2 * 16 * (D + 4) // 256) * 256
        bf = rz.make_config(1, 1, 8, 4, D, "bf16", 4, 1000, 8)
        assert rz.razor_query_bytes(bf, [1000], [100], retr)[1] == ws             # the workspace does not depend on it


@pytest.fixture()
def cache(lib):  # noqa: F811
    lib.fake_reset()
    cfg = rz.make_config(2, 1, 8, 4, 128, "i8", 4, 900, 400)
    h, ws = C.c_void_p(), C.c_size_t()
    pool = C.c_size_t()
    retr, lens, win = np.zeros(4, dtype=np.uint8), np.array([900, 900], dtype=np.int32), np.array([64, 64], dtype=np.int32)
    assert lib.razor_query_bytes(C.byref(cfg), lens.ctypes.data, win.ctypes.data, retr.ctypes.data, C.byref(pool), C.byref(ws)) == 0
    assert lib.razor_cache_create(C.byref(h), C.byref(cfg), PTR, pool, PTR, ws, None) == 0
    assert lib.razor_compress(h, 0, PTR, PTR, 4 * 900 * 128, 900 * 128, 128, lens.ctypes.data, retr.ctypes.data, 4, win.ctypes.data,
                              None) == 0
    yield h
    lib.razor_cache_destroy(h)


def _launches(lib):  # noqa: F811
    seen = (C.c_int * 8)()
    lib.fake_seen(seen)
    return seen[5]


def test_tree_calls_are_refused_and_steps_take_two_launches(lib, cache):  # noqa: F811
    n = np.zeros(2, dtype=np.int32)
    assert lib.razor_decode_attention_tree(cache, 0, PTR, 4096, 1024, PTR, PTR, 4096, 512, PTR, 2, PTR, None) == -3
    assert lib.razor_append_tree(cache, 0, PTR, PTR, 4096, 512, None, 2, n.ctypes.data, None) == -3
    before = _launches(lib)
    assert lib.razor_decode_step(cache, 0, PTR, PTR, PTR, PTR, None) == 0
    assert _launches(lib) == before + 2                                           # append, decode
    before = _launches(lib)
    assert lib.razor_decode_attention_multi(cache, 0, PTR, PTR, 10, None) == 0     # 20 query rows a KV head: blocks of 8
    assert _launches(lib) == before + 3


@pytest.mark.parametrize("kw,code", [(dict(dtype=3), -3), (dict(dtype="i8", head_dim=96), -3), (dict(dtype="i8", n_q_heads=24), -3)])
def test_config_refusals(kw, code):
    a = dict(batch=1, n_layers=1, n_q_heads=8, n_kv_heads=8, head_dim=128, dtype="i8", n_sink=4, max_ctx_len=100, max_new_tokens=0)
    a.update(kw)
    with pytest.raises(rz.RazorError) as e:
        rz.razor_query_bytes(rz.make_config(**a), [10], [5], np.zeros(8, dtype=np.uint8))
    assert e.value.status == code


def test_other_calls_do_not_take_the_type():
    assert rz.load().razor_verify_tree(PTR, 8, 8, None, 0, 0, rz.RAZOR_I8, PTR, PTR, PTR, PTR, 1, 1, 8, PTR, PTR, PTR, None) == -3
    assert rz.load().razor_compensation_mean_static(PTR, PTR, 1 << 20, 128, 1, 128, rz.RAZOR_I8, 10, 0, 5, PTR, PTR, None, None) == -3
