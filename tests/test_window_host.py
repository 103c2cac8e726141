"""CPU tests of the prompt attention: which tiles the kernels walk over, the oracle's pins, the refusals that need no device."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import binding as rz
from paper_2407_15891_b200 import build as rz_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    rz_build.build()


def test_tiles_and_spans_against_single_pairs(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path / "geometry")
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    subprocess.run([gxx, "-std=c++17", "-O2", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(rz_build.CSRC), "-I", cuda,
                    os.path.join(ROOT, "tests", "window_geometry.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout


def test_oracle_window_attention_pins():
    rng = np.random.default_rng(0)
    K, V, q = rng.standard_normal((20, 8)), rng.standard_normal((20, 8)), rng.standard_normal((6, 8))
    full = orc.window_attention(q, K, V, 20, -1, 0, 0.3)
    for t in range(6):
        assert np.abs(full[t] - orc.full_attention(q[t], K[:15 + t], V[:15 + t], 0.3)).max() < 1e-12
    assert np.allclose(orc.window_attention(q, K, V, 20, 100, 0, 0.3), full)      # a window longer than the context
    assert np.allclose(orc.window_attention(q, K, V, 20, 3, 20, 0.3), full)       # sinks that cover it
    assert np.allclose(orc.window_attention(q, K, V, 20, 1, 0, 0.3), V[14:])      # a query that sees itself only
    assert not orc.window_attention(q, K, V, 20, 0, 0, 0.3).any()                 # nothing in sight
    # the last query of a window cache without compensation token is what the decode step over it gives
    hc = orc.compress_head(K, V, 20, 2, 5, False)
    want = orc.full_attention(q[5], hc.K, hc.V, 0.3)
    assert np.abs(orc.window_attention(q, K, V, 20, 5, 2, 0.3)[5] - want).max() < 1e-12


def _call(**kw):
    a = dict(q=1 << 20, q_b=4 * 1024, q_t=1024, K=1 << 21, V=1 << 22, kv_b=1 << 16, kv_h=1 << 14, kv_n=128, window=None, q_len=None,
             ctx_len=None, batch=2, tokens=4, ctx=128, hq=8, hk=4, dim=128, dtype=rz.RAZOR_BF16, n_sink=4, scale=0.0, out=1 << 23,
             ws=1 << 24, ws_bytes=1 << 34, stream=None)
    a.update(kw)
    return rz.load().razor_window_attention(*a.values())


def test_refusals():
    for k in ("q", "K", "V", "out", "ws"):
        assert _call(**{k: None}) == -2, k
    for kw in (dict(batch=0), dict(tokens=-1), dict(ctx=0), dict(hq=6), dict(hk=0), dict(n_sink=-1), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(q_b=64), dict(q_t=64), dict(kv_n=64), dict(kv_h=0),
               dict(kv_b=-128)):
        assert _call(**kw) == -1, kw
    for kw in (dict(dim=96), dict(dim=256), dict(dtype=rz.RAZOR_F32), dict(dtype=9), dict(hq=516, hk=4)):
        assert _call(**kw) == -3, kw
    for kw in (dict(q=(1 << 20) + 8), dict(K=(1 << 21) + 2), dict(out=(1 << 23) + 4), dict(ws=(1 << 24) + 128), dict(q_t=1028),
               dict(kv_n=132), dict(window=2), dict(q_len=1 << 20 | 1), dict(ctx_len=3)):
        assert _call(**kw) == -8, kw
    assert _call(ws_bytes=100) == -4
    assert _call(batch=1 << 24, tokens=1 << 16, hq=8) == -5
    assert _call(tokens=0, q=None) == 0                                           # nothing to do
    assert rz.load().razor_window_attention_workspace_bytes(1, 8, 4, 128, 4, None) == -2
    with pytest.raises(rz.RazorError):
        rz.razor_window_attention_workspace_bytes(1, 8, 3, 128, 4)


def test_workspace_follows_the_rows_of_a_unit():
    small = rz.razor_window_attention_workspace_bytes(4, 32, 8, 128, 1)
    assert small < 2 << 20                                                        # four rows a record
    big = rz.razor_window_attention_workspace_bytes(1, 32, 8, 128, 4096)
    assert 2 * 160 * 256 * 130 * 4 <= big < 2 * 160 * 256 * 130 * 4 + (1 << 16)
    assert rz.razor_window_attention_workspace_bytes(64, 32, 8, 128, 4096) == 256   # whole units from a queue
