"""Rows of V that no query sees may hold anything, and what they hold does not cost a call anything to speak of.

A NaN in sight of some rows of a tile and hidden from others is taken out and put back by a slow look through the tile; the tail
of a buffer behind its context, or what lies before every window, must not set that off."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2407_15891_b200 import binding as rz
from paper_2407_15891_b200 import build as rz_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


def test_which_keys_are_seen(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path / "seen")
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    subprocess.run([gxx, "-std=c++17", "-O2", "-I", os.path.join(ROOT, "include"), "-I", rz_build.CSRC, "-I", cuda,
                    os.path.join(ROOT, "tests", "window_seen.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout


def _fastest(f):
    f()
    best = float("inf")
    for _ in range(30):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,N,Hq,Hk,D,ctx,window", [(4, 1, 8192, 32, 8, 128, 8000, None), (6, 333, 9001, 16, 8, 64, 8000, 500),
                                                      (1, 4096, 4224, 32, 8, 128, 4100, 500), (64, 1, 1024, 64, 32, 128, 1000, 300)])
def test_unseen_rows_cost_nothing(B, T, N, Hq, Hk, D, ctx, window):
    """(Looked through, they took 4 to 700 times as long as the call: three times is far from either.)"""
    g = torch.Generator(DEV).manual_seed(T)
    q, K, V = (torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16) for s in ((B, T, Hq, D), (B, Hk, N, D), (B, Hk, N, D)))
    c, out = torch.full((B,), ctx, dtype=torch.int32, device=DEV), torch.zeros_like(q)
    w = None if window is None else torch.full((B, Hk), window, dtype=torch.int32, device=DEV)
    ws = torch.empty(rz.razor_window_attention_workspace_bytes(B, Hq, Hk, D, T), dtype=torch.uint8, device=DEV)

    def call():
        rz.razor_window_attention(q, K, V, 0, w, None, c, out=out, workspace=ws)

    clean = _fastest(call)
    want = out.clone()
    V[:, :, ctx:] = float("nan")                            # behind the context
    if window is not None:
        V[:, :, :max(0, ctx - T - window + 1)] = float("inf")   # before the first query's window
    assert _fastest(call) <= 3 * clean
    assert torch.equal(out, want)
