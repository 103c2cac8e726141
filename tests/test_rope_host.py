"""CPU tests of the rotary operator: the oracle pinned by what a rotation is, the frequencies against closed forms, the
refusals that need no device."""
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import razor_oracle as orc
from paper_2407_15891_b200 import binding as rz
from paper_2407_15891_b200 import build as rz_build

INVALID, NULL, UNSUPPORTED, MISALIGNED = -1, -2, -3, -8


@pytest.fixture(scope="module", autouse=True)
def _built():
    rz_build.build()


@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_rope_is_a_rotation_by_the_position(interleaved):
    rng = np.random.default_rng(0)
    w = 10000.0 ** (-np.arange(6) / 6)
    x, y = rng.standard_normal((2, 16))
    turn = lambda v, p, **kw: orc.rope(v, np.array(p), w, interleaved, **kw)  # noqa: E731
    assert np.allclose(np.linalg.norm(turn(x, 77)), np.linalg.norm(x))
    assert np.allclose(turn(turn(x, 5), 9), turn(x, 14))
    assert np.allclose(turn(turn(x, 5), 5, inverse=True), x)
    assert np.allclose(turn(x, 103) @ turn(y, 100), turn(x, 3) @ turn(y, 0))      # only the distance counts
    assert np.array_equal(turn(x, 3)[12:], x[12:])                              # what is not rotated is carried over
    a, b = (0, 1) if interleaved else (0, 6)
    assert np.allclose(turn(x, 2)[a], x[a] * math.cos(2) - x[b] * math.sin(2))
    assert np.allclose(turn(x, 2, gain=1.5)[:12], 1.5 * turn(x, 2)[:12])


def test_frequencies_by_closed_form():
    R, base, f, L = 64, 10000.0, 4.0, 8192
    w = base ** (-2.0 * np.arange(R // 2) / R)
    got, gain = rz.razor_rope_frequencies(R, base)
    assert np.allclose(got, w, rtol=1e-14) and gain == 1.0
    assert np.allclose(rz.razor_rope_frequencies(R, base, "linear", f)[0], w / f, rtol=1e-14)
    ntk = rz.razor_rope_frequencies(R, base, "ntk", f)[0]
    assert ntk[0] == 1.0 and np.allclose(ntk[-1], w[-1] / f, rtol=1e-12)         # the slowest pair is stretched by the factor
    yarn, gain = rz.razor_rope_frequencies(R, base, "yarn", f, L)
    turns = L * w / (2 * np.pi)
    assert abs(gain - (0.1 * math.log(f) + 1)) < 1e-6
    # (the ramp's ends are whole pair indices)
    assert np.allclose(yarn[turns > 64], w[turns > 64], rtol=1e-12) and np.allclose(yarn[turns < 0.5], w[turns < 0.5] / f, rtol=1e-12)
    assert ((yarn <= w * (1 + 1e-12)) & (yarn >= w / f * (1 - 1e-12))).all()
    banded = rz.razor_rope_frequencies(R, base, "banded", f, L)[0]
    assert np.allclose(banded[turns >= 4], w[turns >= 4], rtol=1e-12) and np.allclose(banded[turns <= 1], w[turns <= 1] / f, rtol=1e-12)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.allclose(banded[mid], (w / f + (turns - 1) / 3 * (w - w / f))[mid], rtol=1e-12)


@pytest.mark.parametrize("args", [(3, 1e4), (0, 1e4), (258, 1e4), (64, 1.0), (64, float("nan")), (64, 1e4, "linear", 0.5),
                                  (64, 1e4, "yarn", 2.0, 0), (2, 1e4, "ntk", 2.0)])
def test_frequencies_refused(args):
    with pytest.raises(rz.RazorError) as e:
        rz.razor_rope_frequencies(*args)
    assert e.value.status == INVALID


def _rows(**kw):
    base = dict(in_=1 << 20, out=1 << 21, in_stride=(4096, 1024, 128), out_stride=(4096, 1024, 128), n_heads=8)
    base.update(kw)
    return rz.RopeRows.pack(base["in_"], base["out"], *base["in_stride"], *base["out_stride"], base["n_heads"])


def _call(rows, batch=2, tokens=4, dim=128, rotated=128, dtype=rz.RAZOR_BF16, w=None, gain=1.0, positions=None):
    w = np.ones(max(1, rotated // 2)) if w is None else w
    return rz.load().razor_rope(rows, None, positions, batch, tokens, dim, rotated, dtype,
                                w.ctypes.data if w is not False else None, gain, 0, 0, None)


def test_rope_refusals():
    assert _call(_rows(), w=False) == NULL
    assert _call(_rows(out=0)) == NULL
    assert _call(_rows(in_=(1 << 20) + 8)) == MISALIGNED
    assert _call(_rows(in_stride=(4096, 1028, 128))) == MISALIGNED
    assert _call(_rows(), positions=(1 << 20) + 2) == MISALIGNED
    for kw in (dict(batch=0), dict(tokens=-1), dict(rotated=127), dict(rotated=130), dict(rotated=0), dict(gain=float("inf")),
               dict(w=np.full(64, np.nan))):
        assert _call(_rows(), **kw) == INVALID, kw
    for kw in (dict(dim=100, rotated=32), dict(dim=264, rotated=32), dict(dtype=7)):
        assert _call(_rows(), **kw) == UNSUPPORTED, kw
    # rows of the output that meet, or an in-place call whose strides differ
    for stride in ((4096, 1024, 64), (4096, 512, 128), (1024, 1024, 128), (-4096, 1024, 128)):
        assert _call(_rows(out_stride=stride)) == INVALID, stride
    assert _call(_rows(out=1 << 20, out_stride=(8192, 1024, 128))) == INVALID
    assert _call(_rows(n_heads=-1)) == INVALID
    # nothing to do
    assert _call(_rows(), tokens=0) == 0 and _call(None) == 0 and _call(_rows(n_heads=0, in_=0, out=0)) == 0


def test_struct_matches_the_header(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ("in", "out", "in_stride_b", "in_stride_t", "in_stride_h", "out_stride_b", "out_stride_t", "out_stride_h", "n_heads")
    src = '#include <stddef.h>\n#include <stdio.h>\n#include "razor.h"\nint main(void) { printf("%d", (int)sizeof(razor_rope_rows_t)); ' + "".join(
        f'printf(" %d", (int)offsetof(razor_rope_rows_t, {n}));' for n in names) + " return 0; }"
    exe = str(tmp_path / "layout")
    subprocess.run([gcc, "-I", os.path.join(root, "include"), "-x", "c", "-", "-o", exe], input=src, text=True, check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [rz.RopeRows.size] + [8 * i for i in range(9)]
