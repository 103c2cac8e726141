"""How far a value held in 8 bits may be off: half a step, and what the quotients and products of its definition round."""
import numpy as np

from oracle import razor_oracle as orc


def test_rows_are_held_within_the_documented_bound():
    rng = np.random.default_rng(3)
    worst = 0.0
    for _ in range(20):
        top = (rng.uniform(1, 2, (2000, 1)) * 2.0 ** rng.integers(-60, 60, (2000, 1)))
        x = rng.uniform(-1, 1, (2000, 64)) * top
        x[:, :32] = (rng.integers(-127, 127, (2000, 32)) + 0.5) / 127 * top          # next to the ties between two codes
        x[:, 0] = top[:, 0]
        x = x.astype(np.float32)
        held = orc.quantise_rows(x)[2].astype(np.float64)
        top = np.abs(x).max(1, keepdims=True).astype(np.float64)
        off = np.abs(held - x) / top
        assert (off <= 1 / 254 + 2.0 ** -22).all()
        worst = max(worst, off.max())
    assert worst > 1 / 254                                                           # half a step alone would not do
