"""Sizes of the prompt attention's workspace: no wrapped products, and what serves every call."""
import itertools

import pytest

from paper_2407_15891_b200 import binding as rz
from paper_2407_15891_b200 import build as rz_build

BIG = 2 ** 31 - 1


@pytest.fixture(scope="module", autouse=True)
def _built():
    rz_build.build()


@pytest.mark.parametrize("batch,heads,tokens", [(BIG, BIG, 1024), (BIG, BIG, 1000), (BIG, BIG, 1 << 30), (BIG, 1 << 30, 512), (1 << 30, 2, 1),
                                                (1, BIG, 1), (BIG, 1, 1)])
def test_more_work_than_can_be_numbered_is_refused(batch, heads, tokens):
    with pytest.raises(rz.RazorError) as e:
        rz.razor_window_attention_workspace_bytes(batch, heads, heads, 128, tokens)
    assert e.value.status == -5


@pytest.mark.parametrize("D,size", [(64, 21635328), (128, 42607872)])
def test_the_size_that_serves_any_call(D, size):
    needs = [rz.razor_window_attention_workspace_bytes(B, Hk * G, Hk, D, T)
             for B, Hk, G, T in itertools.product((1, 2, 3, 64, 128, 1024, 1025), (1, 2, 8, 1024), (1, 3, 8, 64, 128),
                                                  (0, 1, 2, 3, 100, 127, 128, 129, 256, 4096, 1 << 18, 1 << 20))
             if B * Hk * (T * G // 128 + 1) < 1 << 29]
    # (the table of up to 1024 units, then two records of up to 256 rows for each of 160 spans)
    assert max(needs) <= size and size - max(needs) < 8192
