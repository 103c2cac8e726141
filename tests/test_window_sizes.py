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
