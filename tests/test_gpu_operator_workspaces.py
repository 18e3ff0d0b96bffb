"""One workspace, zero-filled once, for calls of different shapes, one after the other."""
import pytest
import torch

import operator_helpers as H
from paper_2502_19864_gb300 import ringada as R
from test_gpu_attention_decode import Case as Decode

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def share(*cases):
    """All cases in one workspace of the largest need."""
    needs = [R.ra_attention_decode_workspace_bytes(c.a) for c in cases]
    assert min(needs) > 0
    ws = H.workspace(max(needs))
    for c in cases:
        c.ws = ws
        c.a.workspace_dev, c.a.workspace_bytes = ws.data_ptr(), ws.numel()
    return ws


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("few", [([6000], 1), ([3000], 4), ([500, 4000], 2)])
def test_decode_of_many_heads_after_few(dtype, weights, few):
    """A batch that grows and shrinks: a few (sequence, key-value head) pairs, cut over many CTAs, then 96 and 160 of
    them, most of them cut too, and the few again."""
    lens, kv = few
    cases = [Decode(dtype, lens, 1, 2 * kv, kv, 128, 16, weights=weights),
             Decode(dtype, [700 + 13 * i for i in range(24)], 1, 8, 4, 128, 16, weights=weights, seed=1),
             Decode(dtype, [900 - 7 * i for i in range(20)], 2, 8, 8, 64, 24, weights=weights, seed=2)]
    share(*cases)
    for i in (0, 1, 2, 0, 1):
        cases[i].out.fill_(7.0)
        cases[i].lse.fill_(7.0)
        cases[i].check()
