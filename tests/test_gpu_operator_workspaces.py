"""One workspace, zero-filled once, for calls of different shapes and operators, one after the other."""
import pytest
import torch

import operator_helpers as H
from paper_2502_19864_gb300 import ringada as R
from test_gpu_attention_decode import Case as Decode
from test_gpu_attention_window import Case as WindowCase
from test_gpu_verify_draft import model_like, plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def share(*cases):
    """All cases in one workspace of the largest need."""
    size = {R.ra_attention_decode_args: R.ra_attention_decode_workspace_bytes,
            R.ra_attention_window_args: R.ra_attention_window_workspace_bytes,
            R.ra_verify_draft_args: R.ra_verify_draft_workspace_bytes}
    needs = [size[type(c.a)](c.a) for c in cases]
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


class Window(WindowCase):
    def check(self):
        for t in (self.out, self.lse, self.dq, self.dk, self.dv):
            t.fill_(7.0)
        super().check()


class Verify:
    def __init__(self, dtype, B, K, V, seed=0):
        dt = H.DT[dtype]
        target, draft, tokens, uniform, noise = model_like(B, K, V, seed)
        self.target, self.draft, self.tokens = target.to(dt).cuda(), draft.to(dt).cuda(), tokens.to(torch.int32).cuda()
        self.uniform, self.noise = uniform.cuda(), noise.cuda()
        self.accepted = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.out = torch.zeros((B, K + 1), dtype=torch.int32, device="cuda")
        self.a = R.ra_verify_draft_args(
            target_dev=self.target.data_ptr(), target_stride=V, draft_dev=self.draft.data_ptr(), draft_stride=V,
            tokens_dev=self.tokens.data_ptr(), uniform_dev=self.uniform.data_ptr(), noise_dev=self.noise.data_ptr(),
            accepted_dev=self.accepted.data_ptr(), out_tokens_dev=self.out.data_ptr(), batch=B, n_draft=K, vocab=V,
            dtype=H.RA[dtype])

    def check(self):
        self.accepted.fill_(99)
        self.out.fill_(99)
        R.ra_verify_draft(self.a)
        torch.cuda.synchronize()
        K = self.out.shape[1] - 1
        for b in range(len(self.accepted)):
            n, row, apart = plain(self.target[b], self.draft[b], self.tokens[b], self.uniform[b], self.noise[b], K)
            assert apart, "the test's own candidates are too near to each other"
            assert self.accepted[b].item() == n and self.out[b].tolist() == row + [-1] * (K + 1 - len(row)), b


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_all_operators(dtype):
    """Every operator that has a workspace, after every other and again, in shapes that leave much of it in use."""
    cases = [Decode(dtype, [2000, 700, 900], 1, 8, 4, 128, 16, weights=True),
             Window(dtype, 600, [600, 599], 4, 2, 64, 100, 3),
             Verify(dtype, 40, 3, 5000),
             Window(dtype, 1500, [1500], 4, 1, 128, 60, 2),
             Decode(dtype, [300 + 31 * i for i in range(20)], 2, 8, 8, 64, 16, seed=3),
             Verify(dtype, 3, 4, 32000, seed=1)]
    share(*cases)
    for i in (0, 2, 1, 2, 1, 0, 5, 3, 5, 4, 3, 4, 5, 0, 2):
        cases[i].check()


@pytest.mark.parametrize("B", [151, 607, 609, 1300])
def test_verification_of_many_sequences_after_decode(B):
    """As many sequences as are still cut over several CTAs, and more."""
    cases = [Decode("bf16", [2000, 700, 900], 1, 8, 4, 128, 16), Verify("bf16", B, 1, 1100, seed=2)]
    share(*cases)
    for i in (0, 1, 0, 1):
        cases[i].check()
