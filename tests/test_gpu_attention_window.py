"""ra_attention_window_forward and _backward against a plain implementation in 64 bits: types, head layouts, lengths
from one token on, windows and sinks at the edges of the kernels' blocks, strides, and what memory past a
sequence's end holds.  Outputs and log-sum-exps: the bounds of operator_helpers.  Gradients, with p off by dp (and by
e16 where a bf16 kernel rounds it for a product): dS = p (dP - D) is off by
  (dp + e16) |dS| + p (ddP + dD),  ddP = (d + 2) u max |dO| |v|,  dD = sum |dO| bound(o) + (d + 2) u sum |dO| |o|,
dV by (dp + n u + e16) sum p |dO| and dQ, dK by scale (sum err |k| + n u sum |dS| |k|), each with its result's own
rounding, e16 (bf16) or u.  The gradients are also tested against differences of the forward."""
import math

import pytest
import torch

import operator_helpers as H
from paper_2502_19864_gb300 import ringada as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


class Case:
    """q, k and v in one buffer, as a fused projection leaves them (fused), or apart; past a sequence's length every
    input holds NaN."""

    def __init__(self, dtype, S, lens, heads, kv, dh, window, sinks, fused=False, seed=0, poison=True, pad=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt, B = H.DT[dtype], len(lens)
        self.dtype, self.S, self.lens_list, self.heads, self.kv, self.dh, self.window, self.sinks = \
            dtype, S, lens, heads, kv, dh, window, sinks
        rand = lambda n: torch.randn((B, S, n), generator=g, device="cuda").to(dt)  # noqa: E731
        if fused:
            self.buf = rand((heads + 2 * kv) * dh)
            q, k, v = self.buf.split([heads * dh, kv * dh, kv * dh], -1)
        else:
            q, k, v = rand(heads * dh + pad)[..., :heads * dh], rand(kv * dh + pad)[..., :kv * dh], rand(kv * dh)
        q *= 2
        self.do = rand(heads * dh)
        out, dq = (torch.full((B, S, heads * dh), 7.0, dtype=dt, device="cuda") for _ in "od")
        dk, dv = (torch.full((B, S, kv * dh), 7.0, dtype=dt, device="cuda") for _ in "kv")
        if poison:
            for b, n in enumerate(lens):
                for t in (q, k, v, self.do):
                    t[b, n:] = math.nan
        self.q, self.k, self.v, self.out, self.dq, self.dk, self.dv = q, k, v, out, dq, dk, dv
        self.lse = torch.full((B, heads, S), 7.0, device="cuda")
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        ptr = {n + "_dev": getattr(self, m).data_ptr() for n, m in
               (("q", "q"), ("k", "k"), ("v", "v"), ("out", "out"), ("dout", "do"), ("dq", "dq"), ("dk", "dk"), ("dv", "dv"))}
        strides = {n + "_stride": getattr(self, m).stride(1) for n, m in
                   (("q", "q"), ("k", "k"), ("v", "v"), ("out", "out"), ("dout", "do"), ("dq", "dq"), ("dk", "dk"), ("dv", "dv"))}
        self.a = R.ra_attention_window_args(
            lse_dev=self.lse.data_ptr(), lens_dev=self.lens.data_ptr() if min(lens) < S else None, batch=B, seq=S, n_heads=heads,
            n_kv_heads=kv, head_dim=dh, window=window, sinks=sinks, dtype=H.RA[dtype], scale=dh ** -0.5,
            err_dev=self.err.data_ptr(), **ptr, **strides)
        self.ws = H.workspace(R.ra_attention_window_workspace_bytes(self.a))
        self.a.workspace_dev, self.a.workspace_bytes = self.ws.data_ptr(), self.ws.numel()

    def run(self, stream=None, backward=True):
        R.ra_attention_window_forward(self.a, stream)
        if backward:
            R.ra_attention_window_backward(self.a, stream)
        torch.cuda.synchronize()
        assert self.err.item() == 0

    def check(self, backward=True):
        self.run(backward=backward)
        d, scale, e16 = self.dh, self.dh ** -0.5, H.E if self.dtype == "bf16" else 0.0
        group = self.heads // self.kv
        head = lambda t, b, h, n: t[b, :n, h * d:(h + 1) * d].double()  # noqa: E731

        def near(got, ref, bound, what):
            off = ((got.double() - ref).abs() / bound)
            assert (off <= 1).all(), (what, float(off.max()))

        for b, n in enumerate(self.lens_list):
            at = torch.arange(n, device="cuda")
            mask = H.seen(at, at, self.window, self.sinks)
            for t in (self.out,) + ((self.dq, self.dk, self.dv) if backward else ()):
                assert (t[b, n:] == 0).all()
            assert torch.isneginf(self.lse[b, :, n:]).all()
            if n == 0:
                continue
            for e in range(self.kv):
                k, v = head(self.k, b, e, n), head(self.v, b, e, n)
                dk, dv, dk_b, dv_b = (torch.zeros_like(k) for _ in range(4))
                for h in range(e * group, (e + 1) * group):
                    q, do = head(self.q, b, h, n), head(self.do, b, h, n)
                    o, lse, p, bound, dp = H.attention64(q, k, v, mask, scale, self.dtype)
                    near(head(self.out, b, h, n), o, bound, ("out", b, h))
                    near(self.lse[b, h, :n], lse, dp + 4 * H.U * lse.abs() + 1e-7, ("lse", b, h))
                    if not backward:
                        continue
                    ds_ = p * (do @ v.T - (do * o).sum(-1, keepdim=True))
                    ddp = (d + 2) * H.U * float((do.abs() @ v.abs().T).max())
                    dD = (do.abs() * bound).sum(-1, keepdim=True) + (d + 2) * H.U * (do * o).abs().sum(-1, keepdim=True)
                    err = (dp + e16) * ds_.abs() + p * (ddp + dD)
                    dq = scale * ds_ @ k
                    dq_b = scale * (err @ k.abs() + n * H.U * ds_.abs() @ k.abs()) + (e16 + H.U) * dq.abs() + 1e-30
                    near(head(self.dq, b, h, n), dq, dq_b, ("dq", b, h))
                    m = group * n
                    dk += scale * ds_.T @ q
                    dk_b += scale * (err.T @ q.abs() + m * H.U * ds_.abs().T @ q.abs())
                    dv += p.T @ do
                    dv_b += (dp + m * H.U + e16) * (p.T @ do.abs())
                if backward:
                    near(head(self.dk, b, e, n), dk, dk_b + (e16 + H.U) * dk.abs() + 1e-30, ("dk", b, e))
                    near(head(self.dv, b, e, n), dv, dv_b + (e16 + H.U) * dv.abs() + 1e-30, ("dv", b, e))


DIMS = [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)]


@pytest.mark.parametrize("dtype,dh", DIMS)
@pytest.mark.parametrize("S", [1, 2, 63, 64, 65, 127, 128, 129, 255, 257, 300, 520])
def test_lengths(dtype, dh, S):
    Case(dtype, S, [S], 2, 2, dh, 100, 3).check()


@pytest.mark.parametrize("dtype,dh", DIMS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (2, 0), (64, 0), (65, 64), (127, 1), (128, 0), (129, 129),
                                          (200, 400), (256, 4), (300, 256), (4000, 4), (20, 2000)])
def test_windows(dtype, dh, window, sinks):
    Case(dtype, 600, [600, 599], 2, 1, dh, window, sinks).check()


@pytest.mark.parametrize("dtype,dh", DIMS + [("f32", 4), ("f32", 20), ("f32", 32), ("f32", 96), ("f32", 100)])
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (4, 2), (8, 1), (6, 2)])
def test_heads(dtype, dh, heads, kv):
    Case(dtype, 200, [200, 77], heads, kv, dh, 90, 5).check()


@pytest.mark.parametrize("dtype,dh", DIMS)
@pytest.mark.parametrize("fused", [False, True])
def test_ragged_batches_and_strides(dtype, dh, fused):
    """Sequences of no token, of one, and ends on either side of the blocks; NaN past every end."""
    Case(dtype, 400, [400, 0, 1, 128, 129, 127, 64, 256, 257, 399], 4, 2, dh, 130, 2, fused=fused, pad=24).check()


@pytest.mark.parametrize("dtype,dh", DIMS)
def test_many_blocks(dtype, dh):
    Case(dtype, 2100, [2100, 1500], 4, 2, dh, 300, 140).check()


@pytest.mark.parametrize("dtype,dh", DIMS)
def test_again_and_on_another_stream(dtype, dh):
    case = Case(dtype, 700, [700, 311], 4, 2, dh, 200, 4)
    case.run()
    first = [t.clone() for t in (case.out, case.lse, case.dq, case.dk, case.dv)]
    for t in (case.out, case.lse, case.dq, case.dk, case.dv):
        t.fill_(3.0)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    case.run(stream)
    for x, y in zip(first, (case.out, case.lse, case.dq, case.dk, case.dv)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,dh", DIMS)
def test_forward_alone(dtype, dh):
    case = Case(dtype, 300, [300, 100], 2, 2, dh, 50, 1)
    case.check(backward=False)
    out = case.out.clone()
    case.a.lse_dev = None
    case.run(backward=False)
    assert torch.equal(case.out, out)


@pytest.mark.parametrize("dtype,dh", DIMS)
def test_large_scores(dtype, dh):
    """Scores of hundreds, of either sign: the running maximum moves far."""
    case = Case(dtype, 500, [500], 2, 2, dh, 0, 0, poison=False)
    ramp = torch.linspace(-30, 30, 500, device="cuda")[None, :, None].to(case.q.dtype)
    case.k.mul_(ramp)
    case.check()


@pytest.mark.parametrize("dh", [64, 96])
def test_against_differences(dh):
    """(L(x + t r) - L(x - t r)) / 2 t of L = sum out dout along random directions r: the third-order term and the
    forward's rounding over t are both below 1e-3 of |grad| |r| at t = 1e-2."""
    case = Case("f32", 150, [150, 90], 4, 2, dh, 40, 3, poison=False)
    live = (torch.arange(150, device="cuda") < case.lens[:, None])[..., None]
    case.run()
    grads = {n: getattr(case, "d" + n).double().clone() for n in "qkv"}
    g = torch.Generator(device="cuda").manual_seed(5)
    loss = lambda: float((case.out.double() * case.do.double() * live).sum())  # noqa: E731
    for name in "qkv":
        x = getattr(case, name)
        base = x.clone()
        r = torch.randn(x.shape, generator=g, device="cuda")
        sides = []
        for t in (1e-2, -1e-2):
            x.copy_(base + t * r)
            case.run(backward=False)
            sides.append(loss())
        x.copy_(base)
        got = (sides[0] - sides[1]) / 2e-2
        want = float((grads[name] * r.double()).sum())
        assert abs(got - want) <= 1e-3 * float(grads[name].norm() * r.double().norm()), (name, got, want)


def test_lengths_out_of_range_are_reported():
    case = Case("f32", 100, [100, 60], 2, 2, 64, 30, 1)
    case.lens.copy_(torch.tensor([-4, 1000], dtype=torch.int32))
    R.ra_attention_window_forward(case.a)
    torch.cuda.synchronize()
    assert case.err.item() == R.RA_DEV_BOUNDS and (case.out[0] == 0).all()


@pytest.mark.parametrize("dtype,dh", DIMS)
@pytest.mark.parametrize("kv", [4, 2, 1])
def test_more_blocks_than_the_gpu_holds(dtype, dh, kv):
    """Several blocks a CTA, one after the other, among them blocks of sequences that have ended."""
    lens = [(7 * i * i + 13 * i) % 301 for i in range(36)] + [0, 0, 300, 1]
    Case(dtype, 300, lens, 4, kv, dh, 70, 2).check()


@pytest.mark.parametrize("dtype,dh", DIMS)
@pytest.mark.parametrize("sinks", [3, 200])
def test_long_with_few_sinks(dtype, dh, sinks):
    """The first keys are seen from 40 blocks of queries, the others from two or three."""
    Case(dtype, 5000, [5000], 2, 1, dh, 100, sinks).check()


@pytest.mark.parametrize("dtype,dh", DIMS)
def test_lengths_out_of_range_in_the_backward(dtype, dh):
    case = Case(dtype, 200, [200, 60], 2, 2, dh, 30, 1, poison=False)
    case.lens.copy_(torch.tensor([-4, 1000], dtype=torch.int32))
    R.ra_attention_window_forward(case.a)
    R.ra_attention_window_backward(case.a)
    torch.cuda.synchronize()
    assert case.err.item() == R.RA_DEV_BOUNDS
    for t in (case.out, case.dq, case.dk, case.dv):
        assert (t[0] == 0).all() and torch.isfinite(t[1].float()).all() and (t[1] != 7).any()


@pytest.mark.parametrize("dtype,dh", DIMS + [("f32", 20)])
@pytest.mark.parametrize("what", ["query", "key", "value", "infinite query", "infinite value"])
def test_not_finite(dtype, dh, what):
    """A query, or a key or value that is seen, that is not finite: NaN in the rows that see it (infinite where the formula
    says so), in the log-sum-exp as in the output, and never the log-sum-exp of a row that sees nothing.  Rows of other
    sequences, and what came before, are as they are without it."""
    S, at = 300, 140
    case, clean = (Case(dtype, S, [S, 200], 2, 2, dh, 100, 3, poison=False) for _ in "ab")
    clean.run(backward=False)
    x = {"query": case.q, "infinite query": case.q, "key": case.k, "value": case.v, "infinite value": case.v}[what]
    bad = math.inf if "infinite" in what else math.nan
    x[0, at, dh + 3] = bad  # of head 1
    case.run(backward=False)
    rows = [at] if "query" in what else list(range(at, at + 100))  # that see it
    out, lse = case.out[0, :, dh:2 * dh].float(), case.lse[0, 1]
    if "value" in what:
        assert (out[rows, 3].isnan() | out[rows, 3].isinf()).all()
        assert torch.equal(lse, clean.lse[0, 1])
    elif what == "infinite query":  # products of either sign: +-inf, and inf - inf
        assert out[rows].isnan().all() and not lse[rows].isneginf().any() and not lse[rows].isfinite().any()
    else:
        assert out[rows].isnan().all() and lse[rows].isnan().all()
    before = slice(0, at - at % 128)  # (blocks of keys that it is not in)
    for t, c in ((case.out, clean.out), (case.lse[:, :, None, :], clean.lse[:, :, None, :])):
        assert torch.equal(t[1], c[1])
    assert torch.equal(case.out[0, before], clean.out[0, before]) and torch.equal(case.out[0, :, :dh], clean.out[0, :, :dh])
    assert torch.equal(case.lse[0, 0], clean.lse[0, 0]) and torch.equal(case.lse[0, 1, before], clean.lse[0, 1, before])


@pytest.mark.parametrize("dtype,dh", DIMS)
def test_every_key_not_finite(dtype, dh):
    """All scores NaN from the first block on: NaN, not the zero and -inf of a row that sees nothing; gradients are NaN too."""
    case = Case(dtype, 200, [200, 150], 2, 1, dh, 0, 0, poison=False)
    case.k[0] = math.nan
    case.run()
    assert case.out[0].isnan().all() and case.lse[0].isnan().all()
    for t in (case.dq, case.dk):
        assert t[0].isnan().all()
    assert case.out[1, :150].isfinite().all() and case.lse[1, :, :150].isfinite().all()
    for t in (case.dq, case.dk, case.dv):
        assert t[1].isfinite().all()
