"""ra_attention_decode against a plain implementation in 64 bits: types, head layouts, lengths from none to many,
pages of odd sizes, windows and sinks, drafted tokens, accumulated weights, what unused memory holds, and the
indices that the kernel has to refuse.  Bounds: operator_helpers."""
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
    """A cache whose unused slots and pages hold NaN, and the call on it."""

    def __init__(self, dtype, lens, new, heads, kv, dh, page, window=0, sinks=0, weights=False, seed=0, extra=3,
                 q_pad=0, n_pages=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt = H.DT[dtype]
        rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
        B, per = len(lens), max(1, -(-max(lens) // page))
        n_pages = n_pages or B * per + extra
        self.args = dict(dtype=dtype, new=new, heads=heads, kv=kv, dh=dh, page=page, window=window, sinks=sinks)
        self.lens_list = lens
        self.k = torch.full((n_pages, kv, page, dh), math.nan, dtype=dt, device="cuda")
        self.v = self.k.clone()
        order = torch.randperm(n_pages, generator=g, device="cuda") if n_pages < 1 << 19 else torch.arange(n_pages - 1, -1, -1, device="cuda")
        self.table = order[:B * per].to(torch.int32).view(B, per).contiguous()
        for b, n in enumerate(lens):
            at = torch.arange(n, device="cuda")
            where = self.table[b].long()[at // page]
            self.k[where, :, at % page] = rand(n, kv, dh)
            self.v[where, :, at % page] = rand(n, kv, dh)
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        row = heads * dh + q_pad
        self.q_buf = rand(B * new, row) * 2
        self.q = self.q_buf[:, :heads * dh].view(B, new, heads, dh)
        self.out = torch.full((B * new, row), 7.0, dtype=dt, device="cuda")
        self.lse = torch.full((B, new, heads), 7.0, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.a = R.ra_attention_decode_args(
            cache=H.cache(self.k, self.v, self.table, self.err), lens_dev=self.lens.data_ptr(),
            q_dev=self.q_buf.data_ptr(), q_stride=row, out_dev=self.out.data_ptr(), out_stride=row,
            lse_dev=self.lse.data_ptr(), batch=B, n_new=new, n_heads=heads, window=window, sinks=sinks,
            scale=dh ** -0.5)
        self.w_in = self.w_out = None
        if weights:
            n = per * page + 5
            self.w_in = torch.rand((B, kv, n), generator=g, device="cuda")
            self.w_out = torch.full((B, kv, n), 7.0, device="cuda")
            self.a.weights_in_dev, self.a.weights_out_dev = self.w_in.data_ptr(), self.w_out.data_ptr()
            self.a.weights_stride = n
        self.ws = H.workspace(R.ra_attention_decode_workspace_bytes(self.a))
        self.a.workspace_dev, self.a.workspace_bytes = self.ws.data_ptr(), self.ws.numel()

    def run(self, stream=None):
        R.ra_attention_decode(self.a, stream)
        torch.cuda.synchronize()
        return self.out[:, :self.args["heads"] * self.args["dh"]].reshape(self.q.shape)

    def check(self, absent=()):
        """`absent`: {(sequence, page of its table)} that are not there."""
        c = self.args
        out = self.run()
        group = c["heads"] // c["kv"]
        for b, n in enumerate(self.lens_list):
            k, v = H.slots(self.k, self.table.clamp(min=0, max=self.k.shape[0] - 1), b, n), H.slots(
                self.v, self.table.clamp(min=0, max=self.k.shape[0] - 1), b, n)
            query = n - c["new"] + torch.arange(c["new"], device="cuda")
            mask = H.seen(query, torch.arange(n, device="cuda"), c["window"], c["sinks"])
            for bb, page in absent:
                if bb == b:
                    mask[:, page * c["page"]:(page + 1) * c["page"]] = False
                    k, v = k.clone(), v.clone()
                    k[:, page * c["page"]:(page + 1) * c["page"]] = 0
                    v[:, page * c["page"]:(page + 1) * c["page"]] = 0
            total = torch.zeros((c["kv"], n), dtype=torch.float64, device="cuda")
            slack = 0.0
            for h in range(c["heads"]):
                e = h // group
                ref, lse, p, bound, dp = H.attention64(self.q[b, :, h], k[e], v[e], mask, c["dh"] ** -0.5, c["dtype"], H.E / 2)
                assert ((out[b, :, h].double() - ref).abs() <= bound).all(), (b, n, h, float(((out[b, :, h].double() - ref).abs() / bound).max()))
                assert torch.equal(torch.isneginf(self.lse[b, :, h]), torch.isneginf(lse)), (b, h)
                fin = torch.isfinite(lse)
                assert ((self.lse[b, :, h].double() - lse).abs()[fin] <= dp + 4 * H.U * lse.abs()[fin] + 1e-7).all(), (b, h)
                total[e] += p.sum(0)
                slack = max(slack, dp)
            if self.w_out is not None:
                want = self.w_in[b, :, :n].double() + total
                off = (self.w_out[b, :, :n].double() - want).abs()
                # every row's weight is off by dp of itself, and their sum by its roundings
                assert (off <= slack * total + (c["heads"] * c["new"] + 2) * H.U * want + 1e-30).all(), (b, float(off.max()))
                assert (self.w_out[b, :, n:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dh", [(2, 2, 64), (16, 4, 128), (8, 1, 128), (16, 16, 128), (4, 2, 96), (3, 3, 32),
                                         (4, 2, 256), (6, 2, 40), (2, 1, 8), (24, 1, 200)])
def test_heads(dtype, heads, kv, dh):
    Case(dtype, [300, 0, 1, 63, 64, 65, 17], 1, heads, kv, dh, 16, weights=True).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 7, 16, 24, 64, 100, 256])
def test_pages(dtype, page):
    Case(dtype, [129, 1, 500, 31], 1, 4, 2, 64, page).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,heads,kv", [(2, 4, 4), (5, 12, 6), (8, 16, 4), (8, 8, 1), (9, 16, 2), (3, 64, 1), (16, 16, 1)])
def test_drafted_tokens(dtype, new, heads, kv):
    """Several queries a sequence; sequences shorter than the drafts have queries that are not there."""
    Case(dtype, [200, new, 1, 0, new - 1, 1000], new, heads, kv, 64, 16, weights=True).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (63, 0), (64, 64), (100, 130), (500, 4), (5000, 2)])
@pytest.mark.parametrize("new", [1, 5])
def test_window_and_sinks(dtype, window, sinks, new):
    Case(dtype, [1000, 70, 5, 0, 333], new, 8, 4, 128, 24, window, sinks, weights=True).check()


@pytest.mark.parametrize("dtype,lens,heads,kv,dh", [("bf16", [40000, 3, 12345], 16, 2, 128), ("f32", [20000, 7777], 4, 2, 64),
                                                    ("bf16", [70001], 16, 1, 64)])
def test_long(dtype, lens, heads, kv, dh):
    """Sequences that many CTAs share, beside short ones."""
    Case(dtype, lens, 1, heads, kv, dh, 16, weights=True).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(dtype):
    """More sequences than one warp counts at a time, none of them long; empty ones among them."""
    lens = [(37 * i) % 90 for i in range(150)]
    Case(dtype, lens, 1, 4, 2, 64, 16, weights=True).check()
    Case(dtype, [0] * 40 + [5] + [0] * 50, 1, 4, 2, 64, 16).check()
    Case(dtype, [0, 0, 0], 2, 4, 2, 64, 16, weights=True).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype):
    Case(dtype, [77, 300], 3, 4, 2, 64, 16, q_pad=48).check()


def test_far_pages():
    """Values more than 2^31 elements into the pools."""
    n_pages = (1 << 31) // (2 * 16 * 128) + 40
    case = Case("bf16", [300, 100], 1, 4, 2, 128, 16, n_pages=n_pages)
    assert int(case.table.max()) * 2 * 16 * 128 > 1 << 31
    case.check()


def test_in_place_weights_and_none():
    case = Case("bf16", [100, 64, 3], 1, 4, 2, 64, 16, weights=True)
    case.run()
    apart = case.w_out.clone()
    case.a.weights_out_dev = case.w_in.data_ptr()
    case.run()
    for b, n in enumerate(case.lens_list):
        assert torch.equal(case.w_in[b, :, :n], apart[b, :, :n])
    case.a.weights_in_dev = None
    case.run()
    for b, n in enumerate(case.lens_list):
        # one token's weights alone: each head's softmax sums to one
        assert torch.allclose(case.w_in[b, :, :n].sum(-1), torch.full((2,), 2.0, device="cuda"), rtol=0, atol=2e-6 * 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_again_and_on_another_stream(dtype):
    """The same bits again, in a workspace that other shapes have used, and on a stream of its own."""
    case = Case(dtype, [3000, 17, 900], 2, 8, 2, 128, 16, 256, 4, weights=True)
    first, w = case.run().clone(), case.w_out.clone()
    other = Case(dtype, [50], 1, 2, 2, 64, 16)
    other.a.workspace_dev, other.a.workspace_bytes = case.ws.data_ptr(), case.ws.numel()
    if R.ra_attention_decode_workspace_bytes(other.a) <= case.ws.numel():
        other.check()
    stream = torch.cuda.Stream()
    case.out.fill_(3.0)
    torch.cuda.synchronize()
    assert torch.equal(case.run(stream), first) and torch.equal(case.w_out, w)


def test_graph_with_growing_lengths():
    """Captured once, replayed as the lengths on the device grow."""
    case = Case("bf16", [40, 90, 700], 1, 4, 2, 64, 16, weights=True)
    case.run()
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        R.ra_attention_decode(case.a, stream)
    for shorter in ([1, 90, 300], [40, 0, 650], [40, 90, 700]):
        # (slots past a shorter length hold other tokens, which no query may see)
        case.lens.copy_(torch.tensor(shorter, dtype=torch.int32))
        case.lens_list = shorter
        case.w_out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        again = case.out.clone()
        w = case.w_out.clone()
        case.check()
        assert torch.equal(again, case.out) and torch.equal(w, case.w_out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_indices_are_reported_and_not_followed(dtype):
    case = Case(dtype, [200, 90], 1, 4, 2, 64, 16)
    case.check()
    assert case.err.item() == 0
    case.table[0, 3] = 1 << 30
    case.table[1, 0] = -5
    case.check(absent=[(0, 3), (1, 0)])
    assert case.err.item() == R.RA_DEV_BOUNDS
    case = Case(dtype, [64, 32], 1, 4, 2, 64, 16)
    case.lens.copy_(torch.tensor([1 << 30, -3], dtype=torch.int32))
    case.lens_list = [64, 0]  # the table's capacity, and nothing
    case.check()
    assert case.err.item() == R.RA_DEV_BOUNDS


def test_infinite_scores_and_lowest_values():
    """Keys so small that all scores are the type's lowest finite values still share the weight."""
    case = Case("f32", [40], 1, 2, 2, 64, 16)
    case.k.nan_to_num_(nan=0.0)
    case.k.fill_(1e18)
    case.q_buf.fill_(-1e18)
    out = case.run()
    want = H.slots(case.v, case.table, 0, 40).double().mean(1)
    assert torch.allclose(out[0, 0].double(), want, rtol=0, atol=1e-5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[700, 90], [40, 20000]])
def test_not_finite(dtype, lens):
    """A NaN query, key or value: NaN in what sees it, output and log-sum-exp (a value: the output alone), through the parts
    of long sequences too; other heads and sequences are as they are without it."""
    for what in ("q", "k", "v"):
        case, clean = (Case(dtype, lens, 1, 4, 2, 64, 16, weights=True) for _ in "ab")
        clean.run()
        for c in (case, clean):
            c.w_out[:] = 0
        clean.run()
        if what == "q":
            case.q[0, 0, 3, 5] = math.nan
            hit = (3,)
        else:
            slot = lens[0] // 2
            getattr(case, what)[case.table[0].long()[slot // 16], 1, slot % 16, 5] = math.nan
            hit = (2, 3)
        out = case.run()
        want = clean.out[:, :256].reshape(out.shape)
        for h in range(4):
            if h not in hit:
                assert torch.equal(out[0, :, h], want[0, :, h]) and torch.equal(case.lse[0, :, h], clean.lse[0, :, h])
            elif what == "v":
                assert out[0, :, h, 5].isnan().all() and torch.equal(case.lse[0, :, h], clean.lse[0, :, h])
            else:
                assert out[0, :, h].isnan().all() and case.lse[0, :, h].isnan().all()
        assert torch.equal(out[1], want[1]) and torch.equal(case.lse[1], clean.lse[1]) and torch.equal(case.w_out[1], clean.w_out[1])
        if what != "v":
            assert case.w_out[0, 1, :lens[0]].isnan().all()
        assert torch.equal(case.w_out[0, 0], clean.w_out[0, 0])
