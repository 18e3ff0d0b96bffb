"""LayerNorm and RMSNorm with a residual's sum, and their gradients, against 64 bits and against differences.

Bounds, element by element.  u = 2^-24, e = 2^-8 (bf16's rounding; 0 in fp32).  A sum over a row is at most 32 values in turn in
a thread, ten halvings of threads and a few joins: off by c u times the sum of magnitudes, c = 48.  A deviation d = z - mean has the
roundings of z and of the mean (the forward takes the latter out again, the backward reads it rounded) and the
mean's error: dd = 2 u (|z| + |mean|) + c u mean|d|.  rstd is off by r = c u + 2 mean(|d| dd) rstd^2 of itself, the unit row
n = d rstd by dn = dd rstd + (r + 2 u)|n|."""
import pytest
import torch

from paper_2502_19864_gb300 import ringada as R
from tests.operator_helpers import DT, E, RA, U, workspace

pytestmark = pytest.mark.gpu
CU = 48 * U
KIND = {"layer": R.RA_NORM_LAYER, "rms": R.RA_NORM_RMS}


def make(rows, hidden, kind, dtype, wdtype, residual, seed=0, pad=0, gamma=True, beta=True, offset=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = hidden + pad

    def rows_of(scale, shift=0.0):
        return torch.randn(rows, wide, generator=g, device="cuda").mul_(scale).add_(shift).to(DT[dtype])[:, :hidden]
    s = {"x": rows_of(1.5, offset), "dy": rows_of(1.0), "dsum": rows_of(0.5)}
    if residual:
        s["residual"] = rows_of(1.0)
    w = lambda shift: torch.randn(hidden, generator=g, device="cuda").mul_(0.3).add_(shift).to(DT[wdtype])  # noqa: E731
    s["gamma"] = w(1.0) if gamma else None
    s["beta"] = w(0.0) if beta and kind == "layer" else None
    for n in ("y", "sum", "dx"):
        s[n] = torch.full((rows, wide), 7.0, device="cuda", dtype=DT[dtype])[:, :hidden]
    s["stats"] = torch.full((2, max(rows, 1)), 7.0, device="cuda")
    s["dgamma"], s["dbeta"] = (torch.full((hidden,), 7.0, device="cuda", dtype=DT[wdtype]) for _ in "gb")
    at = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    a = R.ra_norm_args(x_dev=at(s["x"]), x_stride=wide, gamma_dev=at(s["gamma"]), beta_dev=at(s["beta"]), y_dev=at(s["y"]),
                       y_stride=wide, mean_dev=at(s["stats"][0]), rstd_dev=at(s["stats"][1]), dy_dev=at(s["dy"]), dy_stride=wide,
                       dx_dev=at(s["dx"]), dx_stride=wide, dgamma_dev=at(s["dgamma"]), rows=rows, hidden=hidden,
                       kind=KIND[kind], dtype=RA[dtype], w_dtype=RA[wdtype], eps=1e-5)
    if kind == "layer":
        a.dbeta_dev = at(s["dbeta"])
    if residual:
        a.residual_dev, a.residual_stride, a.sum_dev, a.sum_stride = at(s["residual"]), wide, at(s["sum"]), wide
        a.dsum_dev, a.dsum_stride = at(s["dsum"]), wide
    n = R.ra_norm_workspace_bytes(a)
    assert n > 0
    s["workspace"] = workspace(n)
    a.workspace_dev, a.workspace_bytes = at(s["workspace"]), n
    return a, s


def near(got, want, bound, what):
    off = (got.double() - want).abs()
    assert bool((off <= bound + 1e-37).all()), (what, float((off / (bound + 1e-37)).max()))


def check(a, s, kind, dtype, wdtype, residual, eps=1e-5):
    e, we = (E if dtype == "bf16" else 0.0), (E if wdtype == "bf16" else 0.0)
    z = s["x"].double() + (s["residual"].double() if residual else 0.0)
    one = z.new_ones(z.shape[1])
    gamma = s["gamma"].double() if s["gamma"] is not None else one
    beta = s["beta"].double() if s["beta"] is not None else one * 0

    def unit(z):
        mean = z.mean(1, keepdim=True) if kind == "layer" else z.new_zeros(z.shape[0], 1)
        d = z - mean
        rstd = (d.square().mean(1, keepdim=True) + eps).rsqrt()
        dd = 2 * U * (z.abs() + mean.abs()) + CU * d.abs().mean(1, keepdim=True)
        r = CU + 2 * (d.abs() * dd).mean(1, keepdim=True) * rstd * rstd
        n = d * rstd
        return mean, rstd, n, dd * rstd + (r + 2 * U) * n.abs(), r
    mean, rstd, n, dn, r = unit(z)
    y = n * gamma + beta
    near(s["y"], y, gamma.abs() * dn + 3 * U * (gamma * n).abs() + U * beta.abs() + (e + U) * y.abs(), "y")
    near(s["stats"][1], rstd[:, 0], ((r + 2 * U) * rstd)[:, 0], "rstd")
    if kind == "layer":
        near(s["stats"][0], mean[:, 0], (CU * z.abs().mean(1) + U * mean[:, 0].abs()), "mean")
    if residual:
        near(s["sum"], z, (e + 2 * U) * z.abs(), "sum")
        kept = s["sum"].double()
        n = (kept - mean) * rstd
        dn = dn + 2 * U * kept.abs() * rstd
    rows = z.shape[0]
    dy = s["dy"].double()
    g = dy * gamma
    mg = g.mean(1, keepdim=True) if kind == "layer" else 0.0 * g[:, :1]
    mgn = (g * n).mean(1, keepdim=True)
    dx = (g - mg - n * mgn) * rstd
    bound = rstd * (4 * U * (g.abs() + mg.abs() + (n * mgn).abs()) + CU * g.abs().mean(1, keepdim=True) + dn * mgn.abs()
                    + n.abs() * ((g.abs() * dn).mean(1, keepdim=True) + CU * (g * n).abs().mean(1, keepdim=True)))
    bound = bound + (r + 2 * U) * dx.abs()
    if residual:
        dx = dx + s["dsum"].double()
    near(s["dx"], dx, bound + (e + U) * dx.abs(), "dx")
    sums = (rows // 608 + 60) * U  # a CTA's rows in turn, then the CTAs
    want = (dy * n).sum(0)
    near(s["dgamma"], want, (dy.abs() * dn).sum(0) + sums * (dy * n).abs().sum(0) + (we + U) * want.abs(), "dgamma")
    if kind == "layer":
        want = dy.sum(0)
        near(s["dbeta"], want, sums * dy.abs().sum(0) + (we + U) * want.abs(), "dbeta")


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("kind,residual", [("layer", False), ("layer", True), ("rms", False), ("rms", True)])
@pytest.mark.parametrize("rows,hidden", [(1, 1), (3, 7), (5, 64), (2, 100), (700, 128), (333, 771), (9, 2048), (1300, 1024), (3, 8200), (2, 20000), (2, 32768), (1, 32767)])
def test_against_64_bits(rows, hidden, kind, residual, dtype, wdtype):
    a, s = make(rows, hidden, kind, dtype, wdtype, residual, seed=rows + hidden)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    check(a, s, kind, dtype, wdtype, residual)


@pytest.mark.parametrize("pad", [1, 8, 24])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype, pad):
    a, s = make(37, 264, "layer", dtype, "f32", True, pad=pad)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    check(a, s, "layer", dtype, "f32", True)
    for n in ("y", "sum", "dx"):  # what lies between rows is left as it was
        whole = torch.as_strided(s[n], (36, pad), (264 + pad, 1), s[n].storage_offset() + 264)
        assert bool((whole == 7.0).all())


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("kind,residual", [("layer", False), ("rms", True)])
@pytest.mark.parametrize("rows,hidden,pad", [(70, 386, 0), (2501, 386, 0), (2501, 1340, 0), (2501, 392, 2), (2501, 392, 4), (2501, 77, 0),
                                             (2501, 2302, 0), (2501, 2300, 4), (2501, 2299, 0), (70, 8198, 0)])
def test_accesses_of_each_width(rows, hidden, pad, kind, residual, dtype, wdtype):
    a, s = make(rows, hidden, kind, dtype, wdtype, residual, seed=rows + hidden, pad=pad)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    check(a, s, kind, dtype, wdtype, residual)
    if pad:
        for n in ("y", "dx") + (("sum",) if residual else ()):
            assert bool((torch.as_strided(s[n], (rows - 1, pad), (hidden + pad, 1), s[n].storage_offset() + hidden) == 7.0).all()), n


def test_a_place_that_is_not_aligned():
    a, s = make(20, 256, "layer", "bf16", "bf16", False)
    buf = torch.zeros(20 * 256 + 1, dtype=torch.bfloat16, device="cuda")
    x = buf[1:].view(20, 256)
    x.copy_(s["x"])
    s["x"], a.x_dev = x, x.data_ptr()
    assert a.x_dev % 16
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    check(a, s, "layer", "bf16", "bf16", False)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_without_weights(kind):
    a, s = make(50, 320, kind, "bf16", "f32", False, gamma=False, beta=False)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    check(a, s, kind, "bf16", "f32", False)


def test_rows_far_from_zero_keep_their_digits():
    a, s = make(64, 1000, "layer", "f32", "f32", False, offset=3000.0)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    check(a, s, "layer", "f32", "f32", False)


def test_equal_values_and_zeros():
    for kind in ("layer", "rms"):
        a, s = make(4, 96, kind, "f32", "f32", False, beta=False)
        s["x"][:2] = 3.25
        s["x"][2:] = 0.0
        R.ra_norm_forward(a)
        R.ra_norm_backward(a)
        torch.cuda.synchronize()
        check(a, s, kind, "f32", "f32", False)


def test_a_row_that_is_not_finite_stays_by_itself():
    a, s = make(6, 200, "layer", "bf16", "bf16", True)
    s["x"][2, 5], s["x"][4, 0] = float("nan"), float("inf")
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    bad = [2, 4]
    ok = [0, 1, 3, 5]
    assert bool(s["y"][bad].isnan().all()) and bool(s["dx"][bad].isnan().all())
    assert bool(s["y"][ok].isfinite().all()) and bool(s["dx"][ok].isfinite().all())


@pytest.mark.parametrize("hidden", [256, 771])
def test_in_place(hidden):
    a, s = make(40, hidden, "rms", "bf16", "bf16", True)
    b, t = make(40, hidden, "rms", "bf16", "bf16", True)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    b.sum_dev, t["sum"] = b.residual_dev, t["residual"]  # the residual stream in its own place
    b.y_dev, t["y"] = b.x_dev, t["x"]
    R.ra_norm_forward(b)
    b.dx_dev, t["dx"] = b.dsum_dev, t["dsum"]
    R.ra_norm_backward(b)
    torch.cuda.synchronize()
    for n in ("y", "sum", "dx", "dgamma"):
        assert torch.equal(s[n], t[n]), n


def test_parts_of_the_backward():
    a, s = make(100, 512, "layer", "bf16", "f32", False)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    want = {n: s[n].clone() for n in ("dx", "dgamma", "dbeta")}
    for keep in want:
        for n in want:
            s[n].fill_(7.0)
            setattr(a, n + "_dev", s[n].data_ptr() if n == keep else None)
        R.ra_norm_backward(a)
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(s[n], want[n]) if n == keep else bool((s[n] == 7.0).all()), (keep, n)


def test_no_rows():
    a, s = make(0, 64, "layer", "bf16", "bf16", False)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    assert bool((s["dgamma"] == 0).all()) and bool((s["dbeta"] == 0).all())


def test_against_differences():
    """The loss sum(y c + sum c2) by steps of 2^-7 in a few values of x, gamma and beta: the difference of two steps is off by
    the third derivative's part, h^2 / 6 |f'''|, which five points along a line bound, and by the loss's rounding."""
    a, s = make(3, 40, "layer", "f32", "f32", True, offset=0.0)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    grads = {n: s[m].clone() for n, m in (("x", "dx"), ("residual", "dx"), ("gamma", "dgamma"), ("beta", "dbeta"))}
    h = 2.0 ** -7

    def loss():
        R.ra_norm_forward(a)
        torch.cuda.synchronize()
        return float((s["y"].double() * s["dy"].double()).sum() + (s["sum"].double() * s["dsum"].double()).sum())
    for name, i in (("x", 3), ("x", 77), ("residual", 50), ("gamma", 11), ("beta", 39)):
        v = s[name].view(-1)
        v0 = float(v[i])
        at = {}
        for k in (-2, -1, 1, 2):
            v[i] = v0 + k * h
            at[k] = loss() / 1.0, float(v[i])
        v[i] = v0
        first = (at[1][0] - at[-1][0]) / (at[1][1] - at[-1][1])
        third = abs(at[2][0] - 2 * at[1][0] + 2 * at[-1][0] - at[-2][0]) / (2 * h ** 3)
        rounding = 120 * 8 * U * 4 / h  # 120 values of at most about 8, each off by a few u
        assert abs(first - float(grads[name].view(-1)[i])) <= third * h * h / 3 + rounding


def test_a_captured_step_and_two_streams():
    a, s = make(900, 768, "layer", "bf16", "f32", True)
    b, t = make(900, 768, "layer", "bf16", "f32", True, seed=5)
    for x in (a, b):
        R.ra_norm_forward(x)
        R.ra_norm_backward(x)
    torch.cuda.synchronize()
    want = [{n: q[n].clone() for n in ("y", "sum", "dx", "dgamma", "dbeta")} for q in (s, t)]
    for q in (s, t):
        for n in want[0]:
            q[n].fill_(7.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st = torch.cuda.current_stream()
        R.ra_norm_forward(a, st)
        R.ra_norm_backward(a, st)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        R.ra_norm_forward(b, other)
        R.ra_norm_backward(b, other)
    torch.cuda.synchronize()
    for q, w in zip((s, t), want):
        for n in w:
            assert torch.equal(q[n], w[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hidden", [40, 77, 250])
def test_many_short_rows_some_outputs_and_in_place(hidden, dtype):
    """Rows of a warp each, eight warps a CTA: any of the outputs may be left out, and dx may take dy's place.  (Without dx a CTA reads
    fewer inputs and more CTAs have room, which add up the weights' sums in another order: within the bounds, not bit for bit.)"""
    a, s = make(5003, hidden, "layer", dtype, "f32", True)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    check(a, s, "layer", dtype, "f32", True)
    names = ("dx", "dgamma", "dbeta")
    want = {n: s[n].clone() for n in names}
    for left in names:
        for n in names:
            s[n].fill_(7.0)
        kept = getattr(a, left + "_dev")
        setattr(a, left + "_dev", None)
        R.ra_norm_backward(a)
        setattr(a, left + "_dev", kept)
        assert bool((s[left] == 7.0).all()), left
        for n in names:
            assert n == left or left == "dx" or torch.equal(s[n], want[n]), (left, n)
        s[left].copy_(want[left])
        check(a, s, "layer", dtype, "f32", True)
    dy = s["dy"].clone()
    a.dx_dev = a.dy_dev
    R.ra_norm_backward(a)
    assert torch.equal(s["dy"], want["dx"]) and torch.equal(s["dbeta"], want["dbeta"]) and not torch.equal(s["dy"], dy)


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("kind,residual", [("layer", False), ("layer", True), ("rms", True)])
@pytest.mark.parametrize("rows,hidden", [(2501, 264), (2433, 520), (5003, 1024), (2501, 2048), (2501, 2056), (2501, 4096), (2433, 8192)])
def test_many_rows_of_several_warps(rows, hidden, kind, residual, dtype, wdtype):
    """Rows in 16-byte pieces, several at a time through the ring, whose sums meet at barriers: from 2432 on."""
    a, s = make(rows, hidden, kind, dtype, wdtype, residual, seed=rows + hidden)
    s["workspace"][16384:] = 255
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    torch.cuda.synchronize()
    check(a, s, kind, dtype, wdtype, residual)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hidden", [1024, 2304, 2302])
def test_many_rows_of_several_warps_in_place(hidden, dtype):
    a, s = make(2501, hidden, "layer", dtype, "f32", True)
    b, t = make(2501, hidden, "layer", dtype, "f32", True)
    R.ra_norm_forward(a)
    R.ra_norm_backward(a)
    b.sum_dev, t["sum"] = b.residual_dev, t["residual"]
    b.y_dev, t["y"] = b.x_dev, t["x"]
    R.ra_norm_forward(b)
    for place in ("dsum", "dy"):
        kept = t[place].clone()
        b.dx_dev = t[place].data_ptr()
        for n in ("dgamma", "dbeta"):
            t[n].fill_(7.0)
        R.ra_norm_backward(b)
        torch.cuda.synchronize()
        for n in ("y", "sum", "dgamma", "dbeta"):
            assert torch.equal(s[n], t[n]), n
        assert torch.equal(s["dx"], t[place]), place
        t[place].copy_(kept)
