"""Orthogonalisation by Newton-Schulz products against 64 bits.

The bound is normwise, from the same steps in 64 bits with every product's elements moved at random by up to rho of
the products' magnitudes (and a normalised input by u): what the roundings of each step may be, carried by the steps that
follow, which raise what lies along small singular values by up to 3.4445 each.  fp32: a sum of K products is off by less than
(sqrt(K) + 2) 2^-23 of their magnitudes; bf16 (operands of 16 bits in two terms): 2^-16.  Four such runs; the largest distance from the undisturbed
result, four times, and the output's rounding."""
import math

import pytest
import torch

from paper_2502_19864_gb300 import ringada as R
from tests.operator_helpers import DT, E, RA, U, orthogonalize_plan, workspace

pytestmark = pytest.mark.gpu
COEF = (3.4445, -4.775, 2.0315)


def make(n, rows, cols, dtype, steps=5, coef=COEF, eps=1e-7, seed=0, pad=0, gap=0, scale=1e-3, fall=-2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    low, row = min(rows, cols), cols + pad
    each = rows * row + gap
    f = torch.logspace(0, fall, low, device="cuda")
    v = (torch.randn(n, rows, low, generator=g, device="cuda") * f) @ torch.randn(n, low, cols, generator=g, device="cuda").mul_(low ** -0.5)
    buf = torch.full((n * each,), 7.0, device="cuda", dtype=DT[dtype])
    s = {"x": torch.as_strided(buf, (n, rows, cols), (each, row, 1))}
    s["x"].copy_(v * scale)
    out = torch.full((n * each,), 7.0, device="cuda", dtype=DT[dtype])
    s["out"], s["whole"] = torch.as_strided(out, (n, rows, cols), (each, row, 1)), out
    s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    a = R.ra_orthogonalize_args(x_dev=buf.data_ptr(), x_stride=row, x_matrix_stride=each, out_dev=out.data_ptr(), out_stride=row,
                                out_matrix_stride=each, n_matrices=n, rows=rows, cols=cols, steps=steps, dtype=RA[dtype],
                                err_dev=s["err"].data_ptr(), a=coef[0], b=coef[1], c=coef[2], eps=eps)
    need = R.ra_orthogonalize_workspace_bytes(a)
    assert need > 0
    s["workspace"] = workspace(need)
    a.workspace_dev, a.workspace_bytes = s["workspace"].data_ptr(), need
    s["buf"] = buf
    return a, s


def steps64(x, steps, coef, eps, rho=0.0, gen=None):
    def mul(p, q):
        r = p @ q
        if rho:
            r = r + rho(p.shape[-1]) * (p.abs() @ q.abs()) * (torch.rand(r.shape, generator=gen, device="cuda", dtype=torch.float64) * 2 - 1)
        return r
    x = x.double()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + eps)
    if rho:
        x = x * (1 + 2 * U * (torch.rand(x.shape, generator=gen, device="cuda", dtype=torch.float64) * 2 - 1))
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    a, b, c = (float(torch.tensor(v, dtype=torch.float32)) for v in coef)
    for _ in range(steps):
        S = mul(x, x.transpose(1, 2))
        x = a * x + mul(b * S + c * mul(S, S), x)
    return x.transpose(1, 2) if tall else x


def check(s, dtype, steps=5, coef=COEF, eps=1e-7):
    assert int(s["err"]) == 0
    eps = float(torch.tensor(eps, dtype=torch.float32))
    want = steps64(s["x"] if "kept" not in s else s["kept"], steps, coef, eps)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rho = (lambda k: (math.sqrt(k) + 2) * 2.0 ** -23) if dtype == "f32" else (lambda k: 2.0 ** -16)
    src = s["x"] if "kept" not in s else s["kept"]
    e = E if dtype == "bf16" else U
    norm = lambda t: t.square().sum((1, 2)).sqrt()  # noqa: E731
    off = torch.stack([norm(steps64(src, steps, coef, eps, rho, gen) - want) for _ in range(4)]).amax(0)
    got = norm(s["out"].double() - want)
    bound = 4 * off + e * norm(want)
    assert bool((got <= bound).all()), float((got / bound).max())


SHAPES = [(1, 1, 1), (2, 1, 9), (3, 9, 1), (1, 5, 7), (4, 16, 128), (4, 128, 16), (2, 64, 64), (3, 65, 127), (2, 200, 130), (48, 96, 40),
          (1, 300, 1000), (1, 513, 257), (2, 128, 128), (1, 777, 640), (1, 31, 4099), (5, 64, 1024), (7, 1024, 64), (3, 321, 33), (1, 2560, 64),
          (2, 63, 2561), (200, 64, 65), (1, 4608, 17), (40, 520, 48), (1, 1100, 600)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,rows,cols", SHAPES)
def test_against_64_bits(n, rows, cols, dtype):
    a, s = make(n, rows, cols, dtype, seed=rows)
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, dtype)


@pytest.mark.parametrize("n,rows,cols", [(2, 777, 1000), (8, 128, 16), (1, 300, 2000)])
def test_fp32_is_no_further_off_than_fp32_products(n, rows, cols):
    """Three times what plain fp32 products on the CUDA cores leave: each of theirs is off by the roundings of K sums, as the planes'
    are, whose accumulators are truncated, which is twice a rounding, and whose smallest terms are left out."""
    a, s = make(n, rows, cols, "f32", seed=3)
    R.ra_orthogonalize(a)
    x = s["x"]
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    tall = rows > cols
    x = x.transpose(1, 2) if tall else x
    for _ in range(5):
        S = x @ x.transpose(1, 2)
        x = COEF[0] * x + (COEF[1] * S + COEF[2] * (S @ S)) @ x
    x = x.transpose(1, 2) if tall else x
    eps = float(torch.tensor(1e-7, dtype=torch.float32))
    want = steps64(s["x"], 5, COEF, eps)
    assert (s["out"].double() - want).norm() <= 3 * (x.double() - want).norm()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("steps", [0, 1, 2, 6])
def test_steps(dtype, steps):
    a, s = make(2, 100, 72, dtype, steps=steps)
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, dtype, steps=steps)


def test_other_coefficients():
    """The cubic (3 X - X X^T X) / 2, which leaves an orthogonal matrix where it is."""
    coef = (1.5, -0.5, 0.0)
    a, s = make(1, 96, 160, "f32", steps=12, coef=coef, fall=-0.5)
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, "f32", steps=12, coef=coef)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,gap", [(3, 0), (8, 5), (0, 1)])
def test_strides(dtype, pad, gap):
    a, s = make(3, 70, 90, dtype, pad=pad, gap=gap)
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, dtype)
    s["out"].fill_(7.0)
    assert bool((s["whole"] == 7.0).all())  # what lies between rows and matrices is left as it was


@pytest.mark.parametrize("dtype,n,rows,cols", [("bf16", 1, 1537, 2050), ("bf16", 1, 2400, 2410), ("f32", 1, 1700, 1701)])
def test_symmetric_products_by_halves(dtype, n, rows, cols):
    """Sizes at which one triangle of the symmetric products' tiles is computed and the other mirrored."""
    a, s = make(n, rows, cols, dtype)
    s["workspace"][16384:] = 255
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,rows,cols", [(1, 3892, 390), (3, 70, 4001), (2, 2050, 129), (1, 20, 30000), (1, 2500, 256), (1, 32768, 65)])
def test_long_sides_in_ranges(n, rows, cols, dtype):
    """Sizes at which S has few tiles and a K that is cut in ranges."""
    a, s = make(n, rows, cols, dtype)
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(90, 72), (72, 90), (300, 40)])
def test_matrices_side_by_side(dtype, rows, cols):
    a, s = make(1, rows, 3 * cols, dtype)
    for name in ("x", "out"):
        s[name] = s[name].view(rows, 3, cols).transpose(0, 1)
    a.n_matrices, a.cols, a.x_matrix_stride, a.out_matrix_stride = 3, cols, cols, cols
    n = R.ra_orthogonalize_workspace_bytes(a)
    s["workspace"] = workspace(n)
    a.workspace_dev, a.workspace_bytes = s["workspace"].data_ptr(), n
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(100, 72), (40, 300)])
def test_in_place(dtype, rows, cols):
    a, s = make(2, rows, cols, dtype)
    s["kept"] = s["x"].clone()
    a.out_dev = a.x_dev
    s["out"] = s["x"]
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, dtype)


@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1e18, 1e34])
def test_values_whose_squares_do_not_fit(scale):
    a, s = make(2, 90, 60, "f32", scale=scale, eps=0.0)
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, "f32", eps=0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 1e-7])
def test_zeros_and_values_that_are_not_finite_stay_in_their_matrix(dtype, eps):
    for steps in (0, 5):
        a, s = make(5, 70, 50, dtype, steps=steps, eps=eps)
        s["x"][1] = 0.0
        s["x"][2, 3, 4] = float("nan")
        s["x"][4, 69, 49] = float("-inf")
        R.ra_orthogonalize(a)
        torch.cuda.synchronize()
        assert bool((s["out"][1] == 0).all())
        assert not bool(s["out"][[2, 4]].isfinite().any())
        s["x"], s["out"] = s["x"][[0, 3]], s["out"][[0, 3]]
        check(s, dtype, steps=steps, eps=eps)


def test_the_same_twice_captured_and_on_two_streams():
    a, s = make(6, 128, 64, "bf16")
    b, t = make(1, 300, 500, "f32")
    for x in (a, b):
        R.ra_orthogonalize(x)
    torch.cuda.synchronize()
    want = [q["out"].clone() for q in (s, t)]
    for q in (s, t):
        q["out"].fill_(7.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.ra_orthogonalize(a, torch.cuda.current_stream())
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        R.ra_orthogonalize(b, other)
    torch.cuda.synchronize()
    for q, w in zip((s, t), want):
        assert torch.equal(q["out"], w)


def test_a_workspace_of_anything_behind_its_zeros():
    a, s = make(3, 90, 200, "bf16")
    s["workspace"][16384:] = 255
    for _ in range(2):
        R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, "bf16")
    assert bool((s["workspace"][:16384] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ranges_keep_matrices_apart(dtype):
    a, s = make(3, 70, 4001, dtype)
    R.ra_orthogonalize(a)
    want = s["out"].clone()
    s["x"][1, 69, 4000] = float("nan")
    s["out"].fill_(7.0)
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    assert torch.equal(s["out"][0], want[0]) and torch.equal(s["out"][2], want[2]) and bool(s["out"][1].isnan().all())


# Sizes and the forms that they run, as orthogonalize_plan has them ("ranges": more than one): tiles' CTAs and columns, and for S and Q
# whether half of the tiles is computed and mirrored.  Between them all the forms of S, Q and X in both directions.
FORMS = [
    ("bf16", 40, 141, 135, {"S0": (1, 128, 1, 1), "S": (1, 128, 1, 1), "Q": (1, 128, 1, 1)}),
    ("bf16", 40, 138, 143, {"S0": (1, 128, 1, 1), "S": (1, 128, 1, 1), "Q": (1, 128, 1, 1)}),
    ("bf16", 16, 280, 259, {"S0": (1, 128, 0, 1), "S": (1, 128, 0, 1), "Q": (1, 128, 0, 1)}),
    ("bf16", 16, 266, 282, {"S0": (1, 128, 0, 1), "S": (1, 128, 0, 1), "Q": (1, 128, 0, 1)}),
    ("bf16", 16, 405, 391, {"S0": (1, 256, 0, 1), "S": (1, 256, 0, 1), "Q": (1, 256, 0, 1)}),
    ("bf16", 16, 385, 386, {"S0": (1, 256, 0, 1), "S": (1, 256, 0, 1), "Q": (1, 256, 0, 1)}),
    ("bf16", 16, 388, 1765, {"S0": (2, 256, 0, 1), "S": (2, 256, 1, 1)}),
    ("bf16", 16, 1736, 405, {"S0": (2, 256, 0, 1), "X": (2, 256)}),
    ("bf16", 16, 2103, 392, {"S": (2, 256, 1, 1), "X": (2, 256)}),
    ("bf16", 3, 1214, 1203, {"Q": (2, 256, 0, 1)}),
    ("bf16", 4, 1405, 1040, {"S0": (2, 256, 1, 1), "S": (2, 256, 1, 1), "Q": (2, 256, 1, 1)}),
    ("bf16", 4, 1057, 1490, {"S0": (2, 256, 1, 1), "S": (2, 256, 1, 1), "Q": (2, 256, 1, 1)}),
    ("bf16", 1, 1038, 1028, {"Q": (1, 128, 1, "ranges")}),
    ("bf16", 1, 1026, 1087, {"Q": (1, 128, 1, "ranges")}),
    ("bf16", 1, 2523, 65, {"S0": (1, 128, 1, "ranges"), "S": (1, 128, 1, "ranges")}),
    ("bf16", 1, 65, 2782, {"S0": (1, 128, 1, "ranges"), "S": (1, 128, 1, "ranges")}),
    ("bf16", 40, 270, 129, {"X": (1, 256)}),
    ("bf16", 40, 66, 1420, {"X0": (1, 256), "X": (1, 256)}),
    ("bf16", 2, 454, 2445, {"X0": (2, 256), "X": (2, 256)}),
    ("bf16", 4, 1198, 450, {"X0": (2, 256)}),
    ("f32", 40, 143, 129, {"S": (1, 128, 1, 1), "Q": (1, 128, 1, 1)}),
    ("f32", 40, 133, 160, {"S": (1, 128, 1, 1), "Q": (1, 128, 1, 1)}),
    ("f32", 16, 280, 258, {"S": (1, 128, 0, 1), "Q": (1, 128, 0, 1), "X": (1, 128)}),
    ("f32", 16, 257, 300, {"S": (1, 128, 0, 1), "Q": (1, 128, 0, 1), "X": (1, 128)}),
    ("f32", 1, 360, 348, {"S": (1, 128, 1, "ranges"), "Q": (1, 128, 1, "ranges")}),
    ("f32", 1, 349, 357, {"S": (1, 128, 1, "ranges"), "Q": (1, 128, 1, "ranges")}),
    ("f32", 1, 67, 65, {"S": (1, 64, 0, 1), "Q": (1, 64, 0, 1), "X": (1, 64)}),
    ("f32", 1, 65, 68, {"S": (1, 64, 0, 1), "Q": (1, 64, 0, 1), "X": (1, 64)}),
]


@pytest.mark.parametrize("dtype,n,rows,cols,forms", FORMS)
def test_each_form(dtype, n, rows, cols, forms):
    a, s = make(n, rows, cols, dtype, seed=cols)
    check_forms(orthogonalize_plan(a), forms)
    s["workspace"][16384:] = 255
    R.ra_orthogonalize(a)
    torch.cuda.synchronize()
    check(s, dtype)


def check_forms(plan, forms):
    for name, want in forms.items():
        got = plan[name]
        if want[-1] == "ranges":
            assert got[-1] > 1, (name, got)
            got, want = got[:-1], want[:-1]
        assert got == want, (name, got, want)
    assert not plan["small"]
