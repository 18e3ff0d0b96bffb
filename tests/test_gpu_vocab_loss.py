"""Cross-entropy over a vocabulary from hidden states, and its gradients, against 64 bits and against differences.

Bounds, element by element.  u = 2^-24, e = 2^-8 (bf16's rounding).  A logit is a sum of H products, off by at most
(H + 8) u sum|x w| =: s.  A weight p = exp(z - lse) is off by dp = 2 max s + 2 u max|z - lse| + 8 u + a u of itself, the sum
of exponentials taking a = 128 + V / 64 steps in turn at most; lse by max s + a u + 4 u + u |lse|, and the loss by s more.
dz = dloss (p - onehot) is off by |dloss| (p dp + 2 u |p - onehot|), and rounded to bf16 by e |dz| more.  A gradient is a
sum of n products with it, off by (n + 8) u of their magnitudes more, and by its rounding."""
import pytest
import torch

from paper_2502_19864_gb300 import ringada as R
from tests.operator_helpers import DT, E, RA, U, vocab_loss_plan, workspace

pytestmark = pytest.mark.gpu


def make(tokens, vocab, hidden, dtype, ignored=0.2, seed=0, pad=0, scale=2.0, word=None, x_scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = hidden + pad
    s = {"x": torch.randn(tokens, wide, generator=g, device="cuda").mul_(x_scale).to(DT[dtype])[:, :hidden],
         "w": torch.randn(vocab, wide, generator=g, device="cuda").mul_(scale * hidden ** -0.5).to(DT[dtype])[:, :hidden]}
    lab = torch.randint(0, vocab, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    if word is not None:
        lab[:] = word
    lab[torch.rand(tokens, generator=g, device="cuda") < ignored] = -100
    s["labels"] = lab
    s["dloss"] = torch.rand(tokens, generator=g, device="cuda").add_(0.5) / max(tokens, 1)
    s["loss"], s["lse"] = (torch.full((tokens,), 7.0, device="cuda") for _ in "ab")
    s["dx"] = torch.full((tokens, wide), 7.0, device="cuda", dtype=DT[dtype])[:, :hidden]
    s["dw"] = torch.full((vocab, wide), 7.0, device="cuda", dtype=DT[dtype])[:, :hidden]
    s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    a = R.ra_vocab_loss_args(x_dev=s["x"].data_ptr(), x_stride=wide, w_dev=s["w"].data_ptr(), w_stride=wide,
                             labels_dev=lab.data_ptr(), loss_dev=s["loss"].data_ptr(), lse_dev=s["lse"].data_ptr(),
                             dloss_dev=s["dloss"].data_ptr(), dx_dev=s["dx"].data_ptr(), dx_stride=wide,
                             dw_dev=s["dw"].data_ptr(), dw_stride=wide, err_dev=s["err"].data_ptr(), tokens=tokens, vocab=vocab,
                             hidden=hidden, dtype=RA[dtype])
    n = R.ra_vocab_loss_workspace_bytes(a)
    assert n > 0
    s["workspace"] = workspace(n)
    a.workspace_dev, a.workspace_bytes = s["workspace"].data_ptr(), n
    return a, s


def both(a, stream=None):
    R.ra_vocab_loss_forward(a, stream)
    R.ra_vocab_loss_backward(a, stream)


def near(got, want, bound, what):
    off = (got.double() - want).abs()
    assert bool((off <= bound + 1e-37).all()), (what, float((off / (bound + 1e-37)).max()))


def check(s, dtype, grads=("dx", "dw")):
    e = E if dtype == "bf16" else 0.0
    lab = s["labels"].long()
    V, H = s["w"].shape
    on = (lab >= 0) & (lab < V)
    off = ~on
    assert bool((s["loss"][off] == 0).all()) and bool((s["lse"][off] == 0).all())
    if "dx" in grads:
        assert bool((s["dx"][off] == 0).all())
    x, w, lab = s["x"][on].double(), s["w"].double(), lab[on]
    row = torch.arange(lab.numel(), device="cuda")
    z = x @ w.T
    dz_ = (H + 8) * U * (x.abs() @ w.abs().T)
    top = dz_.amax(1)
    lse = torch.logsumexp(z, 1)
    chain = (128 + V / 64) * U
    dl = top + chain + 4 * U + U * lse.abs()
    near(s["lse"][on], lse, dl, "lse")
    want = lse - z[row, lab]
    near(s["loss"][on], want, dl + dz_[row, lab] + 2 * U * want.abs(), "loss")
    p = torch.exp(z - lse[:, None])
    dp = 2 * top + 2 * U * (z - lse[:, None]).abs().amax(1) + 8 * U + chain
    d = p.clone()
    d[row, lab] -= 1
    scale = s["dloss"][on].double()[:, None]
    G = d * scale
    dG = scale * (p * dp[:, None] + 2 * U * d.abs()) + e * G.abs()
    if "dx" in grads:
        want = G @ w
        near(s["dx"][on], want, dG @ w.abs() + (V + 8) * U * (G.abs() @ w.abs()) + (e + U) * want.abs(), "dx")
    if "dw" in grads:
        want = G.T @ x
        near(s["dw"], want, dG.T @ x.abs() + (len(row) + 8) * U * (G.abs().T @ x.abs()) + (e + U) * want.abs(), "dw")


SIZES = [(1, 1, 8), (1, 5, 8), (3, 40, 16), (7, 1000, 64), (64, 64, 64), (65, 257, 72), (130, 513, 128), (300, 5003, 136),
         (1025, 300, 256), (513, 2050, 512), (257, 30011, 64), (2, 100000, 32), (4100, 97, 24), (8, 3001, 1000), (9, 77, 2048), (16, 500, 200),
         (17, 1003, 1024), (32, 2000, 136), (33, 2000, 136), (5, 70, 4104), (30, 3, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,hidden", SIZES)
def test_against_64_bits(tokens, vocab, hidden, dtype):
    a, s = make(tokens, vocab, hidden, dtype, ignored=0.0 if tokens < 4 else 0.2, seed=tokens)
    both(a)
    torch.cuda.synchronize()
    check(s, dtype)
    assert int(s["err"]) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ignored", [0.0, 0.9, 1.1])
@pytest.mark.parametrize("tokens", [20, 300])
def test_how_many_are_counted(dtype, ignored, tokens):
    a, s = make(tokens, 700, 64, dtype, ignored=ignored)
    both(a)
    torch.cuda.synchronize()
    check(s, dtype)


def test_one_token_is_counted():
    for at in (0, 150, 299):
        a, s = make(300, 700, 64, "bf16", ignored=1.1)
        s["labels"][at] = 699
        both(a)
        torch.cuda.synchronize()
        check(s, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [20, 300])
def test_what_is_not_counted_does_not_matter(dtype, tokens):
    a, s = make(tokens, 700, 64, dtype, ignored=0.3)
    both(a)
    torch.cuda.synchronize()
    want = {n: s[n].clone() for n in ("loss", "lse", "dx", "dw")}
    skipped = s["labels"] < 0
    s["x"][skipped] = float("nan")
    s["dloss"][skipped] = float("inf")
    s["workspace"][16384:] = 255  # (of a workspace only its start is zeros)
    both(a)
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(s[n], want[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [20, 100, 300])
def test_labels_out_of_range(dtype, tokens):
    for call in ("forward", "backward"):
        a, s = make(tokens, 500, 64, dtype)
        s["labels"][3], s["labels"][10], s["labels"][11] = 500, 2 ** 31 - 1, -2 ** 31
        both(a)
        torch.cuda.synchronize()
        check(s, dtype)
        assert int(s["err"]) == R.RA_DEV_BOUNDS
        s["err"].zero_()
        (R.ra_vocab_loss_forward if call == "forward" else R.ra_vocab_loss_backward)(a)
        torch.cuda.synchronize()
        assert int(s["err"]) == R.RA_DEV_BOUNDS, call


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [8, 56])
@pytest.mark.parametrize("tokens", [12, 150])
def test_strides(dtype, pad, tokens):
    a, s = make(tokens, 333, 64, dtype, pad=pad)
    both(a)
    torch.cuda.synchronize()
    check(s, dtype)
    for n, rows in (("dx", tokens - 1), ("dw", 332)):
        between = torch.as_strided(s[n], (rows, pad), (64 + pad, 1), s[n].storage_offset() + 64)
        assert bool((between == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits(dtype):
    """Logits of hundreds: exponentials of all but a few words vanish, and nothing overflows."""
    for tokens in (7, 200):
        a, s = make(tokens, 900, 64, dtype, scale=150.0)
        both(a)
        torch.cuda.synchronize()
        check(s, dtype)


def test_words_of_the_label_alone():
    a, s = make(500, 1300, 64, "bf16", word=1299)
    both(a)
    torch.cuda.synchronize()
    check(s, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,at", [(20, 7), (100, 77), (300, 77)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_token_that_is_not_finite_stays_by_itself_in_dx(dtype, tokens, at, value):
    a, s = make(tokens, 700, 64, dtype, ignored=0.0)
    s["x"][at, 3] = value
    both(a)
    torch.cuda.synchronize()
    ok = torch.arange(tokens, device="cuda") != at
    assert not bool(s["loss"][at].isfinite()) and not bool(s["dx"][at].isfinite().any())
    assert bool(s["loss"][ok].isfinite().all()) and bool(s["dx"][ok].isfinite().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [25, 200])
def test_parts(dtype, tokens):
    a, s = make(tokens, 700, 64, dtype)
    both(a)
    torch.cuda.synchronize()
    want = {n: s[n].clone() for n in ("loss", "lse", "dx", "dw")}
    for keep in ("dx", "dw"):
        for n in ("dx", "dw"):
            s[n].fill_(7.0)
            setattr(a, n + "_dev", s[n].data_ptr() if n == keep else None)
        R.ra_vocab_loss_backward(a)
        torch.cuda.synchronize()
        for n in ("dx", "dw"):
            assert torch.equal(s[n], want[n]) if n == keep else bool((s[n] == 7.0).all()), (keep, n)
    s["loss"].fill_(7.0)
    a.lse_dev = a.dx_dev = a.dw_dev = None
    R.ra_vocab_loss_forward(a)
    torch.cuda.synchronize()
    assert torch.equal(s["loss"], want["loss"])


def test_no_tokens():
    a, s = make(0, 50, 64, "bf16", pad=8)
    both(a)
    torch.cuda.synchronize()
    assert bool((s["dw"] == 0).all())
    between = torch.as_strided(s["dw"], (49, 8), (72, 1), s["dw"].storage_offset() + 64)
    assert bool((between == 7.0).all())


def test_against_differences():
    """The loss sum(dloss loss) by steps of 2^-5 in x and W: off by h^2 / 6 |f'''|, bounded by the line's third difference,
    and by the losses' rounding."""
    a, s = make(6, 50, 16, "f32", ignored=0.0)
    both(a)
    torch.cuda.synchronize()
    grads = {"x": s["dx"].clone(), "w": s["dw"].clone()}
    h = 2.0 ** -5
    for name, i in (("x", 0), ("x", 95), ("w", 3), ("w", 16 * int(s["labels"][2]) + 5)):
        v = s[name].view(-1)
        v0 = float(v[i])
        at = {}
        for k in (-2, -1, 1, 2):
            v[i] = v0 + k * h
            R.ra_vocab_loss_forward(a)
            torch.cuda.synchronize()
            at[k] = float((s["loss"].double() * s["dloss"].double()).sum()), float(v[i])
        v[i] = v0
        first = (at[1][0] - at[-1][0]) / (at[1][1] - at[-1][1])
        third = abs(at[2][0] - 2 * at[1][0] + 2 * at[-1][0] - at[-2][0]) / (2 * h ** 3)
        # losses of at most 16 of weights that sum to about 1, each off by 32 u of it
        assert abs(first - float(grads[name].view(-1)[i])) <= third * h * h / 3 + 16 * 32 * U * 4 / h


@pytest.mark.parametrize("wide", [True, False])
def test_the_same_twice_captured_and_on_two_streams(wide):
    a, s = make(400 if wide else 90, 3000, 128, "bf16")
    b, t = make(77 if wide else 9, 1500, 64, "f32", seed=5)
    names = ("loss", "lse", "dx", "dw")
    for x in (a, b):
        both(x)
    torch.cuda.synchronize()
    want = [{n: q[n].clone() for n in names} for q in (s, t)]
    for q in (s, t):
        for n in names:
            q[n].fill_(7.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(a, torch.cuda.current_stream())
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        both(b, other)
    torch.cuda.synchronize()
    for q, w in zip((s, t), want):
        for n in names:
            assert torch.equal(q[n], w[n]), n


def test_one_workspace_for_any_shapes():
    cases = [make(5, 3000, 64, "bf16"), make(700, 90, 128, "f32"), make(130, 1025, 64, "bf16"), make(11, 900, 64, "f32")]
    need = max(s["workspace"].numel() for _, s in cases)
    ws = workspace(need)
    ws[16384:] = 255
    for _ in range(2):
        for a, s in cases:
            a.workspace_dev, a.workspace_bytes = ws.data_ptr(), need
            both(a)
    torch.cuda.synchronize()
    assert bool((ws[:16384] == 0).all())
    for (a, s), dtype in zip(cases, ("bf16", "f32", "bf16", "f32")):
        check(s, dtype)


# Sizes and the forms that they run, as vocab_loss_plan has them: pieces of the vocabulary; tiles' CTAs and columns of the logits
# and of the gradients; whether the gradients' sums are cut ("cut": dx's, dW's).  Between them all the tiles of both types.
FORMS = [
    ("bf16", 150, 9923, 960, {"pieces": 1, "forward": (2, 256), "logits": (2, 256)}),
    ("bf16", 38, 36972, 8, {"pieces": 1, "forward": (1, 256), "logits": (1, 256)}),
    ("bf16", 36, 19979, 8, {"pieces": 1, "forward": (1, 160)}),
    ("bf16", 34, 11159, 1264, {"pieces": 1, "forward": (1, 96), "grads": (1, 256), "cut": (True, False)}),
    ("bf16", 999, 839, 1992, {"pieces": 1, "grads": (2, 256), "cut": (False, False)}),
    ("bf16", 134, 4886, 1376, {"pieces": 1, "grads": (2, 256), "cut": (True, False)}),
    ("bf16", 8200, 97, 24, {"pieces": 1, "grads": (1, 64), "cut": (False, True)}),
    ("bf16", 1303, 43550, 8, {"pieces": 2, "grads": (1, 64)}),
    ("bf16", 2100, 40001, 64, {"pieces": 2, "grads": (1, 64)}),
    ("bf16", 1548, 37661, 88, {"pieces": 2, "grads": (1, 128)}),
    ("bf16", 1025, 58697, 528, {"pieces": 2, "grads": (1, 256)}),
    ("bf16", 2060, 40001, 520, {"pieces": 2, "grads": (2, 256)}),
    ("bf16", 3300, 60001, 136, {"pieces": 4}),
    ("f32", 1370, 66, 1296, {"pieces": 1, "grads": (1, 128), "cut": (False, True)}),
    ("f32", 4890, 262, 152, {"pieces": 1, "cut": (True, True)}),
    ("f32", 300, 50003, 64, {"pieces": 2, "grads": (1, 64)}),
    ("f32", 277, 44441, 88, {"pieces": 2, "grads": (1, 128)}),
    ("f32", 4134, 5255, 824, {"pieces": 2, "grads": (1, 128), "cut": (False, False)}),
    ("f32", 2100, 30011, 264, {"pieces": 4, "grads": (1, 128)}),
]


def check_forms(plan, forms):
    for name, want in forms.items():
        got = (plan["splits_x"] > 1, plan["splits_w"] > 1) if name == "cut" else plan[name]
        assert got == want, (name, got, want)
    assert not plan["few"]


@pytest.mark.parametrize("ignored", [0.0, 0.3])
@pytest.mark.parametrize("dtype,tokens,vocab,hidden,forms", FORMS)
def test_each_form(dtype, tokens, vocab, hidden, forms, ignored):
    """With the labels of some tokens at the pieces' borders, a workspace of anything behind its zeros, and each gradient alone."""
    a, s = make(tokens, vocab, hidden, dtype, ignored=ignored, seed=vocab)
    p = vocab_loss_plan(a)
    check_forms(p, forms)
    at = sorted({w for q in range(p["pieces"]) for w in (q * p["width"], q * p["width"] - 1, q * p["width"] + 1)} & set(range(vocab)) | {vocab - 1})
    s["labels"][5:5 + len(at)] = torch.tensor(at, dtype=torch.int32, device="cuda")
    s["workspace"][16384:] = 255
    n = R.ra_kernel_launches()
    R.ra_vocab_loss_forward(a)
    n, n0 = R.ra_kernel_launches(), n
    R.ra_vocab_loss_backward(a)
    launched = n - n0, R.ra_kernel_launches() - n
    torch.cuda.synchronize()
    pieces, cut_w = p["pieces"], p["splits_w"] > 1
    if dtype == "bf16":  # numbering, all logits, join; numbering, dz and gradients a piece, sums
        direct = tokens <= 128
        assert launched == (2 if direct else 3, 2 + 2 * pieces + cut_w)
    else:                # and each piece's logits, the later ones' planes of W
        assert launched == (1 + 2 * pieces, 1 + 3 * pieces + cut_w)
    check(s, dtype)
    assert int(s["err"]) == 0
    want = {g: s[g].clone() for g in ("dx", "dw")}
    for keep in ("dx", "dw"):
        for g in ("dx", "dw"):
            s[g].fill_(7.0)
            setattr(a, g + "_dev", s[g].data_ptr() if g == keep else None)
        s["workspace"][16384:] = 255
        R.ra_vocab_loss_backward(a)
        torch.cuda.synchronize()
        for g in ("dx", "dw"):
            assert torch.equal(s[g], want[g]) if g == keep else bool((s[g] == 7.0).all()), (keep, g)


@pytest.mark.parametrize("dtype,tokens,vocab", [("bf16", 2100, 40001), ("f32", 300, 50003)])
@pytest.mark.parametrize("which", ["none", "first piece", "last word"])
def test_pieces_that_no_label_is_in(dtype, tokens, vocab, which):
    a, s = make(tokens, vocab, 64, dtype, ignored=0.2)
    width = vocab_loss_plan(a)["width"]
    assert width < vocab
    on = s["labels"] >= 0
    s["labels"][on] = {"none": -1, "last word": vocab - 1}.get(which, 0) if which != "first piece" else s["labels"][on] % width
    s["workspace"][16384:] = 255
    both(a)
    torch.cuda.synchronize()
    check(s, dtype)


@pytest.mark.parametrize("dtype,tokens,vocab", [("bf16", 2100, 40001), ("f32", 300, 50003)])
def test_pieces_captured(dtype, tokens, vocab):
    a, s = make(tokens, vocab, 64, dtype)
    assert vocab_loss_plan(a)["pieces"] > 1
    both(a)
    torch.cuda.synchronize()
    want = {n: s[n].clone() for n in ("loss", "lse", "dx", "dw")}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(a, torch.cuda.current_stream())
    for n in want:
        s[n].fill_(7.0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(s[n], want[n]), n


@pytest.mark.parametrize("tokens,vocab,hidden", [(1, 200, 64), (2, 332, 1104), (20, 700, 64), (107, 359, 664), (128, 1003, 256), (100, 140001, 64)])
def test_few_bf16_tokens_keep_16_bits_of_dz(tokens, vocab, hidden):
    """Of up to 128 tokens dz enters its products as two bf16 terms: e^2 |dz| stands in the bounds where e |dz| does for more tokens."""
    a, s = make(tokens, vocab, hidden, "bf16", ignored=0.0, seed=hidden)
    s["workspace"][16384:] = 255
    both(a)
    torch.cuda.synchronize()
    check(s, "bf16")
    x, w, lab = s["x"].double(), s["w"].double(), s["labels"].long()
    row = torch.arange(tokens, device="cuda")
    z = x @ w.T
    top = (hidden + 8) * U * (x.abs() @ w.abs().T).amax(1)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    dp = 2 * top + 2 * U * (z - lse[:, None]).abs().amax(1) + 8 * U + (128 + vocab / 64) * U
    d = p.clone()
    d[row, lab] -= 1
    scale = s["dloss"].double()[:, None]
    G = d * scale
    dG = scale * (p * dp[:, None] + 2 * U * d.abs()) + E * E * G.abs()
    for name, want, bound in (("dx", G @ w, dG @ w.abs() + (vocab + 8) * U * (G.abs() @ w.abs())),
                              ("dw", G.T @ x, dG.T @ x.abs() + (tokens + 8) * U * (G.abs().T @ x.abs()))):
        near(s[name], want, bound + (E + U) * want.abs(), name)
