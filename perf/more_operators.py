"""What the speed of the operators that train all of a decoder's weights is measured on, through the C ABI binding:
the normalisation of a stack's activations, the cross-entropy over a vocabulary straight from hidden states, and the
orthogonalisation of an update, each with the gradients that a training step takes from it.

A case is one call (with ``"train"`` two, forward and backward):

``norm``    ra_norm_forward (LayerNorm or RMSNorm, with ``"residual"`` of a sum that it writes too), and with
            ``"train"`` ra_norm_backward.  Outputs and sums; gradients of the input and of the weights.
``loss``    ra_vocab_loss_forward: the loss of each token under softmax(x W^T), and with ``"train"``
            ra_vocab_loss_backward: gradients of x and W.  Tokens of a negative label are not counted.
``orth``    ra_orthogonalize: matrices whose singular values Newton-Schulz products have brought to about 1.

Values: a residual stream has channels of different sizes, a few of them large, and an offset; hidden states at the
head are normalised, and the logits that they give have a standard deviation of about 2; labels are words of very
different frequency; an update's singular values fall over two orders of magnitude.
"""
import math

import torch

own = False  # True: the framework's operators; False: the same in elementary torch operations

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# the polynomial a X + (b X X^T + c (X X^T)^2) X of the orthogonalisation
A, B, C = 3.4445, -4.775, 2.0315
EPS = {"norm": 1e-5, "orth": 1e-7}


# ---- cases --------------------------------------------------------------------------------

def _norm(name, dtype, wdtype, kind, rows, hidden, residual, train):
    return {"name": name, "op": "norm", "dtype": dtype, "wdtype": wdtype, "kind": kind, "rows": rows, "hidden": hidden,
            "residual": residual, "train": train}


def _loss(name, dtype, tokens, vocab, hidden, train, ignored=0.0):
    return {"name": name, "op": "loss", "dtype": dtype, "tokens": tokens, "vocab": vocab, "hidden": hidden,
            "train": train, "ignored": ignored}


def _orth(name, dtype, n, rows, cols):
    return {"name": name, "op": "orth", "dtype": dtype, "n": n, "rows": rows, "cols": cols, "steps": 5}


def listed():
    return [
        # the newest tokens of four sequences that are being answered, in the LLaMA-style decoder: latency
        _norm("norm_bf16_tokens", "bf16", "bf16", "rms", 4, 2048, True, False),
        # a training step of a small fp32 model, odd sizes
        _norm("norm_f32_train", "f32", "f32", "layer", 333, 771, False, True),
        # the decoder's norm before a block at 8 x 1024 tokens, with the residual's sum, trained
        _norm("norm_bf16_decoder", "bf16", "bf16", "rms", 8192, 2048, True, True),
        # an encoder's LayerNorm over a large batch, 512 x 128 tokens, with fp32 weights, trained
        _norm("norm_bf16_encoder", "bf16", "f32", "layer", 65536, 1024, False, True),
        # the likelihood of a few tokens: the vocabulary's matrix is read for 16 rows
        _loss("loss_bf16_score", "bf16", 16, 32000, 2048, False),
        # a training step of a small fp32 model with padding
        _loss("loss_f32_train", "f32", 333, 5003, 128, True, 0.2),
        # the decoder's training step at 8 x 1024 tokens, the largest
        _loss("loss_bf16_train", "bf16", 8192, 32000, 2048, True),
        # tuning on answers: the prompts' half of the tokens is not counted; a vocabulary of odd size
        _loss("loss_bf16_answers", "bf16", 4096, 50001, 1024, True, 0.5),
        # the adapters of a small fp32 model, two a layer
        _orth("orth_f32_adapters", "f32", 8, 128, 16),
        # the down projections of BERT-large's adapters, two a layer
        _orth("orth_bf16_adapters", "bf16", 48, 1024, 64),
        # weights of an fp32 model, odd sizes
        _orth("orth_f32_odd", "f32", 2, 777, 1000),
        # the decoder's FFN weight
        _orth("orth_bf16_ffn", "bf16", 1, 2048, 5632),
    ]


def _log(rng, lo, hi, to=1):
    """A multiple of ``to`` in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(hi, max(lo, round(v / to) * to)))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    op = rng.choice(["norm", "norm", "loss", "loss", "loss", "orth", "orth"])
    most = max(max(w["flops"] / 250, w["bytes"]) for w in (work(c) for c in listed()))
    while True:
        if op == "norm":
            c = _norm("", dtype, dtype if rng.random() < 0.6 else "f32", rng.choice(["layer", "rms"]), _log(rng, 1, 70000),
                      _log(rng, 30, 9000, rng.choice([1, 8, 8])), rng.random() < 0.4, rng.random() < 0.6)
        elif op == "loss":
            c = _loss("", dtype, _log(rng, 1, 9000), _log(rng, 300, 130000), _log(rng, 64, 4096, 8), rng.random() < 0.7,
                      rng.choice([0.0, 0.0, 0.1, 0.5, 0.9]))
        else:
            c = _orth("", dtype, _log(rng, 1, 64), _log(rng, 8, 4096), _log(rng, 8, 5632))
        w = work(c)
        if op == "norm" and w["bytes"] > 1.2e9 or op == "orth" and w["flops"] > (0.6e12 if dtype == "bf16" else 0.3e12):
            continue
        if op == "loss" and (w["flops"] > (3e12 if dtype == "bf16" else 0.6e12) or c["tokens"] * c["vocab"] > 3e8):
            continue
        if max(w["flops"] / 250, w["bytes"]) <= most:
            del c["name"]
            return c


# ---- inputs -------------------------------------------------------------------------------

def _rand(gen, shape, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale)


def _inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, s = DT[c["dtype"]], {}
    if c["op"] == "norm":
        n, h, wt = c["rows"], c["hidden"], DT[c["wdtype"]]
        size = _rand(gen, (h,), 0.5).exp_()
        size[torch.rand((h,), generator=gen, device="cuda") < 0.01] *= 12
        x = _rand(gen, (n, h)).mul_(size).add_(_rand(gen, (h,), 0.1))
        if c["residual"]:
            s["x"], s["residual"] = _rand(gen, (n, h), 0.3).to(dt), x.to(dt)
        else:
            s["x"] = x.to(dt)
        s["gamma"] = _rand(gen, (h,), 0.1).add_(1).to(wt)
        if c["kind"] == "layer":
            s["beta"] = _rand(gen, (h,), 0.1).to(wt)
        if c["train"]:
            s["dy"] = _rand(gen, (n, h), 1e-3).to(dt)
            if c["residual"]:
                s["dsum"] = _rand(gen, (n, h), 1e-3).to(dt)
        return s
    if c["op"] == "loss":
        n, v, h = c["tokens"], c["vocab"], c["hidden"]
        s["x"] = _rand(gen, (n, h)).to(dt)
        s["w"] = _rand(gen, (v, h), 2 * h ** -0.5).to(dt)
        # words by rank: the k-th as likely as 1 / k
        word = torch.rand((n,), generator=gen, device="cuda").mul_(math.log(v)).exp_().long().clamp_(max=v) - 1
        skip = torch.rand((n,), generator=gen, device="cuda") < c["ignored"]
        s["labels"] = torch.where(skip, -100, word).to(torch.int32)
        if c["train"]:
            # the mean over the counted tokens
            counted = (s["labels"] >= 0).sum().clamp(min=1)
            s["dloss"] = torch.full((n,), 1.0, device="cuda") / counted
        return s
    n, r, k = c["n"], c["rows"], c["cols"]
    low = min(r, k)
    fall = torch.logspace(0, -2, low, device="cuda")
    g = (_rand(gen, (n, r, low)) * fall) @ _rand(gen, (n, low, k), low ** -0.5)
    s["g"] = g.mul_(1e-3).to(dt)
    return s


def _outputs(c, s):
    """The buffers that a user's program keeps for the outputs."""
    like = torch.empty_like
    if c["op"] == "norm":
        o = {"y": like(s["x"])}
        if c["residual"]:
            o["sum"] = like(s["x"])
        if c["train"]:
            o["dx"], o["dgamma"] = like(s["x"]), like(s["gamma"])
            if c["kind"] == "layer":
                o["dbeta"] = like(s["gamma"])
        return o
    if c["op"] == "loss":
        o = {"loss": torch.empty((c["tokens"],), device="cuda")}
        if c["train"]:
            o["dx"], o["dw"] = like(s["x"]), like(s["w"])
        return o
    return {"out": like(s["g"])}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"], s["outputs"] = case, _outputs(case, s)
    if own:  # the argument block, with its workspace, that a program fills in once for its buffers
        s["call"] = _call(case, s)
    return s


# ---- the framework's operators ------------------------------------------------------------

def _call(c, s):
    from paper_2502_19864_gb300 import ringada as R
    o = s["outputs"]
    at = lambda t: t.data_ptr()  # noqa: E731
    dt = {"f32": R.RA_F32, "bf16": R.RA_BF16}
    if c["op"] == "norm":
        n, h = c["rows"], c["hidden"]
        a = R.ra_norm_args(x_dev=at(s["x"]), x_stride=h, gamma_dev=at(s["gamma"]), y_dev=at(o["y"]), y_stride=h, rows=n,
                           hidden=h, kind=R.RA_NORM_LAYER if c["kind"] == "layer" else R.RA_NORM_RMS,
                           dtype=dt[c["dtype"]], w_dtype=dt[c["wdtype"]], eps=EPS["norm"])
        if c["kind"] == "layer":
            a.beta_dev = at(s["beta"])
        if c["residual"]:
            a.residual_dev, a.residual_stride, a.sum_dev, a.sum_stride = at(s["residual"]), h, at(o["sum"]), h
        if not c["train"]:
            return R.ra_norm_forward, (a,)
        s["stats"] = torch.empty((2, n), device="cuda")
        a.mean_dev, a.rstd_dev = at(s["stats"][0]), at(s["stats"][1])
        a.dy_dev, a.dy_stride, a.dx_dev, a.dx_stride, a.dgamma_dev = at(s["dy"]), h, at(o["dx"]), h, at(o["dgamma"])
        if c["kind"] == "layer":
            a.dbeta_dev = at(o["dbeta"])
        if c["residual"]:
            a.dsum_dev, a.dsum_stride = at(s["dsum"]), h
        _workspace(s, a, R.ra_norm_workspace_bytes(a))
        return _both, (R.ra_norm_forward, R.ra_norm_backward, a)
    if c["op"] == "loss":
        h = c["hidden"]
        s["lse"] = torch.empty((c["tokens"],), device="cuda")
        a = R.ra_vocab_loss_args(x_dev=at(s["x"]), x_stride=h, w_dev=at(s["w"]), w_stride=h, labels_dev=at(s["labels"]),
                                 loss_dev=at(o["loss"]), lse_dev=at(s["lse"]), tokens=c["tokens"], vocab=c["vocab"],
                                 hidden=h, dtype=dt[c["dtype"]])
        if c["train"]:
            a.dloss_dev, a.dx_dev, a.dx_stride, a.dw_dev, a.dw_stride = at(s["dloss"]), at(o["dx"]), h, at(o["dw"]), h
        _workspace(s, a, R.ra_vocab_loss_workspace_bytes(a))
        if not c["train"]:
            return R.ra_vocab_loss_forward, (a,)
        return _both, (R.ra_vocab_loss_forward, R.ra_vocab_loss_backward, a)
    r, k = c["rows"], c["cols"]
    a = R.ra_orthogonalize_args(x_dev=at(s["g"]), x_stride=k, x_matrix_stride=r * k, out_dev=at(o["out"]), out_stride=k,
                                out_matrix_stride=r * k, n_matrices=c["n"], rows=r, cols=k, steps=c["steps"],
                                dtype=dt[c["dtype"]], a=A, b=B, c=C, eps=EPS["orth"])
    _workspace(s, a, R.ra_orthogonalize_workspace_bytes(a))
    return R.ra_orthogonalize, (a,)


def _workspace(s, a, n):
    s["workspace"] = torch.zeros(max(n, 256), dtype=torch.uint8, device="cuda")
    a.workspace_dev, a.workspace_bytes = s["workspace"].data_ptr(), n


def _both(forward, backward, a):
    forward(a)
    backward(a)


def run(state):
    if own:
        call, arguments = state["call"]
        call(*arguments)
        return state["outputs"]
    return {"norm": _plain_norm, "loss": _plain_loss, "orth": _plain_orth}[state["case"]["op"]](state["case"], state)


# ---- the plain forms, in 32 bits ----------------------------------------------------------

def _plain_norm(c, s):
    dt, wt = DT[c["dtype"]], DT[c["wdtype"]]
    z = s["x"].float()
    if c["residual"]:
        z = z + s["residual"].float()
    gamma = s["gamma"].float()
    d = z - z.mean(-1, keepdim=True) if c["kind"] == "layer" else z
    rstd = (d.square().mean(-1, keepdim=True) + EPS["norm"]).rsqrt()
    unit = d * rstd
    y = unit * gamma
    if c["kind"] == "layer":
        y = y + s["beta"].float()
    got = {"y": y.to(dt)}
    if c["residual"]:
        got["sum"] = z.to(dt)
    if c["train"]:
        dy = s["dy"].float()
        if c["residual"]:  # a training step keeps the sum as it was written
            unit = got["sum"].float()
            unit = (unit - z.mean(-1, keepdim=True) if c["kind"] == "layer" else unit) * rstd
        got["dgamma"] = (dy * unit).sum(0).to(wt)
        g = dy * gamma
        dx = g - unit * (g * unit).mean(-1, keepdim=True)
        if c["kind"] == "layer":
            got["dbeta"] = dy.sum(0).to(wt)
            dx = dx - g.mean(-1, keepdim=True)
        dx = dx * rstd
        if c["residual"]:
            dx = dx + s["dsum"].float()
        got["dx"] = dx.to(dt)
    return got


def _plain_loss(c, s):
    dt, labels = DT[c["dtype"]], s["labels"].long()
    counted, word = labels >= 0, labels.clamp(min=0)[:, None]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.T
    top = z.amax(-1, keepdim=True)
    chosen = z.gather(1, word)
    p = (z - top).exp_()
    total = p.sum(-1, keepdim=True)
    got = {"loss": (top + total.log() - chosen)[:, 0] * counted}
    if c["train"]:
        scale = (s["dloss"] * counted)[:, None]
        p.mul_(scale / total).scatter_add_(1, word, -scale)
        got["dx"], got["dw"] = (p @ w).to(dt), (p.T @ x).to(dt)
    return got


def _plain_orth(c, s):
    x = s["g"].float()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS["orth"])
    wide = c["rows"] <= c["cols"]
    x = x if wide else x.transpose(1, 2)
    for _ in range(c["steps"]):
        gram = x @ x.transpose(1, 2)
        x = A * x + (B * gram + C * (gram @ gram)) @ x
    return {"out": (x if wide else x.transpose(1, 2)).contiguous().to(DT[c["dtype"]])}


# ---- the work of a call -------------------------------------------------------------------

def work(case):
    c, size = case, {"f32": 4, "bf16": 2}
    es = size[c["dtype"]]
    if c["op"] == "norm":
        n, h, ws = c["rows"], c["hidden"], size[c["wdtype"]]
        weights = h * ws * (2 if c["kind"] == "layer" else 1)
        b = n * h * es * (4 if c["residual"] else 2) + weights
        if c["train"]:  # the backward reads its input and dy again, and what comes back on the residual
            b += n * h * es * (4 if c["residual"] else 3) + 2 * weights
        return {"bytes": b, "flops": n * h * (22 if c["train"] else 8)}
    if c["op"] == "loss":
        n, v, h = max(1, round(c["tokens"] * (1 - c["ignored"]))), c["vocab"], c["hidden"]
        b = es * h * (n + v) + 8 * c["tokens"]
        if c["train"]:
            b += es * h * (c["tokens"] + v) + 4 * c["tokens"]
        # logits; with gradients two products more (and the logits again, where they are not kept)
        return {"bytes": b, "flops": 2 * n * v * h * (3 if c["train"] else 1)}
    low, high = sorted((c["rows"], c["cols"]))
    # of the two symmetric products half
    step = low * low * high + low ** 3 + 2 * low * low * high
    return {"bytes": 2 * es * c["n"] * low * high, "flops": c["n"] * c["steps"] * step}


# ---- the same in 64 bits ------------------------------------------------------------------

def _exact_norm(c, s):
    z = s["x"].double()
    if c["residual"]:
        z = z + s["residual"].double()
    h, layer = c["hidden"], c["kind"] == "layer"
    mean = z.sum(1) / h if layer else torch.zeros(c["rows"], dtype=torch.float64, device="cuda")
    sigma = torch.sqrt(torch.sum((z - mean[:, None]) ** 2, 1) / h + EPS["norm"])
    gamma = s["gamma"].double()
    got = {"y": torch.addcmul(s["beta"].double(), gamma, (z - mean[:, None]) / sigma[:, None]) if layer
           else gamma * z / sigma[:, None]}
    if c["residual"]:
        got["sum"] = z
    if c["train"]:
        # the Jacobian of the unit rows, (I - 1 1^T / h - u u^T / h) / sigma, at the row that the step kept
        kept = z.to(DT[c["dtype"]]).double() if c["residual"] else z
        u = (kept - mean[:, None]) / sigma[:, None]
        dy = s["dy"].double()
        got["dgamma"] = torch.einsum("nh,nh->h", dy, u)
        du = dy * gamma
        along = torch.einsum("nh,nh->n", du, u) / h
        dx = du - along[:, None] * u
        if layer:
            got["dbeta"] = torch.einsum("nh->h", dy)
            dx -= (du.sum(1) / h)[:, None]
        dx /= sigma[:, None]
        got["dx"] = dx + s["dsum"].double() if c["residual"] else dx
    return got


def _exact_loss(c, s):
    w, labels = s["w"].double(), s["labels"].long()
    rows = torch.nonzero(labels >= 0)[:, 0]
    loss = torch.zeros(c["tokens"], dtype=torch.float64, device="cuda")
    dx = torch.zeros(c["tokens"], c["hidden"], dtype=torch.float64, device="cuda") if c["train"] else None
    dw = torch.zeros_like(w) if c["train"] else None
    for part in torch.split(rows, 1024):
        x = s["x"][part].double()
        logp = torch.log_softmax(torch.mm(x, w.t()), 1)
        picked = torch.arange(part.numel(), device="cuda"), labels[part]
        loss[part] = -logp[picked]
        if c["train"]:
            dz = torch.exp(logp)
            dz[picked] -= 1.0
            dz *= s["dloss"][part].double().unsqueeze(1)
            dx[part] = torch.mm(dz, w)
            dw.addmm_(dz.t(), x)
    return {"loss": loss, "dx": dx, "dw": dw} if c["train"] else {"loss": loss}


def _exact_orth(c, s):
    out = []
    for g in s["g"].double():
        x = g / (torch.linalg.vector_norm(g) + EPS["orth"])
        for _ in range(c["steps"]):  # from the side that the plain form does not take where it is no larger
            if c["rows"] > c["cols"]:
                gram = x.t().mm(x)
                x = A * x + x.mm(B * gram + C * gram.mm(gram))
            else:
                gram = x.mm(x.t())
                x = A * x + B * gram.mm(x) + C * gram.mm(gram.mm(x))
        out.append(x)
    return {"out": torch.stack(out)}


def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "loss": _exact_loss, "orth": _exact_orth}[case["op"]](case, s)
