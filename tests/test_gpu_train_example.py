"""The example that trains all of a decoder's weights: a run of the operators together, its gradients and its update against
64 bits."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F = torch.nn.functional


@pytest.fixture(scope="module")
def ex():
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "train.py")
    spec = importlib.util.spec_from_file_location("train_example", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def loss64(ex, m, tokens, labels):
    """The same loss in 64 bits by plain torch, on weights of its own."""
    w = {id(t): t.detach().double().requires_grad_() for t in m.matrices() + m.others()}
    emb = w[id(m.emb)]

    def norm(x, gain):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + ex.EPS) * gain

    def turn(x):
        c, s = m.rope.double()[:x.shape[1], None].chunk(2, -1)
        lo, hi = x.chunk(2, -1)
        return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)
    x = F.embedding(tokens, emb)
    S = tokens.shape[1]
    i, j = torch.arange(S, device="cuda")[:, None], torch.arange(S, device="cuda")
    seen = (j <= i) & ((i - j < m.window) | (j < m.sinks))
    for layer in m.layers:
        g = {k: w[id(t)] for k, t in layer.items()}
        q, k, v = (norm(x, g["before"]) @ g["qkv"].T).unflatten(-1, (-1, m.D)).split([m.H, m.KV, m.KV], 2)
        q, k, v = (t.transpose(1, 2) for t in (turn(q), turn(k), v))
        k, v = (t.repeat_interleave(m.H // m.KV, 1) for t in (k, v))
        p = (q @ k.transpose(2, 3) / math.sqrt(m.D)).masked_fill(~seen, -math.inf).softmax(-1)
        x = x + (p @ v).transpose(1, 2).flatten(2) @ g["o"].T
        x = x + F.silu(norm(x, g["between"]) @ g["up"].T) @ g["down"].T
    z = norm(x, w[id(m.last)]) @ emb.T
    return F.cross_entropy(z.flatten(0, 1), labels.flatten().long(), ignore_index=-1), w


def test_gradients(ex):
    """Of every weight, up to the bf16 rounding of what passes between operators on the way there and back: some sixty
    roundings of 2^-8 relative to a row, added up without correlation: 3 %."""
    m = ex.Decoder(2, seed=3, window=40)
    tokens = torch.randint(0, m.V, (3, 130), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    labels = ex.next_tokens(tokens)
    labels[0, :50] = -1
    loss = m.loss(tokens, labels)
    loss.backward()
    want, w = loss64(ex, m, tokens, labels)
    want.backward()
    assert abs(loss.item() - want.item()) < 3e-2 * want.item()
    for t in m.matrices() + m.others():
        g = w[id(t)].grad
        assert (t.grad.double() - g).norm() <= 3e-2 * g.norm(), tuple(t.shape)
    assert int(m.err) == 0


def test_update(ex):
    """The matrices move by the orthogonalised momentum: singular values of the update as the polynomial has them."""
    m = ex.Decoder(1, seed=2)
    tokens = torch.randint(0, m.V, (2, 100), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    m.loss(tokens, ex.next_tokens(tokens)).backward()
    muon = ex.Muon(m.matrices(), 1.0, m.err)
    for w in m.matrices():
        got = ex.orthogonalize((1.9 * w.grad.float()).to(ex.BF16)[None], m.err)[0].double()
        x = (1.9 * w.grad.float()).to(ex.BF16).double()
        u, s, v = torch.linalg.svd(x / (x.norm() + 1e-7), full_matrices=False)
        for _ in range(5):
            s = s * (3.4445 - 4.775 * s ** 2 + 2.0315 * s ** 4)
        want = (u * s) @ v
        # the output's rounding, and 2^-16 of 17-bit operands raised 3.4445^4 = 141-fold along the smallest singular values
        assert (got - want).norm() <= (2.0 ** -8 + 141 * 2.0 ** -16) * want.norm()
    before = [w.detach().clone() for w in m.matrices()]
    muon.step()
    assert all(bool(torch.isfinite(w).all()) and not torch.equal(w, b) for w, b in zip(m.matrices(), before))


def test_runs(ex):
    m = ex.Decoder(1, seed=4)
    losses = ex.train(m, ex.text(2, 60, m.V), 4)
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses) and int(m.err) == 0
