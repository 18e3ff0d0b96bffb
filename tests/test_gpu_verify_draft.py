"""ra_verify_draft against its definition in 64 bits: the answers are whole numbers and have to be equal.  The
probabilities here are such that no two candidates of a sequence are within 1e-5 of each other (checked), so that the
kernel's one rounded quotient cannot change the order; ties are made exactly equal."""
import pytest
import torch

import operator_helpers as H
from paper_2502_19864_gb300 import ringada as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def plain(target, draft, tokens, uniform, noise, n_drafted):
    """One sequence, in 64 bits, token by token."""
    V = target.shape[1]
    t, d = (x.double().nan_to_num(nan=0.0).clamp(min=0) for x in (target, draft))
    n = 0
    while n < n_drafted:
        x = int(tokens[n])
        if not (0 <= x < V and float(uniform[n]) * float(d[n, x]) < float(t[n, x])):
            break
        n += 1
    r = t[n] if n == n_drafted else (t[n] - d[n]).clamp(min=0)
    if float(r.max()) <= 0:
        r = t[n]
    score = (r / noise.double()).nan_to_num(nan=0.0)
    top = float(score.max())
    best = torch.nonzero(score == top)[0, 0]
    second = score[score < top]
    apart = not len(second) or top == 0 or float(second.max()) < top * (1 - 1e-5)
    return n, [int(x) for x in tokens[:n]] + [int(best)], apart


def check(dtype, target, draft, tokens, uniform, noise, n_drafted=None):
    B, K1, V = target.shape
    K = K1 - 1
    dt = H.DT[dtype]
    pad = 3  # rows that are not next to each other
    t = torch.full((B, K1, V + pad), 9.0, dtype=dt, device="cuda")
    t[..., :V] = target.to(dt)
    d = torch.full((B, max(K, 1), V + pad), 9.0, dtype=dt, device="cuda")
    d[:, :K, :V] = draft.to(dt)
    tok, u, e = tokens.to(torch.int32).cuda(), uniform.float().cuda(), noise.float().cuda()
    nd = torch.tensor(n_drafted, dtype=torch.int32, device="cuda") if n_drafted is not None else None
    accepted = torch.full((B,), 99, dtype=torch.int32, device="cuda")
    out = torch.full((B, K1), 99, dtype=torch.int32, device="cuda")
    a = R.ra_verify_draft_args(target_dev=t.data_ptr(), target_stride=V + pad, draft_dev=d.data_ptr(), draft_stride=V + pad,
                               tokens_dev=tok.data_ptr(), n_drafted_dev=nd.data_ptr() if nd is not None else None,
                               uniform_dev=u.data_ptr(), noise_dev=e.data_ptr(), accepted_dev=accepted.data_ptr(),
                               out_tokens_dev=out.data_ptr(), batch=B, n_draft=K, vocab=V, dtype=H.RA[dtype])
    ws = H.workspace(R.ra_verify_draft_workspace_bytes(a))
    a.workspace_dev, a.workspace_bytes = ws.data_ptr(), ws.numel()
    seen = []
    for again in range(2):  # (the second call finds the workspace as the first left it)
        R.ra_verify_draft(a)
        torch.cuda.synchronize()
        assert (ws == 0).all()
        for b in range(B):
            limit = K if n_drafted is None else min(max(n_drafted[b], 0), K)
            n, row, apart = plain(t[b, :, :V], d[b, :, :V], tok[b], u[b], e[b], limit)
            assert apart, "the test's own candidates are too near to each other"
            assert accepted[b].item() == n, (b, accepted[b].item(), n)
            assert out[b].tolist() == row + [-1] * (K1 - len(row)), (b, n)
            seen.append(n)
        accepted.fill_(99)
        out.fill_(99)
    return seen


def model_like(B, K, V, seed, gap=0.7):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((B, K + 1, V), generator=g) * 3
    target, draft = z.softmax(-1), (z[:, :K] + gap * torch.randn((B, K, V), generator=g)).softmax(-1)
    tokens = (draft / torch.empty((B, K, V)).exponential_(generator=g)).argmax(-1) if K else torch.zeros((B, 0))
    return target, draft, tokens, torch.rand((B, K), generator=g), torch.empty((B, V)).exponential_(generator=g).clamp(min=1e-30)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K,V", [(1, 4, 32000), (7, 1, 50001), (64, 8, 999), (3, 5, 1), (2, 3, 2), (5, 4, 2047), (5, 4, 2049),
                                   (2, 40, 130), (400, 2, 33), (1, 0, 4097)])
def test_batches(dtype, B, K, V):
    check(dtype, *model_like(B, K, V, 3))


def test_all_counts_appear():
    seen = check("f32", *model_like(200, 4, 300, 5, gap=0.4))
    assert set(seen) == {0, 1, 2, 3, 4}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ragged_drafts(dtype):
    check(dtype, *model_like(6, 4, 700, 4), n_drafted=[4, 0, 2, 1, 9, -3])


def test_draft_equal_to_target_and_no_residual():
    target, draft, tokens, u, e = model_like(4, 3, 500, 6)
    draft = target[:, :3].clone()  # every token stands for u < 1 ...
    assert set(check("f32", target, draft, tokens, u, e)) == {3}
    u[:, 1] = 1.0                  # ... and falls for u = 1, with nothing left of p - q: a sample of p
    assert set(check("f32", target, draft, tokens, u, e)) == {1}


def test_zero_probabilities():
    target, draft, tokens, u, e = model_like(3, 2, 64, 7)
    draft[0, 0, tokens[0, 0].long()] = 0       # drafted although the draft gave it none: stands if the target has any
    target[1, 0, tokens[1, 0].long()] = 0      # the target has none: falls, for u = 0 too
    u[1, 0] = 0.0
    target[2] = 0                              # a row of nothing: the lowest token
    check("f32", target, draft, tokens, u, e)


def test_ties_go_to_the_lowest_token():
    V = 20000
    target, draft = torch.zeros(2, 2, V), torch.zeros(2, 1, V)
    target[:, :, [19999, 7001, 12345]] = 0.25
    tokens, u, e = torch.tensor([[5], [7001]]), torch.full((2, 1), 0.5), torch.ones(2, V)
    draft[1, 0, 7001] = 0.25
    assert check("f32", target, draft, tokens, u, e)[:2] == [0, 1]


def test_tokens_outside_the_vocabulary_and_nan():
    target, draft, tokens, u, e = model_like(4, 3, 300, 8)
    tokens[0, 1], tokens[1, 0], tokens[2, 2] = 300, -1, 1 << 30
    target[3, :, ::7] = float("nan")
    draft[3, :, ::5] = float("nan")
    check("f32", target, draft, tokens, u, e)


def test_the_samples_follow_the_target():
    """400000 one-draft verifications: what comes out first is distributed as the target, whatever the draft.  A count
    of n p has a standard deviation below sqrt(n p): six of them, over 12 tokens."""
    B, V = 400000, 12
    g = torch.Generator(device="cuda").manual_seed(11)
    p, q = (torch.randn(V, generator=g, device="cuda").softmax(-1) for _ in "pq")
    tokens = torch.multinomial(q, B, replacement=True, generator=g).to(torch.int32)
    u, e = torch.rand(B, generator=g, device="cuda"), torch.empty((B, V), device="cuda").exponential_(generator=g)
    t, d = p.expand(B, 2, V).contiguous(), q.expand(B, 1, V).contiguous()
    accepted, out = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, 2), dtype=torch.int32, device="cuda")
    a = R.ra_verify_draft_args(target_dev=t.data_ptr(), target_stride=V, draft_dev=d.data_ptr(), draft_stride=V,
                               tokens_dev=tokens.data_ptr(), uniform_dev=u.data_ptr(), noise_dev=e.data_ptr(),
                               accepted_dev=accepted.data_ptr(), out_tokens_dev=out.data_ptr(), batch=B, n_draft=1, vocab=V,
                               dtype=R.RA_F32)
    ws = H.workspace(R.ra_verify_draft_workspace_bytes(a))
    a.workspace_dev, a.workspace_bytes = ws.data_ptr(), ws.numel()
    R.ra_verify_draft(a)
    counts = torch.bincount(out[:, 0].long(), minlength=V).double()
    assert ((counts - B * p.double()).abs() <= 6 * (B * p.double()).sqrt()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("uniform", [0.5, 0.9, 1 - 2.0 ** -24])
def test_acceptance_of_the_smallest_probabilities(dtype, uniform):
    """u q < p where u q - p is far below what 32 bits hold: equal probabilities stand for every u < 1."""
    target, draft, tokens, u, e = model_like(5, 3, 200, 9)
    least = 2.0 ** -149 if dtype == "f32" else 2.0 ** -133
    for b, k in enumerate([1, 2, 3, 7, 100]):
        target[b, :3].scatter_(1, tokens[b, :, None], k * least)
        draft[b].scatter_(1, tokens[b, :, None], k * least)
    u.fill_(uniform)
    assert set(check(dtype, target, draft, tokens, u, e)) == {3}


def test_acceptance_with_small_random_numbers():
    """u q of two ordinary numbers just below and just above a p that 32 bits barely hold."""
    target, draft, tokens, u, e = model_like(2, 1, 200, 10)
    target[:, :1].scatter_(2, tokens[..., None], 2.0 ** -149)
    draft.scatter_(2, tokens[..., None], 2.0 ** -10)
    u[0], u[1] = 2.0 ** -140, 2.0 ** -139 * (1 + 2.0 ** -20)
    assert check("f32", target, draft, tokens, u, e)[:2] == [1, 0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drafted", [0, 1])
def test_race_of_the_smallest_probabilities(dtype, drafted):
    """Rows whose probabilities are all below what 32 bits hold to full precision, with noise that makes their quotients
    ordinary numbers: later tokens win by 1 % to 80 % over earlier ones, at many distances."""
    least = 2.0 ** -149 if dtype == "f32" else 2.0 ** -133
    behind = [1, 32, 64, 128, 128, 128, 256, 512, 640, 1024, 2048]
    B, V = len(behind), 3000
    target, noise = torch.zeros(B, drafted + 1, V), torch.full((B, V), 1.0)
    for b, far in enumerate(behind):
        for i, share in enumerate((1.0, 0.99, 0.9, 0.55)[:4 - b % 3]):
            v = 7 + b + i * far if i * far < 2900 else 2950 + b + i
            target[b, :, v] = least
            noise[b, v] = share * 2.0 ** -30
    draft, tokens, u = torch.zeros(B, drafted, V), torch.zeros(B, drafted), torch.full((B, drafted), 0.5)
    assert set(check(dtype, target, draft, tokens, u, noise)) == {0}
