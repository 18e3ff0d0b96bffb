"""The example that tunes a decoder with windowed attention and answers with it: its pieces against one another."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "answer.py")
    spec = importlib.util.spec_from_file_location("answer_example", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_cache_and_prompt_agree(ex):
    """Logits of tokens fed one to five at a time are those of the whole prompt's windowed attention, up to the bf16
    rounding of each path (some twenty roundings of 2^-8 relative to a row, added up without correlation: 2 %)."""
    m = ex.Decoder(2, seed=3, window=40)
    tokens = ex.text(3, 130, m.V, seed=5)
    whole = ex.Session(m, 3, 160).step(tokens, prompt=True)
    s = ex.Session(m, 3, 160)
    parts, at = [s.step(tokens[:, :60], prompt=True)], 60
    for n in (1, 5, 1, 2, 1, 4, 56):
        parts.append(s.step(tokens[:, at:at + n]))
        at += n
    assert at == 130
    got = torch.cat(parts, 1)
    assert torch.isfinite(whole).all()
    assert (got - whole).norm() / whole.norm() < 2e-2
    assert int(m.err) == 0


def test_tuning_learns_and_answers(ex):
    """A tuned decoder continues its pattern through evictions; drafts by itself stand nearly always."""
    m = ex.Decoder(2, seed=1)
    data = ex.text(4, 200, m.V)
    losses = ex.tune(m, data, 60)
    assert losses[-1] < 0.2 < losses[0]
    answers, stood, evictions = ex.answer(m, m, data[:3, :100], 150, budget=96, limit=128)
    assert evictions >= 1 and stood > 0.9
    want = ex.text(4, 250, m.V)[:3, 100:].tolist()
    right = sum(a == b for row, w in zip(answers, want) for a, b in zip(row, w)) / 450
    assert all(len(a) == 150 and all(0 <= t < m.V for t in a) for a in answers)
    assert right > 0.5


def test_many_prompts(ex):
    """More sequences than the least workspace of the verification has room for."""
    m = ex.Decoder(1, seed=4)
    answers, _, _ = ex.answer(m, m, ex.text(18, 40, m.V, seed=6), 8)
    assert len(answers) == 18 and all(len(a) == 8 and all(0 <= t < m.V for t in a) for a in answers)


def test_sequences_that_end_early(ex):
    """Drafts that often fall: some sequences have all their tokens many rounds before others, and wait."""
    m, draft = ex.Decoder(1, seed=4), ex.Decoder(1, seed=9)
    answers, stood, _ = ex.answer(m, draft, ex.text(12, 40, m.V, seed=6), 207)
    assert all(len(a) == 207 and all(0 <= t < m.V for t in a) for a in answers)
    assert 0 < stood < 1
