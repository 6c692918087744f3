"""Beam search where a step cannot be done: it is done later, or refused, and what was found before stays."""
import pytest

import decode_ref as D
from test_gpu_branching import B, held, model  # noqa: F401

pytestmark = pytest.mark.gpu
VOCAB = 40


def search(pages, max_tokens=60, end=-1, sequences=6, beams=3):
    import torch
    from paper_2401_10652_amd.decode import BeamSearch
    m, _ = model("f32", sequences, max_tokens, pages=pages)
    embedding, head = (torch.from_numpy(D.normal((VOCAB, 128), 60 + i, s)).float() for i, s in enumerate((1.0, 0.4)))
    return BeamSearch(m, embedding, head, beams, end=end)


PROMPTS = [list(range(14)), list(range(30, 0, -1))]                    # (two tokens before a page's end, both)


def state(s):
    return s.scores.clone(), s.logits.clone(), s.found(), list(s.model.lengths)


def equal(a, b):
    import torch
    return all(torch.equal(x, y) if torch.is_tensor(x) else x == y for x, y in zip(a, b))


@pytest.mark.parametrize("end", [-1, 7])
def test_a_step_that_runs_dry_is_done_later(B, end):  # noqa: F811
    """The fork succeeds, the next tokens' pages are missing: called again, the step goes on from there."""
    import torch
    s, other = search(14, end=end), search(60, end=end)
    for a in (s, other):
        a.start(PROMPTS)
        a.step(), a.step()
    assert equal(state(s), state(other)) and s.model.lengths == [16] * 3 + [32] * 3
    before, kept = state(s), (s.model.uses == 0).int()
    s.model.uses += kept                                                # somebody else has the pages that are left
    for _ in range(3):
        with pytest.raises(RuntimeError, match="pages are missing"):
            s.step()
        assert s.scores is not None and s.found() == before[2]
    s.model.uses -= kept
    for _ in range(4):
        got, want = s.step(), other.step()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and equal(state(s), state(other))
        held(s.model)


def test_a_fork_that_runs_dry_is_done_later(B):  # noqa: F811
    import torch
    s, other = search(14), search(60)
    for a in (s, other):
        a.start(PROMPTS)
    kept = (s.model.uses == 0).int()
    s.model.uses += kept
    s.model.ends = [9] * 6                                              # (so that pages are asked for)
    before = state(s)
    for _ in range(2):
        with pytest.raises(RuntimeError, match="pages are missing"):
            s.step()
        assert equal(state(s), before)
    s.model.uses -= kept
    for _ in range(3):
        got, want = s.step(), other.step()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and equal(state(s), state(other))


def test_the_end_of_the_table(B):  # noqa: F811
    """Tokens past the cache's are refused, and a new search starts."""
    s, other = search(60, 33), search(60, 33)
    for a in (s, other):
        a.start(PROMPTS)
        a.step(), a.step(), a.step()
    before = state(s)
    for _ in range(2):
        with pytest.raises(ValueError, match="33"):
            s.step()
        assert s.found() == before[2]
    for a in (s, other):
        a.start([[1, 2], [3]])
        a.step(), a.step()
    assert equal(state(s), state(other))


def test_a_start_that_runs_dry(B):  # noqa: F811
    """The sequences of before are gone, so there is no search until one starts."""
    s, other = search(14), search(60)
    fresh = search(14)
    with pytest.raises(ValueError, match="start"):
        fresh.step()
    for a in (s, other):
        a.start(PROMPTS)
        a.step()
    with pytest.raises((RuntimeError, ValueError)):
        s.start([[1] * 300, [2] * 4])                                   # (more than the table holds)
    with pytest.raises(ValueError, match="start"):
        s.step()
    assert s.found() == [[], []]
    for a in (s, other):
        a.start(PROMPTS)
        a.step(), a.step()
    assert equal(state(s), state(other))


@pytest.mark.parametrize("bad", [VOCAB, VOCAB + 1000, -1, 1 << 40])
def test_tokens_outside_the_vocabulary(B, bad):  # noqa: F811
    """Refused before anything changes: the embedding has no such row."""
    s = search(14)
    s.start(PROMPTS)
    s.step()
    before = state(s)
    for prompts in ([[bad], [1]], [[1, 2], [3, 4, bad, 5]]):
        with pytest.raises(ValueError, match="40"):
            s.start(prompts)
        assert equal(state(s), before)
    s.step()
    s.start([[0], [VOCAB - 1]])
    s.step()
