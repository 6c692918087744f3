"""A model's lengths set back where sequences share pages: what one writes again reaches no other."""
import pytest

from test_gpu_branching import B, held, model  # noqa: F401

pytestmark = pytest.mark.gpu


def pair(pages=40, first=40, sequences=4):
    """A model whose first sequence has read `first` tokens and gone on as the first three, and one whose sequences read them by themselves."""
    m, x = model("f32", sequences, 130, pages=pages)
    own, _ = model("f32", sequences, 130)
    counts = lambda b: [first if i == b else 0 for i in range(sequences)]  # noqa: E731
    m.forward(x[:first], counts(0))
    for b in range(3):
        own.forward(x[:first], counts(b))
    m.fork([0, 0, 0] + [-1] * (sequences - 3))
    assert m.lengths == own.lengths
    return m, own, x


def same(m, own, rows, counts):
    import torch
    assert torch.equal(m.forward(rows, counts), own.forward(rows, counts))
    assert m.lengths == own.lengths
    held(m)


def back(models, lengths):
    for m in models:
        for b, n in lengths.items():
            m.lengths[b] = n


@pytest.mark.parametrize("to", [0, 1, 15, 16, 20, 31, 32, 33])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_behind_a_fork(B, which, to):  # noqa: F811
    """One sequence goes back into what it shares (or up to it), and all read on: the same bits as sequences with pages of their own."""
    m, own, x = pair()
    back((m, own), {which: to})
    for at in range(50, 62, 3):
        same(m, own, x[at:at + 3], [1, 1, 1, 0])
    same(m, own, x[70:123], [17, 2, 34, 0])


def test_several_at_once_and_again(B):  # noqa: F811
    m, own, x = pair()
    back((m, own), {0: 20, 1: 20, 2: 5})                                # (whichever is first, one of them keeps the pages that no other has any more)
    same(m, own, x[50:70], [10, 4, 6, 0])
    back((m, own), {0: 3, 2: 0})
    same(m, own, x[60:100], [30, 9, 1, 0])
    back((m, own), {1: 33})
    same(m, own, x[10:13], [1, 1, 1, 0])
    m.release([0, 1, 2])
    assert held(m) == 0


def test_sequences_that_read_nothing_stay(B):  # noqa: F811
    """A sequence that was set back and has no rows in a call writes nothing, and may go forward again."""
    m, own, x = pair()
    pages = held(m)
    back((m, own), {1: 20})
    same(m, own, x[50:52], [1, 0, 1, 0])
    assert held(m) == pages
    back((m, own), {1: 40})
    same(m, own, x[52:58], [2, 2, 2, 0])
    assert held(m) == pages


@pytest.mark.parametrize("to", [16, 20, 35])
def test_fork_of_a_sequence_that_was_set_back(B, to):  # noqa: F811
    """Its first child does not write into what others have either."""
    m, own, x = pair()
    back((m, own), {1: to})
    m.fork([0, 1, 2, 1])
    for c in own.caches:
        for t in c.keep:
            t4 = t.view(4, -1, *t.shape[1:])
            t4.copy_(t4[[0, 1, 2, 1]].clone())
    own.lengths = [40, to, 40, to]
    for at in range(50, 74, 4):
        same(m, own, x[at:at + 4], [1] * 4)


def test_parents_on_the_device(B):  # noqa: F811
    import torch
    m, own, x = pair()
    back((m, own), {0: 18, 1: 18, 2: 18, 3: 0})
    m.fork(torch.tensor([1, 0, 2, -1], dtype=torch.int32, device="cuda"), [18, 18, 18, 0])
    for at in range(50, 62, 3):
        same(m, own, x[at:at + 3], [1, 1, 1, 0])


def test_from_a_graph(B):  # noqa: F811
    import torch
    m, own, x = pair()
    one, other = m.step_graph(), own.step_graph()
    for at in range(50, 90, 4):
        if at == 54:
            back((m, own), {1: 20})
        if at == 62:
            back((m, own), {0: 8, 2: 31})
        assert torch.equal(one(x[at:at + 4]), other(x[at:at + 4]))
        assert m.lengths == own.lengths
        held(m)


def test_pages_run_out(B):  # noqa: F811
    """Without a page for the copy the call is refused, and nothing changes."""
    import torch
    m, own, x = pair(pages=5)                                           # (two whole pages that are shared, and a part for each of three)
    back((m, own), {0: 20, 1: 20, 2: 20})
    same(m, own, x[50:53], [1, 1, 1, 0])                                # (each of the first two gives up its part for a copy; of the third the page is its own by then)
    assert held(m) == 5
    m, own, x = pair(pages=4, first=32)
    same(m, own, x[50:52], [1, 1, 0, 0])
    back((m, own), {2: 20})
    table, uses = m.table.clone(), m.uses.clone()
    for call in (lambda: m.forward(x[60:61], [0, 0, 1, 0]), lambda: m.fork([0, 1, 2, 2]), lambda: m.step_graph()(x[:4])):
        with pytest.raises(RuntimeError, match="pages are missing"):
            call()
        assert torch.equal(m.table, table) and torch.equal(m.uses, uses) and m.lengths == [33, 33, 20, 0]
    same(m, own, x[60:62], [1, 1, 0, 0])
    m.release([0])
    own.lengths[0] = 0
    same(m, own, x[70:73], [0, 1, 2, 0])


def test_parents_on_the_host(B):  # noqa: F811
    """As tensors too, of either kind of number; lengths, where they are said, have to be the parents'."""
    import torch
    for kind in (torch.int32, torch.int64):
        for said in (None, [40, 40, 40, 40], [40, 40, 40, 0]):
            m, own, x = pair()
            parents = torch.tensor([1, 0, 2, 2 if said and said[3] else -1], dtype=kind)
            m.fork(parents, said)
            same(m, own, x[50:53], [1, 1, 1, 0]) if not said or not said[3] else m.forward(x[50:54], [1] * 4)
            held(m)
    m, own, x = pair()
    table = m.table.clone()
    for parents, lengths in (([0, 1, 2, -1], [20, 40, 40, 0]), ([0, 1, 2, 2], [40, 40, 40, 41]), ([0, 1, 2, 4], [40] * 4), ([0, 1, 2], [40] * 3), ([0, 1, 2, 0], [40] * 3)):
        for kind in (list, torch.tensor):
            with pytest.raises(ValueError):
                m.fork(kind(parents), lengths)
    on_device = torch.tensor([0, 1, 2, 2], device="cuda")
    with pytest.raises(TypeError):
        m.fork(on_device, [40] * 4)
    with pytest.raises(ValueError):
        m.fork(on_device.int()[:3], [40] * 4)
    with pytest.raises(ValueError):
        m.fork(on_device.int(), [40] * 3)
    assert torch.equal(m.table, table) and m.lengths == [40, 40, 40, 0]
    same(m, own, x[50:53], [1, 1, 1, 0])


@pytest.mark.parametrize("graph", [False, True])
def test_a_call_that_fails_behind_a_length_that_was_set_back(B, graph):  # noqa: F811
    """What it gave up, or wrote again, is not taken for the tokens of before."""
    m, own, x = pair(pages=7, first=48)                                 # (three whole pages that are shared)
    step = m.step_graph()
    back((m, own), {1: 20})
    if not graph:                                                       # a page for the copy and three for others, of which there are four
        with pytest.raises(RuntimeError, match="pages are missing"):
            m.forward(x[50:110], [20, 1, 20, 19])
    else:
        m.uses[4:] += 1                                                 # (somebody else has all but one)
        with pytest.raises(RuntimeError, match="pages are missing"):
            step(x[50:54])
        m.uses[4:] -= 1
    assert m.lengths == [48, 20, 48, 0]
    back((m,), {1: 48})
    with pytest.raises(ValueError, match="20 tokens"):
        m.forward(x[60:61], [0, 1, 0, 0])
    with pytest.raises(ValueError, match="20 tokens"):
        m.fork([0, 1, 2, 3])
    back((m,), {1: 20})
    same(m, own, x[60:63], [0, 3, 0, 0])
    same(m, own, x[70:73], [1, 1, 1, 0])


def test_lengths_that_a_sequence_does_not_have(B):  # noqa: F811
    m, own, x = pair()
    step = m.step_graph()
    for b, n in ((0, 41), (1, -1), (3, 1), (2, 100)):
        was = m.lengths[b]
        back((m,), {b: n})
        for call in (lambda: m.forward(x[:1], [int(i == b) for i in range(4)]), lambda: step(x[:4]), lambda: m.fork([0, 1, 2, 3])):
            with pytest.raises(ValueError, match=f"{was} tokens"):
                call()
        back((m,), {b: was})
    back((m, own), {0: 30})
    same(m, own, x[50:52], [0, 2, 0, 0])
    back((m, own), {0: 40})
    same(m, own, x[52:55], [1, 1, 1, 0])
