"""A model that reads on behind a window, branches and searches: the window's attention, the page books and the selection together, as a serving program uses them."""
import numpy as np
import pytest

import decode_ref as D
import test_gpu_beam
import test_gpu_decoder as T
import test_gpu_window
from paper_2401_10652_amd import inputs as I

pytestmark = pytest.mark.gpu
CFG = {dtype: I.TransformerConfig("decoder_2l", 11, 2, 60, 128, 4, 256, True, dtype, None, batch=3) for dtype in ("f32", "bf16")}


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2401_10652_amd import binding
    return binding


def model(dtype, sequences, max_tokens, **more):
    import torch
    from paper_2401_10652_amd.decode import Decoder
    x, layers = I.transformer_inputs(CFG[dtype], bias_std=0.1, ln_jitter=0.1)
    m = Decoder(CFG[dtype], layers, sequences, max_tokens, page=16, group=32, **more)
    return m, torch.as_tensor(x, device="cuda").to(m.dtype)


def held(m):
    """uses has every place that names a page, and no other."""
    table, uses = m.table.cpu().numpy(), m.uses.cpu().numpy()
    assert np.array_equal(np.bincount(table[table >= 0], minlength=len(uses)), uses)
    return int((uses > 0).sum())


@pytest.mark.parametrize("dtype,tol", [("f32", 12 * 2.0 ** -12), ("bf16", 12 * 2.0 ** -8)])      # (as the model without a window: two layers of six operators)
def test_model_behind_a_window(B, monkeypatch, dtype, tol):
    """Each call against the model in 64 bits; pages come back, and no more of them are held than the window, the sinks and the call's rows need."""
    window, sinks = 21, 5
    m, x = model(dtype, 3, 400, window=window, sinks=sinks, pages=14)
    monkeypatch.setattr(D, "attention", lambda q, cache, b, first, length, group, causal, scale: test_gpu_window.attention(q, cache, b, length, group, window, sinks, scale))
    at, step = 0, None
    for counts in ([40, 7, 0], [1, 1, 1], [5, 1, 33], [1, 1, 0], [0, 0, 1], [37, 16, 1], [1, 1, 1], [1, 1, 1], [10, 15, 3]):
        rows = x[at:at + sum(counts)]
        at += sum(counts)
        if counts == [1, 1, 1] and at > 150:
            step = step or m.step_graph()
            y = T.host(step(rows))
        else:
            y = T.host(m.forward(rows, counts))
        ref = T.reference(m, T.host(rows), counts, m.lengths, tol * 4)
        assert np.abs(y - ref).max() <= tol * np.abs(ref).max(), (counts, np.abs(y - ref).max() / np.abs(ref).max())
        assert held(m) <= sum(1 + (window + n + 14) // 16 + 1 for n in counts)
    assert m.lengths == [96, 43, 41] and step is not None
    m.release([0, 2])
    assert m.lengths == [0, 43, 0] and held(m) <= 4
    with pytest.raises(RuntimeError, match="pages are missing"):
        m.forward(x, [170, 5, 5])
    assert m.lengths == [0, 43, 0]
    m.release([0, 1, 2])
    assert held(m) == 0
    m.forward(x[:60], [20, 20, 20])
    held(m)


def test_forks_read_on_as_models_of_their_own(B):
    """The same bits as a model that read each sequence by itself; also after pages moved, and from a graph."""
    import torch
    m, x = model("f32", 4, 130, pages=26)
    own, _ = model("f32", 4, 130)
    read = lambda model, at, counts: model.forward(x[at:at + sum(counts)], counts)  # noqa: E731
    read(m, 0, [37, 16, 0, 0])
    read(own, 0, [37, 16, 0, 0])
    read(own, 0, [0, 0, 37, 16])
    m.fork([0, 1, 0, 1])
    assert m.lengths == [37, 16, 37, 16] and held(m) == 3 + 1 + 1                       # (the second prompt's one page is full, and shared)
    for at in range(53, 53 + 4 * 13, 4):
        assert torch.equal(read(m, at, [1] * 4), read(own, at, [1] * 4))
    m.fork([2, 2, -1, 3])
    for c, o in zip(m.caches, own.caches):                                              # the other model's rows move whole
        for t, u in zip(c.keep, o.keep):
            u4 = u.view(4, -1, *u.shape[1:])
            u4.copy_(u4[[2, 2, 2, 3]].clone())
    own.lengths = [50, 50, 0, 29]
    assert m.lengths == own.lengths
    held(m)
    rows = x[110:140]
    assert torch.equal(m.forward(rows, [13, 2, 9, 6]), own.forward(rows, [13, 2, 9, 6]))
    before = held(m)
    m.release([1])
    own.lengths[1] = 0
    assert m.compact().item() == held(m) < before and int(m.table.max()) == held(m) - 1
    rows = x[10:32]
    assert torch.equal(m.forward(rows, [1, 16, 1, 4]), own.forward(rows, [1, 16, 1, 4]))
    one, other = m.step_graph(), own.step_graph()
    for at in range(0, 24, 4):
        assert torch.equal(one(x[at:at + 4]), other(x[at:at + 4]))
        if at == 8:
            m.fork([0, 1, 2, 3])                                                        # (as they are; every page that is shared is one's own again)
            m.compact()
        if at == 12:
            assert torch.equal(m.forward(x[50:54], [1] * 4), own.forward(x[50:54], [1] * 4))
    held(m)


def test_lengths_set_back_hold_their_pages(B):
    """Places behind a length that was set back name pages still, which are counted where pages run out, and used again."""
    m, x = model("f32", 2, 130, pages=6)
    m.forward(x[:80], [80, 0])
    m.lengths = [10, 0]
    with pytest.raises(RuntimeError, match="1 pages are missing"):
        m.forward(x[:30], [10, 20])
    assert m.lengths == [10, 0] and held(m) == 6
    m.forward(x[:40], [40, 0])
    assert m.lengths == [50, 0] and held(m) == 6
    m.release([0])
    m.forward(x[:60], [30, 30])


def test_forks_want_pages(B):
    m, x = model("f32", 4, 130, pages=5)
    m.forward(x[:40], [40, 0, 0, 0])
    m.fork([0, 0, 0, -1])
    assert m.lengths == [40, 40, 40, 0] and held(m) == 5
    table, uses = m.table.clone(), m.uses.clone()
    with pytest.raises(RuntimeError, match="1 pages are missing"):
        m.fork([0, 1, 2, 0])
    assert m.lengths == [40, 40, 40, 0] and (m.table == table).all() and (m.uses == uses).all()
    for bad in ([0, 1, 2], [0, 1, 2, 4], [-2, 0, 0, 0]):
        with pytest.raises(ValueError):
            m.fork(bad)
    with pytest.raises(ValueError):
        m.release([4])
    own, _ = model("f32", 2, 130)
    for call in (lambda: own.fork([0, 1]), lambda: own.release([0]), own.compact):
        with pytest.raises(ValueError, match="own pages"):
            call()


def test_a_fork_that_fails_leaves_the_sequences(B):
    """Pages that it would have freed and taken for copies are still a sequence's."""
    import torch
    m, x = model("f32", 4, 130, pages=5)
    own, _ = model("f32", 4, 130)
    for a in (m, own):
        a.forward(x[:60], [40, 20, 0, 0])
    before = [t[:5].clone() for c in m.caches for t in c.keep]
    with pytest.raises(RuntimeError, match="1 pages are missing"):
        m.fork([0, 0, 0, 0])
    assert all(torch.equal(t[:5], u) for t, u in zip((t for c in m.caches for t in c.keep), before))
    assert m.lengths == [40, 20, 0, 0] and held(m) == 5
    assert torch.equal(m.forward(x[60:68], [3, 5, 0, 0]), own.forward(x[60:68], [3, 5, 0, 0]))


@pytest.mark.parametrize("end", [-1, 7])
def test_beam_search(B, end):
    """Every step's choice against the definition in 64 bits, from logits of a model that read each beam's tokens by itself."""
    import torch
    from paper_2401_10652_amd.decode import BeamSearch
    vocab, beams, prompts = 40, 3, [[3, 11, 5, 0, 39, 2, 2, 8, 9, 21, 33, 4, 17, 1, 30], [6], [25, 7, 7, 31, 12, 13, 14, 15, 16, 18, 20, 22, 24, 26, 28, 30, 32]]
    m, _ = model("f32", 9, 60, pages=40)
    own, _ = model("f32", 9, 60)
    embedding, head = (torch.from_numpy(D.normal((vocab, 128), 60 + i, s)).float() for i, s in enumerate((1.0, 0.4)))
    bias = torch.from_numpy(D.normal((vocab,), 63, 0.5)).float()
    search = BeamSearch(m, embedding, head, beams, bias, end)
    search.start(prompts, stretch=6)
    table = embedding.cuda()
    tokens = [[p[:], [], []] for p in prompts]                          # (the first beam alone is there)
    scores, ended = np.full((3, beams), -np.inf), np.zeros((3, beams), int)
    scores[:, 0] = 0
    for step in range(12):
        # the other model reads every beam anew: prompts in the same stretches, then token by token
        own.lengths = [0] * 9
        last = torch.zeros((9, 128), device="cuda")
        longest = max(map(len, prompts))
        parts = [[t[b][:len(p)][at:at + 6] for p, t in zip(prompts, tokens) for b in range(beams)] for at in range(0, longest, 6)]
        parts += [[t[b][len(p) + i:len(p) + i + 1] for p, t in zip(prompts, tokens) for b in range(beams)] for i in range(step)]
        for part in parts:
            ids = sum(part, [])
            if not ids:
                continue
            y, at = own.forward(table[torch.tensor(ids, device="cuda")], [len(q) for q in part]), 0
            for b, q in enumerate(part):
                at += len(q)
                if q:
                    last[b] = y[at - 1]
        codes, scale, zero = search.head
        logits = torch.empty((9, vocab), device="cuda")
        B.ac_op_linear_w4(last, codes, scale, logits, 32, zero=zero, bias=search.bias)
        alive = [b for b in range(9) if scores[b // 3, b % 3] > -np.inf]
        # (products of other numbers of rows add up in another order: the model's tolerance)
        assert (logits - search.logits)[alive].abs().max() <= 12 * 2.0 ** -12 * logits[alive].abs().max()
        want, near = test_gpu_beam.select(search.logits.double().cpu().numpy().reshape(3, beams, vocab), scores, ended if end >= 0 else None, end, beams)
        assert (near > 2.0 ** -20).all()
        parent, token = search.step()
        assert np.array_equal(parent.cpu().numpy(), want[1]) and np.array_equal(token.cpu().numpy(), want[2])
        scores, ended = search.scores.double().cpu().numpy(), want[3]
        tokens = [[tokens[p][want[1][p, i] % 3] + [int(want[2][p, i])] for i in range(beams)] for p in range(3)]
        held(m)
    found = search.found()
    for p in range(3):
        for i, (score, got) in enumerate(found[p]):
            text = tokens[p][i][len(prompts[p]):]
            assert score == scores[p, i] and got == (text[:text.index(end) + 1] if end in text else text)
    if end >= 0:
        assert ended.any()
    with pytest.raises(ValueError):
        search.start(prompts[:2])
    with pytest.raises(ValueError):
        BeamSearch(m, embedding, head, 2)


def test_command(B, monkeypatch, capsys):
    import json
    from paper_2401_10652_amd import decode
    monkeypatch.setattr("sys.argv", ["decode", "--config", "C2", "--batch", "2", "--prompt", "200", "--stretch", "90", "--steps", "6", "--window", "70", "--sinks", "4", "--beams", "3", "--vocab", "500"])
    decode.main()
    got = json.loads(capsys.readouterr().out)
    assert got["finite"] and got["beams"] == 3 and got["beam_tokens"] == [6, 3] and got["ms_per_step"] > 0
