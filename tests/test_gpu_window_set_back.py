"""A model's lengths set back behind a window: only as far as it still has what its rows see."""
import numpy as np
import pytest

import decode_ref as D
import test_gpu_decoder as T
import test_gpu_window
from test_gpu_branching import B, held, model  # noqa: F401

pytestmark = pytest.mark.gpu
TOL = 12 * 2.0 ** -12                                                   # (as the model without a window: two layers of six operators)


class Reader:
    """A model whose rows are compared with the same in 64 bits, from the tokens that its cache holds."""

    def __init__(self, monkeypatch, window, sinks, sequences=1, pages=60):
        self.m, self.x = model("f32", sequences, 200, window=window, sinks=sinks, pages=pages)
        self.at, self.step = 0, None
        monkeypatch.setattr(D, "attention", lambda q, cache, b, first, length, group, causal, scale: test_gpu_window.attention(q, cache, b, length, group, window, sinks, scale))

    def rows(self, n):
        self.at = self.at + n if self.at + 2 * n <= len(self.x) else 0
        return self.x[self.at:self.at + n]

    def read(self, *counts, graph=False):
        rows = self.rows(sum(counts))
        if graph:
            self.step = self.step or self.m.step_graph()
        y = T.host(self.step(rows) if graph else self.m.forward(rows, list(counts)))
        ref = T.reference(self.m, T.host(rows), list(counts), self.m.lengths, TOL * 4)
        assert np.abs(y - ref).max() <= TOL * np.abs(ref).max(), (counts, self.m.lengths, np.abs(y - ref).max() / np.abs(ref).max())
        held(self.m)

    def refused(self, call):
        import torch
        table, uses, lengths = self.m.table.clone(), self.m.uses.clone(), list(self.m.lengths)
        with pytest.raises(ValueError, match="window"):
            call()
        assert torch.equal(self.m.table, table) and torch.equal(self.m.uses, uses) and self.m.lengths == lengths


# (pages of 16 tokens, 60 tokens read one by one: the last call, behind 59, gave up the pages before token 60 - window, whole ones and but for the sinks')
@pytest.mark.parametrize("window,sinks,to,fine", [
    (4, 0, 59, True), (4, 0, 51, True), (4, 0, 50, False), (4, 0, 48, False), (4, 0, 3, False), (4, 0, 1, False), (4, 0, 0, True),
    (4, 20, 51, True), (4, 20, 50, False), (4, 20, 33, False), (4, 20, 32, True), (4, 20, 20, True), (4, 20, 2, True),
    (1, 0, 10, True), (1, 0, 47, True), (1, 5, 1, True), (2, 0, 47, False), (2, 0, 49, True), (0, 7, 30, True), (100, 0, 3, True), (28, 3, 43, False), (28, 3, 59, True)])
@pytest.mark.parametrize("graph", [False, True])
def test_one_by_one(B, monkeypatch, window, sinks, to, fine, graph):  # noqa: F811
    r = Reader(monkeypatch, window, sinks)
    for _ in range(60):
        r.m.forward(r.rows(1), [1])
    if graph:
        r.step = r.m.step_graph()
    r.m.lengths = [to]
    if not fine:
        r.refused(lambda: r.step(r.rows(1)) if graph else r.m.forward(r.rows(3), [3]))
        r.m.lengths = [60]
    for _ in range(3):
        r.read(1, graph=graph)
    r.read(20)


def test_what_one_call_read_is_all_there(B, monkeypatch):  # noqa: F811
    r = Reader(monkeypatch, 4, 0)
    r.read(60)
    for to in (5, 33, 0):
        r.m.lengths = [to]
        r.read(30)
    r.read(1)                                                           # (the first call that has left something)
    r.m.lengths = [3]
    r.refused(lambda: r.m.forward(r.rows(1), [1]))


def test_tokens_that_were_written_again_are_there(B, monkeypatch):  # noqa: F811
    r = Reader(monkeypatch, 4, 20)
    for _ in range(60):
        r.m.forward(r.rows(1), [1])
    r.m.lengths = [32]                                                  # (the sinks' pages are there, and nothing behind them)
    for _ in range(10):
        r.read(1)
    r.m.lengths = [36]
    for _ in range(40):
        r.read(1)
    r.m.lengths = [61]
    r.refused(lambda: r.m.forward(r.rows(1), [1]))
    r.m.lengths = [40]
    r.refused(lambda: r.m.forward(r.rows(1), [1]))
    r.m.lengths = [69]
    r.read(3)


def test_forks_releases_and_sequences_without_rows(B, monkeypatch):  # noqa: F811
    import torch
    r = Reader(monkeypatch, 4, 0, 4)
    for _ in range(60):
        r.m.forward(r.rows(2), [1, 0, 0, 1])
    r.m.fork([0, 0, -1, 3])
    r.m.lengths = [60, 50, 0, 60]
    r.refused(lambda: r.m.forward(r.rows(1), [0, 1, 0, 0]))
    r.read(1, 0, 2, 1)                                                  # (that one reads nothing)
    r.m.lengths[1] = 60
    r.read(1, 1, 1, 1)
    r.m.fork(torch.tensor([0, 1, 3, -1], dtype=torch.int32, device="cuda"), [62, 61, 62, 0])
    for b in (0, 1, 2):
        was = list(r.m.lengths)
        r.m.lengths[b] = 50
        r.refused(lambda: r.m.forward(r.rows(1), [int(i == b) for i in range(4)]))
        r.refused(lambda: r.m.step_graph()(r.rows(4)))
        r.m.lengths = was
    r.read(1, 1, 1, 1)
    r.m.release([1, 2])
    r.read(1, 5, 2, 40)


@pytest.mark.parametrize("device", [False, True])
def test_fork_of_sequences_that_were_set_back(B, monkeypatch, device):  # noqa: F811
    """Their children have what they have; what those read again is there, and a parent that cannot go on is refused."""
    import torch
    r = Reader(monkeypatch, 4, 20, 3)

    def fork(parents):
        r.m.fork(torch.tensor(parents, dtype=torch.int32, device="cuda"), [r.m.lengths[p] if p >= 0 else 0 for p in parents]) if device else r.m.fork(parents)
    for _ in range(60):
        r.m.forward(r.rows(2), [1, 1, 0])
    r.m.lengths = [32, 60, 0]
    fork([0, 0, 1])
    for _ in range(10):
        r.read(1, 1, 1)
    r.m.lengths = [36, 42, 70]
    for _ in range(30):
        r.read(1, 0, 2) if _ % 3 else r.read(1, 1, 0)
    r.m.lengths[1] = 45                                                 # (its last token, behind 51, left those before 48)
    r.refused(lambda: r.m.forward(r.rows(2), [0, 1, 1]))
    r.m.lengths[1] = 51
    r.read(0, 1, 1)
    r.m.lengths[1] = 32
    r.read(0, 2, 1)
    r.m.lengths[1] = 33
    r.read(0, 1, 1)
    r.m.lengths[2] = 60
    r.refused(lambda: fork([0, 1, 2]))
    r.refused(lambda: r.m.forward(r.rows(1), [0, 0, 1]))
    r.m.lengths[0] = 33
    r.refused(lambda: fork([0, 0, 1]))
    r.m.lengths = [66, 34, 0]
    r.m.release([2])
    r.read(1, 1, 1)
