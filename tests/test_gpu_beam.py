"""Beam search's selection against its definition in 64 bits: which candidates come out, and in which order, has to be equal."""
import numpy as np
import pytest

import decode_ref as D

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2401_10652_amd import binding
    binding.lib()
    return binding


def select(x, scores, ended, end, keep):
    """x [batch, beams, vocab] -> (scores, parents, tokens, ended), and for each prompt how near its totals are to each other: the least difference of
    two beams' candidates of which one comes out."""
    batch, beams, vocab = x.shape
    out = np.full((batch, keep), -np.inf), np.full((batch, keep), -1), np.full((batch, keep), -1), np.zeros((batch, keep), int)
    near = np.full(batch, np.inf)
    for b in range(batch):
        value, beam, token, logit = [], [], [], []
        for i in range(beams):
            s = float(scores[b, i])
            if ended is not None and ended[b, i]:
                v, t, a = np.array([s]), np.array([end]), np.array([0.0])
            else:
                a, t = x[b, i], np.arange(vocab)
                m = a.max() if not np.isnan(a).any() else np.nan
                with np.errstate(invalid="ignore", divide="ignore"):
                    d = np.where(a == m, 0.0, a - m) if m > -np.inf else np.full(vocab, -np.inf)
                    v = d - np.log(np.exp(d).sum()) + s
                v = np.where((a > -np.inf) & ~np.isnan(v), v, -np.inf)
                top = np.lexsort((t, -a, -v))[:keep + 1]
                v, t, a = v[top], t[top], a[top]
            value.append(v), beam.append(np.full(len(v), i)), token.append(t), logit.append(a)
        v, i, t, a = (np.concatenate(z) for z in (value, beam, token, logit))
        order = np.lexsort((t, -a, i, -v))
        v, i, t = v[order], i[order], t[order]
        n = min(keep, int((v > -np.inf).sum()))
        for k in range(min(n, len(v) - 1)):
            if i[k] != i[k + 1] and v[k + 1] > -np.inf:
                near[b] = min(near[b], v[k] - v[k + 1])
        out[0][b, :n], out[1][b, :n], out[2][b, :n] = v[:n], b * beams + i[:n], t[:n]
        out[3][b, :n] = (t[:n] == end) | (False if ended is None else ended[b, i[:n]] != 0)
    return out, near


def run(B, x, scores, dtype, keep, ended=None, end=-1, pad=0, shift=0):
    """x [batch, beams, vocab]; pad: elements between rows; shift: of the first row from a multiple of 16 bytes."""
    import torch
    batch, beams, vocab = x.shape
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    room = torch.full((shift + batch * beams * (vocab + pad),), float("nan"), dtype=kind, device="cuda")
    rows = room[shift:].view(batch * beams, vocab + pad)[:, :vocab]
    rows.copy_(torch.from_numpy(x.reshape(batch * beams, vocab).astype(np.float32)))
    rows = rows if vocab + pad > 1 else rows
    x = rows.double().cpu().numpy().reshape(x.shape)
    s = torch.from_numpy(np.asarray(scores, np.float32)).cuda().view(batch, beams)
    i32 = dict(dtype=torch.int32, device="cuda")
    e = None if ended is None else torch.tensor(np.asarray(ended), **i32)
    whole = [torch.full((batch * keep + 8,), 7, dtype=torch.float32 if n == 0 else torch.int32, device="cuda") for n in range(4)]
    out = [w[:batch * keep].view(batch, keep) for w in whole]
    need = B.ac_beam_select_workspace_bytes(rows, beams, keep)
    ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")
    B.ac_op_beam_select(rows, s, out[0], out[1], out[2], ws[:need], ended=e, ended_out=out[3], end=end)
    assert all((w[batch * keep:] == 7).all() for w in whole) and (ws[need:] == 0xff).all()
    return x, s.double().cpu().numpy(), [o.cpu().numpy() for o in out], (rows, s, e)


def check(B, x, scores, dtype, keep, ended=None, end=-1, sure=True, **more):
    """Exponentials, their sum and its logarithm in 32 bits, of terms that are at most 1: an error of 2^-21 of the sum; a total in 64 bits is rounded once.  Where two beams' totals are nearer
    to each other than that (which the seeds avoid, sure) their order is not said."""
    x, scores, got, _ = run(B, x, scores, dtype, keep, ended, end, **more)
    want, near = select(x, scores, ended, end, keep)
    sum_error = 2.0 ** -21
    clear = (near > 2 * sum_error) | (near == 0)
    assert clear.all() or not sure, near.min()
    for g, w in zip(got[1:], want[1:]):
        assert np.array_equal(g[clear], w[clear]), np.argwhere(g != w)[:5]
    fine = np.isfinite(want[0])
    assert np.array_equal(got[0][~fine], want[0][~fine].astype(np.float32))
    assert (np.abs(got[0] - want[0])[fine] <= sum_error + 2.0 ** -24 * np.abs(want[0][fine])).all()
    return got


def logits(batch, beams, vocab, seed, std=2.5):
    return D.normal((batch, beams, vocab), seed, std)


def past(batch, beams, seed):
    return -np.cumsum(np.abs(D.normal((batch, beams), seed + 50, 1.5)), 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,beams,vocab,keep", [
    (1, 1, 1, 1), (1, 1, 1, 4), (2, 3, 2, 8), (1, 4, 7, 4), (3, 2, 63, 5), (5, 4, 1000, 4), (2, 5, 4097, 10), (1, 4, 49999, 8), (3, 8, 8192, 16), (2, 16, 3001, 32), (1, 64, 500, 64),
    (1, 3, 200001, 64), (40, 8, 20000, 8), (1, 1, 100, 64)])
def test_select(B, dtype, batch, beams, vocab, keep):
    check(B, logits(batch, beams, vocab, vocab + keep), past(batch, beams, vocab), dtype, keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 1, 3, 64])
@pytest.mark.parametrize("shift", [0, 1, 5])
def test_rows_anywhere(B, dtype, pad, shift):
    for vocab in (1, 9, 2049, 5003):
        check(B, logits(2, 3, vocab, vocab + pad), past(2, 3, shift), dtype, 4, pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_beams_that_ended_and_beams_that_are_none(B, dtype):
    x, s = logits(4, 4, 700, 3), past(4, 4, 4)
    ended = np.array([[0, 1, 0, 0], [1, 1, 1, 1], [0, 0, 0, 0], [1, 0, 0, 1]])
    s[0, 2] = s[1, 3] = s[3, 0] = -np.inf
    s[2] = [0, -np.inf, -np.inf, -np.inf]                                # a search's first step
    for keep in (4, 8):
        got = check(B, x, s, dtype, keep, ended, 5)
        assert (got[2][1, :3] == 5).all() and (got[1][1, 3:] == -1).all() and (got[1][2] == 8).all()
    x[2, 0, 5] = 30                                                      # this one ends now
    got = check(B, x, s, dtype, 4, ended, 5)
    assert got[2][2, 0] == 5 and got[3][2, 0] == 1
    check(B, x, s, dtype, 4, None, 5)
    s[:] = -np.inf
    got = check(B, x, s, dtype, 4, ended, 0)
    assert (got[1] == -1).all() and (got[3] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [50, 3000, 40000])
def test_equal_ones_go_by_their_numbers(B, dtype, vocab):
    """All logits the same (more of them than there is room for at the border), the same beams twice, few different values."""
    for keep in (1, 4, 32):
        x, s = np.zeros((2, 3, vocab)), np.zeros((2, 3))
        got = check(B, x, s, dtype, keep)
        assert (got[1][0] == 0).all() and (got[2][0] == np.arange(keep)).all()
        x, s = np.round(logits(2, 4, vocab, 8) / 2.5), np.full((2, 4), -3.0)
        x[:, 1], x[:, 3] = x[:, 0], x[:, 2]
        check(B, x, s, dtype, keep)
        x = np.full((1, 2, vocab), -1.0)
        x[0, 0, vocab // 2:], x[0, 1, -3:] = 2.0, 7.0
        check(B, x, [[-1.0, -30.0]], dtype, keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite(B, dtype):
    """Tokens that may not come, whole rows of them, infinities, NaN."""
    vocab = 5000
    x, s = logits(6, 3, vocab, 21), past(6, 3, 22)
    x[0][np.abs(x[0]) > 0.01] = -np.inf                                  # few are left
    x[1, 0], x[1, 2, 100:] = -np.inf, -np.inf
    x[2] = -np.inf
    x[3, 1, [7, 4000, 4999]] = np.inf
    x[4, 0, 3333], x[4, 1] = np.nan, np.nan
    x[5, 0] = 3e38
    x[5, 1, :4], x[5, 1, 4:] = -3e38, -np.inf
    for keep in (3, 40):
        got = check(B, x, s, dtype, keep)
        assert (got[1][2] == -1).all() and set(got[1][4]) == {14}
    assert np.isfinite(got[0][3, :3]).all()
    s[0] = [np.nan, np.inf, -1]
    x, s, got, _ = run(B, x[:1], s[:1], dtype, 2)
    assert (got[1] == 1).all() and (got[0] == np.inf).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 40, 3001])
def test_one_token_that_may_come_is_certain(B, dtype, vocab):
    """The logarithm of its probability is 0, not nearly so."""
    x, s = np.full((3, 4, vocab), -np.inf), np.zeros((3, 4))
    for i, v in enumerate(D.normal((12,), 5, 9.0)):
        x[i // 4, i % 4, i * 7 % vocab] = v
    s[1], s[2, 1:] = [-1.5, -2.25, -3.0, -11.0], -np.inf
    got = check(B, x, s, dtype, 4)
    assert (got[0][0] == 0).all() and (got[0][1] == s[1]).all() and (got[0][2] == [0, -np.inf, -np.inf, -np.inf]).all()


def test_ascending_rows(B):
    """The largest logits side by side at the end of a row, and rows in order: every candidate of a run is in the last one's place."""
    for dtype in ("f32", "bf16"):
        for keep in (4, 64):
            x = np.sort(logits(1, 2, 30000, 6), 2)
            check(B, x, [[-1.0, -1.3]], dtype, keep)
            check(B, x[:, :, ::-1], [[-1.0, -1.3]], dtype, keep)


def test_select_twice_and_from_a_graph(B):
    """The same bits again; replays with other logits."""
    import torch
    _, _, first, (rows, s, _) = run(B, logits(3, 4, 9000, 1), past(3, 4, 2), "bf16", 8)
    out = [torch.empty((3, 8), dtype=torch.float32 if n == 0 else torch.int32, device="cuda") for n in range(3)]
    ws = B.empty_workspace(B.ac_beam_select_workspace_bytes(rows, 4, 8))
    B.ac_op_beam_select(rows, s, *out, ws)
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(out, first))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ac_op_beam_select(rows, s, *out, ws)
    for seed in range(4):
        rows.copy_(torch.from_numpy(logits(3, 4, 9000, 30 + seed).reshape(12, 9000).astype(np.float32)))
        s.copy_(torch.from_numpy(past(3, 4, seed).astype(np.float32)))
        graph.replay()
        got = [o.cpu().numpy() for o in out]
        B.ac_op_beam_select(rows, s, *out, ws)
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(out, got))
        want, _ = select(rows.double().cpu().numpy().reshape(3, 4, 9000), s.double().cpu().numpy(), None, -1, 8)
        assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
