"""The order of beam candidates whose totals are equal in 64 bits though their logits are not: within a beam that of the logits."""
import numpy as np
import pytest

from test_gpu_beam import B, check, logits, run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [50, 3000, 40000])
@pytest.mark.parametrize("keep", [8, 32, 64])
def test_scores_that_swallow_the_logits(B, dtype, vocab, keep):  # noqa: F811
    """-3.4e38 for a beam that is none yet: all its candidates have the same total."""
    x, s = logits(3, 3, vocab, vocab + keep), np.full((3, 3), -3.4e38)
    s[0, 0] = s[1, 1] = 0
    for b, i in ((0, 0), (1, 1)):                                       # few tokens may come
        allowed = np.argsort(x[b, i])[[3, vocab // 2, vocab - 1]]
        row = np.full(vocab, -np.inf)
        row[allowed] = x[b, i, allowed]
        x[b, i] = row
    got = check(B, x, s, dtype, keep)
    assert (got[1][0, :3] == 0).all() and (got[1][0, 3:] == 1).any()
    for _ in range(8):                                                  # (what waves find of each other's borders in time must not show)
        again = run(B, x, s, dtype, keep)[2]
        assert all(np.array_equal(a, b) for a, b in zip(again, got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 5000, 70000])
def test_logits_closer_than_a_step_of_the_total(B, dtype, vocab):  # noqa: F811
    x = np.full((1, 2, vocab), -4.0)
    x[0, :, 7] = 5
    x[0, :, 9:21] = 0.0
    x[0, 0, [vocab - 1, vocab - 3, 13]] = 1e-30, 2e-30, 5e-31
    x[0, 1, [11, vocab - 2]] = -1e-30, 3e-30
    for score in ([0.0, 0.0], [-1.0, -1.0], [-3.0, -2.5]):
        check(B, x, [score], dtype, 20)
    x[0, :, 20:] = D_steps(vocab - 20)                                  # so many that all entries are gone through one after another
    got = check(B, x, [[-1.0, -1.0]], dtype, 64)
    assert len(set(got[0][0])) < 64


def D_steps(n):
    return 1e-30 * (1 + np.arange(n) * 7 % 64)


def test_ended_beams_among_them(B):  # noqa: F811
    x, s = logits(1, 4, 2000, 5), np.full((1, 4), -3.4e38)
    check(B, x, s, "f32", 32, np.array([[0, 1, 0, 1]]), 1500)
    check(B, x, s, "f32", 64, np.array([[1, 1, 1, 0]]), 0)
