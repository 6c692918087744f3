"""Reads, lengths set, forks, releases and moves in any order: what a sequence's next row sees is what it read, or the call is refused."""
import random

import pytest

from test_gpu_branching import B, held, model  # noqa: F401

pytestmark = pytest.mark.gpu
SEQUENCES, MOST, PAGE = 5, 150, 16


def keys(m):
    """The first layer's keys of every place of the table, as numbers: they depend on a token's row and place alone."""
    import torch
    k, _, scale, _ = m.caches[0].keep
    numbers = k.view(torch.float8_e4m3fn).float() * scale.repeat_interleave(16, 2)[..., None]
    return numbers[m.table.clamp(min=0).long()].transpose(2, 3).reshape(SEQUENCES, -1, numbers.shape[1] * numbers.shape[3]), m.table.repeat_interleave(PAGE, 1) >= 0


def whole(m, other, texts, x, window, sinks):
    """Of each sequence, whether the tokens that its next row sees are those of its text: as near to another model's, which read the text at once, as codes of 8 bits with other scales are."""
    other.release(range(SEQUENCES))
    other.forward(x[sum(texts, [])], [len(t) for t in texts]) if any(texts) else None
    (got, there), (want, _) = keys(m), keys(other)
    near = (((got - want).norm(dim=2) < 0.25 * want.norm(dim=2)) & there).tolist()
    return [all(near[b][t] for t in range(n) if window is None or t < sinks or n - t < window) for b, n in enumerate(map(len, texts))]


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("window,sinks,pages", [(None, 0, 60), (None, 0, 12), (17, 5, 60), (20, 40, 13), (3, 0, 60), (7, 20, 9), (40, 3, 10)])
def test_any_order(B, window, sinks, pages, seed):  # noqa: F811
    import torch
    rng = random.Random(f"{seed} {window} {pages}")
    m, x = model("f32", SEQUENCES, MOST, pages=pages, window=window, sinks=sinks)
    other, _ = model("f32", SEQUENCES, MOST, pages=60, window=window, sinks=sinks)
    step = m.step_graph() if seed % 2 else None
    texts, done, refused, dry = [[] for _ in range(SEQUENCES)], 0, 0, 0
    for _ in range(60):
        fine = whole(m, other, texts, x, window, sinks)
        op = rng.choice(["read", "read", "step", "step", "step", "set", "set", "fork", "fork on device", "release", "compact"])
        if op in ("read", "step"):
            counts = [rng.choice((0, 1, 1, 3, rng.randint(0, 40))) for _ in texts] if op == "read" else [1] * SEQUENCES
            counts = [min(c, MOST - len(t)) for c, t in zip(counts, texts)]
            if sum(counts) == 0 or (op == "step" and min(counts) == 0):
                continue
            new = [[rng.randrange(len(x)) for _ in range(c)] for c in counts]
            rows = x[sum(new, [])]
            can = all(f for f, c in zip(fine, counts) if c)
            try:
                step(rows) if op == "step" and step else m.forward(rows, counts)
            except ValueError:
                assert not can
                refused += 1
                if refused % 4 == 0:                                    # (or it may stay as it is for long)
                    m.release(range(SEQUENCES))
                    texts = [[] for _ in texts]
            except RuntimeError:
                assert can and pages < 60
                dry += 1
                if dry % 3 == 0:
                    gone = rng.sample(range(SEQUENCES), 3)
                    m.release(gone)
                    texts = [[] if b in gone else t for b, t in enumerate(texts)]
            else:
                assert can
                texts = [t + n for t, n in zip(texts, new)]
                done += 1
        elif op == "set":
            b = rng.randrange(SEQUENCES)
            texts[b] = texts[b][:max(0, len(texts[b]) - rng.choice((1, 2, 5, 17, 60)))]
            m.lengths[b] = len(texts[b])
        elif op in ("fork", "fork on device"):
            parents = [rng.choice((j, j, rng.randrange(-1, SEQUENCES))) for j in range(SEQUENCES)]
            new = [texts[p][:] if p >= 0 else [] for p in parents]
            try:
                m.fork(torch.tensor(parents, dtype=torch.int32, device="cuda"), [len(t) for t in new]) if "device" in op else m.fork(parents)
            except ValueError:
                assert not all(f for b, f in enumerate(fine) if "device" in op or b in parents)
                refused += 1
            except RuntimeError:
                assert pages < 60
                dry += 1
            else:
                assert all(f for b, f in enumerate(fine) if b in parents)
                texts = new
        elif op == "release":
            gone = rng.sample(range(SEQUENCES), 1)
            m.release(gone)
            texts = [[] if b in gone else t for b, t in enumerate(texts)]
        else:
            m.compact()
        assert m.lengths == [len(t) for t in texts]
        held(m)
    assert done >= 8
