"""The decoding operators at their edges, on the host: no GPU, no pointer followed."""
import random

import pytest

import w4_steps as W


def test_scales_have_landed_before_they_are_read():
    rng = random.Random(5)
    cases = [(k, g) for g in (32, 64, 128, 256, 384, 512) for k in range(8, 14000, 8 if g == 256 else 104)]
    cases += [(8 * rng.randint(1, 1 << 13), 128 * rng.randint(1, 12)) for _ in range(300)]
    for k, group in cases:
        for block in range(0, 256, 8):                            # (blocks of eight begin at the same step)
            for half in (0, 1):
                assert W.late_chunks(k, group, block, half, True) == [], (k, group, block, half)


@pytest.mark.parametrize("m,n,k,group,pad", W.SHORT_CHUNKS)
def test_cases_of_short_chunks_need_the_wait(m, n, k, group, pad):
    """Without the wait a block of this product would read scales that are on their way; a row of them is a multiple of 16 bytes, whole chunks come by direct loads."""
    groups = -(-k // group)
    assert m >= 96 and m * n > 64 * 128 * 128 and (groups + pad) % 8 == 0 and groups > 8
    assert any(W.late_chunks(k, group, block, half, False) for block in range(-(-n // 128)) for half in (0, 1))
