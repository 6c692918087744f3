"""The decoding operators at the edges of what they accept, against their definitions in 64 bits: chunks of scales of one step, rows of scales that lie apart."""
import math

import numpy as np
import pytest

import decode_ref as D
import w4_steps as W
from test_gpu_decode import B, torch_dtype, up  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- linear layers ----------------------------------------------------------------------------------------------------

def apart(t, pad):
    """The same matrix with `pad` NaNs behind each row."""
    import torch
    if not pad:
        return t
    spread = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    spread[:, :t.shape[1]] = t
    return spread[:, :t.shape[1]]


def linear_case(B, dtype, m, n, k, group, pad=(0, 0), seed=0):
    """(what comes out, the definition's, the bound): sums in 32 bits, at most 8 roundings of the magnitudes that they are made of, and the result
    rounded once.  pad: elements between rows of scales and of zeros."""
    import torch
    groups = -(-k // group)
    xt, x = up(D.normal((m, k), seed), dtype)
    codes = D.uniform_ints(0, 16, (n, k), seed + 1)
    st, s = up((D.uniform_ints(50, 150, (n, groups), seed + 2) / 100.0) / (4.6 * math.sqrt(k)), dtype)
    zt, z = up(D.uniform_ints(0, 16, (n, groups), seed + 3), dtype)
    out = torch.full((m, n), float("nan"), dtype=xt.dtype, device="cuda")
    B.ac_op_linear_w4(xt, torch.from_numpy(D.pack(codes)).cuda(), apart(st, pad[0]), out, group, zero=apart(zt, pad[1]))
    ref, size = D.linear(x, codes, s, z, group)
    return out.double().cpu().numpy(), ref, 8 * D.U["f32"] * size + 1.01 * D.U[dtype] * np.abs(ref) + 1e-30


@pytest.mark.parametrize("m,n,k,group,pad", W.SHORT_CHUNKS)
def test_linear_w4_of_tiles_chunks_of_one_step(B, m, n, k, group, pad):
    got, ref, bound = linear_case(B, "bf16", m, n, k, group, (pad, pad), seed=k + group)
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [(1, 3), (8, 0), (0, 5)])
@pytest.mark.parametrize("m,n,k,group", [(1, 50, 200, 32), (40, 300, 2300, 64), (300, 700, 900, 128), (500, 2200, 520, 32)])
def test_linear_w4_scales_and_zeros_apart(B, dtype, m, n, k, group, pad):
    got, ref, bound = linear_case(B, dtype, m, n, k, group, pad, seed=m)
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)
