"""The decoding operators at the edges of what they accept, against their definitions in 64 bits: chunks of scales of one step, rows of scales that lie apart."""
import math

import numpy as np
import pytest

import decode_ref as D
import w4_steps as W
from paper_2401_10652_amd import inputs as I
from test_gpu_decode import B, attention_case, torch_dtype, up  # noqa: F401
from test_gpu_decoder import host, reference

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


def linear_case(B, dtype, m, n, k, group, pad=(0, 0), seed=0, zeros=None, x=None):
    """(what comes out, the definition's, the bound): sums in 32 bits, at most 8 roundings of the magnitudes that they are made of, and the result
    rounded once.  pad: elements between rows of scales and of zeros."""
    import torch
    groups = -(-k // group)
    xt, x = up(D.normal((m, k), seed) if x is None else x, dtype)
    codes = D.uniform_ints(0, 16, (n, k), seed + 1)
    st, s = up((D.uniform_ints(50, 150, (n, groups), seed + 2) / 100.0) / (4.6 * math.sqrt(k)), dtype)
    zt, z = up(D.uniform_ints(0, 16, (n, groups), seed + 3) if zeros is None else zeros(n, groups), dtype)
    out = torch.full((m, n), float("nan"), dtype=xt.dtype, device="cuda")
    B.ac_op_linear_w4(xt, torch.from_numpy(D.pack(codes)).cuda(), apart(st, pad[0]), out, group, zero=apart(zt, pad[1]))
    ref, size = D.linear(x, codes, s, z, group)
    return out.double().cpu().numpy(), ref, 8 * D.U["f32"] * size + 1.01 * D.U[dtype] * np.abs(ref) + 2.0 ** -126


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


# Zeros that are no whole numbers from 0 to 15.  32nds leave differences of up to 9 bits, numbers below 1 longer ones, and whole numbers beyond 240 ones of 9 and more.
ZEROS = {"fractions": lambda n, g: D.uniform_ints(0, 15 * 32, (n, g), 91) / 32.0, "any": lambda n, g: D.normal((n, g), 92, 5.0) + 7.5, "small": lambda n, g: D.normal((n, g), 93, 0.01),
         "hundreds": lambda n, g: D.normal((n, g), 94, 300.0), "whole": lambda n, g: D.uniform_ints(-260, 270, (n, g), 95), "mixed": lambda n, g: np.where(
             D.uniform_ints(0, 40, (n, g), 96) == 0, 7.53125, 8.0)}


@pytest.mark.parametrize("zeros", ZEROS)
@pytest.mark.parametrize("dtype,m,n,k,group", [("f32", 5, 100, 200, 32), ("f32", 150, 300, 520, 64), ("bf16", 1, 100, 200, 32), ("bf16", 150, 300, 520, 64), ("bf16", 500, 2200, 328, 32),
                                               ("bf16", 1000, 1160, 520, 64), ("bf16", 500, 2200, 1000, 256)])
def test_linear_w4_zeros_that_are_not_whole(B, dtype, m, n, k, group, zeros):
    got, ref, bound = linear_case(B, dtype, m, n, k, group, seed=m, zeros=ZEROS[zeros])
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)


@pytest.mark.parametrize("zeros", [None, "fractions"])
@pytest.mark.parametrize("dtype,m,n,k,group", [("f32", 3, 60, 256, 32), ("f32", 200, 700, 256, 128), ("bf16", 3, 60, 256, 32), ("bf16", 64, 2100, 256, 64), ("bf16", 500, 2200, 256, 32),
                                               ("bf16", 1000, 1160, 256, 128)])
def test_linear_w4_rows_near_the_ends_of_the_range(B, dtype, m, n, k, group, zeros):
    """Rows whose sums are a tenth of fp32's range, and rows of its least numbers (as far as an output of their size is one)."""
    x = D.normal((m, k), 41)
    x[0] = np.abs(x[0]) * (3.4e38 / 10 / (0.8 * group))
    x[1] *= -2.0 ** 90
    x[2] *= 2.0 ** -100
    got, ref, bound = linear_case(B, dtype, m, n, k, group, seed=m, zeros=ZEROS[zeros] if zeros else None, x=x)
    assert np.isfinite(got).all() and np.isfinite(ref).all()
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)


@pytest.mark.parametrize("act", ["none", "relu", "sigmoid", "silu", "gelu_erf", "gelu_tanh"])
@pytest.mark.parametrize("dtype,m,n", [("f32", 20, 40), ("f32", 200, 1500), ("bf16", 20, 40), ("bf16", 1000, 1160)])
def test_linear_w4_nan_passes_activations(B, dtype, m, n, act):
    """Where the definition's product is NaN, so is the result; where it is an infinity, what the activation makes of it, or NaN; elsewhere neither."""
    import torch
    k, group = 160, 32
    x = D.normal((m, k), 3)
    x[3, 7], x[17, 159], x[5, 40], x[11, 0], x[11, 90] = np.nan, np.inf, -np.inf, np.inf, -np.inf
    xt, x = up(x, dtype)
    codes, zero = D.uniform_ints(0, 16, (n, k), 4), D.uniform_ints(0, 16, (n, k // group), 5)
    st, s = up(np.full((n, k // group), 0.01), dtype)
    zt, z = up(zero, dtype)
    out = torch.empty((m, n), dtype=xt.dtype, device="cuda")
    B.ac_op_linear_w4(xt, torch.from_numpy(D.pack(codes)).cuda(), st, out, group, zero=zt, activation=getattr(B, "AC_ACT_" + act.upper()))
    got = out.double().cpu().numpy()
    with np.errstate(all="ignore"):
        y = D.linear(x, codes, s, z, group)[0]
        of = {"none": lambda v: v, "relu": lambda v: np.where(v < 0, 0.0, v), "sigmoid": lambda v: 1 / (1 + np.exp(-v)), "silu": lambda v: v / (1 + np.exp(-v)),
              "gelu_erf": lambda v: np.where(v > 0, v, np.nan), "gelu_tanh": lambda v: np.where(v > 0, v, np.nan)}[act]       # (of infinities)
        far = np.isinf(y)
        assert far.any() and np.isnan(got[np.isnan(y)]).all()
        assert (np.isnan(got) | (got == of(y)))[far].all()
    assert np.isfinite(got[np.isfinite(y)]).all()


# ---- attention ---------------------------------------------------------------------------------------------------------

def bound_of_few_rows(out, size, reach, dtype):
    """As for rows in fp32, but probabilities of two bf16 terms, each of half a unit of 2^-8: 2^-16 of them is lost; and the result rounded once."""
    p = 4 * 8 * D.U["f32"] * reach + 16 * D.U["f32"]
    return (p + D.U["bf16"] ** 2) * size + 1.01 * D.U["bf16"] * np.abs(out) + 1e-30


@pytest.mark.parametrize("counts,lengths,heads,heads_kv,d,page", [
    ([1], [40], 4, 4, 32, 16), ([1], [1000], 4, 2, 64, 16), ([1], [4099], 4, 2, 128, 32), ([1, 1, 1], [700, 0, 3000], 8, 2, 96, 16), ([5, 3], [900, 2500], 8, 1, 64, 32),
    ([7], [600], 2, 1, 192, 16), ([16], [333], 2, 2, 256, 64)])
def test_attention_of_few_rows_rounds_once(B, monkeypatch, counts, lengths, heads, heads_kv, d, page):
    """What bf16 rows come out as is the fp32 result, rounded to bf16."""
    monkeypatch.setattr(D, "attention_bound", bound_of_few_rows)
    attention_case(B, "bf16", counts, lengths, heads, heads_kv, d, page, seed=sum(lengths) + d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pages,places", [(0, 3), (4, 0), (0, 0)])
def test_no_pages_and_no_places(B, dtype, pages, places):
    """Queries are rotated, keys and values dropped, rows see nothing."""
    import torch
    heads, heads_kv, d, n = 4, 2, 64, 9
    u8, i32 = dict(dtype=torch.uint8, device="cuda"), dict(dtype=torch.int32, device="cuda")
    k, v = torch.full((pages, heads_kv, 32, d), 0x7f, **u8), torch.full((pages, heads_kv, 2, d, 16), 0x7f, **u8)
    ks, vs = (torch.full((pages, heads_kv, 2), float("nan"), device="cuda") for _ in "kv")
    cache = B.kv_cache(k, v, ks, vs)
    rows = B.cache_rows(torch.tensor([0, 5, n], **i32), torch.tensor([20, 4], **i32), torch.zeros((2, places), **i32), 5, 20)
    xt, x = up(D.normal((n, (heads + 2 * heads_kv) * d), 6), dtype)
    q, kn, vn = xt.split([heads * d, heads_kv * d, heads_kv * d], 1)
    q_out, out = (torch.full((n, heads * d), float("nan"), dtype=xt.dtype, device="cuda") for _ in "qo")
    cos, sin = torch.zeros((20, 32), device="cuda"), torch.ones((20, 32), device="cuda")
    B.ac_op_cache_append(kn, vn, cache, rows, q=q, q_out=q_out, rotary=B.rotary(cos, sin))
    turned = D.rotate(x[:, :heads * d].reshape(n, heads, d), np.zeros((n, 32)), np.ones((n, 32)), False)
    assert np.array_equal(host(q_out).reshape(n, heads, d), turned)
    for causal in (True, False):
        B.ac_op_cache_attention(q_out, out.fill_(float("nan")), cache, rows, causal, workspace=B.empty_workspace(B.ac_cache_attention_workspace_bytes(q_out, cache, rows, causal)))
        assert (out == 0).all()
    assert (k == 0x7f).all() and (v == 0x7f).all() and torch.isnan(ks).all() and torch.isnan(vs).all()


# ---- the model -----------------------------------------------------------------------------------------------------------

def small_model(sequences=3, max_tokens=200, **more):
    """(a decoder of two fp32 layers, rows for it)"""
    import torch
    from paper_2401_10652_amd.decode import Decoder
    cfg = I.TransformerConfig("decoder_2l", 11, 2, 60, 128, 4, 256, True, "f32", None, batch=3)
    x, layers = I.transformer_inputs(cfg, bias_std=0.1, ln_jitter=0.1)
    return Decoder(cfg, layers, sequences, max_tokens, page=16, group=32, **more), torch.as_tensor(x, device="cuda")


MODEL_TOL = 12 * 2.0 ** -12       # two layers of six operators, each off by 2^-16 of magnitudes that are about 16 times its sums


def test_steps_from_a_graph_after_lengths_changed_in_place(B):
    """A sequence cut short, and one begun anew, between two replays: each replay against the model in 64 bits."""
    model, x = small_model()
    model.forward(x[:80], [40, 25, 15])
    step = model.step_graph()
    for i, (b, n) in enumerate(((None, 0), (1, 0), (None, 0), (0, 17), (2, 0), (None, 0))):
        if b is not None:
            model.lengths[b] = n
        lengths = [t + 1 for t in model.lengths]
        y = step(x[80 + 3 * i:83 + 3 * i])
        assert model.lengths == lengths
        ref = reference(model, host(x[80 + 3 * i:83 + 3 * i]), [1, 1, 1], lengths, MODEL_TOL * 4)
        assert np.abs(host(y) - ref).max() <= MODEL_TOL * np.abs(ref).max(), (i, np.abs(host(y) - ref).max() / np.abs(ref).max())


def test_model_without_tokens(B):
    model, x = small_model()
    model.forward(x[:5], [2, 0, 3])
    assert model.forward(x[:0], [0, 0, 0]).shape == (0, 128) and model.lengths == [2, 0, 3]


def test_model_reads_rows_of_any_layout(B):
    """Column by column, and every other row."""
    import torch
    model, x = small_model()
    y = model.forward(x[:30], [20, 0, 10])
    for rows in (x[:30].T.contiguous().T, x[:30].repeat_interleave(2, 0)[::2]):
        assert torch.equal(rows, x[:30])
        model.lengths = [0, 0, 0]
        assert torch.equal(model.forward(rows, [20, 0, 10]), y)
