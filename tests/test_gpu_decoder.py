"""The decoding operators together, as a model reads prompts and single tokens, against the same model in 64 bits."""
import numpy as np
import pytest

import decode_ref as D
from paper_2401_10652_amd import inputs as I

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2401_10652_amd import binding
    return binding


def host(t):
    return t.double().cpu().numpy()


def gelu(x):
    from scipy.special import erf
    return 0.5 * x * (1 + erf(x / np.sqrt(2)))


def norm(x, g, b, eps):
    x = x - x.mean(1, keepdims=True)
    return x / np.sqrt((x * x).mean(1, keepdims=True) + eps) * g + b


class Held(D.Cache):
    """The model's cache as it stands."""

    def __init__(self, cache, table):
        k, v, ks, vs = (t.cpu().numpy() for t in cache.keep)
        self.k, self.v, self.k_scale, self.v_scale = k, v, ks.astype(np.float64), vs.astype(np.float64)
        self.pages, self.heads, self.page, self.d = k.shape
        self.table = table


def reference(model, x, counts, lengths, tol):
    """The same rows in 64 bits, from the model's codes.  New keys and values have to be in its cache, from which the rows then read: how
    they round there is the append's own test's matter, and a number next to a rounding's edge may go either way."""
    cfg, d, h, hk = model.cfg, model.cfg.head_dim, model.cfg.heads, model.heads_kv
    table, n = model.table.cpu().numpy(), sum(counts)
    place = np.concatenate([np.arange(t - c, t) for c, t in zip(counts, lengths)])
    cos, sin = (host(t)[place] for t in model.rotary.keep[:2])

    def linear(w, name, x, **more):
        codes, scale, zero = w["w_" + name]
        codes = codes.cpu().numpy()
        codes = np.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1)[:, :x.shape[1]].astype(np.float64)
        return D.linear(x, codes, host(scale), host(zero), model.group, host(w["b_" + name]), **more)[0]

    for w, cache in zip(model.layers, model.caches):
        qkv = linear(w, "qkv", norm(x, host(w["ln1_g"]), host(w["ln1_b"]), cfg.ln_eps)).reshape(n, h + 2 * hk, d)
        q, k, v = D.rotate(qkv[:, :h], cos, sin, False), D.rotate(qkv[:, h:h + hk], cos, sin, False), qkv[:, h + hk:]
        held, ctx, at = Held(cache, table), np.zeros((n, h, d)), 0
        for b, c in enumerate(counts):
            for i in range(hk):
                for name, y in (("k", k), ("v", v)):
                    y, got = y[at:at + c, i], held.tokens(name, b, i, lengths[b])[lengths[b] - c:]
                    assert (np.abs(got - y) <= np.abs(y) / 16 + (2.0 ** -8 + tol) * np.abs(qkv).max()).all(), (name, b, i)
            if c:
                ctx[at:at + c] = D.attention(q[at:at + c], held, b, lengths[b] - c, lengths[b], h // hk, True, d ** -0.5)[0]
            at += c
        x = linear(w, "o", ctx.reshape(n, -1), residual=x)
        x = linear(w, "2", linear(w, "1", norm(x, host(w["ln2_g"]), host(w["ln2_b"]), cfg.ln_eps), act=gelu), residual=x)
    return x


# Two layers of six operators.  f32: an operator's sums of up to 256 products are off by 2^-16 of their magnitudes at most, which are about 16 times
# the sums: 2 * 6 * 2^-12.  bf16: each operator's result is rounded to 2^-8 of itself, and the norms keep that: 2 * 6 * 2^-8.
@pytest.mark.parametrize("dtype,tol", [("f32", 12 * 2.0 ** -12), ("bf16", 12 * 2.0 ** -8)])
@pytest.mark.parametrize("heads_kv", [4, 2])
def test_model(B, dtype, tol, heads_kv):
    import torch
    from paper_2401_10652_amd.decode import Decoder
    cfg = I.TransformerConfig("decoder_2l", 11, 2, 60, 128, 4, 256, True, dtype, None, batch=3)
    x, layers = I.transformer_inputs(cfg, bias_std=0.1, ln_jitter=0.1)
    for w in layers:                                                    # keys' and values' heads: the first ones of each
        w["w_qkv"], w["b_qkv"] = (np.concatenate([t[:128], t[128:128 + 32 * heads_kv], t[256:256 + 32 * heads_kv]]) for t in (w["w_qkv"], w["b_qkv"]))
    model = Decoder(cfg, layers, 3, 130, page=16, group=32)
    assert model.heads_kv == heads_kv
    at, x = 0, torch.as_tensor(x, device="cuda").to(model.dtype)
    for counts in ([40, 7, 0], [1, 1, 1], [5, 1, 33], [1, 1, 0], [0, 0, 1], [17, 16, 1]):
        rows = x[at:at + sum(counts)]
        at += sum(counts)
        y = host(model.forward(rows, counts))
        ref = reference(model, host(rows), counts, model.lengths, tol * 4)
        assert np.abs(y - ref).max() <= tol * np.abs(ref).max(), (counts, np.abs(y - ref).max() / np.abs(ref).max())
    assert model.lengths == [64, 26, 36]
    with pytest.raises(ValueError):
        model.forward(x[:140], [67, 0, 73])
    with pytest.raises(ValueError):
        model.forward(x[:3], [1, 1, 0])
    assert model.lengths == [64, 26, 36]


def test_steps_from_a_graph(B):
    """Replays with eager calls and other lengths between them, each against the model in 64 bits and against an eager call from the same state."""
    import torch
    from paper_2401_10652_amd.decode import Decoder
    cfg, tol = I.TransformerConfig("decoder_2l", 11, 2, 60, 128, 4, 256, True, "f32", None, batch=3), 12 * 2.0 ** -12
    x, layers = I.transformer_inputs(cfg, bias_std=0.1, ln_jitter=0.1)
    model = Decoder(cfg, layers, 3, 1500, page=16, group=32)
    x = torch.as_tensor(x, device="cuda")
    model.forward(x[:47], [40, 0, 7])
    step = model.step_graph()
    assert model.lengths == [40, 0, 7]
    at = 47
    for eager in (None, [1, 1, 1], None, [5, 17, 0], None, None):
        n = 3 if eager is None else sum(eager)
        rows = x[at:at + n]
        at += n
        if eager is None:
            before = [[t.clone() for t in c.keep] for c in model.caches], list(model.lengths)
            y = step(rows).clone()
            ref = reference(model, host(rows), [1, 1, 1], model.lengths, tol * 4)
            assert np.abs(host(y) - ref).max() <= tol * np.abs(ref).max()
            after = [[t.clone() for t in c.keep] for c in model.caches], list(model.lengths)
            for c, held in zip(model.caches, before[0]):
                for t, u in zip(c.keep, held):
                    t.copy_(u)
            model.lengths = before[1]
            assert np.abs(host(model.forward(rows, [1, 1, 1])) - ref).max() <= tol * np.abs(ref).max()
            assert model.lengths == after[1]
            # (the first layer's keys and values do not depend on how its attention is split)
            assert all(torch.equal(t, u) for t, u in zip(model.caches[0].keep, after[0][0]))
        else:
            model.forward(rows, eager)
    with pytest.raises(ValueError):
        step(x[:2])
    model.lengths[1] = 1500
    with pytest.raises(ValueError):
        step(x[:3])


def test_codes_of_weights(B):
    import torch
    from paper_2401_10652_amd.decode import quantize_w4
    w = torch.from_numpy(D.normal((20, 100), 5)).float().cuda()
    w[3], w[4], w[5, :32] = 0, w[4].abs(), 7.0
    codes, scale, zero = quantize_w4(w, 32, torch.float32)
    assert codes.shape == (20, 64) and scale.shape == zero.shape == (20, 4)
    c = torch.stack([codes & 15, codes >> 4], 2).view(20, -1)[:, :100].float()
    over = lambda t: t.repeat_interleave(32, 1)[:, :100]  # noqa: E731
    # half a step, and half a step more at the ends of a group, whose zero is rounded
    assert ((((c - over(zero)) * over(scale) - w).abs()) <= over(scale) * 1.001).all() and (c[3] == over(zero)[3]).all()
