"""The decoding operators against their definitions in 64 bits, at the sizes, layouts, masks and values where they can go wrong."""
import math

import numpy as np
import pytest

import decode_ref as D
from oracle import transformer as O
from util import host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2401_10652_amd import binding
    binding.lib()
    return binding


def torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def up(x, dtype):
    """(device tensor, its values in 64 bits)"""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch_dtype(dtype)).cuda()
    return t, t.double().cpu().numpy()


# ---- linear layers ----------------------------------------------------------------------------------------------------

def linear_case(B, dtype, m, n, k, group, zero=True, bias=True, residual=True, act="none", seed=0, pad=0, wide=0, x=None):
    """pad: elements between rows of x, out and residual; wide: further bytes of a row of codes."""
    import torch
    groups = -(-k // group)
    xt, x = up(D.normal((m, k), seed) if x is None else x, dtype)
    codes = D.uniform_ints(0, 16, (n, k), seed + 1)
    st, s = up((D.uniform_ints(50, 150, (n, groups), seed + 2) / 100.0) / (4.6 * math.sqrt(k)), dtype)
    zt, z = up(D.uniform_ints(0, 16, (n, groups), seed + 3), dtype) if zero else (None, None)
    bt, b = up(D.normal((n,), seed + 4), dtype) if bias else (None, None)
    rt, r = up(D.normal((m, n), seed + 5), dtype) if residual else (None, None)
    w = torch.from_numpy(D.pack(codes, -(-k // 32) * 16 + wide)).cuda()
    if pad:
        spread = torch.full((m, k + pad), float("nan"), dtype=xt.dtype, device="cuda")
        spread[:, :k] = xt
        xt = spread[:, :k]
    out = torch.full((m, n + pad), float("nan"), dtype=xt.dtype, device="cuda")[:, :n]
    B.ac_op_linear_w4(xt, w, st, out, group, zero=zt, bias=bt, residual=rt, activation=B.ACTIVATIONS[act])
    fn = {"none": None, "gelu_erf": O.gelu_erf, "gelu_tanh": O.gelu_tanh, "relu": O.relu}[act]
    ref, size = D.linear(x, codes, s, z, group, b, fn, r)
    # sums in 32 bits: at most 8 roundings of the magnitudes they are made of; the erf form's own error; the result rounded once
    bound = 8 * D.U["f32"] * size + 2e-7 * np.abs(ref) + (2e-7 * size if act != "none" else 0) + 1.01 * D.U[dtype] * np.abs(ref) + 1e-30
    got = host(out) if dtype == "f32" else out.double().cpu().numpy()
    return got, ref, bound


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k,group", [
    (1, 16, 32, 32), (1, 1, 1, 32), (1, 17, 129, 64), (2, 33, 100, 32), (3, 250, 1000, 128), (15, 48, 256, 64), (16, 64, 2048, 256),
    (17, 130, 384, 128), (33, 95, 513, 64), (64, 256, 640, 32), (65, 70, 300, 128), (130, 200, 1030, 384), (1, 4096, 96, 32)])
def test_linear_w4(B, dtype, m, n, k, group):
    got, ref, bound = linear_case(B, dtype, m, n, k, group, seed=m + n + k)
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)


@pytest.mark.parametrize("m,n,k,group", [(96, 8192, 64, 32), (6200, 129, 8, 64), (1029, 800, 200, 128), (2600, 310, 520, 64), (257, 3100, 1000, 32), (512, 1600, 1032, 256),
                                          (1500, 600, 100, 32), (128, 6500, 333, 64), (300, 384, 1024, 256), (40, 2050, 96, 32), (70, 8200, 200, 64), (130, 5000, 160, 128)])
def test_linear_w4_of_many_rows(B, m, n, k, group):
    for zero in (False, True):
        got, ref, bound = linear_case(B, "bf16", m, n, k, group, zero, seed=m + n)
        assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)


@pytest.mark.parametrize("m,n,k,group", [(96, 11000, 64, 32), (8200, 129, 8, 64), (1029, 1100, 200, 128), (3500, 310, 520, 64), (257, 4200, 1000, 32), (512, 2100, 1032, 256),
                                         (300, 3600, 2112, 32), (1100, 1000, 1096, 64), (128, 8300, 4096, 512)])
def test_linear_w4_of_tiles(B, m, n, k, group):
    for zero in (False, True):
        got, ref, bound = linear_case(B, "bf16", m, n, k, group, zero, seed=m + n)
        assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)


@pytest.mark.parametrize("act,bias,residual,pad,wide", [("none", False, False, 8, 16), ("gelu_erf", True, False, 1, 0), ("gelu_tanh", False, True, 24, 0), ("relu", True, True, 8, 48)])
def test_linear_w4_of_tiles_forms(B, act, bias, residual, pad, wide):
    got, ref, bound = linear_case(B, "bf16", 130, 8300, 320, 64, True, bias, residual, act, seed=7, pad=pad, wide=wide)
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)


def test_linear_w4_of_tiles_rows_keep_to_themselves(B):
    m, n, k = 130, 8300, 160
    x = D.normal((m, k), 31)
    x[3, 7], x[17, 159], x[5] = np.nan, np.inf, x[5] * 1e30
    x[6] *= 1e-30
    got, ref, bound = linear_case(B, "bf16", m, n, k, 32, bias=False, residual=False, x=x)
    assert not np.isfinite(got[[3, 17]]).any()
    rest = [i for i in range(m) if i not in (3, 17)]
    assert (np.abs(got - ref)[rest] <= bound[rest]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k,group", [(33, 4110, 200, 32), (64, 2048, 130, 128), (70, 2801, 96, 256), (47, 8200, 129, 64), (90, 11000, 160, 128), (300, 700, 72, 64),
                                         (1, 33, 30100, 32), (3, 20, 20000, 64), (20, 8200, 2300, 32), (17, 70, 9000, 384)])
def test_linear_w4_of_some_rows(B, dtype, m, n, k, group):
    got, ref, bound = linear_case(B, dtype, m, n, k, group, seed=m + n)
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("act,bias,residual", [("none", False, False), ("gelu_erf", True, False), ("gelu_tanh", False, True), ("relu", True, True)])
def test_linear_w4_epilogues(B, dtype, zero, act, bias, residual):
    for m, n in ((1, 72), (20, 72), (130, 6148)):
        got, ref, bound = linear_case(B, dtype, m, n, 320, 64, zero, bias, residual, act, seed=m)
        assert (np.abs(got - ref) <= bound).all(), (m, np.max(np.abs(got - ref) / bound))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,wide", [(1, 0), (8, 16), (5, 48)])
def test_linear_w4_strides(B, dtype, pad, wide):
    for m, n in ((1, 50), (7, 50), (40, 50), (200, 4001)):
        got, ref, bound = linear_case(B, dtype, m, n, 200, 32, seed=m, pad=pad, wide=wide)
        assert (np.abs(got - ref) <= bound).all(), (m, np.max(np.abs(got - ref) / bound))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_w4_rows_keep_to_themselves(B, dtype):
    """NaN and infinities of one row reach no other; large and tiny rows keep their precision."""
    for m, n in ((20, 40), (130, 6500)):
        k = 160
        x = D.normal((m, k), 3)
        x[3, 7], x[17, 159], x[5] = np.nan, np.inf, x[5] * 1e30
        x[6] *= 1e-30
        got, ref, bound = linear_case(B, dtype, m, n, k, 32, bias=False, residual=False, x=x)
        assert not np.isfinite(got[[3, 17]]).any()
        rest = [i for i in range(m) if i not in (3, 17)]
        assert (np.abs(got - ref)[rest] <= bound[rest]).all()


def test_linear_w4_in_place_residual_and_no_rows(B):
    import torch
    x = torch.randn(5, 64, device="cuda")
    w = torch.randint(0, 256, (32, 32), dtype=torch.uint8, device="cuda")
    scale = torch.rand(32, 2, device="cuda")
    y = torch.randn(5, 32, device="cuda")
    apart = torch.empty_like(y)
    B.ac_op_linear_w4(x, w, scale, apart, 32, residual=y)
    B.ac_op_linear_w4(x, w, scale, y, 32, residual=y)
    assert torch.equal(y, apart)
    B.ac_op_linear_w4(x[:0], w, scale, y[:0], 32)
    assert torch.equal(y, apart)


# ---- the cache on the device -----------------------------------------------------------------------------------------------

class Device:
    """A host cache's tensors on the device; gap: further bytes (and floats) between pages."""

    def __init__(self, B, cache, gap=0):
        import torch
        self.B, self.host, t = B, cache, {}
        for name, x, kind in (("k", cache.k, np.uint8), ("v", cache.v, np.uint8), ("k_scale", cache.k_scale, np.float32),
                              ("v_scale", cache.v_scale, np.float32)):
            flat = x.reshape(cache.pages, -1).astype(kind)
            spread = torch.zeros((cache.pages, flat.shape[1] + gap), dtype=torch.from_numpy(flat).dtype, device="cuda")
            spread[:, :flat.shape[1]] = torch.from_numpy(flat).cuda()
            t[name] = spread[:, :flat.shape[1]].unflatten(1, x.shape[1:])
        self.t = t
        self.desc = B.kv_cache(t["k"], t["v"], t["k_scale"], t["v_scale"])

    def rows(self, counts, lengths, max_rows=None, max_length=None):
        import torch
        begin = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
        length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        table = torch.from_numpy(self.host.table).cuda()
        return self.B.cache_rows(begin, length, table, max(counts) if max_rows is None else max_rows,
                                 max(lengths) if max_length is None else max_length)

    def down(self):
        return {n: x.cpu().numpy() for n, x in self.t.items()}


# ---- append --------------------------------------------------------------------------------------------------------------------

def tables(length, pairs, seed=0):
    angle = np.arange(length)[:, None] * 10000.0 ** (-np.arange(pairs) / max(pairs, 1))
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def append_case(B, dtype, counts, befores, heads, heads_kv, d, page, pairs, interleaved=False, sections=None, positions=True, seed=0, gap=0,
                lie=False, in_place=False, alter=None, louder=1.0):
    """Appends to a device cache and to the host's; checks both.  befores: tokens held before; lie: sizes that the host states too small."""
    import torch
    lengths = [b + n for b, n in zip(befores, counts)]
    cache = D.Cache(lengths, heads_kv, d, page, seed)
    for b, n in enumerate(befores):
        cache.fill(b, n, seed + 1000)
    total = sum(counts)
    packed = D.normal((total, (heads + 2 * heads_kv) * d), seed + 5, louder)
    if alter is not None:
        alter(packed)
    pt, packed = up(packed, dtype)
    dev = Device(B, cache, gap)
    rows = dev.rows(counts, lengths, *((1, 1) if lie else (None, None)))
    table_rows = max(lengths) + 3
    cos, sin = tables(table_rows, pairs)
    place = np.concatenate([np.arange(b, b + n) for b, n in zip(befores, counts)]) if total else np.zeros(0, int)
    sections = (pairs,) if sections is None else sections
    where = np.stack([place] + [D.uniform_ints(-2, table_rows + 2, (total,), seed + 60 + a) for a in range(1, len(sections))]) if positions else place[None]
    rot = B.rotary(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(),
                   torch.from_numpy(where.astype(np.int32)).cuda() if positions else None, sections, interleaved)
    q, k, v = (pt[:, a * d:b * d] for a, b in ((0, heads), (heads, heads + heads_kv), (heads + heads_kv, heads + 2 * heads_kv)))
    q_out = q if in_place else torch.full((total, heads * d), float("nan"), dtype=pt.dtype, device="cuda")
    B.ac_op_cache_append(k, v, dev.desc, rows, q=q if heads else None, q_out=q_out if heads else None, rotary=rot if pairs or positions else None)

    axis = np.repeat(np.arange(len(sections)), sections)
    at = np.clip(where[axis], 0, table_rows - 1).T if pairs else np.zeros((total, 0), int)      # [rows, pairs]
    c, s = cos[at, np.arange(pairs)], sin[at, np.arange(pairs)]
    packed = packed.reshape(total, heads + 2 * heads_kv, d)
    turned = D.rotate(packed, c.astype(np.float64), s.astype(np.float64), interleaved)
    # codes are compared with those of the products and sums rounded one by one to 32 bits, as the operator's definition has them
    single = D.rotate(packed.astype(np.float32), c, s, interleaved).astype(np.float64)
    got = q_out.double().cpu().numpy().reshape(total, heads, d)
    bound = 1.01 * D.U[dtype] * np.abs(turned[:, :heads]) + 3 * D.U["f32"] * np.sqrt(2) * np.abs(packed[:, :heads]).max(initial=0.0)
    assert (np.abs(got - turned[:, :heads])[np.isfinite(turned[:, :heads])] <= bound[np.isfinite(turned[:, :heads])]).all()
    at = 0
    for b, n in enumerate(counts):
        cache.append(b, single[at:at + n, heads:heads + heads_kv], packed[at:at + n, heads + heads_kv:], lengths[b])
        at += n
    down = dev.down()
    for name in ("k_scale", "v_scale"):
        assert np.array_equal(down[name], getattr(cache, name).astype(np.float32)), name
    for name in ("k", "v"):
        a, b = down[name], getattr(cache, name)
        assert np.array_equal(np.isnan(D.VALUE[a]), np.isnan(D.VALUE[b])), name
        fine = ~np.isnan(D.VALUE[b])
        assert np.array_equal(D.VALUE[a][fine], D.VALUE[b][fine]), name
    # and in 64 bits: a new element is within half a step of what it stands for
    at = 0
    for b, n in enumerate(counts):
        for h in range(heads_kv):
            for name, x in (("k", turned[at:at + n, heads + h]), ("v", packed[at:at + n, heads + heads_kv + h])):
                held = cache.tokens(name, b, h, lengths[b])[befores[b]:]
                scales = np.array([cache.get(name, cache.block(b, t // 16), h)[1] for t in range(befores[b], lengths[b])])[:, None]
                step = np.maximum(2.0 ** np.floor(np.log2(np.maximum(np.abs(x), 1e-300))) / 8, scales * 2.0 ** -9)
                fine = np.isfinite(x)
                assert (np.abs(held - x)[fine] <= (0.5 * step * (1 + 1e-5) + 1e-6 * np.abs(x))[fine]).all(), name
        at += n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,befores,heads,heads_kv,d,page,pairs", [
    ([1], [0], 1, 1, 32, 16, 16), ([1], [15], 2, 1, 64, 16, 32), ([1], [16], 3, 3, 128, 32, 64), ([1, 1, 1, 1], [3, 0, 31, 64], 8, 2, 64, 64, 32),
    ([16], [0], 4, 4, 96, 16, 48), ([17], [15], 4, 2, 128, 128, 64), ([40, 1, 0, 5], [7, 100, 20, 0], 5, 5, 64, 32, 16), ([33], [31], 7, 1, 192, 48, 96),
    ([200, 3], [0, 250], 2, 2, 256, 64, 128)])
def test_append(B, dtype, counts, befores, heads, heads_kv, d, page, pairs):
    append_case(B, dtype, counts, befores, heads, heads_kv, d, page, pairs, seed=sum(counts) + d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pairs,sections", [(0, None), (4, None), (8, (4, 4)), (32, (8, 12, 12)), (32, (1, 30, 0, 1)), (20, (3, 17))])
def test_append_rotations(B, dtype, interleaved, pairs, sections):
    append_case(B, dtype, [9, 20], [13, 2], 4, 2, 64, 16, pairs, interleaved, sections, seed=pairs)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_forms(B, dtype):
    append_case(B, dtype, [5, 30], [30, 2], 4, 2, 64, 32, 32, positions=False, seed=1)                  # places in the sequence
    append_case(B, dtype, [5, 30], [30, 2], 0, 2, 64, 32, 32, seed=2)                                   # no queries
    append_case(B, dtype, [5, 30], [30, 2], 4, 2, 64, 32, 32, seed=3, gap=32)                           # pages apart
    append_case(B, dtype, [5, 90], [30, 2], 4, 2, 64, 32, 32, seed=4, lie=True)                         # more rows than the host said
    append_case(B, dtype, [5, 30], [30, 2], 4, 2, 64, 32, 32, seed=5, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("louder", [1e-35, 1e-28, 0.01, 700.0, 1e30])
def test_append_moves_the_scale(B, dtype, louder):
    """Quieter rows keep the block's scale, louder ones raise it and move the older tokens' codes."""
    append_case(B, dtype, [3, 1, 20], [5, 15, 9], 2, 2, 64, 16, 0, positions=False, seed=9, louder=louder)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_values_that_are_not_finite(B, dtype):
    """They are stored as NaN, and neither their block's scale nor its other tokens see them."""
    def alter(x):
        x[2, 130], x[4, 200], x[7, 300] = np.inf, -np.inf, np.nan     # keys and values of heads that are not rotated
        x[11] = 0.0
    append_case(B, dtype, [12], [5], 2, 2, 64, 16, 0, positions=False, seed=10, alter=alter)


def test_append_with_tables_of_no_pairs(B):
    import torch
    for cos in (torch.empty((70, 0), device="cuda"), torch.empty((70, 9), device="cuda")[:, 9:]):
        x, host = up(D.normal((40, 96), 12), "f32")
        cache = D.Cache([40], 1, 32, 16, 4)
        dev, out = Device(B, cache), torch.empty((40, 32), device="cuda")
        where = torch.arange(40, dtype=torch.int32, device="cuda")[None]
        B.ac_op_cache_append(x[:, 32:64], x[:, 64:], dev.desc, dev.rows([40], [40]), q=x[:, :32], q_out=out, rotary=B.rotary(cos, cos, where))
        assert torch.equal(out, x[:, :32])
        cache.append(0, host[:, 32:64].reshape(40, 1, 32), host[:, 64:].reshape(40, 1, 32), 40)
        down = dev.down()
        assert all(np.array_equal(down[n], getattr(cache, n)) for n in ("k", "v", "k_scale", "v_scale"))


def test_append_of_zeros_and_what_is_dropped(B):
    import torch
    cache = D.Cache([40, 8], 1, 32, 16, 3, fill=0x7f)
    cache.table[0, 1] = cache.pages + 5                               # names no page
    dev = Device(B, cache)
    rows = dev.rows([40, 12], [40, 8])                                # the second has rows in front of token 0
    k, v = torch.zeros((52, 32), device="cuda"), torch.zeros((52, 32), device="cuda")
    v[40:44] = 1e6                                                    # dropped: in front of token 0
    before = dev.down()
    B.ac_op_cache_append(k, v, dev.desc, rows)
    down, unused = dev.down(), [p for p in range(cache.pages) if p not in cache.table]
    for p in (cache.table[0, 0], cache.table[1, 0]):
        assert (down["k_scale"][p] == 2.0 ** -100).all() and (down["v_scale"][p] == 2.0 ** -100).all()
    assert (down["k"][cache.table[0, 0]] == 0).all() and (down["v"][cache.table[1, 0]][..., :8] == 0).all()
    for p in unused:
        assert all(np.array_equal(down[n][p], before[n][p], equal_nan=n.endswith("scale")) for n in down)
    assert (down["k"][cache.table[1, 0]][:, 8:] == 0x7f).all() and (down["v"][cache.table[1, 0]][..., 8:] == 0x7f).all()


# ---- attention -------------------------------------------------------------------------------------------------------------------

def attention_case(B, dtype, counts, lengths, heads, heads_kv, d, page, causal=True, scale=None, seed=0, gap=0, lie=False, pad=0, alter=None,
                   std=1.0, pages_of_a_sequence=None, fill=0x7f, longest=None):
    """What lies behind a sequence's last token, and in pages that no sequence has, is NaN, codes and scales."""
    import torch
    cache = D.Cache(lengths, heads_kv, d, page, seed, pages_of_a_sequence, fill=fill)
    for b, n in enumerate(lengths):
        cache.fill(b, n, seed + 1000)
    if alter is not None:
        alter(cache)
    total = sum(counts)
    qt, q = up(D.normal((total, heads * d), seed + 7, std), dtype)
    if pad:
        spread = torch.full((total, heads * d + pad), float("nan"), dtype=qt.dtype, device="cuda")
        spread[:, :heads * d] = qt
        qt = spread[:, :heads * d]
    dev = Device(B, cache, gap)
    rows = dev.rows(counts, lengths, *((1, 1) if lie else (None, longest)))
    out = torch.full((total, heads * d + pad), float("nan"), dtype=qt.dtype, device="cuda")[:, :heads * d]
    need = B.ac_cache_attention_workspace_bytes(qt, dev.desc, rows, causal)
    ws = torch.full((max(need, 16),), 0xff, dtype=torch.uint8, device="cuda")
    B.ac_op_cache_attention(qt, out, dev.desc, rows, causal, scale, ws)
    got = out.double().cpu().numpy().reshape(total, heads, d)
    scale, at = d ** -0.5 if scale is None else scale, 0
    for b, n in enumerate(counts):
        if n:
            ref, size, reach = D.attention(q[at:at + n].reshape(n, heads, d), cache, b, lengths[b] - n, lengths[b], heads // heads_kv, causal, scale)
            mine, poisoned = got[at:at + n], np.isnan(ref)
            assert np.array_equal(np.isnan(mine), poisoned), (b, np.argwhere(np.isnan(mine) != poisoned)[:5])
            bound = D.attention_bound(ref, size, reach, dtype)
            assert (np.abs(mine - ref)[~poisoned] <= bound[~poisoned]).all(), (b, np.max((np.abs(mine - ref) / bound)[~poisoned]))
        at += n
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,lengths,heads,heads_kv,d,page", [
    ([1], [1], 1, 1, 32, 16), ([1], [15], 2, 2, 64, 16), ([1], [16], 4, 1, 128, 32), ([1], [17], 7, 1, 96, 48), ([1], [64], 8, 2, 64, 64),
    ([1], [65], 16, 1, 64, 16), ([1], [1000], 4, 4, 128, 32), ([1], [777], 17, 1, 192, 16), ([1], [300], 6, 2, 256, 128),
    ([1, 1, 1, 1], [5, 0, 130, 260], 8, 2, 64, 16), ([3], [3], 4, 2, 64, 16), ([5, 2, 0, 9], [200, 2, 40, 9], 12, 4, 64, 32),
    ([33], [33], 2, 2, 32, 16), ([40], [500], 3, 1, 128, 64), ([130, 1, 64], [130, 90, 100], 4, 2, 64, 16), ([70], [400], 2, 1, 256, 16),
    ([50], [150], 2, 2, 96, 16), ([29], [333], 5, 1, 192, 32)])
@pytest.mark.parametrize("causal", [True, False])
def test_attention(B, dtype, counts, lengths, heads, heads_kv, d, page, causal):
    attention_case(B, dtype, counts, lengths, heads, heads_kv, d, page, causal, seed=sum(lengths) + d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,lengths", [([1], [4099]), ([1, 1], [3000, 17]), ([4], [2500]), ([200], [1300])])
def test_attention_over_many_tokens(B, dtype, counts, lengths):
    attention_case(B, dtype, counts, lengths, 4, 2, 64, 32, seed=31)


@pytest.mark.parametrize("d", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("counts,lengths,heads,heads_kv,page,causal", [
    ([65], [65], 1, 1, 16, True), ([150], [700], 2, 1, 48, True), ([128], [333], 1, 1, 32, False), ([257, 3, 0, 90], [257, 1400, 0, 95], 2, 2, 64, True),
    ([31], [1029], 9, 3, 16, True)])
def test_attention_prompts(B, d, counts, lengths, heads, heads_kv, page, causal):
    attention_case(B, "bf16", counts, lengths, heads, heads_kv, d, page, causal, seed=d)


@pytest.mark.parametrize("d", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("counts,lengths,heads,heads_kv,page,causal", [
    ([65], [65], 1, 1, 16, True), ([150], [700], 2, 1, 48, True), ([128], [333], 1, 1, 32, False), ([257, 3, 0, 90], [257, 1400, 0, 95], 2, 2, 64, True),
    ([31], [1029], 9, 3, 16, True), ([33, 5] + [0, 34] * 34, [40, 100] + [0, 34] * 34, 2, 2, 16, True)])
def test_attention_prompts_of_long_caches(B, d, counts, lengths, heads, heads_kv, page, causal):
    """Where the host knows of the lengths only that they are no more than 2^19, work is laid out for these."""
    attention_case(B, "bf16", counts, lengths, heads, heads_kv, d, page, causal, seed=d, longest=1 << 19)


@pytest.mark.parametrize("longest", [None, 1 << 19])
@pytest.mark.parametrize("counts,lengths", [([400], [900]), ([90, 0, 300], [2000, 7, 301])])
def test_attention_prompts_forms(B, counts, lengths, longest):
    for i, more in enumerate((dict(gap=48), dict(pad=8), dict(scale=0.37), dict(std=30.0), dict(pages_of_a_sequence=160), dict(causal=False))):
        attention_case(B, "bf16", counts, lengths, 4, 2, 64, 32, seed=i, longest=longest, **more)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_forms(B, dtype):
    attention_case(B, dtype, [3, 20], [90, 50], 4, 2, 64, 32, seed=1, gap=48)                           # pages apart
    attention_case(B, dtype, [3, 20], [90, 50], 4, 2, 64, 32, seed=2, pad=8)                            # rows apart
    attention_case(B, dtype, [3, 20], [900, 50], 4, 2, 64, 32, seed=3, lie=True)                        # more than the host said
    attention_case(B, dtype, [3, 40], [90, 50], 4, 2, 64, 32, seed=4, scale=0.37)
    attention_case(B, dtype, [3, 20], [90, 50], 4, 2, 64, 32, seed=5, std=30.0)                         # one key takes it all
    attention_case(B, dtype, [3, 140], [90, 500], 4, 2, 64, 32, seed=6, pages_of_a_sequence=40)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,lengths", [([1, 1], [100, 3]), ([70, 4], [100, 9])])
def test_attention_rows_that_see_nothing(B, dtype, counts, lengths):
    """More rows than tokens, pages that are not there, lengths of zero."""
    import torch

    def alter(cache):
        cache.table[0, 0], cache.table[0, 3] = -1, cache.pages
        cache.table[1] = -7
    got = attention_case(B, dtype, counts, lengths, 4, 2, 64, 16, seed=8, alter=alter)
    assert (got[counts[0]:] == 0).all()
    got = attention_case(B, dtype, [9, 1], [4, 0], 4, 2, 64, 16, seed=9)
    assert (got[:5] == 0).all() and (got[9] == 0).all() and (got[5:9] != 0).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts,length", [([30], 100), ([130], 200), ([1], 100)])
def test_attention_nan_reaches_only_the_rows_that_see_it(B, dtype, d, counts, length):
    """A NaN key: every row from its token on.  A NaN value: its element of these rows."""
    def alter(cache):
        for name, token, head, e in (("k", 95, 0, 3), ("v", 80, 1, 5), ("v", 99, 0, 2), ("v", 40, 1, 31), ("v", 99, 1, d - 1)):
            where = cache.block(0, token // 16)
            codes, s = cache.get(name, where, head)
            codes = codes.copy()
            codes[token % 16, e] = 0xff
            cache.put(name, where, head, codes, s, length - token // 16 * 16)
    got = attention_case(B, dtype, counts, [length], 4, 2, d, 16, seed=10, alter=alter)
    if counts[0] == 30:
        assert np.isnan(got[25:, :2]).all() and not np.isnan(got[:25, :2]).any() and np.isnan(got[10:, 2:, 5]).all() and not np.isnan(got[:10, 2:, 5]).any()


def test_attention_prompts_with_nan_and_missing_pages(B):
    def nan(cache):
        for name, token, head, e in (("k", 95, 0, 3), ("v", 80, 1, 5), ("v", 199, 0, 2), ("v", 40, 1, 31), ("v", 199, 1, 63)):
            where = cache.block(0, token // 16)
            codes, s = cache.get(name, where, head)
            codes = codes.copy()
            codes[token % 16, e] = 0xff
            cache.put(name, where, head, codes, s, 200 - token // 16 * 16)
    got = attention_case(B, "bf16", [130], [200], 4, 2, 64, 16, seed=10, alter=nan, longest=1 << 19)
    assert np.isnan(got[25:, :2]).all() and not np.isnan(got[:25, :2]).any() and np.isnan(got[10:, 2:, 5]).all() and np.isnan(got[:, 2:, 31]).all()

    def missing(cache):
        cache.table[0, 0], cache.table[0, 3] = -1, cache.pages
        cache.table[1] = -7
    got = attention_case(B, "bf16", [70, 4], [100, 9], 4, 2, 64, 16, seed=8, alter=missing, longest=1 << 19)
    assert (got[70:] == 0).all()
    got = attention_case(B, "bf16", [90, 1], [60, 0], 4, 2, 64, 16, seed=9, longest=1 << 19)
    assert (got[:30] == 0).all() and (got[90] == 0).all() and (got[30:90] != 0).any()


def test_far_pages(B):
    """Pages that begin past 2^32 bytes of codes."""
    import torch
    pages, heads, page, d = 1 << 15, 2, 128, 256
    k, v = (torch.zeros((pages, 2 * heads * page * d), dtype=torch.uint8, device="cuda") for _ in "kv")      # 4 GiB each: as much between pages as in them
    k, v = k[:, :heads * page * d].unflatten(1, (heads, page, d)), v[:, :heads * page * d].unflatten(1, (heads, page // 16, d, 16))
    ks, vs = (torch.zeros((pages, heads, page // 16), device="cuda") for _ in "kv")
    cache = B.kv_cache(k, v, ks, vs)
    assert cache.stride_page * (pages - 1) >= (1 << 32) - (1 << 18)
    table = torch.tensor([[pages - 1, 5]], dtype=torch.int32, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    n = 200
    rows = B.cache_rows(torch.tensor([0, n], **i32), torch.tensor([n], **i32), table, n, n)
    xt, x = up(D.normal((n, 3 * heads * d), 77), "f32")
    q, kn, vn = xt.split(heads * d, 1)
    B.ac_op_cache_append(kn, vn, cache, rows)
    out = torch.empty((n, heads * d), device="cuda")
    B.ac_op_cache_attention(q, out, cache, rows, workspace=B.empty_workspace(B.ac_cache_attention_workspace_bytes(q, cache, rows)))
    assert (ks[pages - 1] > 0).all() and int((ks > 0).sum()) == heads * (8 + 5)
    held = D.Cache([n], heads, d, page, 0)
    held.table[0] = [0, 1]
    for name, t in (("k", k), ("v", v), ("k_scale", ks), ("v_scale", vs)):
        getattr(held, name)[:2] = t[[pages - 1, 5]].cpu().numpy()
    fresh = D.Cache([n], heads, d, page, 0)
    fresh.table[0] = [0, 1]
    fresh.append(0, *(x[:, a * heads * d:(a + 1) * heads * d].reshape(n, heads, d) for a in (1, 2)), n)
    assert all(np.array_equal(D.VALUE[getattr(held, name)[:2]], D.VALUE[getattr(fresh, name)[:2]]) for name in "kv")
    ref, size, reach = D.attention(x[:, :heads * d].reshape(n, heads, d), held, 0, 0, n, 1, True, d ** -0.5)
    got = out.double().cpu().numpy().reshape(n, heads, d)
    assert (np.abs(got - ref) <= D.attention_bound(ref, size, reach, "f32")).all()
