"""Attention through a sliding window with sinks, over the 8-bit cache, against its definition in 64 bits, at the windows, lengths and values where it can go wrong."""
import numpy as np
import pytest

import decode_ref as D
from test_gpu_decode import B, Device, up  # noqa: F401

pytestmark = pytest.mark.gpu


def attention(q, cache, b, length, group, window, sinks, scale):
    """(out, the bound's sizes) of the last rows q [rows, heads, d] of a sequence of `length` tokens: see decode_ref.attention."""
    rows, heads, d = q.shape
    out, size, reach = np.zeros((rows, heads, d)), np.zeros((rows, heads, d)), 0.0
    held = max(0, min(length, cache.table.shape[1] * cache.page))
    there = np.array([cache.block(b, t // D.BLOCK) is not None for t in range(held)], bool)
    t, place = np.arange(held), np.arange(length - rows, length)[:, None]
    see = there & (t <= place) & ((place - t < window) | (t < sinks))
    some = see.any(1)
    if not some.any():
        return out, size, reach
    for h in range(heads):
        if h % group == 0:
            k, v = (cache.tokens(n, b, h // group, held) for n in "kv")
            k[~see.any(0)] = 0
            nan = np.isnan(v)
            v[nan] = 0
            poison = see.astype(float) @ nan > 0 if nan[see.any(0)].any() else np.zeros((rows, d), bool)
        s = np.where(see, q[:, h] @ k.T * scale, -np.inf)
        reach = max(reach, float(np.nanmax(np.where(see, np.abs(q[:, h]) @ np.abs(k).T, 0.0))) * scale)
        p = np.exp(s - np.where(some, s.max(1), 0.0)[:, None])
        p /= np.where(some, p.sum(1), 1.0)[:, None]
        out[:, h], size[:, h] = np.where(poison, np.nan, p @ v), p @ np.abs(v)
    return out, size, reach


def case(B, dtype, counts, lengths, heads, heads_kv, d, page, window, sinks, seed=0, gap=0, lie=False, pad=0, scale=None, std=1.0, alter=None,
         gone=True, places=None):
    """What no row sees is NaN, codes and scales, and (gone) pages of which no row sees a token have no number."""
    import torch
    cache = D.Cache(lengths, heads_kv, d, page, seed, places, fill=0x7f)
    for b, n in enumerate(lengths):
        cache.fill(b, n, seed + 1000)
        first = n - counts[b]
        for i in range(-(-n // page)):
            hidden = i * page >= sinks and ((i + 1) * page <= first - window + 1 or not counts[b])
            if hidden:
                cache.k[cache.table[b, i]], cache.v[cache.table[b, i]] = 0xff, 0x7f
                if gone:
                    cache.table[b, i] = -1 if i % 2 else cache.pages + i
    if alter is not None:
        alter(cache)
    total = sum(counts)
    qt, q = up(D.normal((total, heads * d), seed + 7, std), dtype)
    if pad:
        spread = torch.full((total, heads * d + pad), float("nan"), dtype=qt.dtype, device="cuda")
        spread[:, :heads * d] = qt
        qt = spread[:, :heads * d]
    dev = Device(B, cache, gap)
    rows = dev.rows(counts, lengths, *((1, 1) if lie else (None, None)))
    whole = torch.full((total + 2, heads * d + pad), 7.0, dtype=qt.dtype, device="cuda")
    out = whole[:total, :heads * d]
    need = B.ac_cache_attention_window_workspace_bytes(qt, dev.desc, rows, window, sinks)
    ws = torch.full((max(need, 16),), 0xff, dtype=torch.uint8, device="cuda")
    B.ac_op_cache_attention_window(qt, out, dev.desc, rows, window, sinks, scale, ws)
    got = out.double().cpu().numpy().reshape(total, heads, d)
    assert (whole[total:] == 7).all() and (whole[:, heads * d:] == 7).all()
    scale, at = d ** -0.5 if scale is None else scale, 0
    for b, n in enumerate(counts):
        if n:
            ref, size, reach = attention(q[at:at + n].reshape(n, heads, d), cache, b, lengths[b], heads // heads_kv, window, sinks, scale)
            mine, poisoned = got[at:at + n], np.isnan(ref)
            assert np.array_equal(np.isnan(mine), poisoned), (b, np.argwhere(np.isnan(mine) != poisoned)[:5])
            bound = D.attention_bound(ref, size, reach, dtype)
            assert (np.abs(mine - ref)[~poisoned] <= bound[~poisoned]).all(), (b, np.max((np.abs(mine - ref) / bound)[~poisoned]))
        at += n
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 16), (17, 5), (64, 33), (100, 4), (400, 0), (1 << 30, 7), (0, 20), (3, 1 << 30)])
@pytest.mark.parametrize("counts,lengths,heads,heads_kv,d,page", [
    ([1], [1], 1, 1, 32, 16), ([1], [130], 4, 1, 128, 32), ([1, 1, 1, 1], [5, 0, 130, 333], 8, 2, 64, 16), ([5, 2, 0, 9], [200, 2, 40, 9], 12, 4, 64, 32),
    ([40], [300], 3, 1, 96, 64), ([33], [33], 2, 2, 32, 16)])
def test_window(B, dtype, window, sinks, counts, lengths, heads, heads_kv, d, page):  # noqa: F811
    case(B, dtype, counts, lengths, heads, heads_kv, d, page, window, sinks, seed=sum(lengths) + d + sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 192, 256])
def test_window_head_widths(B, dtype, d):  # noqa: F811
    case(B, dtype, [1, 20, 3], [400, 333, 90], 6, 2, d, 16, 50, 6, seed=d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,lengths,window,sinks", [([1], [9000], 2500, 4), ([1, 1], [3000, 17], 1500, 40), ([4], [9000], 1200, 0), ([200], [1300], 700, 10),
                                                         ([1, 7, 1], [70, 5000, 2000], 4000, 1000)])
def test_window_in_runs(B, dtype, counts, lengths, window, sinks):  # noqa: F811
    """Windows of several runs of keys."""
    case(B, dtype, counts, lengths, 4, 2, 64, 32, window, sinks, seed=31)


def tiles_of_128(counts, heads, heads_kv, lengths, window, sinks):
    """Whether these bf16 calls go by tiles of 128 rows: more than 32 rows of a key head, and heads x rows x the tokens that a tile reads."""
    rows, total, group = max(counts), sum(counts), heads // heads_kv
    tokens = min(max(lengths), -(-sinks // 16) * 16 + window + 16 + min(rows, -(-128 // group) + 1))
    all_rows = rows * len(counts) if rows < total // len(counts) else total
    return rows * group > 32 and all_rows * heads * tokens >= 1 << 24


PROMPTS = [([1100], [1300], 64, 2, 16, 240, 20), ([1900], [2000], 128, 32, 32, 5, 3), ([2100], [2100], 64, 64, 48, 1, 0), ([700, 3, 0, 1100], [800, 1400, 0, 1101], 64, 8, 64, 100, 33),
           ([1400], [2500], 32, 32, 16, 300, 129)]


@pytest.mark.parametrize("counts,lengths,heads,heads_kv,page,window,sinks", PROMPTS)
def test_window_prompts(B, counts, lengths, heads, heads_kv, page, window, sinks):  # noqa: F811
    """Tiles of 128 rows, whose windows begin and end inside tiles of keys."""
    assert tiles_of_128(counts, heads, heads_kv, lengths, window, sinks)
    case(B, "bf16", counts, lengths, heads, heads_kv, 64, page, window, sinks, seed=window)


@pytest.mark.parametrize("d", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("counts,lengths,heads,heads_kv,page,window,sinks", [
    ([1100], [1300], 64, 2, 16, 240, 20), ([600, 600], [900, 2500], 16, 2, 64, 1000, 64), ([512], [4600], 8, 1, 32, 7000, 0)])
def test_window_prompts_head_widths(B, d, counts, lengths, heads, heads_kv, page, window, sinks):  # noqa: F811
    assert tiles_of_128(counts, heads, heads_kv, lengths, window, sinks)
    case(B, "bf16", counts, lengths, heads, heads_kv, d, page, window, sinks, seed=d)


@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 200), (1 << 30, 0), (63, 1), (65, 63)])
def test_window_prompts_windows(B, window, sinks):  # noqa: F811
    counts, lengths = [2048], [2200]
    assert tiles_of_128(counts, 128, 4, lengths, window, sinks) == (window + sinks > 0)
    got = case(B, "bf16", counts, lengths, 128, 4, 32, 16, window, sinks, seed=window % 100)
    assert (got == 0).all() == (window + sinks == 0)


@pytest.mark.parametrize("d,window,sinks", [(64, 9, 40), (256, 120, 41), (32, 300, 0)])
def test_window_prompts_nan_and_missing_pages(B, d, window, sinks):  # noqa: F811
    def alter(cache):
        rng = np.random.default_rng(window)
        for i in range(60):
            name, token, head, e = ("v", "k")[i % 20 == 0], int(rng.integers(0, 2000)), int(rng.integers(0, 2)), int(rng.integers(0, 6))
            where = cache.block(0, token // 16)
            if where is not None:
                codes, s = cache.get(name, where, head)
                codes = codes.copy()
                codes[token % 16, e] = 0xff
                cache.put(name, where, head, codes, s, 2000 - token // 16 * 16)
        cache.table[0, 60], cache.table[0, 70] = -1, cache.pages
    assert tiles_of_128([1900], 128, 4, [2000], window, sinks)
    got = case(B, "bf16", [1900], [2000], 128, 4, d, 16, window, sinks, seed=10, alter=alter)
    assert np.isnan(got).any() and not np.isnan(got).all()


@pytest.mark.parametrize("more", [dict(gap=48), dict(pad=8), dict(scale=0.37), dict(std=30.0), dict(places=160), dict(gone=False)])
def test_window_prompts_forms(B, more):  # noqa: F811
    case(B, "bf16", [1100, 4], [1300, 90], 64, 2, 32, 16, 240, 20, seed=2, **more)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_window_forms(B, dtype):  # noqa: F811
    for i, more in enumerate((dict(gap=48), dict(pad=8), dict(lie=True), dict(scale=0.37), dict(std=30.0), dict(places=40), dict(gone=False))):
        case(B, dtype, [3, 140], [900, 500], 4, 2, 64, 32, 100, 20, seed=i, **more)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_window_rows_that_see_nothing(B, dtype):  # noqa: F811
    """More rows than tokens, pages of the window and of the sinks that are not there, lengths of zero, no window and no sinks."""
    got = case(B, dtype, [9, 1], [4, 0], 4, 2, 64, 16, 3, 1, seed=9)
    assert (got[:5] == 0).all() and (got[9] == 0).all() and (got[5:9] != 0).any()

    def missing(cache):
        cache.table[0, 0], cache.table[0, 5] = -1, cache.pages
        cache.table[1] = -7
    got = case(B, dtype, [70, 4], [100, 9], 4, 2, 64, 16, 10, 5, seed=8, alter=missing)
    assert (got[70:] == 0).all()
    assert (case(B, dtype, [50], [80], 4, 2, 64, 16, 0, 0, seed=3) == 0).all()


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 64), ("bf16", 128), ("bf16", 256)])
@pytest.mark.parametrize("counts,window,sinks", [([30], 20, 4), ([130], 9, 0), ([130], 50, 41), ([180], 7, 45), ([1], 20, 3)])
def test_window_nan_reaches_only_the_rows_that_see_it(B, dtype, d, counts, window, sinks):  # noqa: F811
    """NaN keys and values, several of an element, between which rows see none."""
    def alter(cache):
        for name, token, head, e in (("k", 95, 0, 3), ("v", 80, 1, 5), ("v", 150, 1, 5), ("v", 199, 0, 2), ("v", 40, 1, 31), ("v", 42, 0, 30), ("v", 2, 1, 7), ("v", 120, 1, d - 1),
                                     ("v", 60, 0, 1), ("v", 100, 0, 1), ("v", 140, 0, 1)):
            where = cache.block(0, token // 16)
            if where is None:
                continue
            codes, s = cache.get(name, where, head)
            codes = codes.copy()
            codes[token % 16, e] = 0xff
            cache.put(name, where, head, codes, s, 200 - token // 16 * 16)
    got = case(B, dtype, counts, [200], 4, 2, d, 16, window, sinks, seed=10, alter=alter)
    assert np.isnan(got).any() and not np.isnan(got).all()


def test_window_that_reaches_all_is_causal_attention(B):  # noqa: F811
    """The same bits where the window holds every token (and the split is the same)."""
    import torch
    for dtype, counts, lengths in (("bf16", [1, 1], [3000, 700]), ("f32", [5], [900]), ("bf16", [600], [2000])):
        cache = D.Cache(lengths, 2, 64, 32, 5)
        for b, n in enumerate(lengths):
            cache.fill(b, n, 1005)
        dev = Device(B, cache, 0)
        rows = dev.rows(counts, lengths, None, None)
        q, _ = up(D.normal((sum(counts), 8 * 64), 12), dtype)
        a, b = torch.empty_like(q), torch.empty_like(q)
        need = B.ac_cache_attention_workspace_bytes(q, dev.desc, rows)
        assert need == B.ac_cache_attention_window_workspace_bytes(q, dev.desc, rows, 1 << 30, 3)
        ws = B.empty_workspace(need)
        B.ac_op_cache_attention(q, a, dev.desc, rows, workspace=ws)
        B.ac_op_cache_attention_window(q, b, dev.desc, rows, 1 << 30, 3, workspace=ws)
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,counts,length", [("f32", [9], 350), ("bf16", [60], 345), ("bf16", [3], 900)])
@pytest.mark.parametrize("window,sinks", [(30, 20), (500, 0), (70, 300)])
def test_window_of_a_text_longer_than_its_table(B, dtype, counts, length, window, sinks):  # noqa: F811
    """Tokens without a place (the table has 304) count as masked."""
    import torch
    cache = D.Cache([300], 2, 64, 16, 3)
    cache.fill(0, 300, 1003)
    dev = Device(B, cache, 0)
    q, q64 = up(D.normal((counts[0], 4 * 64), 4), dtype)
    rows = dev.rows(counts, [length])
    out = torch.full_like(q, float("nan"))
    B.ac_op_cache_attention_window(q, out, dev.desc, rows, window, sinks, workspace=B.empty_workspace(B.ac_cache_attention_window_workspace_bytes(q, dev.desc, rows, window, sinks)))
    got = out.double().cpu().numpy().reshape(counts[0], 4, 64)
    ref, size, reach = attention(q64.reshape(counts[0], 4, 64), cache, 0, length, 2, window, sinks, 64 ** -0.5)
    assert (np.abs(got - ref) <= D.attention_bound(ref, size, reach, dtype)).all()


def test_window_of_a_long_text(B):  # noqa: F811
    """Places near 2^30, of which only the pages in the window are there; launches of such tables read nothing behind them."""
    import torch
    length, window, sinks, page, d = (1 << 30) - 5, 100, 20, 128, 64
    cache = D.Cache([300], 1, d, page, 3)
    cache.fill(0, 300, 1003)
    dev = Device(B, cache, 0)
    places = (1 << 30) // page
    table = torch.full((1, places), -1, dtype=torch.int32, device="cuda")
    used = [0, places - 2, places - 1]
    table[0, torch.tensor(used, device="cuda")] = torch.from_numpy(cache.table[0].copy()).cuda()
    q, q64 = up(D.normal((3, 2 * d), 4), "f32")
    i32 = dict(dtype=torch.int32, device="cuda")
    rows = B.cache_rows(torch.tensor([0, 3], **i32), torch.tensor([length], **i32), table, 3, length)
    out = torch.empty_like(q)
    ws = B.empty_workspace(B.ac_cache_attention_window_workspace_bytes(q, dev.desc, rows, window, sinks))
    B.ac_op_cache_attention_window(q, out, dev.desc, rows, window, sinks, workspace=ws)
    got = out.double().cpu().numpy().reshape(3, 2, d)
    # the three pages as a text of 384 places, of which the last five are not written
    near = D.Cache([300], 1, d, page, 3)
    near.fill(0, 300, 1003)
    for r in range(3):
        place = 3 * page - 5 - 3 + r
        see = [t for t in range(place + 1) if t < sinks or place - t < window]
        k, v = (near.tokens(n, 0, 0, 3 * page)[see] for n in "kv")
        for h in range(2):
            s = k @ q64[r].reshape(2, d)[h] * d ** -0.5
            p = np.exp(s - s.max())
            p /= p.sum()
            bound = D.attention_bound(p @ v, p @ np.abs(v), float((np.abs(k) @ np.abs(q64[r].reshape(2, d)[h])).max()) * d ** -0.5, "f32")
            assert (np.abs(got[r, h] - p @ v) <= bound).all()
