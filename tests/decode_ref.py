"""What the decoding operators compute, in 64 bits on the host, and small inputs for them (test infrastructure only)."""
import math

import numpy as np

from paper_2401_10652_amd import inputs as I

BLOCK = 16
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}       # half a unit in the last place, relative


def normal(shape, seed, std=1.0):
    n = int(np.prod(shape))
    return (I.standard_normal(700000 + seed, n) * std).reshape(shape)


def uniform_ints(low, high, shape, seed):
    """Whole numbers in [low, high)."""
    n = int(np.prod(shape))
    u = (I.splitmix64(np.arange(n, dtype=np.uint64) + np.uint64((800000 + seed) << 32)) >> np.uint64(11)).astype(np.float64) * 2.0 ** -53
    return (low + np.floor(u * (high - low))).astype(np.int64).reshape(shape)


# ---- e4m3 --------------------------------------------------------------------------------------------------------

def _values():
    v = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = math.nan if c & 127 == 127 else -x if c >> 7 else x
    return v


VALUE = _values()
_POS = VALUE[:127]                                # ascending


def to_codes(x):
    """The nearest e4m3 codes of 64-bit numbers, ties to the even code; what is not finite, or past 464, is NaN."""
    x = np.asarray(x, np.float64)
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(_POS, a), 1, 126)
    lo = hi - 1
    up, down = _POS[hi] - a, a - _POS[lo]
    c = np.where(up < down, hi, np.where(down < up, lo, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(a == 0, 0, np.where(a > 464, 127, np.where(a > 448, 126, c)))
    c = np.where(np.isfinite(x), c, 127)
    return (c + 128 * np.signbit(x)).astype(np.uint8)


def scale_of(largest):
    """The least power of two s >= 2^-100 with largest <= 448 s."""
    e = -100
    if largest > 448 * 2.0 ** -100:
        e = math.ceil(math.log2(largest / 448))
        e += int(448 * 2.0 ** e < largest) - int(448 * 2.0 ** (e - 1) >= largest)
    return 2.0 ** e


# ---- linear layer -----------------------------------------------------------------------------------------------------

def pack(codes, ldw=None):
    """uint8 [n, ldw] of codes [n, k]; what lies past column k is all ones."""
    n, k = codes.shape
    ldw = ldw or -(-k // 32) * 16
    full = np.full((n, 2 * ldw), 15, np.uint8)
    full[:, :k] = codes
    return full[:, 0::2] | full[:, 1::2] << 4


def linear(x, codes, scale, zero, group, bias=None, act=None, residual=None):
    """(out, the sum of the magnitudes that the products are made of: what rounding errors are relative to)."""
    k = codes.shape[1]
    over = lambda t: np.repeat(np.asarray(t, np.float64), group, 1)[:, :k]  # noqa: E731
    z = np.full(codes.shape, 8.0) if zero is None else over(zero)
    w = (codes - z) * over(scale)
    y = x @ w.T + (0.0 if bias is None else bias)
    size = np.abs(x) @ ((32.0 + codes + np.abs(z)) * np.abs(over(scale))).T + (0.0 if bias is None else np.abs(bias))
    if act is not None:
        y = act(y)
    return (y, size) if residual is None else (y + residual, size + np.abs(residual))


# ---- cache ------------------------------------------------------------------------------------------------------------------

def rotate(x, c, s, interleaved):
    """x [rows, heads, width]; c, s [rows, pairs]."""
    x, p = x.copy(), c.shape[1]
    one, two = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if interleaved else (slice(0, p), slice(p, 2 * p))
    a, b = x[..., one].copy(), x[..., two].copy()
    x[..., one], x[..., two] = a * c[:, None] - b * s[:, None], a * s[:, None] + b * c[:, None]
    return x


class Cache:
    """A host cache: codes [pages, heads, page, d] and [pages, heads, page / 16, d, 16], scales, page table and lengths."""

    def __init__(self, lengths, heads, d, page, seed, pages_of_a_sequence=None, spare=1, fill=0):
        self.page, self.heads, self.d = page, heads, d
        need = [-(-n // page) for n in lengths]
        self.pages = sum(need) + spare
        order = np.argsort(uniform_ints(0, 1 << 40, (self.pages,), seed), kind="stable")
        self.table = np.full((len(lengths), pages_of_a_sequence or max(max(need), 1)), -1, np.int32)
        at = 0
        for b, c in enumerate(need):
            self.table[b, :c] = order[at:at + c]
            at += c
        self.k = np.full((self.pages, heads, page, d), fill, np.uint8)
        self.v = np.full((self.pages, heads, page // BLOCK, d, BLOCK), fill, np.uint8)
        self.k_scale = np.full((self.pages, heads, page // BLOCK), np.nan if fill else 1.0)
        self.v_scale = self.k_scale.copy()

    def block(self, b, j):
        """(page, block in it) of block j of sequence b, or None."""
        n = j * BLOCK // self.page
        if n >= self.table.shape[1] or not 0 <= self.table[b, n] < self.pages:
            return None
        return int(self.table[b, n]), j % (self.page // BLOCK)

    def fill(self, b, tokens, seed, std=1.0):
        """Sequence b's first tokens: normal numbers, each block with its own scale."""
        for j in range(-(-tokens // BLOCK)):
            where = self.block(b, j)
            for h in range(self.heads):
                for i, name in enumerate("kv"):
                    x = normal((BLOCK, self.d), seed + ((b * 4096 + j) * 64 + h) * 2 + i, std)
                    x[max(0, tokens - j * BLOCK):] = 0
                    s = scale_of(np.abs(x).max())
                    self.put(name, where, h, to_codes(x / s), s, tokens - j * BLOCK)

    def put(self, name, where, h, codes, s, tokens=BLOCK):
        p, i = where
        n = min(tokens, BLOCK)
        if name == "k":
            self.k[p, h, i * BLOCK:i * BLOCK + n] = codes[:n]
            self.k_scale[p, h, i] = s
        else:
            self.v[p, h, i, :, :n] = codes[:n].T
            self.v_scale[p, h, i] = s

    def get(self, name, where, h):
        p, i = where
        if name == "k":
            return self.k[p, h, i * BLOCK:(i + 1) * BLOCK], self.k_scale[p, h, i]
        return self.v[p, h, i].T, self.v_scale[p, h, i]

    def tokens(self, name, b, h, n):
        """[n, d] values of sequence b's tokens (NaN where there is no page)."""
        out = np.full((-(-n // BLOCK) * BLOCK, self.d), np.nan)
        for j in range(-(-n // BLOCK)):
            where = self.block(b, j)
            if where is not None:
                c, s = self.get(name, where, h)
                out[j * BLOCK:(j + 1) * BLOCK] = VALUE[c] * s
        return out[:n]

    def append(self, b, k, v, length):
        """Rows k, v [rows, heads, d] (already rotated) become the last of sequence b's `length` tokens."""
        first = length - k.shape[0]
        for name, x in (("k", k), ("v", v)):
            for j in range(max(first, 0) // BLOCK, -(-length // BLOCK)):
                where = self.block(b, j)
                if where is None:
                    continue
                at = np.arange(j * BLOCK, (j + 1) * BLOCK)
                new, old = (at >= max(first, 0)) & (at < length), at < max(first, 0)
                for h in range(self.heads):
                    rows = x[at[new] - first, h]
                    fine = np.abs(rows[np.isfinite(rows)])
                    s = scale_of(fine.max() if fine.size else 0.0)
                    codes, before = self.get(name, where, h)
                    codes = codes.copy()
                    if old.any():
                        s = max(s, before)
                        codes[old] = to_codes(VALUE[codes[old]] * (before / s))
                    codes[new] = to_codes(rows / s)
                    self.put(name, where, h, codes, s)


def attention(q, cache, b, first, length, group, causal, scale):
    """(out, and what its rounding errors are relative to: sum p |v|, the largest |q| . |k| scale) of rows q [rows, heads, d]."""
    rows, heads, d = q.shape
    out, size, reach = np.zeros((rows, heads, d)), np.zeros((rows, heads, d)), 0.0
    held = min(length, cache.table.shape[1] * cache.page)
    for h in range(heads):
        k, v = (cache.tokens(n, b, h // group, max(held, 0)) for n in "kv")
        there = np.array([cache.block(b, j // BLOCK) is not None for j in range(max(held, 0))], bool)
        for r in range(rows):
            n = min(max(first + r + 1, 0), max(held, 0)) if causal else max(held, 0)
            see = np.flatnonzero(there[:n])
            if not see.size:
                continue
            s = k[see] @ q[r, h] * scale
            reach = max(reach, float(np.nanmax(np.abs(k[see]) @ np.abs(q[r, h]) * scale, initial=0.0)))
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h], size[r, h] = p @ v[see], p @ np.abs(v[see])
    return out, size, reach


def attention_bound(out, size, reach, dtype):
    """Scores: products summed in 32 bits and scaled, at most 8 roundings of what they are made of; a relative error of twice that in
    each probability and as much in their sum; sums of the products with the values and the joins, 16 roundings; probabilities (bf16 only) and result rounded once."""
    u = U["f32"]
    p = 4 * 8 * u * reach + 16 * u
    return (p + (U["bf16"] if dtype == "bf16" else 0.0)) * size + U[dtype] * np.abs(out) * 1.01 + 1e-30
