"""The decoding operators at their edges, on the host: no GPU, no pointer followed."""
import os
import random
import subprocess
import sys

import pytest

import launch_stub
import w4_steps as W
from paper_2401_10652_amd import inputs as I


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


def test_attention_workspace_stays_small(tmp_path):
    """The parts of rows over split keys: no more than what fills the chip once (256 tiles of 128 rows), or, of rows that are few in a sequence (32 of a key head), a part for every
    2048 tokens, which is a 31st of the codes that they read."""
    launch_stub.run(launch_stub.build(str(tmp_path)), """
rng, split = random.Random(3), 0
def need(dtype, batch, rows, total, length, heads, group, d):
    c = B.ac_kv_cache(k=X, v=Y, k_scale=W, v_scale=W + 4096, pages=10, stride_page=heads * 64 * d, stride_scale=heads * 4, page=64, heads=heads, head_dim=d)
    r = B.ac_cache_rows(row_begin=X, length=Y, page_table=W, ld_page_table=1 << 14, batch=batch, max_rows=rows, max_length=length)
    return L.ac_cache_attention_workspace_bytes(total, heads * group, ctypes.byref(c), ctypes.byref(r), 1, dtype)
for dtype in (B.AC_F32, B.AC_BF16):
    for i in range(3000):
        batch, rows, length = (int(2 ** rng.uniform(0, e)) for e in (8, 13, 18))
        heads, group, d = rng.choice((1, 2, 8, 16)), rng.choice((1, 4, 7)), rng.choice((32, 64, 128, 256))
        total = rng.randint(rows, rows * batch)
        got = need(dtype, batch, rows, total, length, heads, group, d)
        split += got > 0
        fill, runs = 256 * 128 * (d + 2) * 4, batch * heads * length * (d + 2) // 16
        # (rows of a tile that is not full are counted by their tile, and where sequences differ the longest's count is taken for all)
        assert got <= max(fill, runs), (dtype, batch, rows, total, length, heads, group, d, got)
    assert split > 100
assert need(B.AC_F32, 2, 8192, 16384, 8192, 16, 1, 128) == 0 and need(B.AC_F32, 8, 512, 4096, 65536, 16, 1, 128) == 0 and need(B.AC_F32, 2, 65536, 131072, 65536, 16, 1, 128) == 0
""")


@pytest.mark.parametrize("name", ["C1", "C3"])
def test_decoder_refuses_models_that_are_not_causal(name):
    from paper_2401_10652_amd.decode import Decoder
    with pytest.raises(ValueError, match="not causal"):
        Decoder(I.CONFIGS[name], [], 1, 16)
    r = subprocess.run([sys.executable, "-m", "paper_2401_10652_amd.decode", "--config", name], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True)
    assert r.returncode == 2 and "invalid choice" in r.stderr


def test_calls_with_nothing_in_them(tmp_path):
    """No sequences, no rows, sequences without places, a cache without pages: empty tensors, whose addresses are NULL."""
    launch_stub.run(launch_stub.build(str(tmp_path)), """
import torch
B._stream = lambda: 0
i = lambda *x: torch.tensor(x, dtype=torch.int32)
u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
table = lambda *s: torch.zeros(s, dtype=torch.int32)
def cache(pages): return B.kv_cache(u8(pages, 2, 32, 64), u8(pages, 2, 2, 64, 16), torch.ones(pages, 2, 2), torch.ones(pages, 2, 2))
x = torch.zeros(2, 128)
for c, begin, length, t, n, launches in ((cache(3), i(0), i(), table(0, 3), 0, 0), (cache(3), i(0, 0), i(5), table(1, 3), 0, 0), (cache(3), i(0, 1, 2), i(1, 1), table(2, 0), 2, 1),
                                         (cache(0), i(0, 1, 2), i(1, 1), table(2, 3), 2, 1)):
    rows = B.cache_rows(begin, length, t, 1, 1)
    assert rows.ld_page_table == t.shape[1] and B.ac_cache_attention_workspace_bytes(x[:n], c, rows) == 0
    B.ac_op_cache_append(x[:n], x[:n], c, rows)
    assert len(kernels()) == launches
    B.ac_op_cache_attention(x[:n], x[:n], c, rows)
    assert len(kernels()) == launches
assert B.cache_rows(i(0, 1), i(1), table(4, 8)[1:2, 3:5], 1, 1).ld_page_table == 2         # one row's places, not those between it and the next
""")


def test_cache_of_other_formats_is_refused():
    import torch
    from paper_2401_10652_amd import binding as B
    k, v, s = torch.zeros((3, 2, 32, 64), dtype=torch.uint8), torch.zeros((3, 2, 2, 64, 16), dtype=torch.uint8), torch.ones(3, 2, 2)
    B.kv_cache(k, v, s, s)
    B.kv_cache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), s, s)
    for other in (torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz):
        for bad in ((k.view(other), v), (k, v.view(other))):
            with pytest.raises(TypeError):
                B.kv_cache(*bad, s, s)


def test_decoder_asks_for_a_workspace_without_making_rows():
    import torch
    from paper_2401_10652_amd import binding as B
    from paper_2401_10652_amd.decode import Decoder
    model = object.__new__(Decoder)
    model.cfg, model.dtype, model.heads_kv = I.C2, torch.bfloat16, 16
    model.caches = [B.kv_cache(torch.zeros((3, 16, 32, 64), dtype=torch.uint8), torch.zeros((3, 16, 2, 64, 16), dtype=torch.uint8), *(torch.ones(3, 16, 2) for _ in "kv"))]
    i32 = dict(dtype=torch.int32)
    rows = B.cache_rows(torch.zeros(2, **i32), torch.zeros(1, **i32), torch.zeros((1, 2048), **i32), 1, 65536)
    q = torch.empty((1, 1024), dtype=torch.bfloat16)
    assert model._workspace_bytes(1, rows) == B.ac_cache_attention_workspace_bytes(q, model.caches[0], rows) > 0
    rows = B.cache_rows(torch.zeros(2, **i32), torch.zeros(1, **i32), torch.zeros((1, 2048), **i32), 1 << 26, 65536)
    assert model._workspace_bytes(1 << 26, rows) == 0                 # (128 GiB of queries)


def test_launches_of_the_largest_calls(tmp_path, monkeypatch):
    """A launch has less than 2^32 threads along each side: the stub refuses others, as the runtime does."""
    source = launch_stub.SOURCE
    for old, new in (("__hipPushCallConfiguration(grid3 g, grid3 b, size_t lds, void* stream) { return 0; }",
                      "__hipPushCallConfiguration(grid3 g, grid3 b, size_t lds, void* stream) { grid = g; block = b; return 0; }"),
                     ("__hipPopCallConfiguration(grid3* g, grid3* b, size_t* lds, void** stream) { return 0; }",
                      "__hipPopCallConfiguration(grid3* g, grid3* b, size_t* lds, void** stream) { *g = grid; *b = block; return 0; }"),
                     ("  int i = 0;\n", "  int i = 0;\n  if ((unsigned long long)g.x * b.x >> 32 || g.y > 65535 || g.z > 65535) return error = 9;\n"),
                     ("static int n_known", "static int error;\nstatic grid3 grid, block;\nstatic int n_known"),
                     ("int hipGetLastError(void) { return 0; }", "int hipGetLastError(void) { int e = error; error = 0; return e; }")):
        assert source.count(old) == 1
        source = source.replace(old, new)
    monkeypatch.setattr(launch_stub, "SOURCE", source)
    launch_stub.run(launch_stub.build(str(tmp_path)), """
N = 1 << 30
def cache(d): return B.ac_kv_cache(k=X, v=Y, k_scale=W, v_scale=W + 4096, pages=1 << 24, stride_page=16 * d, stride_scale=1, page=16, heads=1, head_dim=d)
def rows(batch, most, length): return B.ac_cache_rows(row_begin=X, length=Y, page_table=W, ld_page_table=1 << 26, batch=batch, max_rows=most, max_length=length)
for d in (32, 256):
    for batch, most in ((1, N), (2, N), (65535, 1 << 15)):
        for dtype in (B.AC_BF16, B.AC_F32):
            c, r = cache(d), rows(batch, most, N)
            assert L.ac_op_cache_append(None, 0, None, 0, 0, X, d, Y, d, N, ctypes.byref(c), ctypes.byref(r), None, dtype, None) == 0, L.ac_last_error()
            for most in (most, 1):                                 # few rows of a sequence, many of the matrices
                r = rows(batch, most, N)
                need = L.ac_cache_attention_workspace_bytes(N, 1, ctypes.byref(c), ctypes.byref(r), 1, dtype)
                assert L.ac_op_cache_attention(X, d, Y, d, N, 1, ctypes.byref(c), ctypes.byref(r), 1, 0.1, W, need, dtype, None) == 0, L.ac_last_error()
for m, n in ((1, 1 << 26), (16 * 65535, 1 << 26), (200, 1 << 26), (16 * 65535, 16)):
    for dtype in (B.AC_BF16, B.AC_F32):
        for group in (32, 128):
            assert L.ac_op_linear_w4(X, 64, Y, 32, W, 2, None, 0, group, None, None, 0, W + 4096, 1 << 26, m, n, 64, 0, dtype, None) == 0, L.ac_last_error()
assert L.ac_op_linear_w4(X, 64, Y, 32, W, 2, None, 0, 32, None, None, 0, W + 4096, 1 << 27, 1, (1 << 26) + 1, 64, 0, B.AC_BF16, None) == B.AC_ERR_UNSUPPORTED
assert kernels()
""")


def test_workspace_of_calls_that_are_refused(tmp_path):
    """Rows times heads past what a call takes: no size, as no launch could use it."""
    launch_stub.run(launch_stub.build(str(tmp_path)), """
c = B.ac_kv_cache(k=X, v=Y, k_scale=W, v_scale=W + 4096, pages=10, stride_page=64 * 64, stride_scale=4, page=64, heads=1, head_dim=64)
for rows, heads in ((1 << 30, 64), (1 << 30, 2), (1 << 20, 1 << 11), (1 << 16, 1 << 17)):
    for dtype in (B.AC_F32, B.AC_BF16):
        r = B.ac_cache_rows(row_begin=X, length=Y, page_table=W, ld_page_table=1 << 14, batch=2, max_rows=rows, max_length=1 << 20)
        assert L.ac_cache_attention_workspace_bytes(rows, heads, ctypes.byref(c), ctypes.byref(r), 1, dtype) == 0
        assert L.ac_op_cache_attention(X, heads * 64, Y, heads * 64, rows, heads, ctypes.byref(c), ctypes.byref(r), 1, 0.1, W, 1 << 62, dtype, None) < 0
""")
