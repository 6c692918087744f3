"""The decoding operators' refusals and launches, on the host: no GPU, no pointer followed."""
import pytest

import launch_stub

SETUP = """
def cache(**kw):
    d = dict(k=1 << 40, v=1 << 41, k_scale=1 << 42, v_scale=1 << 43, pages=10, stride_page=2 * 32 * 64, stride_scale=4, page=32, heads=2, head_dim=64)
    return B.ac_kv_cache(**{**d, **kw})

def rows(**kw):
    d = dict(row_begin=1 << 44, length=1 << 45, page_table=1 << 46, ld_page_table=4, batch=3, max_rows=1, max_length=100)
    return B.ac_cache_rows(**{**d, **kw})

def rot(sections=(32,), **kw):
    import ctypes
    d = dict(cos=1 << 40, sin=1 << 41, table_rows=100, ld_table=32, positions=None, ld_positions=0, pairs=32, interleaved=0, axes=len(sections))
    r = B.ac_rotary(**{**d, **kw})
    for i, s in enumerate(sections): r.section[i] = s
    return r

def byref(x):
    import ctypes
    return None if x is None else ctypes.byref(x)

def attention(c=None, r=None, q=X, ldq=256, out=Y, ldo=256, n=3, heads=4, causal=1, scale=0.1, ws=W, ws_bytes=1 << 40, dtype=B.AC_BF16, no=()):
    return L.ac_op_cache_attention(q, ldq, out, ldo, n, heads, None if "cache" in no else byref(c or cache()), None if "rows" in no else byref(r or rows()),
                                   causal, scale, ws, ws_bytes, dtype, None)

def append(c=None, r=None, ro=None, n=3, q=X, ldq=512, q_out=Y, ldqo=256, heads=4, k=W, ldk=512, v=W + 4096, ldv=512, dtype=B.AC_BF16):
    return L.ac_op_cache_append(q, ldq, q_out, ldqo, heads, k, ldk, v, ldv, n, byref(c or cache()), byref(r or rows()), byref(ro), dtype, None)

def linear(x=X, ldx=256, w=Y, ldw=128, scale=W, lds=2, zero=None, ldz=0, group=128, bias=None, residual=None, ldr=0, out=W + 4096, ldo=64, m=4, n=64,
           k=256, act=0, dtype=B.AC_BF16):
    return L.ac_op_linear_w4(x, ldx, w, ldw, scale, lds, zero, ldz, group, bias, residual, ldr, out, ldo, m, n, k, act, dtype, None)

def refused(status, **kw):
    what = kw.pop("what")
    got = what(**kw)
    assert got == status, (what.__name__, kw, got, L.ac_last_error())
    assert kernels() == [] and L.ac_last_error()
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return launch_stub.build(str(tmp_path_factory.mktemp("stub")))


def test_linear_w4_refusals(lib):
    launch_stub.run(lib, SETUP + """
assert linear() == 0 and len(kernels()) == 1
assert linear(m=0) == 0 and linear(n=0) == 0 and kernels() == []
for kw in (dict(x=None), dict(w=None), dict(scale=None), dict(out=None), dict(m=-1), dict(n=-1), dict(k=0), dict(ldx=255), dict(ldo=63), dict(lds=1),
           dict(zero=X, ldz=1), dict(residual=X, ldr=63), dict(group=0), dict(group=-32), dict(act=-1), dict(act=6), dict(dtype=2), dict(ldw=112)):
    refused(B.AC_ERR_ARG, what=linear, **kw)
for kw in (dict(group=16, lds=16), dict(group=96, lds=3), dict(group=192), dict(m=1 << 21)):
    refused(B.AC_ERR_UNSUPPORTED, what=linear, **kw)
for kw in (dict(w=Y + 8), dict(ldw=136)):
    refused(B.AC_ERR_ALIGN, what=linear, **kw)
""")


def test_cache_refusals(lib):
    launch_stub.run(lib, SETUP + """
for what in (attention, append):
    assert what() == 0, L.ac_last_error()
    assert kernels()
    assert what(r=rows(batch=0)) == 0 and what(n=0) == 0 and kernels() == []
    for c in (dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(pages=-1), dict(page=0), dict(page=24), dict(heads=0), dict(head_dim=0),
              dict(stride_page=2 * 32 * 64 - 16), dict(stride_scale=3)):
        refused(B.AC_ERR_ARG, what=what, c=cache(**c))
    for r in (dict(row_begin=None), dict(length=None), dict(page_table=None), dict(ld_page_table=-1), dict(batch=-1), dict(max_rows=-1),
              dict(max_length=-1)):
        refused(B.AC_ERR_ARG, what=what, r=rows(**r))
    for r in (dict(batch=65536), dict(max_length=(1 << 30) + 1), dict(ld_page_table=(1 << 25) + 1)):
        refused(B.AC_ERR_UNSUPPORTED, what=what, r=rows(**r))
    refused(B.AC_ERR_ARG, what=what, n=-1)
    refused(B.AC_ERR_UNSUPPORTED, what=what, n=(1 << 30) + 1)
    refused(B.AC_ERR_UNSUPPORTED, what=what, c=cache(head_dim=80, stride_page=1 << 20))
    for c in (dict(k=(1 << 40) + 8), dict(v=(1 << 40) + 8), dict(stride_page=2 * 32 * 64 + 8)):
        refused(B.AC_ERR_ALIGN, what=what, c=cache(**c))
    refused(B.AC_ERR_ARG, what=what, dtype=2)
for no in ("cache", "rows"):
    refused(B.AC_ERR_ARG, what=attention, no=(no,))
""")


def test_append_refusals(lib):
    launch_stub.run(lib, SETUP + """
assert append(q=None, q_out=None, heads=0) == 0 and append(ro=rot()) == 0 and append(ro=rot((), pairs=0, axes=1, cos=None, sin=None)) == 0 and kernels()
for kw in (dict(k=None), dict(v=None), dict(ldk=127), dict(ldv=127), dict(q_out=None), dict(heads=0), dict(ldq=255), dict(ldqo=255)):
    refused(B.AC_ERR_ARG, what=append, **kw)
for kw in (dict(q=X + 4), dict(q_out=Y + 2), dict(k=W + 4), dict(v=W + 2), dict(ldk=514), dict(ldqo=258)):
    refused(B.AC_ERR_ALIGN, what=append, **kw)
refused(B.AC_ERR_ALIGN, what=append, k=W + 8, dtype=B.AC_F32)
for kw in (dict(cos=None), dict(sin=None), dict(pairs=-4), dict(pairs=36, sections=(36,)), dict(sections=(31,)), dict(sections=(40, -8)), dict(table_rows=0),
           dict(ld_table=28), dict(axes=0), dict(axes=5), dict(sections=(16, 16), positions=X, ld_positions=2)):
    refused(B.AC_ERR_ARG, what=append, ro=rot(**kw))
refused(B.AC_ERR_UNSUPPORTED, what=append, ro=rot(pairs=30, sections=(30,)))
for no_pairs in (dict(ld_table=1), dict(cos=X + 4, sin=X + 8, ld_table=3), dict(table_rows=1 << 40)):
    assert append(ro=rot(**{**dict(sections=(0,), pairs=0, axes=1), **no_pairs})) == 0 and kernels()
assert append(ro=rot(table_rows=1 << 25)) == 0 and append(ro=rot((), pairs=0, axes=1, cos=None, sin=None, ld_table=0)) == 0 and kernels()
refused(B.AC_ERR_UNSUPPORTED, what=append, ro=rot(table_rows=(1 << 25) + 1))
for kw in (dict(cos=X + 4), dict(sin=X + 8), dict(ld_table=34)):
    refused(B.AC_ERR_ALIGN, what=append, ro=rot(**kw))
""")


def test_attention_refusals(lib):
    launch_stub.run(lib, SETUP + """
for kw in (dict(q=None), dict(out=None), dict(heads=0), dict(heads=3), dict(ldq=255), dict(ldo=255), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
           dict(scale=float("inf"))):
    refused(B.AC_ERR_ARG, what=attention, **kw)
for kw in (dict(q=X + 8), dict(out=Y + 8), dict(ldq=260), dict(ldo=260)):
    refused(B.AC_ERR_ALIGN, what=attention, **kw)
r = rows(batch=1, max_length=65536, ld_page_table=2048)
need = L.ac_cache_attention_workspace_bytes(3, 4, byref(cache()), byref(r), 1, B.AC_BF16)
if need:
    for kw in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=W + 8)):
        refused(B.AC_ERR_WORKSPACE, what=attention, r=r, **kw)
    assert attention(r=r, ws_bytes=need) == 0
assert L.ac_cache_attention_workspace_bytes(3, 3, byref(cache()), byref(r), 1, B.AC_BF16) == 0
assert L.ac_cache_attention_workspace_bytes(3, 4, None, byref(r), 1, B.AC_BF16) == 0
""")


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    from paper_2401_10652_amd import binding as B
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    k, v, s = u8(3, 2, 32, 64), u8(3, 2, 2, 64, 16), torch.ones(3, 2, 2)
    B.kv_cache(k, v, s, s)
    for bad in ((k, v[:, :, :1], s, s), (k, v, s[:2], s), (k.transpose(2, 3), v, s, s)):
        with pytest.raises(ValueError):
            B.kv_cache(*bad)
    with pytest.raises(TypeError):
        B.kv_cache(k, v, s.double(), s)
    with pytest.raises(TypeError):
        B.kv_cache(k.float(), v, s, s)
    i = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    table = torch.zeros((2, 3), dtype=torch.int32)
    cache, rows = B.kv_cache(k, v, s, s), B.cache_rows(i(0, 1, 2), i(1, 1), table, 1, 1)
    with pytest.raises(TypeError):
        B.cache_rows(i(0, 1, 2).long(), i(1, 1), table, 1, 1)
    with pytest.raises(ValueError):
        B.cache_rows(i(0, 1), i(1, 1), table, 1, 1)
    x = torch.zeros(2, 128)
    with pytest.raises(TypeError):
        B.ac_op_cache_append(x, x.bfloat16(), cache, rows)
    with pytest.raises(ValueError):
        B.ac_op_cache_append(x, x[:1], cache, rows)
    with pytest.raises(ValueError):
        B.ac_op_cache_append(x[:, :100], x, cache, rows)
    with pytest.raises(ValueError):
        B.ac_op_cache_attention(x, x[:1], cache, rows)
    with pytest.raises(ValueError):
        B.rotary(torch.zeros(4, 8), torch.zeros(4, 4))
    with pytest.raises(ValueError):
        B.rotary(torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros((2, 5), dtype=torch.int32))
    with pytest.raises(ValueError):
        B.ac_op_cache_attention(x[:, ::2], x[:, ::2], B.kv_cache(u8(3, 2, 32, 32), u8(3, 2, 2, 32, 16), s, s), rows)
    w, sc, y = u8(8, 16), torch.ones(8, 1), torch.zeros(2, 8)
    for kw in (dict(scale=sc[:4]), dict(out=y[:, :4]), dict(zero=sc[:4]), dict(bias=torch.zeros(3)), dict(w=u8(8, 8))):
        a = {**dict(x=torch.zeros(2, 32), w=w, scale=sc, out=y, group=32), **kw}
        with pytest.raises(ValueError):
            B.ac_op_linear_w4(**a)
    with pytest.raises(TypeError):
        B.ac_op_linear_w4(torch.zeros(2, 32), w.to(torch.int8), sc, y, 32)
    with pytest.raises(TypeError):
        B.ac_op_linear_w4(torch.zeros(2, 32), w, sc.bfloat16(), y, 32)
