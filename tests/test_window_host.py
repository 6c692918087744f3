"""Attention through a window: refusals, launches and workspaces, on the host: no GPU, no pointer followed."""
import pytest

import launch_stub

SETUP = """
from test_decode_host import SETUP
exec(SETUP)

def window(c=None, r=None, q=X, ldq=256, out=Y, ldo=256, n=3, heads=4, window=50, sinks=4, scale=0.1, ws=W, ws_bytes=1 << 40, dtype=B.AC_BF16, no=()):
    return L.ac_op_cache_attention_window(q, ldq, out, ldo, n, heads, None if "cache" in no else byref(c or cache()), None if "rows" in no else byref(r or rows()),
                                          window, sinks, scale, ws, ws_bytes, dtype, None)

def need(r, n=3, heads=4, window=50, sinks=4, dtype=B.AC_BF16):
    return L.ac_cache_attention_window_workspace_bytes(n, heads, byref(cache()), byref(r), window, sinks, dtype)
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    lib = launch_stub.build(str(tmp_path_factory.mktemp("stub")))
    return lambda code: launch_stub.run(lib, "import sys; sys.path.insert(0, 'tests')\n" + SETUP + code)


def test_refusals(run):
    run("""
assert window() == 0 and len(kernels()) == 1
assert window(r=rows(batch=0)) == 0 and window(n=0) == 0 and kernels() == []
for kw in (dict(window=-1), dict(sinks=-1), dict(window=(1 << 30) + 1), dict(sinks=(1 << 30) + 1), dict(q=None), dict(out=None), dict(heads=0), dict(heads=3),
           dict(ldq=255), dict(ldo=255), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(dtype=2), dict(n=-1), dict(no=("cache",)),
           dict(no=("rows",)), dict(c=cache(page=24)), dict(c=cache(k=None)), dict(r=rows(length=None))):
    refused(B.AC_ERR_ARG, what=window, **kw)
for kw in (dict(q=X + 8), dict(out=Y + 8), dict(ldq=260), dict(ldo=260), dict(c=cache(k=(1 << 40) + 8))):
    refused(B.AC_ERR_ALIGN, what=window, **kw)
for kw in (dict(n=(1 << 28) + 1), dict(r=rows(batch=65536)), dict(c=cache(head_dim=80, stride_page=1 << 20))):
    refused(B.AC_ERR_UNSUPPORTED, what=window, **kw)
assert b"window" in L.ac_last_error()
r = rows(batch=1, max_length=65536, ld_page_table=2048)
size = need(r, window=4096)
assert size > 0
for kw in (dict(ws=None), dict(ws_bytes=size - 1), dict(ws=W + 8)):
    refused(B.AC_ERR_WORKSPACE, what=window, r=r, window=4096, **kw)
assert window(r=r, window=4096, ws_bytes=size) == 0 and len(kernels()) == 2
""")


def test_work_goes_by_the_window(run):
    """Parts and tiles by what rows read, not by how long the text is; all of it where the window is longer."""
    run("""
far = rows(batch=1, max_length=1 << 30, ld_page_table=1 << 25)
assert need(far, window=500) == 0 and window(r=far, window=500, ws=None, ws_bytes=0) == 0
assert need(far, window=4096) == need(rows(batch=1, max_length=70000, ld_page_table=1 << 25), window=4096) > 0
assert 0 < need(far, window=4096) < L.ac_cache_attention_workspace_bytes(3, 4, byref(cache()), byref(far), 1, B.AC_BF16)
for length in (1, 100, 5000, 1 << 20):
    r = rows(batch=1, max_length=length, ld_page_table=1 << 20)
    assert need(r, window=1 << 30, sinks=1 << 30) == L.ac_cache_attention_workspace_bytes(3, 4, byref(cache()), byref(r), 1, B.AC_BF16)
for bad in (dict(window=-1), dict(sinks=-1), dict(heads=3), dict(dtype=2), dict(n=-1)):
    assert need(far, **{**dict(window=4096), **bad}) == 0
kernels()
big = rows(batch=1, max_rows=2048, max_length=16384, ld_page_table=1 << 20)
assert window(r=big, n=2048, heads=16, ldq=1024, ldo=1024, window=4096) == 0 and any("prefill" in k for k in kernels())
assert window(r=big, n=2048, heads=16, ldq=1024, ldo=1024, window=16) == 0 and not any("prefill" in k for k in kernels())
""")


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    from paper_2401_10652_amd import binding as B
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    i = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    cache = B.kv_cache(u8(3, 2, 32, 64), u8(3, 2, 2, 64, 16), torch.ones(3, 2, 2), torch.ones(3, 2, 2))
    rows = B.cache_rows(i(0, 1, 2), i(1, 1), torch.zeros((2, 3), dtype=torch.int32), 1, 1)
    x = torch.zeros(2, 128)
    for q, out in ((x, x[:1]), (x[:, :100], x), (x[:, ::2], x[:, ::2])):
        with pytest.raises(ValueError):
            B.ac_op_cache_attention_window(q, out, cache, rows, 10)
    with pytest.raises(TypeError):
        B.ac_op_cache_attention_window(x, x.bfloat16(), cache, rows, 10)
