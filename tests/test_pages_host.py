"""The page books' refusals and launches, on the host: no GPU, no pointer followed."""
import pytest

import launch_stub

SETUP = """
import ctypes

def cache(**kw):
    d = dict(k=1 << 40, v=1 << 41, k_scale=1 << 42, v_scale=1 << 43, pages=10, stride_page=2 * 32 * 64, stride_scale=4, page=32, heads=2, head_dim=64)
    return B.ac_kv_cache(**{**d, **kw})

def caches(*found):
    return (B.ac_kv_cache * max(1, len(found)))(*found), len(found)

def books(**kw):
    d = dict(uses=1 << 44, page_table=1 << 45, pages=10, ld_page_table=6, batch=3, page=32)
    return B.ac_page_books(**{**d, **kw})

def other(**kw):
    return books(**{**dict(uses=1 << 46, page_table=1 << 47), **kw})

byref = lambda x: None if x is None else ctypes.byref(x)
NONE = object()
P = 1 << 38
SPACE = dict(ws=W, size=1 << 40)

def update(a=None, b=None, drop=(P, P + 64), take=(P + 128, P + 192), missing=None, ws=W, size=1 << 40):
    return L.ac_op_pages_update(byref(None if a is NONE else a or books()), byref(None if b is NONE else b or other()), *drop, *take, missing, ws, size, None)

def fork(c=None, a=None, b=None, parent=P, length=P + 64, length_to=P + 128, missing=None, ws=W, size=1 << 40):
    array, n = c or caches(cache(), cache(heads=1))
    return L.ac_op_cache_fork(array, n, byref(None if a is NONE else a or books()), byref(None if b is NONE else b or other()), parent, length, length_to, missing, ws, size, None)

def compact(c=None, a=None, b=None, used=None, ws=W, size=1 << 40):
    array, n = c or caches(cache())
    return L.ac_op_cache_compact(array, n, byref(None if a is NONE else a or books()), byref(None if b is NONE else b or other()), used, ws, size, None)

def copy(c=None, source=P, target=P + 64, tokens=None, n=5):
    array, count = c or caches(cache())
    return L.ac_op_cache_copy_pages(array, count, source, target, tokens, n, None)

def refused(status, what, **kw):
    got = what(**kw)
    assert got == status, (what.__name__, kw, got, L.ac_last_error())
    assert kernels() == [] and L.ac_last_error()

need = L.ac_pages_workspace_bytes(byref(books()))
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    lib = launch_stub.build(str(tmp_path_factory.mktemp("stub")))
    return lambda code: launch_stub.run(lib, SETUP + code)


def test_books(run):
    run("""
assert need > 0
for what in (update, fork, compact):
    assert what() == 0, L.ac_last_error()
    assert what(size=need) == 0 and what(b=books() if what is not fork else other(uses=1 << 44)) == 0 and kernels()
    for a in (dict(uses=None), dict(page_table=None), dict(pages=-1), dict(ld_page_table=-1), dict(batch=-1), dict(page=0), dict(page=24)):
        refused(B.AC_ERR_ARG, what, a=books(**a))
        refused(B.AC_ERR_ARG, what, b=other(**a))
    for a in (dict(pages=11), dict(ld_page_table=5), dict(batch=2), dict(page=16)):                       # not of the same sizes
        refused(B.AC_ERR_ARG, what, b=other(**a))
    for a in (dict(uses=(1 << 44) + 36), dict(uses=(1 << 44) - 4), dict(page_table=(1 << 45) + 68), dict(page_table=(1 << 45) - 4)):       # overlapping in part
        refused(B.AC_ERR_ARG, what, b=other(**a))
    assert what(b=other(uses=(1 << 44) + 40, page_table=(1 << 45) + 72)) == 0 and kernels()
    for a in (NONE,):
        refused(B.AC_ERR_ARG, what, a=a)
        refused(B.AC_ERR_ARG, what, b=a)
    for a in (dict(pages=(1 << 24) + 1), dict(batch=65536), dict(ld_page_table=(1 << 25) + 1)):
        refused(B.AC_ERR_UNSUPPORTED, what, a=books(**a), b=other(**a))
    for a in (dict(uses=(1 << 44) + 2), dict(page_table=(1 << 45) + 1)):
        refused(B.AC_ERR_ALIGN, what, a=books(**a))
    for kw in (dict(ws=None), dict(ws=W + 8), dict(size=need - 1)):
        refused(B.AC_ERR_WORKSPACE, what, **kw)
for kw in (dict(drop=(P, None)), dict(drop=(None, P)), dict(take=(P, None)), dict(take=(None, P))):
    refused(B.AC_ERR_ARG, update, **kw)
assert update(drop=(None, None), take=(None, None)) == 0
assert L.ac_pages_workspace_bytes(None) == 0 and L.ac_pages_workspace_bytes(byref(books(page=24))) == 0
""")


def test_uses_and_tables_apart_and_ranks_in_32_bits(run):
    run("""
for what in (update, fork, compact):
    for a, b in ((dict(), dict(uses=(1 << 45) + 68)), (dict(), dict(page_table=(1 << 44) - 68)), (dict(uses=(1 << 45) - 36), dict()), (dict(), dict(page_table=(1 << 46) + 36))):
        refused(B.AC_ERR_ARG, what, a=books(**a), b=other(**b))
    assert what(b=other(uses=(1 << 45) + 72, page_table=(1 << 44) - 72)) == 0 and kernels()
    # entries of a table: 65535 x 16385 is more than 2^30, 65535 x 16384 is less
    large, rest = dict(batch=65535, ld_page_table=16384, uses=1 << 50), dict(length_to=P + (1 << 20)) if what is fork else {}
    assert what(a=books(**large, page_table=1 << 52), b=other(**{**large, "uses": 1 << 51}, page_table=1 << 53), **rest) == 0 and kernels(), L.ac_last_error()
    large["ld_page_table"] += 1
    refused(B.AC_ERR_UNSUPPORTED, what, a=books(**large, page_table=1 << 52), b=other(**{**large, "uses": 1 << 51}, page_table=1 << 53), **rest)
assert L.ac_pages_workspace_bytes(byref(books(**large, page_table=1 << 52))) == 0
""")


def test_caches(run):
    run("""
for what in (fork, compact, copy):
    for c in (dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(pages=-1), dict(page=24), dict(heads=0), dict(head_dim=0),
              dict(stride_page=2 * 32 * 64 - 16), dict(stride_scale=3)):
        refused(B.AC_ERR_ARG, what, c=caches(cache(), cache(**c)))
    refused(B.AC_ERR_ARG, what, c=(None, 1))
    refused(B.AC_ERR_ARG, what, c=(caches(cache())[0], -1))
    refused(B.AC_ERR_ARG, what, c=caches(cache(), cache(pages=11)))
    refused(B.AC_ERR_ARG, what, c=caches(cache(), cache(page=16)))
    refused(B.AC_ERR_UNSUPPORTED, what, c=caches(cache(head_dim=80, stride_page=1 << 20)))
    for c in (dict(k=(1 << 40) + 8), dict(v=(1 << 40) + 8), dict(stride_page=2 * 32 * 64 + 8)):
        refused(B.AC_ERR_ALIGN, what, c=caches(cache(**c)))
    many = caches(*[cache()] * 40)
    assert what(c=many) == 0 and len([k for k in kernels() if "pages_copy" in k and "uses" not in k]) == 3
    assert what(c=caches()) == 0 and not [k for k in kernels() if "pages_copy" in k and "uses" not in k]
for what in (fork, compact):
    refused(B.AC_ERR_ARG, what, c=caches(cache(pages=11)))
    refused(B.AC_ERR_ARG, what, c=caches(cache(page=64, stride_page=1 << 20, stride_scale=64)))
big = dict(page=1 << 25, heads=2, head_dim=256, stride_page=1 << 40, stride_scale=1 << 30)
refused(B.AC_ERR_UNSUPPORTED, copy, c=caches(cache(**big)))
""")


def test_fork_and_copy(run):
    run("""
for kw in (dict(parent=None), dict(length=None), dict(length_to=None), dict(length_to=P + 64), dict(length_to=P + 68), dict(length_to=P), dict(b=other(page_table=1 << 45))):
    refused(B.AC_ERR_ARG, fork, **kw)
assert fork(b=other(uses=1 << 44)) == 0
empty = dict(batch=0, page_table=None)
kernels()
assert fork(a=books(**empty), b=other(**empty), parent=None, length=None, length_to=None) == 0 and kernels()
for kw in (dict(source=None), dict(target=None), dict(n=-1)):
    refused(B.AC_ERR_ARG, copy, **kw)
refused(B.AC_ERR_UNSUPPORTED, copy, n=(1 << 24) + 1)
assert copy(n=0, source=None, target=None) == 0 and copy(c=caches(cache(pages=0, k=None, v=None, k_scale=None, v_scale=None))) == 0 and kernels() == []
assert copy(tokens=P + 128) == 0 and len(kernels()) == 1
""")


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    from paper_2401_10652_amd import binding as B
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    books = B.page_books(i(8), i(2, 3), 16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    assert B.ac_pages_workspace_bytes(books) <= ws.numel()
    for uses, table, error in ((i(8).long(), i(2, 3), TypeError), (i(8), i(2, 3).long(), TypeError), (i(8), i(2, 6)[:, ::2], ValueError), (i(16)[::2], i(2, 3), ValueError)):
        with pytest.raises(error):
            B.page_books(uses, table, 16)
    for kw, error in ((dict(drop=(i(2), i(3))), ValueError), (dict(take=(i(2).long(), i(2))), TypeError), (dict(missing=i(2)), ValueError), (dict(drop=(i(4)[::2], i(2))), ValueError)):
        with pytest.raises(error):
            B.ac_op_pages_update(books, books, ws, **kw)
    none = B.kv_caches([])
    for parent, length, out, error in ((i(3), i(2), i(2), ValueError), (i(2), i(2).long(), i(2), TypeError), (i(2), i(2), i(1), ValueError)):
        with pytest.raises(error):
            B.ac_op_cache_fork(none, books, books, parent, length, out, ws)
    with pytest.raises(ValueError):
        B.ac_op_cache_compact(none, books, books, ws, used=i(2))
    with pytest.raises(ValueError):
        B.ac_op_cache_copy_pages(none, i(3), i(2))
    with pytest.raises(TypeError):
        B.ac_op_cache_copy_pages(none, i(3), i(3), i(3).float())
