"""Copies of pages of more than 2^32 codes a head, and forks of books without pages."""
import pytest

pytestmark = pytest.mark.gpu


def test_copy_of_a_large_page():
    import torch
    from paper_2401_10652_amd import binding as B
    page, d = (1 << 26) + 16, 64                                        # 4 GiB of keys, and as many of values
    cache = B.kv_cache(torch.empty((2, 1, page, d), dtype=torch.uint8, device="cuda"), torch.empty((2, 1, page // 16, d, 16), dtype=torch.uint8, device="cuda"),
                       torch.empty((2, 1, page // 16), device="cuda"), torch.empty((2, 1, page // 16), device="cuda"))
    of = [t.view(2, page // 16, -1) for t in cache.keep]
    for t in of:
        t[0, :4], t[1, :4] = 3, 5
        t[0, -2:], t[1, -2:] = 7, 9
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    B.ac_op_cache_copy_pages(B.kv_caches([cache]), ints(0), ints(1), ints(40))
    for t in of:
        assert (t[1, :3] == 3).all() and (t[1, 3] == 5).all() and (t[1, -2:] == 9).all()
    B.ac_op_cache_copy_pages(B.kv_caches([cache]), ints(0), ints(1))
    for t in of:
        assert (t[1, :4] == 3).all() and (t[1, -2:] == 7).all()


def test_fork_without_pages():
    import torch
    from paper_2401_10652_amd import binding as B
    page, none = 1 << 26, lambda *s, dtype=torch.uint8: torch.empty((0, 1, *s), dtype=dtype, device="cuda")
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = B.kv_cache(none(page, 64), none(page // 16, 64, 16), none(page // 16, dtype=torch.float32), none(page // 16, dtype=torch.float32))
    books, out = (B.page_books(ints(), torch.full((2, 3), -1, dtype=torch.int32, device="cuda"), page) for _ in range(2))
    length, missing = ints(-1, -1), ints(-1)
    B.ac_op_cache_fork(B.kv_caches([cache]), books, out, ints(1, 1), ints(20, 30), length, B.empty_workspace(B.ac_pages_workspace_bytes(books)), missing)
    assert length.tolist() == [30, 30] and out.keep[1].tolist() == [[-1] * 3] * 2 and missing.item() == 0
