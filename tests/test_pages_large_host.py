"""Pages of so many tokens that a head's codes pass 32 bits, on the host: no GPU, no pointer followed."""
import launch_stub

from test_pages_host import SETUP


def test_copies_of_large_pages(tmp_path):
    launch_stub.run(launch_stub.build(str(tmp_path)), SETUP + """
for page in (1 << 26, (1 << 26) + 16, 1 << 27):
    big = dict(page=page, heads=1, head_dim=64, stride_page=page * 64, stride_scale=page // 16)
    assert copy(c=caches(cache(pages=2, **big))) == 0 and len(kernels()) == 1, L.ac_last_error()
    size = dict(page=page, ld_page_table=4)
    assert fork(c=caches(cache(**big)), a=books(**size), b=other(**size)) == 0 and compact(c=caches(cache(**big)), a=books(**size), b=other(**size)) == 0
    # without pages there is nothing to copy
    kernels()
    empty, size["pages"] = cache(pages=0, k=None, v=None, k_scale=None, v_scale=None, **big), 0
    for what in (fork, compact):
        assert what(c=caches(empty), a=books(**size), b=other(**size)) == 0 and not [k for k in kernels() if "pages_copy" in k and "uses" not in k]
""")
