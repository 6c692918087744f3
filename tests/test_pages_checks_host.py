"""The page calls' arrays beside the books: where they lie, on the host: no GPU, no pointer followed."""
import launch_stub

from test_pages_host import SETUP


def test_arrays_that_overlap_or_lie_between_elements(tmp_path):
    launch_stub.run(launch_stub.build(str(tmp_path)), SETUP + """
U, T, V, S = 1 << 44, 1 << 45, 1 << 46, 1 << 47        # uses (40 bytes) and tables (72) before and after; of three sequences
inside = (V, V + 36, V - 8, S, S + 68, S - 8)          # of three numbers one at least among what comes out
for at in inside:
    for kw in (dict(drop=(at, P)), dict(drop=(P, at)), dict(take=(at, P)), dict(take=(P, at))):
        refused(B.AC_ERR_ARG, update, **kw)
        refused(B.AC_ERR_ARG, update, b=other(uses=U), **{k: tuple(at + U - V if x == at and at - V in (0, 36, -8) else x for x in v) for k, v in kw.items()})
    refused(B.AC_ERR_ARG, fork, parent=at)
    refused(B.AC_ERR_ARG, fork, length=at)
for at in (U, U + 36, T, T + 68, V, V + 36, S, S + 68):                  # one number that comes out
    refused(B.AC_ERR_ARG, update, missing=at)
    refused(B.AC_ERR_ARG, fork, missing=at)
    refused(B.AC_ERR_ARG, compact, used=at)
    refused(B.AC_ERR_ARG, fork, length_to=at)
for at in (P, P + 8, P + 72, P + 128, P + 200):
    refused(B.AC_ERR_ARG, update, missing=at)
for at in (P + 4, P + 64, P + 128, P + 136):                             # parents, lengths, the new lengths
    refused(B.AC_ERR_ARG, fork, missing=at)
for kw in (dict(length_to=P + 8), dict(length_to=P - 8), dict(length_to=P + 56), dict(length_to=P + 72)):
    refused(B.AC_ERR_ARG, fork, **kw)
# side by side, and what is only read as often as wanted
for at in (U + 40, U - 4, T + 72, T - 4, V + 40, V - 4, S + 72, S - 4, P + 12, P + 76):
    assert update(missing=at) == 0 and fork(missing=at) == 0 and compact(used=at) == 0, (hex(at), L.ac_last_error())
assert update(drop=(P, P), take=(P, P)) == 0 and update(drop=(U, T), take=(T + 4, T + 8)) == 0 and fork(parent=T, length=U) == 0 and fork(length=P) == 0 and kernels()
assert update(drop=(V + 40, V - 12), take=(S + 72, S - 12)) == 0 and fork(parent=V - 12, length=S + 72, length_to=V + 40) == 0 and kernels()
for odd in (1, 2, 3):
    for kw in (dict(drop=(P + odd, P)), dict(drop=(P, P + odd)), dict(take=(P + odd, P)), dict(take=(P, P + odd)), dict(missing=(1 << 37) + odd)):
        refused(B.AC_ERR_ALIGN, update, **kw)
    for kw in (dict(parent=P + 256 + odd), dict(length=P + 256 + odd), dict(length_to=P + 256 + odd), dict(missing=P + 256 + odd)):
        refused(B.AC_ERR_ALIGN, fork, **kw)
    refused(B.AC_ERR_ALIGN, compact, used=P + odd)
    for kw in (dict(source=P + odd), dict(target=P + odd), dict(tokens=P + odd)):
        refused(B.AC_ERR_ALIGN, copy, **kw)
""")
