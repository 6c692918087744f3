"""Beam selection: refusals and launches, on the host: no GPU, no pointer followed."""
import pytest

import launch_stub

SETUP = """
P = 1 << 38
def select(logits=X, ld=1000, batch=2, beams=4, vocab=1000, scores=P, ended=None, keep=4, end=-1, scores_out=P + 4096, parent=P + 8192, token=P + 12288, ended_out=None, ws=W,
           size=1 << 40, dtype=B.AC_BF16):
    return L.ac_op_beam_select(logits, ld, batch, beams, vocab, scores, ended, keep, end, scores_out, parent, token, ended_out, ws, size, dtype, None)

def refused(status, **kw):
    got = select(**kw)
    assert got == status, (kw, got, L.ac_last_error())
    assert kernels() == [] and L.ac_last_error()
"""


def test_refusals(tmp_path):
    launch_stub.run(launch_stub.build(str(tmp_path)), SETUP + """
assert select() == 0 and kernels()
assert select(batch=0) == 0 and kernels() == []
assert select(ended=P + 64, end=999, ended_out=P + 16384) == 0 and select(end=0) == 0 and select(ld=5000) == 0 and select(logits=X + 2) == 0 and kernels()
for kw in (dict(logits=None), dict(scores=None), dict(scores_out=None), dict(parent=None), dict(token=None), dict(ld=999), dict(batch=-1), dict(beams=0), dict(vocab=0), dict(keep=0),
           dict(dtype=2), dict(end=1000), dict(end=-2), dict(ended=P + 64), dict(ended=P + 64, end=1000),
           dict(scores_out=P), dict(scores_out=P + 28), dict(parent=P + 4096), dict(token=P + 8192 + 28), dict(ended=P + 8192, end=1), dict(ended_out=P + 12288 - 4)):
    refused(B.AC_ERR_ARG, **kw)
for kw in (dict(batch=65536), dict(beams=65), dict(keep=65), dict(vocab=(1 << 24) + 1, ld=1 << 25)):
    refused(B.AC_ERR_UNSUPPORTED, **kw)
for kw in (dict(logits=X + 1), dict(logits=X + 2, dtype=B.AC_F32), dict(scores=P + 2), dict(ended=P + 66, end=1), dict(scores_out=P + 4098), dict(parent=P + 8193), dict(token=P + 12290),
           dict(ended_out=P + 16386)):
    refused(B.AC_ERR_ALIGN, **kw)
need = L.ac_beam_select_workspace_bytes(2, 4, 1000, 4, B.AC_BF16)
assert need > 0 and select(size=need) == 0 and kernels()
for kw in (dict(ws=None), dict(ws=W + 8), dict(size=need - 1)):
    refused(B.AC_ERR_WORKSPACE, **kw)
for bad in ((-1, 4, 1000, 4, 1), (2, 65, 1000, 4, 1), (2, 4, 0, 4, 1), (2, 4, 1000, 65, 1), (2, 4, 1000, 4, 2), (0, 4, 1000, 4, 1)):
    assert L.ac_beam_select_workspace_bytes(*bad) == 0
""")


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    from paper_2401_10652_amd import binding as B
    f, i = (lambda *s: torch.zeros(s)), (lambda *s: torch.zeros(s, dtype=torch.int32))  # noqa: E731
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    good = dict(logits=f(8, 50), scores=f(2, 4), scores_out=f(2, 3), parent=i(2, 3), token=i(2, 3), workspace=ws)
    for kw, error in ((dict(logits=f(7, 50)), ValueError), (dict(logits=f(8, 100)[:, ::2]), ValueError), (dict(logits=f(8, 50).double()), TypeError), (dict(scores=f(2, 4).double()), TypeError),
                      (dict(scores_out=f(2, 3).bfloat16()), TypeError), (dict(scores_out=f(3, 3)), ValueError), (dict(parent=i(2, 4)), ValueError), (dict(token=i(2, 3).long()), TypeError),
                      (dict(ended=i(2, 3)), ValueError), (dict(ended_out=i(2, 4)), ValueError), (dict(scores=f(2, 8)[:, ::2]), ValueError)):
        with pytest.raises(error):
            B.ac_op_beam_select(**{**good, **kw})
