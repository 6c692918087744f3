import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def pytest_sessionstart(session):
    """The suite loads the built library; it compiles it only when none is there."""
    from paper_2401_10652_amd.build import ensure_built
    ensure_built()


def pytest_collection_modifyitems(config, items):
    """GPU tests are skipped (not failed) when no device is visible."""
    need_gpu = [it for it in items if "gpu" in it.keywords]
    if not need_gpu:
        return
    import torch
    if torch.cuda.is_available():
        return
    skip = pytest.mark.skip(reason="no GPU visible")
    for it in need_gpu:
        it.add_marker(skip)


@pytest.fixture(autouse=True, scope="module")
def _cycles_of_other_modules_are_gone():
    """Tensors that an earlier module's tests left in reference cycles (a refusal's traceback holds its frame) are freed here, and not by chance while a test
    reads how much memory is allocated."""
    import gc
    gc.collect()
