import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_sessionstart(session):
    # the tests load the library that is built; only if there is none it is built now
    from paper_2303_06324_amd import build as _b
    _b.ensure_built()


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu on the GPU box)")


def _has_gpu():
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:
        return False


@pytest.hookimpl(trylast=True)
def pytest_collection_modifyitems(config, items):
    # files named test_zz_* last, by name, in whatever order the others come: what runs before must not find the streams that they have used
    items.sort(key=lambda it: it.path.name if it.path.name.startswith("test_zz_") else "")
    if _has_gpu():
        return
    skip = pytest.mark.skip(reason="no GPU in this environment")
    for it in items:
        if "gpu" in it.keywords:
            it.add_marker(skip)
