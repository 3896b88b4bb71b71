import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def pytest_collection_modifyitems(items):
    """Tests without the gpu marker in files named *_host.py, and in test_zz_no_alloc.py, give entry points made-up addresses, in calls that have
    to be refused: where a GPU is visible, one that is not refused would run on them."""
    host = [i for i in items if (i.path.name.endswith("_host.py") or i.path.name == "test_zz_no_alloc.py") and not i.get_closest_marker("gpu")]
    if not host:
        return
    import torch
    if torch.cuda.device_count() == 0:
        return
    skip = pytest.mark.skip(reason="made-up addresses: runs where no GPU is visible (HIP_VISIBLE_DEVICES=-1)")
    for item in host:
        item.add_marker(skip)


@pytest.fixture(scope="session")
def oracle():
    import oracle as _oracle
    _oracle.build()
    return _oracle
