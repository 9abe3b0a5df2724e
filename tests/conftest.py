import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA GPU (GB300) and the built CUDA library")


def pytest_collection_modifyitems(items):
    """Tests of a machine without a device hand the library addresses that are none and count on the call's failing for
    want of a device: with one they would read there."""
    apart = [i for i in items if i.name.endswith("_without_device")]
    if apart:
        import torch

        if torch.cuda.is_available():
            for item in apart:
                item.add_marker(pytest.mark.skip(reason="for machines without a GPU: passes addresses that are none"))


@pytest.fixture(scope="session")
def oracle_mod():
    import oracle
    oracle.build()
    return oracle
