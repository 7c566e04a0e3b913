import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(autouse=True)
def noted_addresses_stay(request, monkeypatch):
    """A test that compares addresses of tensors that were alive at different times needs every tensor whose address it notes to stay: memory
    that was freed is given out again, and whether it is depends on what ran before."""
    if request.node.name != "test_acting_shares_no_scratch_with_segments":
        return
    import torch
    kept, storage = [], torch.Tensor.untyped_storage

    def noting(self):
        kept.append(self)
        return storage(self)

    monkeypatch.setattr(torch.Tensor, "untyped_storage", noting)
