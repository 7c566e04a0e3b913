"""The memory's entry points at the ends of what they serve."""
import pytest

from paper_2603_09237_amd import binding

pytestmark = pytest.mark.gpu


def test_convolution_of_as_many_environments_as_there_may_be():
    """N next to 2^31 with a single channel: gradients of every environment, none beyond.  (Sums of ones below 2^24 a workgroup and of whole
    millions over them: exact but for the last, short workgroup.)"""
    import torch
    N = 2 ** 31 - 1
    x = torch.ones(1, N, 1, dtype=torch.bfloat16, device="cuda")
    dy = torch.ones_like(x)
    out = torch.full((N + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    w, b = torch.full((1, 1), 0.5, device="cuda"), torch.full((1,), 1.0, device="cuda")
    dims = binding.ConvDims(1, N, 1, 1, 0, 1)
    binding.conv_fwd(dims, x, w, b, None, None, out, None)
    assert bool((out[:N] == 1.5).all()) and bool((out[N:] == 7.0).all())
    out.fill_(7.0)
    ws = torch.empty(binding.conv_workspace_bytes(dims), dtype=torch.uint8, device="cuda")
    dw, db = torch.full((1, 1), 7.0, device="cuda"), torch.full((1,), 7.0, device="cuda")
    binding.conv_bwd(dims, x, w, b, None, None, dy, None, out, dw, db, None, ws)
    assert bool((out[:N] == 0.5).all()) and bool((out[N:] == 7.0).all())
    assert abs(float(dw) - N) <= 256 and abs(float(db) - N) <= 256
