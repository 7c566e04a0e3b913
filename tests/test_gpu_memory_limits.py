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


def test_scan_and_step_of_as_many_heads_as_there_may_be():
    """N * heads next to 2^25, a wave each: every one gets h = e^(-ln 2) 1 + ln 2 (a step of softplus(0), a = -1), and y = h; in the step x, B and C
    have been through SiLU."""
    import math
    import torch
    N, H = 8191, 4096
    xbc = torch.ones(1, N, H + 2, device="cuda")
    dt, a_log = torch.zeros(1, N, H, device="cuda"), torch.zeros(H, device="cuda")
    y, state, out = torch.empty(1, N, H, device="cuda"), torch.ones(N, H, 1, 1, device="cuda"), torch.full((N * H + 64,), 7.0, device="cuda")
    dims = binding.ScanDims(1, N, H, 1, 1, 1, 0)
    ws = torch.empty(binding.scan_workspace_bytes(dims), dtype=torch.uint8, device="cuda")
    binding.scan_fwd(dims, xbc, xbc[..., H:], xbc[..., H + 1:], dt, None, a_log, None, None, None, state, y, out, None, ws)
    want = 0.5 + math.log(2)
    assert float((y - want).abs().max()) < 1e-6 and float((out[:N * H] - want).abs().max()) < 1e-6
    assert bool((out[N * H:] == 7.0).all())
    y.zero_()
    w = torch.ones(H + 2, 1, device="cuda")
    binding.memory_step(dims, 1, xbc, dt, None, w, None, a_log, None, None, None, None, state, y, None, out)
    s = 1 / (1 + math.exp(-1))
    h = 0.5 + math.log(2) * s * s
    assert float((out[:N * H] - h).abs().max()) < 1e-6 and float((y - h * s).abs().max()) < 1e-6
    assert bool((out[N * H:] == 7.0).all())
