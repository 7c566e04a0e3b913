"""Gradients that are sums over every step: what the steps' own gradients are off by has no common sign that would add up in them."""
import pytest

pytestmark = pytest.mark.gpu


def test_errors_of_the_steps_do_not_add_up():
    """Inputs of a positive mean, as SiLU leaves them, where sums that are always cut the same way show.  n steps' errors of a common size
    and independent signs add up to sqrt(n) of it, four standard deviations to four times that; an error of a state stays in it for as many
    steps as it decays in, some 16 here, which makes four times sixteen's root of it: 16.  What is always 3 % of their size low in half of
    the 65536 steps adds up to as much, and an error of a tenth to 25."""
    from test_gpu_memory import F32, run_scan, run_scan_bwd, scan_problem, scan_truth
    import torch
    T, N, H = 64, 1024, 2
    dims, h, d = scan_problem(T, N, H, 64, 1, 32, F32, 0.0, True, seed=1)
    h["xbc"] = torch.nn.functional.silu(h["xbc"])
    d["xbc"].copy_(h["xbc"])
    _, _, want = scan_truth(dims, {k: v.cuda() if v is not None else None for k, v in h.items()}, True)
    _, _, saved = run_scan(dims, d, saved=True)
    got = run_scan_bwd(dims, d, saved)
    off = got["dt"].double() - want["dt"]
    ratio = off.sum((0, 1)).abs() / off.square().sum((0, 1)).sqrt()
    assert (ratio <= 16).all(), ratio.tolist()
    off = (got["bias"].double() - want["bias"]).abs() / (got["dt"].double() - want["dt"]).square().sum((0, 1)).sqrt()
    assert (off <= 16).all(), off.tolist()
