"""A row's result among other rows: its own x and adapter decide it, bit for bit in small calls and where few adapters lie together, up to the
rounding of u's sums where many do."""
import pytest

from paper_2603_09237_amd import binding

pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1


def setup(M, I, O, r, P, dtype):
    """rows in groups, of which the first eight of every sixteen keep their adapter"""
    import torch
    from test_gpu_adapter import problem
    dims, d, ref = problem(M, I, O, r, P, dtype, "grouped", seed=M + P)
    keep = torch.arange(M, device="cuda") // 8 % 2 == 0
    return dims, d, ref, keep


def others(d, keep, P, together):
    """indices of the other rows: of each 32 the same one, or any"""
    import torch
    g = torch.Generator().manual_seed(3)
    M = keep.numel()
    new = torch.randint(0, P, (M // 32 + 1,), generator=g).repeat_interleave(32)[:M] if together else torch.randint(0, P, (M,), generator=g)
    return torch.where(keep, d["index"], new.to(torch.int32).cuda())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,I,O,r,P", [(200, 264, 392, 16, 20), (300, 27, 130, 5, 24)])
@pytest.mark.parametrize("together", [True, False])
def test_small_calls(M, I, O, r, P, together, dtype):
    import torch
    from test_gpu_adapter import run_bwd, run_fwd
    dims, d, _, keep = setup(M, I, O, r, P, dtype)
    y, dx = run_fwd(dims, d).clone(), run_bwd(dims, d, ("dx",))["dx"].clone()
    d["index"] = others(d, keep, P, together)
    assert torch.equal(run_fwd(dims, d)[keep], y[keep])
    assert torch.equal(run_bwd(dims, d, ("dx",))["dx"][keep], dx[keep])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,I,O,r,P", [(4200, 520, 520, 16, 40), (6000, 515, 523, 12, 40)])
def test_large_calls(M, I, O, r, P, dtype):
    import torch
    from test_gpu_adapter import check, definition, run_bwd, run_fwd
    dims, d, ref, keep = setup(M, I, O, r, P, dtype)
    y, dx = run_fwd(dims, d).clone(), run_bwd(dims, d, ("dx",))["dx"].clone()
    start = d["index"]
    d["index"] = others(d, keep, P, True)      # never more than four adapters among 32 rows
    assert torch.equal(run_fwd(dims, d)[keep], y[keep])
    for together in (True, False):             # (sorted for dx, few lie together either way)
        d["index"] = others(dict(index=start), keep, P, together)
        assert torch.equal(run_bwd(dims, d, ("dx",))["dx"][keep], dx[keep])
        ref["index"] = d["index"].cpu().numpy()
        want = definition(ref, P)
        check(run_fwd(dims, d), want["y"], want["yabs"], max(I, r), dtype == BF16, "y")
