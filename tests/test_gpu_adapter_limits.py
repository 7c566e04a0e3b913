"""The adapters' entry points at the ends of what they serve."""
import pytest

from paper_2603_09237_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P", [1, 3])    # one walk over all rows for every adapter, and chunks of rows
def test_as_many_rows_as_there_may_be(P):
    """2^28 rows of one value: outputs exact, sums within 2^-20 (sums of 32 products, then of workgroups, all of one sign)."""
    import torch
    M = 1 << 28
    m = torch.arange(M, device="cuda", dtype=torch.int32)
    x, index = (m % 5 + 1).float()[:, None], m % (P + 1) - 1
    w0, A, B = torch.full((1, 1), 2.0, device="cuda"), torch.arange(1.0, P + 1, device="cuda")[:, None, None].clone(), torch.full((P, 1, 1), 0.5, device="cuda")
    factor = torch.where(index >= 0, 0.5 * (index + 1), 0.0)[:, None]
    dims = binding.AdapterDims(M, 1, 1, 1, P, 0)
    y = torch.empty(M, 1, device="cuda")
    ws = torch.empty(binding.adapter_workspace_bytes(dims, True), dtype=torch.uint8, device="cuda")
    binding.adapter_fwd(dims, x, w0, None, A, B, index, y, ws)
    assert torch.equal(y, x * (2.0 + factor))
    dy = torch.ones_like(x)
    dw0, db, dA, dB = (torch.empty(s, device="cuda") for s in ((1, 1), (1,), (P, 1, 1), (P, 1, 1)))
    binding.adapter_bwd(dims, x, w0, A, B, index, dy, y, dw0, db, dA, dB, ws)
    assert torch.equal(y, 2.0 + factor)
    near = lambda a, b: abs(float(a) - float(b)) <= 2.0 ** -20 * abs(float(b))  # noqa: E731
    assert near(dw0, x.double().sum()) and near(db, M)
    for p in range(P):
        s = x[index == p].double().sum()
        assert near(dA[p], 0.5 * s) and near(dB[p], (p + 1) * s), p
