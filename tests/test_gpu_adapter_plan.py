"""Rows sorted by adapter where rows times adapters are many: the same order as of few, and work that goes by the rows and the adapters, not by
their product."""
import pytest

from paper_2603_09237_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,P,more", [(9000, 30, 60000), (70000, 24, 8000), (4097, 4000, 130000), (600, 5, 900000), (66000, 1, 8200)])
def test_adapters_without_rows_change_nothing(M, P, more):
    """The gradients of the first P adapters and of x, bit for bit, with and without `more` adapters that no row names."""
    import torch
    from test_gpu_adapter import F32, check, definition, problem, run_bwd
    I, O, r = 24, 16, 2
    dims, d, ref = problem(M, I, O, r, P, F32, "mixed", seed=M)
    d["index"][d["index"] >= P] = -1
    few = {k: v.clone() for k, v in run_bwd(dims, d).items()}
    wide = binding.AdapterDims(M, I, O, r, P + more, F32)
    for k in ("A", "B"):
        d[k] = torch.cat([d[k], torch.full((more, *d[k].shape[1:]), float("nan"), device="cuda")])
    many = run_bwd(wide, d)
    again = {k: v.clone() for k, v in many.items()}
    many = run_bwd(wide, d)
    for k in ("dx", "dw0"):
        assert torch.equal(many[k], few[k]), k
    for k in ("dA", "dB"):
        assert torch.equal(many[k][:P], few[k]), k
        assert (many[k][P:] == 0).all(), k
    for k in many:
        assert torch.equal(many[k], again[k]), k
    if P <= 30:
        want = definition(ref, P)
        check(many["dbias"], want["dbias"], want["dbiasabs"], M, False, "dbias")
        for k in ("dA", "dB"):
            check(many[k][:P], want[k], want[k + "abs"], max(M, I), False, k)


def test_rows_times_adapters_do_not_count():
    """2^22 rows of 2^18 adapters: two walks of every adapter over every row were 2^41 reads, over a second; rows and adapters once are 20 MB."""
    import torch
    M, P = 1 << 22, 1 << 18
    dims = binding.AdapterDims(M, 8, 8, 1, P, 0)
    x, dy = torch.ones(M, 8, device="cuda"), torch.ones(M, 8, device="cuda")
    w0, A, B = torch.ones(8, 8, device="cuda"), torch.ones(P, 8, 1, device="cuda"), torch.ones(P, 1, 8, device="cuda")
    index = (torch.arange(M, device="cuda") * 7919 % P).to(torch.int32)
    dA, dB = torch.empty_like(A), torch.empty_like(B)
    ws = torch.empty(binding.adapter_workspace_bytes(dims, True), dtype=torch.uint8, device="cuda")
    run = lambda: binding.adapter_bwd(dims, x, w0, A, B, index, dy, None, None, None, dA, dB, ws)  # noqa: E731
    run()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    a.record()
    run()
    b.record()
    torch.cuda.synchronize()
    assert (dA == 16 * 8).all() and (dB == 16 * 8).all()   # sixteen rows each, u = v = 8
    assert a.elapsed_time(b) < 250, a.elapsed_time(b)
