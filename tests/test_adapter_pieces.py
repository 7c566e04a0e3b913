"""The factors' gradients in pieces of 256 sorted rows: adapters that begin and end at a piece's edge, inside one, or take many; and scratch
that goes by the rows, not by the adapters that could have some."""
import os

import pytest

from paper_2603_09237_amd import binding

F32, BF16 = 0, 1


def test_scratch_goes_by_the_rows():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_09237_amd import build
        build.build(verbose=False)
    wide = lambda rows, adapters: binding.adapter_workspace_bytes(binding.AdapterDims(rows, 2048, 2048, 32, adapters, BF16), True)  # noqa: E731
    # an adapter more costs its place in the sums of the bias, 8 KB here, not a place in those of its factors (512 KB)
    assert wide(4096, 4096) - wide(4096, 1) <= 4095 * (2048 * 4 + 64)
    assert wide(1, 1024) <= 16 << 20


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [(512, 512), (256, 256, 256), (255, 1, 256, 257), (100, 412, 0, 0, 1000, 3), (1, 2000, 1), (256, 0, 300, 724, 0), (40,) * 30])
def test_gradients(rows, dtype):
    import torch
    from test_gpu_adapter import check, definition, problem, run_bwd
    M, P = sum(rows), len(rows)
    dims, d, ref = problem(M, 136, 72, 8, P, dtype, "grouped", seed=M)
    index = torch.repeat_interleave(torch.arange(P), torch.tensor(rows)).to(torch.int32)
    for at in (index, index[torch.randperm(M, generator=torch.Generator().manual_seed(1))]):
        d["index"], ref["index"] = at.cuda(), at.numpy()
        want, got = definition(ref, P), run_bwd(dims, d)
        for k in ("dA", "dB", "dbias"):
            check(got[k], want[k], want[k + "abs"], max(M, 136), False, k)
