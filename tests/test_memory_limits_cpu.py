"""Sizes next to the limits of the memory's entry points, without a GPU: what no launch could hold is refused on the host."""
import os

import pytest

from paper_2603_09237_amd import binding

GOOD = 0x10000


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_09237_amd import build
        build.build(verbose=False)
    return binding.load()


def dims(N, heads, groups, dtype):
    return binding.ScanDims(1, N, heads, 1, groups, 1, dtype)


def test_scan_backward_beyond_a_launch():
    """2^24 workgroups of 256 threads, one for every head where no heads share a group, are 2^32 threads."""
    d, ws = dims(1 << 12, 1 << 12, 1 << 12, 1), (GOOD, 1 << 62)
    with pytest.raises(binding.MorlaxError) as e:
        binding.scan_bwd(d, GOOD, GOOD, GOOD, GOOD, None, GOOD, None, None, None, GOOD, GOOD, None, GOOD + 64, GOOD + 64, GOOD + 64, GOOD + 64, None, None, None,
                         None, None, ws, stream=0)
    assert e.value.code == binding.ERR_UNSUPPORTED and "2^24" in str(e.value)
    for query in (lambda: binding.scan_workspace_bytes(d, True), lambda: binding.scan_saved_bytes(d)):
        with pytest.raises(binding.MorlaxError):
            query()
    assert binding.scan_workspace_bytes(d) > 0      # the forward takes a wave a head


@pytest.mark.parametrize("N,heads,groups,dtype", [((1 << 12) - 1, 1 << 12, 1 << 12, 1), (1 << 12, 1 << 12, 1 << 11, 1), (1 << 12, 1 << 12, 1 << 12, 0),
                                                  ((1 << 13) - 1, 1 << 12, 1 << 12, 0), ((1 << 13) - 1, 1 << 12, 1 << 10, 1)])
def test_scan_backward_within_a_launch(N, heads, groups, dtype):
    d = dims(N, heads, groups, dtype)
    assert binding.scan_workspace_bytes(d, True) > 0 and binding.scan_saved_bytes(d) > 0


def refused_as_its_input(call):
    with pytest.raises(binding.MorlaxError) as e:
        call()
    assert e.value.code == binding.ERR_SHAPE and "an output is its input" in str(e.value)


def test_outputs_over_inputs():
    """Other workgroups read what an output over its input would have overwritten."""
    d, ws = binding.AdapterDims(8, 16, 16, 4, 3, 1), (GOOD, 1 << 40)
    refused_as_its_input(lambda: binding.adapter_fwd(d, GOOD, GOOD, None, GOOD, GOOD, GOOD, GOOD, ws, stream=0))
    for dx in (GOOD, GOOD + 64):
        refused_as_its_input(lambda: binding.adapter_bwd(d, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD + 64, dx, None, None, None, None, ws, stream=0))
    d = binding.ScanDims(1, 3, 4, 16, 2, 8, 1, z_n=72)
    for y in (GOOD, GOOD + 64):
        refused_as_its_input(lambda: binding.memory_step(d, 4, GOOD, GOOD, GOOD + 64, GOOD, None, GOOD, None, None, None, None, None, y, None, GOOD, stream=0))
