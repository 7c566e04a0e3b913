"""What the entry points of the adapters and of the memory refuse, and what they ask for, without a GPU: every check is made on the host
before the first launch (the addresses here are fake)."""
import os

import pytest

from paper_2603_09237_amd import binding

GOOD, ODD = 0x10000, 0x10002
NULL, SHAPE, UNSUPPORTED, WORKSPACE = binding.ERR_NULL, binding.ERR_SHAPE, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_09237_amd import build
        build.build(verbose=False)
    return binding.load()


def refused(code, call):
    with pytest.raises(binding.MorlaxError) as e:
        call()
    assert e.value.code == code, str(e.value)
    assert str(e.value)


def adapter(**over):
    d = dict(rows=8, d_in=16, d_out=24, rank=4, adapters=3, dtype=1)
    d.update(over)
    return binding.AdapterDims(**d)


ADAPTER_BAD = [(dict(rows=-1), SHAPE), (dict(d_in=0), SHAPE), (dict(d_out=0), SHAPE), (dict(rank=0), SHAPE), (dict(adapters=0), SHAPE),
               (dict(dtype=2), UNSUPPORTED), (dict(rank=33), UNSUPPORTED), (dict(d_in=65537), UNSUPPORTED), (dict(adapters=(1 << 20) + 1), UNSUPPORTED),
               (dict(ld_x=15), SHAPE), (dict(ld_y=23), SHAPE), (dict(rows=1 << 24, d_out=65536), UNSUPPORTED),
               (dict(rows=(1 << 28) + 1, d_out=1), UNSUPPORTED)]


@pytest.mark.parametrize("over,code", ADAPTER_BAD)
def test_adapter_dimensions(over, code):
    d, ws = adapter(**over), (GOOD, 1 << 50)
    refused(code, lambda: binding.adapter_fwd(d, GOOD, GOOD, None, GOOD, GOOD, GOOD, GOOD, ws, stream=0))
    refused(code, lambda: binding.adapter_bwd(d, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, ws, stream=0))
    with pytest.raises(binding.MorlaxError):
        binding.adapter_workspace_bytes(d)


def test_adapter_pointers_and_workspace():
    d = adapter()
    fwd = dict(x=GOOD, w0=GOOD, bias=GOOD, A=GOOD, B=GOOD, index=GOOD, y=GOOD)
    need = binding.adapter_workspace_bytes(d)

    def call(ws=(GOOD, need), **over):
        binding.adapter_fwd(d, **dict(fwd, **over), ws=ws, stream=0)

    for k in fwd:
        if k != "bias":
            refused(NULL, lambda: call(**{k: None}))
        refused(SHAPE, lambda: call(**{k: GOOD + 1}))
        if k not in ("x", "y"):      # rows may begin at any element, everything else at 16 bytes
            refused(SHAPE, lambda: call(**{k: GOOD + 4}))
    refused(WORKSPACE, lambda: call(ws=(GOOD, need - 1)))
    refused(NULL, lambda: call(ws=None))
    back = dict(x=GOOD, w0=GOOD, A=GOOD, B=GOOD, index=GOOD, dy=GOOD, dx=GOOD, dw0=GOOD, dbias=GOOD, dA=GOOD, dB=GOOD)
    need = binding.adapter_workspace_bytes(d, True)
    assert need > binding.adapter_workspace_bytes(d)

    def bwd(ws=(GOOD, need), **over):
        binding.adapter_bwd(d, **dict(back, **over), ws=ws, stream=0)

    for k in back:
        if k not in ("dx", "dw0", "dbias", "dA", "dB"):
            refused(NULL, lambda: bwd(**{k: None}))
        refused(SHAPE, lambda: bwd(**{k: GOOD + 1}))
    refused(WORKSPACE, lambda: bwd(ws=(GOOD, need - 1)))
    # no rows: nothing is read, so nothing of them has to be there (and the forward launches nothing)
    binding.adapter_fwd(adapter(rows=0), None, GOOD, None, GOOD, GOOD, None, None, (GOOD, 1 << 20), stream=0)


def conv(**over):
    d = dict(T=5, N=3, channels=16, width=4, act=1, dtype=1)
    d.update(over)
    return binding.ConvDims(**d)


@pytest.mark.parametrize("over,code", [(dict(T=0), SHAPE), (dict(N=0), SHAPE), (dict(channels=0), SHAPE), (dict(width=0), SHAPE),
                                       (dict(width=5), UNSUPPORTED), (dict(act=2), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(x_t=15), SHAPE),
                                       (dict(y_n=8), SHAPE), (dict(channels=(1 << 20) + 1), UNSUPPORTED),
                                       (dict(channels=1 << 20, N=1 << 11), UNSUPPORTED)])
def test_convolution_dimensions(over, code):
    d = conv(**over)
    refused(code, lambda: binding.conv_fwd(d, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD + 64, GOOD + 64, stream=0))
    with pytest.raises(binding.MorlaxError):
        binding.conv_workspace_bytes(d)


def test_convolution_pointers_and_workspace():
    d = conv()
    fwd = dict(x=GOOD, w=GOOD, b=GOOD, first=GOOD, state_in=GOOD, y=GOOD + 64, state_out=GOOD + 64)

    def call(**over):
        binding.conv_fwd(d, **dict(fwd, **over), stream=0)

    for k in ("x", "w", "y"):
        refused(NULL, lambda: call(**{k: None}))
    for k in ("x", "w", "b", "state_in", "y", "state_out"):
        refused(SHAPE, lambda: call(**{k: GOOD + 1}))
    refused(SHAPE, lambda: call(y=GOOD))           # in place
    refused(SHAPE, lambda: call(state_out=GOOD))
    need = binding.conv_workspace_bytes(d)
    back = dict(x=GOOD, w=GOOD, b=GOOD, first=GOOD, state_in=GOOD, dy=GOOD, dstate_out=GOOD, dx=GOOD + 64, dw=GOOD, db=GOOD, dstate_in=GOOD + 64)

    def bwd(ws=(GOOD, need), **over):
        binding.conv_bwd(d, **dict(back, **over), ws=ws, stream=0)

    for k in ("x", "w", "dy", "dx"):
        refused(NULL, lambda: bwd(**{k: None}))
    for k in back:
        if k != "first":
            refused(SHAPE, lambda: bwd(**{k: GOOD + 1}))
    refused(SHAPE, lambda: bwd(dx=GOOD))
    refused(WORKSPACE, lambda: bwd(ws=(GOOD, need - 1)))


def scan(**over):
    d = dict(T=5, N=3, heads=4, head_dim=16, groups=2, state=8, dtype=1)
    d.update(over)
    return binding.ScanDims(**d)


SCAN_BAD = [(dict(T=0), SHAPE), (dict(N=0), SHAPE), (dict(heads=0, groups=1), SHAPE), (dict(head_dim=0), SHAPE), (dict(state=0), SHAPE), (dict(groups=3), SHAPE),
            (dict(dtype=2), UNSUPPORTED), (dict(head_dim=65), UNSUPPORTED), (dict(state=65), UNSUPPORTED), (dict(x_n=63), SHAPE), (dict(y_t=1), SHAPE),
            (dict(dt_n=3), SHAPE), (dict(heads=1 << 16, groups=1 << 16, head_dim=1, state=1, N=1 << 9), UNSUPPORTED)]


@pytest.mark.parametrize("over,code", SCAN_BAD)
def test_scan_dimensions(over, code):
    d, ws = scan(**over), (GOOD, 1 << 50)
    refused(code, lambda: binding.scan_fwd(d, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD + 64, GOOD, None, ws, stream=0))
    for query in (binding.scan_saved_bytes, binding.scan_workspace_bytes):
        with pytest.raises(binding.MorlaxError):
            query(d)


def test_scan_pointers_and_workspace():
    d = scan()
    fwd = dict(x=GOOD, b=GOOD, c=GOOD, dt=GOOD, z=GOOD, a_log=GOOD, d_skip=GOOD, dt_bias=GOOD, first=GOOD, state_in=GOOD, y=GOOD + 64, state_out=GOOD,
               saved=GOOD)
    need = binding.scan_workspace_bytes(d)

    def call(ws=(GOOD, need), dims=d, **over):
        binding.scan_fwd(dims, **dict(fwd, **over), ws=ws, stream=0)

    for k in ("x", "b", "c", "dt", "a_log", "y"):
        refused(NULL, lambda: call(**{k: None}))
    for k in fwd:
        if k != "first":
            refused(SHAPE, lambda: call(**{k: GOOD + 1}))
    for k in ("a_log", "state_in", "state_out", "saved"):
        refused(SHAPE, lambda: call(**{k: GOOD + 4}))
    refused(SHAPE, lambda: call(y=GOOD))
    refused(SHAPE, lambda: call(dims=scan(z_n=10)))
    refused(WORKSPACE, lambda: call(ws=(GOOD, need - 1)))
    back = dict(x=GOOD, b=GOOD, c=GOOD, dt=GOOD, z=GOOD, a_log=GOOD, d_skip=GOOD, dt_bias=GOOD, first=GOOD, saved=GOOD, dy=GOOD, dstate_out=GOOD,
                dx=GOOD + 64, db=GOOD + 64, dc=GOOD + 64, ddt=GOOD + 64, dz=GOOD + 64, da_log=GOOD, dd_skip=GOOD, ddt_bias=GOOD, dstate_in=GOOD)
    need = binding.scan_workspace_bytes(d, True)

    def bwd(ws=(GOOD, need), **over):
        binding.scan_bwd(d, **dict(back, **over), ws=ws, stream=0)

    for k in ("x", "b", "c", "dt", "a_log", "saved", "dy", "dx", "db", "dc", "ddt"):
        refused(NULL, lambda: bwd(**{k: None}))
    refused(NULL, lambda: bwd(dz=None))            # a gate has a gradient
    refused(NULL, lambda: bwd(z=None))
    refused(SHAPE, lambda: bwd(dx=GOOD))
    refused(WORKSPACE, lambda: bwd(ws=(GOOD, need - 1)))
    # many heads a group: sums of several workgroups need room; few heads and a long segment: states between spans of time
    assert binding.scan_workspace_bytes(scan(heads=16, groups=1), True) > binding.scan_workspace_bytes(scan(heads=4, groups=1), True)
    assert binding.scan_workspace_bytes(scan(T=4096)) > binding.scan_workspace_bytes(scan(T=32))


def test_step_refusals():
    d = scan(T=1)
    args = dict(xbc=GOOD, dt=GOOD, z=GOOD, conv_w=GOOD, conv_b=GOOD, a_log=GOOD, d_skip=GOOD, dt_bias=GOOD, first=GOOD, conv_in=GOOD, state_in=GOOD, y=GOOD,
                conv_out=GOOD + 64, state_out=GOOD)

    def call(dims=d, width=4, **over):
        binding.memory_step(dims, width, **dict(args, **over), stream=0)

    for k in ("xbc", "dt", "conv_w", "a_log", "y", "state_out"):
        refused(NULL, lambda: call(**{k: None}))
    refused(SHAPE, lambda: call(conv_out=GOOD))
    refused(SHAPE, lambda: call(width=0))
    refused(UNSUPPORTED, lambda: call(width=5))
    refused(SHAPE, lambda: call(dims=scan(T=2)))
    refused(SHAPE, lambda: call(dims=scan(T=1, x_n=64)))
