"""Which buffers the memory block's calls use, without a GPU: the entry points are replaced by ones that note what they are given."""
import pytest

torch = pytest.importorskip("torch")

from paper_2603_09237_amd import memory  # noqa: E402

CALLS = ("adapter_fwd", "adapter_bwd", "conv_fwd", "conv_bwd", "scan_fwd", "scan_bwd", "memory_step")
SIZES = {"adapter_workspace_bytes": 640, "conv_workspace_bytes": 320, "scan_saved_bytes": 512, "scan_workspace_bytes": 256}


class Noted:
    """The binding's functions as the block calls them; `calls`: (name, tensors)."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name in SIZES:
            return lambda d, *a: SIZES[name]
        if name in CALLS:
            return lambda *a, **k: self.calls.append((name, [t for t in a if isinstance(t, torch.Tensor)]))
        import paper_2603_09237_amd.binding as real
        return getattr(real, name)


@pytest.fixture
def noted(monkeypatch):
    n = Noted()
    monkeypatch.setattr(memory, "binding", n)
    return n


def block(**over):
    return memory.MemoryBlock(**{**dict(preferences=3, width=8, heads=2, head_dim=4, state=4, rank=2, device="cpu", dtype=torch.float32), **over})


def inputs(b, T=4, N=5):
    return torch.zeros(T, N, b.width, dtype=b.dtype), torch.zeros(N, dtype=torch.int32), b.new_state(N)


def memory_of(calls):
    """storage addresses of everything that the calls were given"""
    return {t.untyped_storage().data_ptr() for _, ts in calls for t in ts if t.numel()}


def test_acting_shares_no_scratch_with_segments(noted):
    b = block()
    x, index, state = inputs(b)
    b.segment(x, index, None, state, train=True)
    b.backward(torch.zeros_like(x))
    update, noted.calls = memory_of(noted.calls), []
    after = b.new_state(5)
    given = [x[0].clone(), index.clone(), *b.new_state(5)]
    b.act(given[0], given[1], None, (given[2], given[3]), after)
    acting = memory_of(noted.calls)
    parameters = {t.untyped_storage().data_ptr() for t in b.p.values()}
    assert update & acting <= parameters


def test_captured_buffers_stay(noted, monkeypatch):
    """A call that is captured, then calls of other sizes, which take buffers of their own: the captured call's are still there."""
    import gc
    import weakref
    b = block()
    x, index, state = inputs(b)

    def work(x, index, state):
        b.segment(x, index, None, state, train=True)
        b.backward(torch.zeros_like(x))
        b.act(x[0].clone(), index, None, state, b.new_state(x.shape[1]))

    work(x, index, state)       # as before a capture
    noted.calls = []
    monkeypatch.setattr(b, "_capturing", lambda: True, raising=False)
    work(x, index, state)
    buffers = {id(t): t for t in b.b.values()}
    used = memory_of(noted.calls)
    mine = [weakref.ref(t) for t in buffers.values() if t.untyped_storage().data_ptr() in used]
    assert len(mine) >= 10
    monkeypatch.setattr(b, "_capturing", lambda: False, raising=False)
    before = dict(SIZES)
    try:
        SIZES.update({k: 4 * v for k, v in SIZES.items()})
        del buffers
        noted.calls = []
        work(*inputs(b, T=6, N=7))
        work(*inputs(b, T=3, N=2))
    finally:
        SIZES.update(before)
    noted.calls = []
    gc.collect()
    assert all(r() is not None for r in mine)


def test_backward_needs_its_segment(noted):
    """After a segment that kept nothing, or whose inputs have changed, there is no backward."""
    b = block()
    x, index, state = inputs(b)
    first = torch.zeros(4, 5, dtype=torch.uint8)
    dy = torch.zeros_like(x)
    with pytest.raises(RuntimeError, match="train=True"):
        b.backward(dy)
    b.segment(x, index, first, state, train=True)
    b.backward(dy)
    b.segment(x, index, first, state)
    with pytest.raises(RuntimeError, match="train=True"):
        b.backward(dy)
    for t in (x, first):
        b.segment(x, index, first, state, train=True)
        t.zero_()
        with pytest.raises(RuntimeError, match="written to"):
            b.backward(dy)
    with torch.inference_mode():
        y = x.clone()
        b.segment(y, index, None, b.new_state(5), train=True)
        b.backward(dy)


def bad(t):
    """the tensor in other types, shapes and orders"""
    wide = torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype)
    yield t.to(torch.int64 if t.dtype == torch.int32 else torch.float64)
    yield torch.cat([t, t])
    yield wide[..., ::2]


def test_arguments_that_are_refused(noted):
    b = block()
    x, index, state = inputs(b)
    first, after, dy = torch.zeros(4, 5, dtype=torch.uint8), b.new_state(5), torch.zeros_like(x)
    good = dict(x=x, first=first, state0=state[0], state1=state[1])
    for k in good:
        for t in bad(good[k]):
            a = dict(good, **{k: t})
            if k == "x" and t.shape[0] == 8:
                continue        # a longer segment
            with pytest.raises(ValueError, match=k.rstrip("01")):
                b.segment(a["x"], index, a["first"], (a["state0"], a["state1"]))
    good = dict(x=x[0].clone(), index=index, first=first[0].clone(), state0=state[0], state1=state[1], after0=after[0], after1=after[1])
    for k in good:
        for t in bad(good[k]):
            a = dict(good, **{k: t})
            with pytest.raises(ValueError):
                b.act(a["x"], a["index"], a["first"], (a["state0"], a["state1"]), (a["after0"], a["after1"]))
    b.segment(x, index, first, state, train=True)
    for t in bad(dy):
        with pytest.raises(ValueError, match="dy"):
            b.backward(t)
    assert [c for c, _ in noted.calls] == ["adapter_fwd", "conv_fwd", "scan_fwd", "adapter_fwd"]
    b.act(good["x"], index, None, state, after)
    b.segment(x, index.long(), first.bool(), state)     # (the index is copied for every step, from any type)
