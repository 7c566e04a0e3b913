"""Which buffers the attention block's calls use and which arguments it refuses, without a GPU: the entry points are replaced by ones that note what they
are given."""
import pytest

torch = pytest.importorskip("torch")

from paper_2603_09237_amd import attention, memory  # noqa: E402

CALLS = ("adapter_fwd", "adapter_bwd", "attn_fwd", "attn_bwd", "norm_fwd", "norm_bwd", "cache_pages", "attn_step")
SIZES = {"adapter_workspace_bytes": 640, "attn_workspace_bytes": 320, "attn_saved_bytes": 512, "norm_workspace_bytes": 256, "pages_workspace_bytes": 128,
         "attn_step_workspace_bytes": 192}


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
    monkeypatch.setattr(memory, "binding", n)       # (the projections)
    monkeypatch.setattr(attention, "binding", n)
    return n


def block(**over):
    return attention.AttentionBlock(**{**dict(preferences=3, width=8, heads=4, kv_heads=2, head_dim=4, buckets=3, window=6, rank=2, device="cpu",
                                              dtype=torch.float32), **over})


def inputs(b, T=4, N=5):
    x = torch.zeros(T, N, b.width, dtype=b.dtype)
    return x, x.clone(), torch.zeros(N, dtype=torch.int32), b.new_state(N)


def memory_of(calls):
    """storage addresses of everything that the calls were given"""
    return {t.untyped_storage().data_ptr() for _, ts in calls for t in ts if t.numel()}


def test_acting_shares_no_scratch_with_segments(noted):
    b = block()
    x, h, index, state = inputs(b)
    alive = [b.segment(x, h, index, None, state, train=True), b.backward(torch.zeros_like(x), torch.zeros_like(x))]
    update, noted.calls = noted.calls, []
    given = [x[0].clone(), h[0].clone(), index.clone()]
    alive.append(b.act(*given, None, b.new_cache(5, page=2)))
    parameters = {t.untyped_storage().data_ptr() for t in list(b.p.values()) + [b.edges]}
    assert memory_of(update) & memory_of(noted.calls) <= parameters
    del alive


def test_captured_buffers_stay(noted, monkeypatch):
    """A call that is captured, then calls of other sizes, which take buffers of their own: the captured call's are still there."""
    import gc
    import weakref
    b = block()
    first = torch.zeros(4, 5, dtype=torch.uint8)

    def work(x, h, index, state, first=None):
        y, nxt, after = b.segment(x, h, index, first, state, train=True)
        b.backward(torch.zeros_like(x), torch.zeros_like(x))
        b.segment(x, h, index, first, after, train=True)                # (with past steps)
        b.backward(torch.zeros_like(x), torch.zeros_like(x))
        b.act(x[0].clone(), h[0].clone(), index, None, b.new_cache(x.shape[1], page=2))

    case = inputs(b)
    work(*case, first)       # as before a capture
    noted.calls = []
    monkeypatch.setattr(b, "_capturing", lambda: True, raising=False)
    work(*case, first)
    buffers = {id(t): t for t in list(b.b.values()) + list(b.captured.values())}
    used = memory_of(noted.calls)
    mine = [weakref.ref(t) for t in buffers.values() if t.untyped_storage().data_ptr() in used]
    assert len(mine) >= 15
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
    x, h, index, state = inputs(b)
    first = torch.zeros(4, 5, dtype=torch.uint8)
    dy = torch.zeros_like(x)
    with pytest.raises(RuntimeError, match="train=True"):
        b.backward(dy, dy)
    b.segment(x, h, index, first, state, train=True)
    b.backward(dy, dy)
    b.segment(x, h, index, first, state)
    with pytest.raises(RuntimeError, match="train=True"):
        b.backward(dy, dy)
    for t in (x, h, first):
        b.segment(x, h, index, first, state, train=True)
        t.zero_()
        with pytest.raises(RuntimeError, match="written to"):
            b.backward(dy, dy)


def test_state_behind_a_segment(noted):
    """The last window - 1 steps' keys and values and begins, of the past's too, whatever the segment's length."""
    b = block()
    state = b.new_state(5)
    for T, steps in ((1, 1), (2, 3), (4, 5), (9, 5), (1, 5)):
        x, h, index, _ = inputs(b, T=T)
        first = torch.ones(T, 5, dtype=torch.bool)
        _, _, state = b.segment(x, h, index, first, state)
        assert state[0].shape == (steps, 5, 2 * b.E) and state[1].shape == (steps, 5) and bool(state[1].all())
    b = block(window=1)
    x, h, index, state = inputs(b)
    _, _, state = b.segment(x, h, index, None, state)
    assert state[0].shape == (0, 5, 2 * b.E) and state[1].shape == (0, 5)


def bad(t):
    """the tensor in other types, shapes and orders"""
    wide = torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype)
    yield t.to(torch.int64 if t.dtype == torch.int32 else torch.float64)
    yield torch.cat([t, t])
    yield wide[..., ::2]


def test_arguments_that_are_refused(noted):
    b = block()
    x, h, index, state = inputs(b)
    first, dy = torch.zeros(4, 5, dtype=torch.uint8), torch.zeros_like(x)
    state = (torch.zeros(3, 5, 2 * b.E), torch.zeros(3, 5, dtype=torch.uint8))
    good = dict(x=x, h=h, first=first, state0=state[0], state1=state[1])
    for k in good:
        for t in bad(good[k]):
            a = dict(good, **{k: t})
            with pytest.raises(ValueError):
                b.segment(a["x"], a["h"], index, a["first"], (a["state0"], a["state1"]))
    good = dict(x=x[0].clone(), h=h[0].clone(), index=index, first=first[0].clone())
    cache = b.new_cache(5, page=2)
    for k in good:
        for t in bad(good[k]):
            a = dict(good, **{k: t})
            with pytest.raises(ValueError):
                b.act(a["x"], a["h"], a["index"], a["first"], cache)
    for other in (b.new_cache(6), block(kv_heads=4).new_cache(5), block(head_dim=8).new_cache(5), block(dtype=torch.bfloat16).new_cache(5)):
        with pytest.raises(ValueError, match="cache"):
            b.act(good["x"], good["h"], index, None, other)
    b.segment(x, h, index, first, state, train=True)
    for t in bad(dy):
        with pytest.raises(ValueError, match="dy"):
            b.backward(t, dy)
        with pytest.raises(ValueError, match="dh"):
            b.backward(dy, t)
    assert [c for c, _ in noted.calls] == ["adapter_fwd", "attn_fwd", "adapter_fwd", "norm_fwd"]
    b.act(good["x"], good["h"], index, None, cache)
    b.segment(x, h, index.long(), first.bool(), state)     # (the index is copied for every step, from any type)


def test_edges_rise():
    for buckets in (1, 2, 3, 8, 32, 64):
        for reach in (1, 5, 64, 8192, 1 << 20):
            e = attention.distance_edges(buckets, reach)
            assert len(e) == buckets and e[0] == 0 and all(a < b for a, b in zip(e, e[1:]))
    assert attention.distance_edges(0, 10) == []
