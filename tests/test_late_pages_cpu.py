"""Entry points and block for caches whose pages may come late, without a GPU: what is refused, and what the block hands on."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2603_09237_amd import attention, binding, memory  # noqa: E402

GOOD = 0x10000


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
    assert "_since" in str(e.value)


def places(*names):
    return {n: GOOD + 256 * (i + 1) for i, n in enumerate(names)}


def test_pages_pointers():
    d = binding.PagesDims(5, 4, 3, 15)
    f = places("first", "length_in", "table_in", "queue_in", "state_in", "since_in", "length", "table", "queue", "state", "since", "slot")
    need = binding.pages_workspace_bytes(d)

    def call(ws=(GOOD, need), **over):
        binding.cache_pages(d, **dict(f, **over), ws=ws, stream=0)

    for k in f:
        if k != "first":
            refused(binding.ERR_NULL, lambda: call(**{k: None}))
            refused(binding.ERR_SHAPE, lambda: call(**{k: f[k] + 4}))
    ins, outs = ("length_in", "table_in", "queue_in", "state_in", "since_in"), ("length", "table", "queue", "state", "since", "slot")
    for i, o in enumerate(outs):
        for j, n in enumerate(ins):
            if i != j:
                refused(binding.ERR_SHAPE, lambda: call(**{o: f[n]}))
        for other in outs[:i]:
            refused(binding.ERR_SHAPE, lambda: call(**{o: f[other]}))
        refused(binding.ERR_SHAPE, lambda: call(**{o: f["first"]}))
    refused(binding.ERR_WORKSPACE, lambda: call(ws=(GOOD, need - 1)))


def test_step_pointers():
    d = binding.CacheDims(3, 4, 2, 16, 8, 12, 4, 3, 9, 1)
    f = places("q", "k", "v", "bias", "edges", "table", "length", "since", "k_cache", "v_cache", "y")
    need = binding.attn_step_workspace_bytes(d)

    def call(ws=(GOOD, need), **over):
        binding.attn_step(d, **dict(f, **over), ws=ws, stream=0)

    for k in f:
        if k != "since":
            refused(binding.ERR_NULL, lambda: call(**{k: None}))
        refused(binding.ERR_SHAPE, lambda: call(**{k: f[k] + 1}))
    refused(binding.ERR_SHAPE, lambda: call(y=f["q"]))
    refused(binding.ERR_WORKSPACE, lambda: call(ws=(GOOD, need - 1)))


def test_the_block_keeps_and_hands_on_since(monkeypatch):
    calls = []

    class Noted:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *a: 256
            if name in ("adapter_fwd", "norm_fwd", "cache_pages", "attn_step"):
                return lambda *a, **k: calls.append((name, k))
            return getattr(binding, name)

    monkeypatch.setattr(memory, "binding", Noted())
    monkeypatch.setattr(attention, "binding", Noted())
    b = attention.AttentionBlock(3, 8, heads=4, kv_heads=2, head_dim=4, buckets=3, window=6, rank=2, device="cpu", dtype=torch.float32)
    cache, x = b.new_cache(5, page=2, pages=4), torch.zeros(5, 8)
    assert cache.since.shape == (5, 3) and cache.since.dtype is torch.int32
    b.act(x, x.clone(), torch.zeros(5, dtype=torch.int32), None, cache)
    given = dict(calls)
    assert given["cache_pages"]["since_in"] is cache.since and given["cache_pages"]["since"] is cache.since and given["attn_step"]["since"] is cache.since
