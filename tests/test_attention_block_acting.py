"""Acting refuses a cache before its books move, without a GPU: launches are noted, sizes are asked of the library."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2603_09237_amd import attention, binding, memory  # noqa: E402


@pytest.fixture
def calls(monkeypatch):
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_09237_amd import build
        build.build(verbose=False)
    names = []

    class Noted:
        def __getattr__(self, name):
            if name in ("adapter_fwd", "norm_fwd", "cache_pages", "attn_step"):
                return lambda *a, **k: names.append(name)
            return getattr(binding, name)

    monkeypatch.setattr(memory, "binding", Noted())
    monkeypatch.setattr(attention, "binding", Noted())
    return names


def block(**over):
    return attention.AttentionBlock(**{**dict(preferences=3, width=8, heads=4, kv_heads=2, head_dim=4, buckets=3, window=6, rank=2, device="cpu",
                                              dtype=torch.float32), **over})


def act(b, cache, N=5):
    x = torch.zeros(N, b.width, dtype=b.dtype)
    return b.act(x, x.clone(), torch.zeros(N, dtype=torch.int32), None, cache)


def test_a_cache_of_another_window(calls):
    """Its slots hold fewer steps than this block looks back over."""
    b = block()
    with pytest.raises(ValueError, match="cache"):
        act(b, block(window=4).new_cache(5, page=2))
    assert calls == []
    act(b, block(window=9).new_cache(5, page=2))    # (more of them do no harm)
    assert calls == ["adapter_fwd", "cache_pages", "attn_step", "adapter_fwd", "norm_fwd"]


def test_sizes_that_the_step_refuses(calls):
    for b, page in ((block(), 3), (block(head_dim=129), 2), (block(buckets=65), 2)):
        with pytest.raises(binding.MorlaxError):
            act(b, b.new_cache(5, page=page))
    assert "cache_pages" not in calls


@pytest.mark.parametrize("name", ["length", "table", "since", "queue", "state", "slot", "k", "v"])
def test_books_of_other_sizes_and_types(calls, name):
    b = block()
    good = getattr(b.new_cache(5, page=2), name)
    for t in (good.double(), torch.cat([good, good]), good[:-1], torch.stack([good, good], -1)[..., 0]):
        cache = b.new_cache(5, page=2)
        setattr(cache, name, t)
        with pytest.raises(ValueError, match="cache"):
            act(b, cache)
    assert calls == []
