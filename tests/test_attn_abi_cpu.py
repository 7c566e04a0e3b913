"""What the entry points of the memory by attention refuse, and what they ask for, without a GPU: every check is made on the host before the first
launch (the addresses here are fake)."""
import os

import pytest

from paper_2603_09237_amd import binding

GOOD = 0x10000
NULL, SHAPE, UNSUPPORTED, WORKSPACE = binding.ERR_NULL, binding.ERR_SHAPE, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE
BIG = (GOOD, 1 << 50)


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


def places(*names):
    """A place of its own for each"""
    return {n: GOOD + 256 * (i + 1) for i, n in enumerate(names)}


HEADS_BAD = [(dict(N=0), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=129), UNSUPPORTED),
             (dict(buckets=-1), SHAPE), (dict(buckets=65), UNSUPPORTED), (dict(window=0), SHAPE), (dict(dtype=2), UNSUPPORTED), (dict(scale=float("nan")), SHAPE),
             (dict(scale=float("inf")), SHAPE), (dict(heads=2048, kv_heads=2048, head_dim=1), UNSUPPORTED)]


# ---- segments ----
def attn(**over):
    return binding.AttnDims(**{**dict(T=5, S=9, N=3, heads=4, kv_heads=2, head_dim=16, buckets=8, window=6, dtype=1), **over})


@pytest.mark.parametrize("over,code", HEADS_BAD + [(dict(T=0), SHAPE), (dict(S=4), SHAPE), (dict(S=(1 << 20) + 1), UNSUPPORTED), (dict(q_t=63), SHAPE), (dict(q_n=63), SHAPE),
                                                   (dict(k_t=31), SHAPE), (dict(k_n=31), SHAPE), (dict(y_t=63), SHAPE), (dict(y_n=63), SHAPE),
                                                   (dict(N=1 << 22), UNSUPPORTED), (dict(T=1, S=1 << 20, N=1024, heads=2), UNSUPPORTED)])
def test_attention_dimensions(over, code):
    d, f = attn(**over), places("q", "k", "v", "bias", "edges", "first", "y", "saved")
    b = dict(f, **{k: v + 8192 for k, v in places("dy", "dq", "dk", "dv", "dbias").items()})
    refused(code, lambda: binding.attn_fwd(d, **f, ws=BIG, stream=0))
    refused(code, lambda: binding.attn_bwd(d, **b, ws=BIG, stream=0))
    for call in (lambda: binding.attn_saved_bytes(d), lambda: binding.attn_workspace_bytes(d), lambda: binding.attn_workspace_bytes(d, True)):
        with pytest.raises(binding.MorlaxError):
            call()


def test_attention_pointers_and_workspace():
    d, f = attn(), places("q", "k", "v", "bias", "edges", "first", "y", "saved")
    need = binding.attn_workspace_bytes(d)

    def fwd(ws=(GOOD, need), **over):
        binding.attn_fwd(d, **dict(f, **over), ws=ws, stream=0)

    for k in ("q", "k", "v", "y", "bias", "edges"):
        refused(NULL, lambda: fwd(**{k: None}))
    for k in ("q", "k", "v", "y", "bias", "edges", "saved"):
        refused(SHAPE, lambda: fwd(**{k: f[k] + 1}))
    for k in ("q", "k", "v"):
        refused(SHAPE, lambda: fwd(y=f[k]))
    refused(WORKSPACE, lambda: fwd(ws=(GOOD, need - 1), saved=None))
    refused(NULL, lambda: fwd(ws=None, saved=None))
    b = dict(f, **{k: v + 8192 for k, v in places("dy", "dq", "dk", "dv", "dbias").items()})
    need = binding.attn_workspace_bytes(d, True)

    def bwd(ws=(GOOD, need), **over):
        binding.attn_bwd(d, **dict(b, **over), ws=ws, stream=0)

    for k in ("q", "k", "v", "y", "dy", "dq", "dk", "dv", "saved", "bias", "edges"):
        refused(NULL, lambda: bwd(**{k: None}))
    for k in ("q", "k", "v", "y", "dy", "dq", "dk", "dv", "saved", "bias", "edges", "dbias"):
        refused(SHAPE, lambda: bwd(**{k: b[k] + 1}))
    for k in ("dq", "dk", "dv"):
        for other in ("q", "k", "v", "y", "dy"):
            refused(SHAPE, lambda: bwd(**{k: b[other]}))
    for k, other in (("dq", "dk"), ("dk", "dv"), ("dq", "dv")):
        refused(SHAPE, lambda: bwd(**{k: b[other]}))
    refused(WORKSPACE, lambda: bwd(ws=(GOOD, need - 1)))


def test_attention_sizes_grow_with_the_rows():
    """No product of sizes that need not be together (rows by rows, buckets by steps)."""
    d = attn(T=4096, S=4096, N=16, heads=8, kv_heads=8, head_dim=64, buckets=32, window=4096)
    rows = 4096 * 16 * 8
    assert binding.attn_saved_bytes(d) <= rows * (4 + 128) + 4 * 4096 * (16 + 8 + 1) + 4096
    assert binding.attn_workspace_bytes(d, True) <= rows * 4 + rows / 64 * 32 * 4 + 4096


# ---- pages ----
def pages(**over):
    return binding.PagesDims(**{**dict(N=5, page=4, slots=3, pages=15), **over})


@pytest.mark.parametrize("over,code", [(dict(N=0), SHAPE), (dict(page=0), SHAPE), (dict(slots=0), SHAPE), (dict(pages=0), SHAPE), (dict(page=3), UNSUPPORTED),
                                       (dict(page=8192), UNSUPPORTED), (dict(pages=1 << 29), UNSUPPORTED), (dict(N=1 << 20, slots=1 << 11), UNSUPPORTED),
                                       (dict(N=1, slots=(1 << 30) + 1), UNSUPPORTED),
                                       (dict(N=(1 << 24) + 1), UNSUPPORTED)])
def test_pages_dimensions(over, code):
    d, f = pages(**over), places("first", "length_in", "table_in", "queue_in", "state_in", "length", "table", "queue", "state", "slot")
    refused(code, lambda: binding.cache_pages(d, **f, ws=BIG, stream=0))
    with pytest.raises(binding.MorlaxError):
        binding.pages_workspace_bytes(d)


def test_pages_pointers_and_workspace():
    d, f = pages(), places("first", "length_in", "table_in", "queue_in", "state_in", "length", "table", "queue", "state", "slot")
    need = binding.pages_workspace_bytes(d)

    def call(ws=(GOOD, need), **over):
        binding.cache_pages(d, **dict(f, **over), ws=ws, stream=0)

    for k in f:
        if k != "first":
            refused(NULL, lambda: call(**{k: None}))
            refused(SHAPE, lambda: call(**{k: f[k] + 4}))
    ins, outs = ("length_in", "table_in", "queue_in", "state_in"), ("length", "table", "queue", "state", "slot")
    for i, o in enumerate(outs):
        for j, n in enumerate(ins):
            if i != j:
                refused(SHAPE, lambda: call(**{o: f[n]}))
        for other in outs[:i]:
            refused(SHAPE, lambda: call(**{o: f[other]}))
        refused(SHAPE, lambda: call(**{o: f["first"]}))
    refused(WORKSPACE, lambda: call(ws=(GOOD, need - 1)))


# ---- one step ----
def cache(**over):
    return binding.CacheDims(**{**dict(N=3, heads=4, kv_heads=2, head_dim=16, buckets=8, window=12, page=4, slots=3, pages=9, dtype=1), **over})


@pytest.mark.parametrize("over,code", HEADS_BAD + [(dict(page=6), UNSUPPORTED), (dict(slots=0), SHAPE), (dict(pages=0), SHAPE), (dict(window=13), SHAPE), (dict(q_n=63), SHAPE),
                                                   (dict(k_n=31), SHAPE), (dict(y_n=63), SHAPE), (dict(N=1 << 20), UNSUPPORTED)])
def test_step_dimensions(over, code):
    d, f = cache(**over), places("q", "k", "v", "bias", "edges", "table", "length", "k_cache", "v_cache", "y")
    refused(code, lambda: binding.attn_step(d, **f, ws=BIG, stream=0))
    with pytest.raises(binding.MorlaxError):
        binding.attn_step_workspace_bytes(d)


def test_step_pointers_and_workspace():
    d, f = cache(window=12), places("q", "k", "v", "bias", "edges", "table", "length", "k_cache", "v_cache", "y")
    need = binding.attn_step_workspace_bytes(d)

    def call(ws=(GOOD, need), **over):
        binding.attn_step(d, **dict(f, **over), ws=ws, stream=0)

    for k in f:
        refused(NULL, lambda: call(**{k: None}))
        refused(SHAPE, lambda: call(**{k: f[k] + 1}))
    for a, b in (("y", "q"), ("y", "k"), ("y", "v"), ("k_cache", "v_cache"), ("k_cache", "y"), ("v_cache", "y"), ("k_cache", "k"), ("v_cache", "v"), ("k_cache", "q")):
        refused(SHAPE, lambda: call(**{a: f[b]}))
    refused(WORKSPACE, lambda: call(ws=(GOOD, need - 1)))
    # few environments with a long window share its length: parts of it are kept
    assert binding.attn_step_workspace_bytes(cache(N=1, window=8192, slots=2048, pages=2048)) > need


# ---- norms ----
def norm(**over):
    return binding.NormDims(**{**dict(rows=5, width=24, dtype=1), **over})


NORM = ("x", "u", "gate", "scale", "w_post", "w_pre")


@pytest.mark.parametrize("over,code", [(dict(rows=-1), SHAPE), (dict(width=0), SHAPE), (dict(width=8193), UNSUPPORTED), (dict(rows=(1 << 28) + 1), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
                                       (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(ld_x=23), SHAPE), (dict(ld_u=23), SHAPE), (dict(ld_g=23), SHAPE),
                                       (dict(ld_h=23), SHAPE)])
def test_norm_dimensions(over, code):
    d = norm(**over)
    refused(code, lambda: binding.norm_fwd(d, **places(*NORM, "y", "h"), stream=0))
    refused(code, lambda: binding.norm_bwd(d, **places(*NORM, "dy", "dh", "dx", "du", "dgate", "dscale", "dw_post", "dw_pre"), ws=BIG, stream=0))
    with pytest.raises(binding.MorlaxError):
        binding.norm_workspace_bytes(d)


def test_norm_pointers_and_workspace():
    d, f = norm(), places(*NORM, "y", "h")

    def fwd(**over):
        binding.norm_fwd(d, **dict(f, **over), stream=0)

    for over in (dict(x=None), dict(y=None), dict(h=None), dict(w_pre=None), dict(u=None), dict(u=None, gate=None), dict(u=None, gate=None, scale=None)):
        refused(NULL, lambda: fwd(**over))
    for k in f:
        refused(SHAPE, lambda: fwd(**{k: f[k] + 1}))
    for a, b in (("h", "x"), ("h", "u"), ("h", "gate"), ("h", "y"), ("y", "u"), ("y", "gate")):
        refused(SHAPE, lambda: fwd(**{a: f[b]}))
    b = places(*NORM, "dy", "dh", "dx", "du", "dgate", "dscale", "dw_post", "dw_pre")
    need = binding.norm_workspace_bytes(d)

    def bwd(ws=(GOOD, need), **over):
        binding.norm_bwd(d, **dict(b, **over), ws=ws, stream=0)

    for over in (dict(x=None), dict(w_pre=None), dict(gate=None), dict(u=None, gate=None, scale=None, w_post=None)):
        refused(NULL, lambda: bwd(**over))
    for k in b:
        refused(SHAPE, lambda: bwd(**{k: b[k] + 1}))
    for a in ("dx", "du", "dgate"):
        for o in ("x", "u", "gate", "dh") + (("dy",) if a != "dx" else ()):
            refused(SHAPE, lambda: bwd(**{a: b[o]}))
    refused(SHAPE, lambda: bwd(du=b["dx"]))
    refused(WORKSPACE, lambda: bwd(ws=(GOOD, need - 1)))
    refused(NULL, lambda: bwd(ws=None))
    binding.norm_fwd(norm(rows=0), None, None, None, None, None, None, None, None, stream=0)   # no rows: nothing launched
