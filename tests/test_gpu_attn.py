"""Attention over an episode's past and its gradients against the definition in 64 bits (environment by environment, on the CPU, gradients from the
formulas), and those gradients against differences.

Tolerances, from the arithmetic: a product of two vectors of n elements in fp32 is off by n 2^-24 of the sum of its terms' magnitudes, an
exponential by 4 2^-24 of itself and by what its argument is off; a probability that is multiplied in bf16 is held in two parts, off by 2^-17
of itself, and so is what y was before its rounding; a rounding to bf16 by 2^-8 of the value."""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _torch():
    import torch
    return torch


def make(dtype, T, S, N, H, KV, D, B, window, p_first, seed=0, scale=None):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    c = dict(T=T, S=S, N=N, H=H, KV=KV, D=D, B=B, window=window, dtype=dtype, scale=D ** -0.5 if scale is None else scale)
    for n, shape in (("q", (T, N, H, D)), ("k", (S, N, KV, D)), ("v", (S, N, KV, D)), ("dy", (T, N, H, D))):
        c[n] = torch.randn(*shape, generator=g).to(dtype)
    c["bias"] = torch.randn(H, B, generator=g) if B else None
    c["edges"] = None
    if B:
        half = max(1, B // 2)
        c["edges"] = torch.tensor([j if j < half else half + 3 * (j - half) for j in range(B)], dtype=torch.int32)
    c["first"] = (torch.rand(S, N, generator=g) < p_first).to(torch.uint8) if p_first else None
    return c


def seen_and_bucket(c, n):
    torch = _torch()
    T, S = c["T"], c["S"]
    gap = torch.arange(S - T, S)[:, None] - torch.arange(S)
    see = (gap >= 0) & (gap < c["window"])
    if c["first"] is not None:
        e = c["first"][:, n].long().cumsum(0)
        see = see & (e[S - T:, None] == e[None])
    bucket = torch.zeros_like(gap)
    for j in range(1, c["B"]):
        bucket += (gap >= c["edges"][j]).long()
    return see, bucket


def define(c, gradients=True, eps=None):
    """Results and the error bounds of each (`half` is left to the caller); eps: (tensor name, place, difference) for the value alone."""
    torch = _torch()
    T, S, N, H, KV, D, B = (c[k] for k in ("T", "S", "N", "H", "KV", "D", "B"))
    share, sc, two = H // KV, c["scale"], 2.0 ** -17 if c["dtype"] == torch.bfloat16 else 0.0
    x = {k: c[k].double().clone() for k in ("q", "k", "v", "dy")}
    bias = c["bias"].double().clone() if B else None
    if eps is not None:
        where = bias if eps[0] == "bias" else x[eps[0]]
        where[eps[1]] += eps[2]
    out = {k: torch.zeros_like(x[k]) for k in ("q", "k", "v")}
    out["y"], out["bias"] = torch.zeros_like(x["dy"]), torch.zeros(H, max(B, 1), dtype=torch.float64)
    bound = {k: torch.zeros_like(v) for k, v in out.items()}
    dot = lambda a, b: torch.bmm(a, b.transpose(1, 2).contiguous())  # noqa: E731
    for n in range(N):
        see, bucket = seen_and_bucket(c, n)
        q, dy = (x[k][:, n].transpose(0, 1).contiguous() for k in ("q", "dy"))
        k, v = (x[m][:, n].transpose(0, 1).repeat_interleave(share, 0) for m in ("k", "v"))
        a = dot(q, k) * sc
        if B:
            a = a + bias[:, bucket]
        a = a.masked_fill(~see, float("-inf"))
        p = torch.softmax(a, -1)
        y = torch.bmm(p, v)
        out["y"][:, n] = y.transpose(0, 1)
        if not gradients:
            continue
        fin = torch.where(see, a, 0.0)
        e_a = (D + 4) * U * abs(sc) * float(dot(q.abs(), k.abs()).max()) + 4 * U * float(fin.abs().max())
        e_p = 2 * e_a + (S + 12) * U
        bound["y"][:, n] = ((e_p + two + S * U) * torch.bmm(p, v.abs())).transpose(0, 1)
        dp, delta = dot(dy, v), (dy * y).sum(-1, keepdim=True)
        e_dp, e_delta = (D + 2) * U * dot(dy.abs(), v.abs()), ((e_p + 2 * two + (D + 2 + S) * U) * (dy.abs() * torch.bmm(p, v.abs())).sum(-1, keepdim=True))
        da = p * (dp - delta)
        e_da = p * ((e_p + 2 * U) * (dp - delta).abs() + e_dp + e_delta)
        group = lambda t: t.reshape(KV, share, S, D).sum(1).transpose(0, 1)  # noqa: E731
        turn = lambda t: t.transpose(1, 2).contiguous()  # noqa: E731
        out["q"][:, n] = sc * torch.bmm(da, k).transpose(0, 1)
        bound["q"][:, n] = abs(sc) * torch.bmm(e_da + (two + (S + 2) * U) * da.abs(), k.abs()).transpose(0, 1)
        rows = T * share
        out["k"][:, n] = sc * group(torch.bmm(turn(da), q))
        bound["k"][:, n] = abs(sc) * group(torch.bmm(turn(e_da + (two + (rows + 2) * U) * da.abs()), q.abs()))
        out["v"][:, n] = group(torch.bmm(turn(p), dy))
        bound["v"][:, n] = group(torch.bmm(turn((e_p + two + (rows + 2) * U) * p), dy.abs()))
        if B:
            out["bias"].index_add_(1, bucket.reshape(-1), da.reshape(H, -1))
            bound["bias"].index_add_(1, bucket.reshape(-1), (e_da + (T + S + N * T / 64 + 70) * U * da.abs()).reshape(H, -1))
    return out, bound


def place(t, pad, order):
    """On the device with rows `pad` elements longer and time or environments outermost; returns the view and its strides."""
    torch = _torch()
    L, N, H, D = t.shape
    shape = (L, N, H * D + pad) if order == "time" else (N, L, H * D + pad)
    whole = torch.full(shape, 7.0, dtype=t.dtype, device="cuda")
    view = whole if order == "time" else whole.transpose(0, 1)
    view[..., :H * D] = t.reshape(L, N, H * D).cuda()
    return whole, view[..., :H * D], view.stride(0), view.stride(1)


def run(c, pad=0, order="time", train=True, first="as it is"):
    from paper_2603_09237_amd import binding
    torch = _torch()
    T, S, N, H, KV, D, B = (c[k] for k in ("T", "S", "N", "H", "KV", "D", "B"))
    t = {n: place(c[n], pad, order) for n in ("q", "k", "v", "dy")}
    y = place(torch.zeros(T, N, H, D, dtype=c["dtype"]), pad, order)
    d = binding.AttnDims(T, S, N, H, KV, D, B, c["window"], 1 if c["dtype"] == torch.bfloat16 else 0, c["scale"], q_t=t["q"][2], q_n=t["q"][3],
                         k_t=t["k"][2], k_n=t["k"][3], y_t=y[2], y_n=y[3])
    bias, edges, first = (None if v is None else v.cuda() for v in (c["bias"], c["edges"], c["first"]))
    n = max(binding.attn_workspace_bytes(d), binding.attn_workspace_bytes(d, True))
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")   # (undefined whatever type it is read as)
    saved = torch.full((binding.attn_saved_bytes(d),), 0xff, dtype=torch.uint8, device="cuda") if train else None
    binding.attn_fwd(d, t["q"][1], t["k"][1], t["v"][1], bias, edges, first, y[1], saved, ws)
    got = {"y": y}
    if train:
        g = {m: place(torch.zeros_like(c[m]), pad, order) for m in ("q", "k", "v")}
        dbias = torch.full((H, B), 7.0, device="cuda") if B else None
        ws.fill_(0xff)
        binding.attn_bwd(d, t["q"][1], t["k"][1], t["v"][1], bias, edges, first, y[1], saved, t["dy"][1], g["q"][1], g["k"][1], g["v"][1], dbias, ws)
        got.update(g)
        if B:
            got["bias"] = dbias
    torch.cuda.synchronize()
    res = {}
    for k, v in got.items():
        if k == "bias":
            res[k] = v.cpu()
            continue
        whole, view = v[0], v[1]
        if pad:
            assert bool((whole[..., view.shape[-1]:] == 7.0).all()), f"{k}: behind its rows"
        L = S if k in ("k", "v") else T
        res[k] = view.cpu().reshape(L, N, -1, D)
    return res


def near(got, want, bound, what):
    torch = _torch()
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
    err, tol = (got.double() - want).abs(), bound + half * (want.abs() + bound) + 1e-30
    bad = ~(err <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), bad.numel(), float((err / tol).max()))


SHAPES = [  # T, S, N, H, KV, D, B, window, p_first
    (1, 1, 1, 1, 1, 1, 0, 1, 0.0),          # one step sees itself
    (1, 70, 3, 4, 2, 16, 5, 70, 0.05),      # one query, a past longer than a tile
    (3, 3, 2, 2, 1, 8, 4, 2, 0.4),
    (17, 17, 2, 3, 3, 33, 7, 17, 0.1),      # rows that are no whole pieces
    (64, 64, 2, 4, 1, 64, 8, 64, 0.02),
    (65, 130, 2, 6, 3, 40, 17, 50, 0.03),   # two heads to a head of keys, a window that ends inside tiles
    (70, 70, 1, 8, 2, 128, 64, 70, 0.0),
    (100, 333, 1, 5, 1, 127, 3, 1000, 0.01),
    (129, 200, 2, 2, 2, 20, 1, 200, 1.0),   # every step begins an episode
    (200, 200, 1, 4, 4, 72, 32, 130, 0.0),  # tiles that all rows see, beyond the last edge
    (300, 300, 1, 4, 1, 64, 6, 300, 0.0),   # four heads to a head of keys, beyond the last edge
    (40, 41, 70, 2, 1, 24, 9, 41, 0.1),
    (2, 128, 3, 2, 2, 128, 32, 128, 0.0),   # few rows that end with a tile of keys
    (70, 192, 2, 3, 3, 16, 16, 192, 0.0),   # a last block of few rows, the same
    (256, 400, 1, 2, 2, 64, 4, 300, 0.0),   # tiles at the window's begin, then ones beyond the last edge
    (9, 9, 2, 2, 1, 8, 3, 1, 0.0),          # rows that see themselves only
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(v) for v in s))
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_values_and_gradients(kind, shape):
    c = make(getattr(_torch(), kind), *shape)
    want, bound = define(c)
    got = run(c)
    for k in got:
        near(got[k], want[k], bound[k], k)


# walks of so many tiles, by so few workgroups, that they are cut into chunks whose parts are joined
LONG = [
    (1100, 1100, 1, 2, 1, 40, 17, 1100, 0.002),   # forward and queries in two chunks, keys in four; chunks behind an episode's end
    (1, 1200, 2, 4, 1, 64, 8, 1200, 0.0),
    (600, 600, 1, 4, 1, 128, 8, 600, 0.01),       # keys only
    (130, 1300, 2, 2, 2, 33, 0, 1025, 0.0),       # forward only, no bias, rows that are no whole pieces
    (1030, 1031, 1, 1, 1, 8, 3, 1000, 0.3),       # most chunks see nothing
    (3, 1100, 20, 1, 1, 8, 2, 1100, 0.004),       # long histories of some environments, of more
    (2, 1100, 70, 1, 1, 8, 2, 1100, 0.004),
    (1100, 1150, 1, 1, 1, 64, 40, 1150, 0.0),     # a chunk's end among the distances that have buckets of their own
]


@pytest.mark.parametrize("shape", LONG, ids=lambda s: "x".join(str(v) for v in s))
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_long_walks_of_few_workgroups(kind, shape):
    torch = _torch()
    c = make(getattr(torch, kind), *shape)
    want, bound = define(c)
    got, again, strided = run(c), run(c), run(c, 5, "environments")
    for k in got:
        near(got[k], want[k], bound[k], k)
        assert torch.equal(got[k], again[k]) and torch.equal(got[k], strided[k]), k


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_undefined_in_a_chunk(kind):
    """An undefined value, key, query or gradient in a cut walk reaches what sees it and nothing else."""
    torch = _torch()
    c = make(getattr(torch, kind), 1100, 1100, 1, 1, 1, 16, 0, 600, 0.0)
    clean, t = run(c), torch.arange(1100)
    sees, seen = (t >= 30) & (t < 630), (t <= 900) & (t > 300)
    for name, at, affected in (("v", 30, {"y": sees}), ("k", 30, {"y": sees, "q": sees}), ("q", 900, {"y": t == 900, "k": seen, "v": seen}),
                               ("dy", 900, {"q": t == 900, "k": seen})):
        d = dict(c, **{name: c[name].clone()})
        d[name][at, 0, 0] = float("nan")
        got = run(d)
        for k, rows in affected.items():
            assert not bool(torch.isfinite(got[k][rows].float()).any()), (name, k)
            assert torch.equal(got[k][~rows], clean[k][~rows]), (name, k)


@pytest.mark.parametrize("pad,order", [(3, "time"), (8, "environments"), (5, "environments")])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_strides(kind, pad, order):
    """Rows that begin anywhere, time or environments outermost: bit for bit what contiguous rows give, and nothing written behind them."""
    torch = _torch()
    for shape in (SHAPES[4], SHAPES[5], SHAPES[3]):
        c = make(getattr(torch, kind), *shape)
        a, b = run(c), run(c, pad, order)
        for k in a:
            assert torch.equal(a[k], b[k]), k


def test_rows_that_see_themselves_only():
    """Their probability is one whatever the scores are: their scores' gradients are zeros, not what two sums' roundings leave."""
    torch = _torch()
    for kind in (torch.float32, torch.bfloat16):
        got = run(make(kind, 70, 75, 3, 4, 2, 40, 6, 1, 0.0))
        for k in ("q", "k", "bias"):
            assert not bool(got[k].any()), k


def test_definition_against_differences():
    torch = _torch()
    c = make(torch.float64, 6, 9, 2, 4, 2, 5, 4, 7, 0.2)
    want, _ = define(c)
    value = lambda eps: float((define(c, False, eps)[0]["y"] * c["dy"]).sum())  # noqa: E731
    for k, at in (("q", (2, 1, 3, 4)), ("k", (4, 0, 1, 2)), ("v", (7, 1, 0, 0)), ("bias", (2, 1)), ("bias", (0, 0))):
        h = 1e-5
        slope = (value((k, at, h)) - value((k, at, -h))) / (2 * h)
        assert abs(slope - float(want[k][at])) < 1e-7 * (1 + abs(slope)), (k, at)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_seen_never_counts(kind, what):
    """Environment 0's episode begins at step 30: infinite and undefined keys, values, queries and gradients before it change nothing behind it, and
    the other way round, in tiles that both lie in."""
    torch = _torch()
    c = make(getattr(torch, kind), 50, 60, 2, 4, 2, 32, 6, 60, 0.0)
    c["first"] = torch.zeros(60, 2, dtype=torch.uint8)
    c["first"][30, 0] = 1
    clean = run(c)
    for names, times in ((("q", "k", "v", "dy"), slice(0, 30)), (("q", "k", "v", "dy"), slice(30, 60))):
        for name in names:
            d = dict(c, **{name: c[name].clone()})
            past = 10 if name in ("q", "dy") else 0
            lo, hi = max(times.start - past, 0), times.stop - past
            d[name][lo:hi, 0, :, 3] = what
            got = run(d)
            for k in ("y", "q", "k", "v"):
                other = torch.ones(got[k].shape[0], dtype=torch.bool)
                off = 10 if k in ("y", "q") else 0
                other[max(times.start - off, 0):times.stop - off] = False
                assert torch.equal(got[k][other][:, 0], clean[k][other][:, 0]), (name, k)
                assert torch.equal(got[k][:, 1], clean[k][:, 1]), (name, k)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_undefined_inputs_show(kind):
    """What depends on an infinite or undefined element is not finite."""
    torch = _torch()
    c = make(getattr(torch, kind), 20, 20, 1, 2, 1, 16, 4, 20, 0.0)
    for name, at, affected in (("v", (5, 0, 0, 3), {"y": lambda t: t[5:, 0, :, 3], "q": lambda t: t[5:, 0]}),
                               ("k", (5, 0, 0, 3), {"q": lambda t: t[5:, 0], "bias": lambda t: t[:, 0]}),
                               ("q", (7, 0, 1, 2), {"y": lambda t: t[7, 0, 1], "q": lambda t: t[7, 0, 1], "k": lambda t: t[:8, 0], "v": lambda t: t[:8, 0]}),
                               ("dy", (7, 0, 1, 2), {"q": lambda t: t[7, 0, 1], "k": lambda t: t[:8, 0], "v": lambda t: t[:8, 0, 0, 2]})):
        d = dict(c, **{name: c[name].clone()})
        d[name][at] = float("nan")
        got = run(d)
        for k, part in affected.items():
            assert not bool(torch.isfinite(part(got[k]).float()).any()), (name, k)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_bias_of_minus_infinity(kind):
    """A bucket whose bias is -infinity (or the type's lowest value) is not looked at; a row that has no other is undefined and no other row is."""
    torch = _torch()
    lowest = float(torch.finfo(torch.float32).min)
    for low in (-float("inf"), lowest):
        c = make(getattr(torch, kind), 90, 90, 1, 2, 2, 16, 6, 90, 0.0)
        c["bias"][0, 4] = low
        want, bound = define(c)
        got = run(c)
        for k in ("y", "v"):
            ok = torch.isfinite(want[k])
            assert bool(ok.all())
            near(got[k], want[k], torch.nan_to_num(bound[k], 1e-4, 1e-4).clamp(max=1e-4 if kind == "float32" else 1e-3), k)
        c["bias"][1, 0] = -float("inf")    # head 1 does not see itself: its first row sees nothing
        got = run(c)
        assert bool(torch.isnan(got["y"][0, 0, 1].float()).all()) and bool(torch.isfinite(got["y"][1:].float()).all())
        assert bool(torch.isfinite(got["y"][0, 0, 0].float()).all())


def test_large_scores():
    """Scores of some thousands: one key takes all, no overflow."""
    torch = _torch()
    c = make(torch.float32, 70, 70, 1, 1, 1, 16, 0, 70, 0.0, scale=300.0)
    want, _ = define(c)
    got = run(c)
    assert bool(torch.isfinite(got["y"]).all())
    # (scores of up to 2^13 are off by 16 2^-24 2^13 = 0.008, probabilities by as much of themselves)
    assert float((got["y"].double() - want["y"]).abs().max()) < 0.03


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_same_again_without_saving_and_on_another_stream(kind):
    torch = _torch()
    c = make(getattr(torch, kind), *SHAPES[5])
    a, b, alone = run(c), run(c), run(c, train=False)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = run(c)
    for k in a:
        assert torch.equal(a[k], b[k]) and torch.equal(a[k], other[k]), k
    # (a bf16 pass that saves holds its probabilities in more bits: its y is the same up to what two parts leave, and a rounding)
    if kind == "float32":
        assert torch.equal(a["y"], alone["y"])
    want, bound = define(c)
    near(alone["y"], want["y"], bound["y"], "y without saving")


def test_without_the_bias_gradient():
    from paper_2603_09237_amd import binding
    torch = _torch()
    c = make(torch.bfloat16, *SHAPES[5])
    want = run(c)
    T, S, N, H, KV, D, B = (c[k] for k in ("T", "S", "N", "H", "KV", "D", "B"))
    d = binding.AttnDims(T, S, N, H, KV, D, B, c["window"], 1)
    x = {k: c[k].cuda() for k in ("q", "k", "v", "dy", "bias", "edges", "first")}
    y, saved = torch.empty_like(x["q"]), torch.empty(binding.attn_saved_bytes(d), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(binding.attn_workspace_bytes(d), binding.attn_workspace_bytes(d, True)), dtype=torch.uint8, device="cuda")
    binding.attn_fwd(d, x["q"], x["k"], x["v"], x["bias"], x["edges"], x["first"], y, saved, ws)
    g = [torch.empty_like(x[k]) for k in ("q", "k", "v")]
    binding.attn_bwd(d, x["q"], x["k"], x["v"], x["bias"], x["edges"], x["first"], y, saved, x["dy"], *g, None, ws)
    for t, k in zip(g, ("q", "k", "v")):
        assert torch.equal(t.cpu().reshape(want[k].shape), want[k]), k


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_chunks_whose_scores_are_minus_infinity(kind):
    """Distances from five on are not looked at: most chunks of a cut walk are there and hold nothing of a row."""
    torch = _torch()
    c = make(getattr(torch, kind), 1100, 1100, 1, 2, 1, 16, 4, 1100, 0.0)
    c["bias"][:, 3] = -float("inf")
    want, bound = define(c)
    got = run(c)
    for k in ("y", "v"):
        near(got[k], want[k], torch.nan_to_num(bound[k], 1e-4, 1e-4).clamp(max=1e-4 if kind == "float32" else 1e-3), k)
    assert all(bool(torch.isfinite(got[k].float()).all()) for k in got) and bool((got["bias"][:, 3] == 0).all())


@pytest.mark.parametrize("shape", [(1100, 1100, 1, 2, 1, 40, 17, 1100, 0.002), (70, 192, 3, 3, 3, 16, 16, 192, 0.02)], ids=["cut", "whole"])
def test_replays(shape):
    """Forward and backward recorded once, replayed with changed inputs and other calls between, against the calls themselves."""
    from paper_2603_09237_amd import binding
    torch = _torch()
    c = make(torch.bfloat16, *shape)
    T, S, N, H, KV, D, B = (c[k] for k in ("T", "S", "N", "H", "KV", "D", "B"))
    d = binding.AttnDims(T, S, N, H, KV, D, B, c["window"], 1)
    x = {k: c[k].cuda() for k in ("q", "k", "v", "dy", "bias", "edges", "first")}
    out = {k: torch.empty_like(v) for k, v in x.items() if k in ("q", "k", "v", "bias")}
    out["y"], saved = torch.empty_like(x["q"]), torch.empty(binding.attn_saved_bytes(d), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(binding.attn_workspace_bytes(d), binding.attn_workspace_bytes(d, True)), dtype=torch.uint8, device="cuda")

    def work():
        binding.attn_fwd(d, x["q"], x["k"], x["v"], x["bias"], x["edges"], x["first"], out["y"], saved, ws)
        binding.attn_bwd(d, x["q"], x["k"], x["v"], x["bias"], x["edges"], x["first"], out["y"], saved, x["dy"], out["q"], out["k"], out["v"], out["bias"], ws)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        work()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in range(4):
        x["k"].normal_()
        x["first"].copy_(torch.rand(S, N, device="cuda") < 0.01)
        work()
        want = {k: v.clone() for k, v in out.items()}
        for t in (*out.values(), saved, ws):
            t.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k], want[k]), (i, k)
