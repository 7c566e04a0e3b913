"""Norms, gate and residual scale between two blocks against the definition in 64 bits, gradients from the formulas and those against differences.

Tolerances: every result is a sum of a few terms, each a product of up to eight factors, and two means over a row: fp32 arithmetic is off by
(16 + width / 32 + |gate|) 2^-24 of the sum of the terms' magnitudes (a lane adds up at most width / 64 x 2 elements and then six steps; an exponential is off by its
argument's 2^-24), columns by the number of rows that one thread adds up besides; a rounding to bf16 by 2^-8 of the value."""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5


def _torch():
    import torch
    return torch


def make(dtype, rows, width, parts="u gate scale w_post w_pre", seed=0):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    c = {k: None for k in ("u", "gate", "scale", "w_post", "w_pre")}
    for k in ("x", "u", "gate", "dy", "dh"):
        v = (torch.randn(rows, width, generator=g) * (2 if k in ("x", "gate") else 1)).to(dtype)
        if k in ("x", "dy") or k in parts.split() or (k == "dh" and "w_pre" in parts):
            c[k] = v
    c.setdefault("dh", None)
    for k in ("scale", "w_post", "w_pre"):
        v = 1 + 0.3 * torch.randn(width, generator=g)
        if k in parts.split():
            c[k] = v
    return c


def define(c, move=None):
    """Results and the sums of their terms' magnitudes."""
    torch = _torch()
    x = {k: None if v is None else v.double().clone() for k, v in c.items()}
    if move is not None:
        x[move[0]][move[1]] += move[2]
    X, W = x["x"], x["x"].shape[1]
    one = torch.ones_like(X)
    sc, wo, wi = (one[0] if x[k] is None else x[k] for k in ("scale", "w_post", "w_pre"))
    u = torch.zeros_like(X) if x["u"] is None else x["u"]
    s = one if x["gate"] is None else torch.sigmoid(x["gate"])
    less = 0 * one if x["gate"] is None else torch.sigmoid(-x["gate"])   # what s lacks to one, all digits of it
    ru = one[:, :1] if x["w_post"] is None else (u.square().mean(1, keepdim=True) + EPS) ** -0.5
    n = u * ru * wo
    y = X + sc * s * n
    ay = X.abs() + (sc * s * n).abs()
    ry = (y.square().mean(1, keepdim=True) + EPS) ** -0.5
    h = y * ry * wi
    out, mag = {"y": y, "h": h}, {"y": ay, "h": ay * ry * wi.abs() * 2}
    dy, ady = x["dy"], x["dy"].abs()
    if x["dh"] is not None:
        g = x["dh"] * wi
        m = (g * y).mean(1, keepdim=True)
        am = (g.abs() * ay).mean(1, keepdim=True)
        dy = dy + ry * g - y * ry ** 3 * m
        ady = ady + 3 * ry * g.abs() + 5 * ay * ry ** 3 * am
        out["dw_pre"], mag["dw_pre"] = (x["dh"] * y * ry).sum(0), 3 * (x["dh"].abs() * ay * ry).sum(0)
    out["dx"], mag["dx"] = dy, ady
    if x["u"] is not None:
        out["dscale"], mag["dscale"] = (dy * s * n).sum(0), (ady * s * n.abs()).sum(0)
        if x["gate"] is not None:
            out["dgate"], mag["dgate"] = dy * sc * n * s * less, ady * (sc * n).abs() * s * less
        t, at = dy * sc * s * wo, ady * (sc * s * wo).abs()
        if x["w_post"] is not None:
            out["dw_post"], mag["dw_post"] = (dy * sc * s * u * ru).sum(0), (ady * (sc * s * u).abs() * ru).sum(0)
            out["du"] = ru * t - u * ru ** 3 * (t * u).mean(1, keepdim=True)
            mag["du"] = ru * at + 3 * u.abs() * ru ** 3 * (at * u.abs()).mean(1, keepdim=True)
        else:
            out["du"], mag["du"] = t, at
    return out, mag


def run(c, pad=0, in_place=False):
    from paper_2603_09237_amd import binding
    torch = _torch()
    rows, width = c["x"].shape
    kind = 1 if c["x"].dtype == torch.bfloat16 else 0
    d = binding.NormDims(rows, width, kind, EPS, *[width + pad] * 4)

    def dev(v):
        if v is None:
            return None
        if v.dim() == 1:
            return v.cuda()
        t = torch.full((rows, width + pad), 7.0, dtype=v.dtype, device="cuda")
        t[:, :width] = v.cuda()
        return t

    x = {k: dev(v) for k, v in c.items()}
    new = lambda: torch.full((rows, width + pad), 7.0, dtype=c["x"].dtype, device="cuda")  # noqa: E731
    col = lambda: torch.full((width,), 7.0, device="cuda")  # noqa: E731
    o = {"y": x["x"].clone() if in_place else new(), "h": new() if c["w_pre"] is not None else None}
    binding.norm_fwd(d, o["y"] if in_place else x["x"], x["u"], x["gate"], x["scale"], x["w_post"], x["w_pre"], o["y"], o["h"])
    o["dx"] = x["dy"].clone() if in_place else new()
    for k, src in (("du", "u"), ("dgate", "gate")):
        o[k] = new() if c[src] is not None else None
    for k, there in (("dscale", c["u"]), ("dw_post", c["w_post"]), ("dw_pre", c["w_pre"])):
        o[k] = col() if there is not None else None
    ws = torch.full((binding.norm_workspace_bytes(d),), 0xff, dtype=torch.uint8, device="cuda")
    binding.norm_bwd(d, x["x"], x["u"], x["gate"], x["scale"], x["w_post"], x["w_pre"], o["dx"] if in_place else x["dy"], x["dh"], o["dx"], o["du"],
                     o["dgate"], o["dscale"], o["dw_post"], o["dw_pre"], ws)
    res = {}
    for k, v in o.items():
        if v is None:
            continue
        if v.dim() == 2:
            assert bool((v[:, width:] == 7.0).all()), k
            v = v[:, :width]
        res[k] = v.cpu()
    return res


def compare(c, got):
    torch = _torch()
    want, mag = define(c)
    rows, width = c["x"].shape
    gate = 0.0 if c["gate"] is None else float(c["gate"].float().abs().max())
    assert set(got) == set(k for k in want if k != "h" or c["w_pre"] is not None)
    for k in got:
        n = 16 + width / 32 + gate + (rows / 64 + 64 if want[k].dim() == 1 else 0)
        half = 2.0 ** -8 if got[k].dtype == torch.bfloat16 else U
        err, tol = (got[k].double() - want[k]).abs(), n * U * mag[k] + half * want[k].abs() * (1 + n * U) + 1e-30
        assert bool((err <= tol).all()), (k, int((err > tol).sum()), float((err / tol).max()))


ALL = "u gate scale w_post w_pre"


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,width,parts", [(1, 1, ALL), (1, 8, ALL), (3, 13, ALL), (70, 64, ALL), (257, 256, ALL), (5000, 40, ALL), (33, 512, "u scale w_pre"),
                                              (9, 513, "u w_post w_pre"), (20, 1024, "u gate w_post"), (7, 1999, ALL), (6, 2056, ALL), (5, 4099, "u"),
                                              (4, 8192, ALL), (12, 300, "w_pre"), (1100, 3, "u gate scale")])
def test_values_and_gradients(kind, rows, width, parts):
    c = make(getattr(_torch(), kind), rows, width, parts)
    compare(c, run(c))


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_strides_and_in_place(kind):
    torch = _torch()
    for rows, width in ((9, 24), (5, 515)):
        c = make(getattr(torch, kind), rows, width)
        a = run(c)
        for b in (run(c, pad=3), run(c, pad=8), run(c, in_place=True)):
            for k in a:
                assert torch.equal(a[k], b[k]), k


def test_definition_against_differences():
    torch = _torch()
    c = make(torch.float64, 3, 5)
    want, _ = define(c)

    def value(move):
        o, _ = define(c, move)
        return float((o["y"] * c["dy"]).sum() + (o["h"] * c["dh"]).sum())

    for k, g, at in (("x", "dx", (1, 2)), ("u", "du", (0, 4)), ("gate", "dgate", (2, 0)), ("scale", "dscale", (3,)), ("w_post", "dw_post", (1,)), ("w_pre", "dw_pre", (2,))):
        h = 1e-6
        slope = (value((k, at, h)) - value((k, at, -h))) / (2 * h)
        assert abs(slope - float(want[g][at])) < 1e-6 * (1 + abs(slope)), k


def test_gates_at_the_ends():
    """Gates so large that the sigmoid is 0 or 1: no overflow, and its slope keeps its digits."""
    torch = _torch()
    c = make(torch.float32, 4, 12)
    c["gate"][:] = torch.tensor([-200.0, -100.0, -88.0, -30.0, -5.0, 0.0, 5.0, 20.0, 30.0, 88.0, 100.0, 200.0])
    got = run(c)
    want, mag = define(c)
    # (exponentials of up to 200 are off by 200 2^-24 2 of themselves; below 2^-126 they are zero)
    err, tol = (got["dgate"].double() - want["dgate"]).abs(), 500 * U * mag["dgate"] + 2e-38
    assert bool((err <= tol).all())
    assert bool(torch.isfinite(got["y"]).all())


def test_rows_are_their_own():
    """An undefined or infinite row leaves the others alone (but for the columns' sums, which it is in)."""
    torch = _torch()
    for kind in (torch.float32, torch.bfloat16):
        c = make(kind, 6, 40)
        clean = run(c)
        for k, v in (("x", float("nan")), ("u", float("inf")), ("gate", float("nan")), ("dy", float("inf")), ("dh", float("nan"))):
            d = dict(c, **{k: c[k].clone()})
            d[k][2, 7] = v
            got = run(d)
            for name in ("y", "h", "dx", "du", "dgate"):
                keep = torch.arange(6) != 2
                assert torch.equal(got[name][keep], clean[name][keep]), (k, name)
            assert not bool(torch.isfinite(got["dx" if k in ("dy", "dh") else "y"][2, 7].float()))


def test_no_rows_and_zero_rows():
    from paper_2603_09237_amd import binding
    torch = _torch()
    d = binding.NormDims(0, 16, 0, EPS)
    cols = [torch.full((16,), 7.0, device="cuda") for _ in range(3)]
    ws = torch.empty(binding.norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    w = torch.ones(16, device="cuda")
    binding.norm_fwd(d, None, None, None, w, w, w, None, None)
    binding.norm_bwd(d, None, None, None, w, w, w, None, None, None, None, None, *cols, ws)
    assert all(bool((t == 0).all()) for t in cols)
    c = make(torch.float32, 3, 16)
    for k in ("x", "u"):
        c[k][:] = 0
    got = run(c)
    assert all(bool(torch.isfinite(v.float()).all()) for v in got.values()) and bool((got["y"] == 0).all())


def test_repeats_and_replays():
    from paper_2603_09237_amd import binding
    torch = _torch()
    c = make(torch.bfloat16, 3000, 512)
    a, b = run(c), run(c)
    assert all(torch.equal(a[k], b[k]) for k in a)
    d = binding.NormDims(3000, 512, 1, EPS)
    x = {k: v.cuda() for k, v in c.items()}
    o = {k: torch.empty_like(x["x"]) for k in ("y", "h", "dx", "du", "dgate")}
    cols = {k: torch.empty(512, device="cuda") for k in ("dscale", "dw_post", "dw_pre")}
    ws = torch.empty(binding.norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")

    def work():
        binding.norm_fwd(d, x["x"], x["u"], x["gate"], x["scale"], x["w_post"], x["w_pre"], o["y"], o["h"])
        binding.norm_bwd(d, x["x"], x["u"], x["gate"], x["scale"], x["w_post"], x["w_pre"], x["dy"], x["dh"], o["dx"], o["du"], o["dgate"], *cols.values(), ws)

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in range(4):
        x["x"].normal_()
        work()
        want = [t.clone() for t in (*o.values(), *cols.values())]
        for t in (*o.values(), *cols.values()):
            t.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((*o.values(), *cols.values()), want)), i
