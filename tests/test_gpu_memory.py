"""The causal convolution, the selective scan and the single step against their definitions in 64 bits, one time step after the
other, with gradients by differentiation of that definition (and that against differences)."""
import numpy as np
import pytest

from paper_2603_09237_amd import binding

pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1


def _torch():
    import torch
    return torch


def _kind(dtype):
    torch = _torch()
    return torch.bfloat16 if dtype == BF16 else torch.float32


# ---- definitions (float64, CPU) ----
def conv_definition(x, w, b, first, state, act):
    torch = _torch()
    T = x.shape[0]
    seen, ys = state, []
    for t in range(T):
        if first is not None:
            seen = torch.where(first[t].bool()[:, None, None], torch.zeros((), dtype=x.dtype), seen)
        win = torch.cat([seen, x[t][:, None]], 1)
        y = (win * w.t()).sum(1) + (b if b is not None else 0)
        ys.append(y * torch.sigmoid(y) if act else y)
        seen = win[:, 1:]
    return torch.stack(ys), seen


def scan_definition(x, b, c, dt, z, a_log, d, bias, first, h):
    """x [T, N, H, P], b and c [T, N, G, S], dt [T, N, H], z like x, h [N, H, P, S]"""
    torch = _torch()
    T, N, H, P = x.shape
    rep = H // b.shape[2]
    ys = []
    for t in range(T):
        if first is not None:
            h = torch.where(first[t].bool()[:, None, None, None], torch.zeros((), dtype=x.dtype), h)
        step = torch.nn.functional.softplus(dt[t] + (bias if bias is not None else 0))
        bt, ct = (v[t].repeat_interleave(rep, 1)[:, :, None] for v in (b, c))
        h = torch.exp(-step * torch.exp(a_log))[..., None, None] * h + (step[..., None] * x[t])[..., None] * bt
        y = (h * ct).sum(-1) + (d[:, None] * x[t] if d is not None else 0)
        ys.append(y * z[t] * torch.sigmoid(z[t]) if z is not None else y)
    return torch.stack(ys), h


def close(got, want, chain, rounded, what, scale=None):
    """fp32 results: up to four chained sums (scores, decays, states, outputs) of `chain` products, each off by chain 2^-24 of its largest
    partial sum at the very most, taken as the largest value of the tensor (or `scale`, where sums cancel).  bf16 outputs: 2^-8 of
    themselves more."""
    torch = _torch()
    got, want = got.double().cpu(), want.detach()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    top = max(float(want.abs().max()), scale or 0.0)
    err = (got - want).abs()
    tol = 4 * chain * 2.0 ** -24 * top + (2.0 ** -8 * want.abs() if rounded else 0) + 1e-30
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.numel(), float(err[bad].max()), top)


def strided(v, pad, order, fill=7.0):
    """A device tensor [T, N, C] with the values of v: rows `pad` elements longer, and time or environments outermost in memory."""
    torch = _torch()
    T, N, C = v.shape
    if order == "tn":
        return torch.full((T, N, C + pad), fill, dtype=v.dtype, device="cuda")[:, :, :C].copy_(v)
    return torch.full((N, T, C + pad), fill, dtype=v.dtype, device="cuda").transpose(0, 1)[:, :, :C].copy_(v)


# ---- convolution ----
def conv_problem(T, N, C, W, dtype, p_first, pad, order, seed, state=True, bias=True):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    td = _kind(dtype)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    h = dict(x=r(T, N, C).to(td), dy=r(T, N, C).to(td), w=r(C, W) * W ** -0.5, b=r(C) if bias else None, state=r(N, W - 1, C).to(td) if state else None,
             dstate=r(N, W - 1, C).to(td), first=(torch.rand(T, N, generator=g) < p_first).to(torch.uint8) if p_first > 0 else None)
    d = {k: (strided(v, pad, order) if k in ("x", "dy") else v.cuda()) if v is not None else None for k, v in h.items()}
    d["y"], d["dx"] = (strided(torch.zeros(T, N, C, dtype=td), pad, order) for _ in range(2))
    dims = binding.ConvDims(T, N, C, W, 1, dtype, d["x"].stride(0), d["x"].stride(1), d["y"].stride(0), d["y"].stride(1))
    return dims, h, d


CONV = [(1, 1, 1, 1, 0.0, 0, "tn"), (1, 3, 8, 4, 0.5, 0, "tn"), (2, 5, 24, 4, 0.3, 8, "nt"), (3, 2, 9, 3, 0.0, 1, "tn"), (37, 6, 640, 4, 0.05, 0, "tn"),
        (130, 2, 33, 2, 0.1, 3, "nt"), (70, 9, 40, 4, 1.0, 0, "tn"), (64, 33, 16, 3, 0.02, 16, "tn")]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("T,N,C,W,p,pad,order", CONV)
def test_convolution(T, N, C, W, p, pad, order, act, dtype):
    torch = _torch()
    dims, h, d = conv_problem(T, N, C, W, dtype, p, pad, order, seed=T + C, state=N != 6, bias=C != 9)
    dims.act = act
    out = torch.full((N, W - 1, C), 7.0, dtype=_kind(dtype), device="cuda")
    binding.conv_fwd(dims, d["x"], d["w"], d["b"], d["first"], d["state"], d["y"], out if W > 1 else None)
    names = ["x", "w", "state"] + (["b"] if h["b"] is not None else [])
    ins = {k: (h[k] if h[k] is not None else torch.zeros(N, W - 1, C)).double().requires_grad_() for k in names}
    y, last = conv_definition(ins["x"], ins["w"], ins.get("b"), h["first"], ins["state"], act)
    close(d["y"], y, 8, dtype == BF16, "y")
    if W > 1:
        assert torch.equal(out.double().cpu(), last.detach())
    ws = torch.full((binding.conv_workspace_bytes(dims),), 255, dtype=torch.uint8, device="cuda")
    dw, db = torch.full((C, W), 7.0, device="cuda"), torch.full((C,), 7.0, device="cuda")
    dstate = torch.full((N, W - 1, C), 7.0, dtype=_kind(dtype), device="cuda") if W > 1 else None
    with_out = N != 5
    for _ in range(2):
        binding.conv_bwd(dims, d["x"], d["w"], d["b"], d["first"], d["state"], d["dy"], d["dstate"] if with_out and W > 1 else None, d["dx"], dw, db,
                         dstate, ws)
    loss = (y * h["dy"].double()).sum() + ((last * h["dstate"].double()).sum() if with_out else 0)
    want = dict(zip(names, torch.autograd.grad(loss, [ins[k] for k in names], allow_unused=True)))
    close(d["dx"], want["x"], 16, dtype == BF16, "dx")
    close(dw, want["w"], 16 + T * N, False, "dw")
    if "b" in want:
        close(db, want["b"], 16 + T * N, False, "db")
    if W > 1:
        close(dstate, want["state"] if want["state"] is not None else torch.zeros(N, W - 1, C).double(), 16, dtype == BF16, "dstate_in")
    if pad:  # nothing between the rows was written
        for v in (d["y"], d["dx"]):
            assert (v.as_strided((T, N, pad), (v.stride(0), v.stride(1), 1), C) == 7.0).all()


def test_convolution_keeps_episodes_apart():
    """Infinite and undefined inputs of an episode stay in it, forward and backward."""
    torch = _torch()
    dims, h, d = conv_problem(20, 4, 16, 4, F32, 0.0, 0, "tn", seed=3)
    first = torch.zeros(20, 4, dtype=torch.uint8, device="cuda")
    first[7, :2] = 1
    ws = torch.empty(binding.conv_workspace_bytes(dims), dtype=torch.uint8, device="cuda")
    args = lambda: (dims, d["x"], d["w"], d["b"], first, d["state"])  # noqa: E731
    dw, db, dst = torch.empty(16, 4, device="cuda"), torch.empty(16, device="cuda"), torch.empty(4, 3, 16, device="cuda")
    res = []
    for bad in (False, True):
        if bad:
            d["x"][6, 0, 3], d["x"][5, 1, 5], d["dy"][7, 1] = float("nan"), float("inf"), float("nan")
        binding.conv_fwd(*args(), d["y"], None)
        binding.conv_bwd(*args(), d["dy"], None, d["dx"], dw, db, dst, ws)
        res.append((d["y"].clone(), d["dx"].clone()))
    assert torch.equal(res[0][0][7:], res[1][0][7:]) and torch.equal(res[0][0][:5], res[1][0][:5])
    # (the infinite x[5] makes the derivatives of steps 5 and 6 undefined, and the first of them reaches back to dx[2])
    assert torch.equal(res[0][1][:2, 1], res[1][1][:2, 1]) and not torch.isfinite(res[1][0][6, 0, 3])
    assert torch.isfinite(res[1][1][4:7, 1][:, 0]).all()  # dy of the next episode does not reach the one before


# ---- scan ----
def scan_problem(T, N, H, P, G, S, dtype, p_first, gate, seed, pad=0, order="tn", state=True):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    td = _kind(dtype)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    D, GS = H * P, G * S
    h = dict(xbc=r(T, N, D + 2 * GS).to(td), dt=(0.5 * r(T, N, H)).to(td), z=r(T, N, D).to(td) if gate else None, a_log=torch.log(1 + 15 * torch.rand(H, generator=g)),
             d=r(H), bias=torch.log(torch.expm1(torch.exp(torch.rand(H, generator=g) * 4.6 - 6.9))), dy=r(T, N, D).to(td),
             first=(torch.rand(T, N, generator=g) < p_first).to(torch.uint8) if p_first > 0 else None,
             state=0.3 * r(N, H, P, S) if state else None, dstate=0.1 * r(N, H, P, S))
    d = {k: (strided(v, pad, order) if k in ("xbc", "dt", "z", "dy") else v.cuda()) if v is not None else None for k, v in h.items()}
    for k, like in (("y", "dy"), ("dxbc", "xbc"), ("ddt", "dt"), ("dz", "z")):
        d[k] = strided(torch.zeros_like(h[like]), pad, order) if h[like] is not None else None
    st = lambda k: (d[k].stride(0), d[k].stride(1)) if d[k] is not None else (0, 0)  # noqa: E731
    dims = binding.ScanDims(T, N, H, P, G, S, dtype, *st("xbc"), *st("z"), *st("dt"), *st("y"))
    return dims, h, d


def parts(v, dims):
    D, GS = dims.heads * dims.head_dim, dims.groups * dims.state
    return v[..., :D], v[..., D:D + GS], v[..., D + GS:D + 2 * GS]


def run_scan(dims, d, saved=False, state_out=None):
    torch = _torch()
    x, b, c = parts(d["xbc"], dims)
    out = torch.full((dims.N, dims.heads, dims.head_dim, dims.state), 7.0, device="cuda") if state_out is None else state_out
    sv = torch.full((binding.scan_saved_bytes(dims),), 255, dtype=torch.uint8, device="cuda") if saved else None
    ws = torch.full((binding.scan_workspace_bytes(dims),), 255, dtype=torch.uint8, device="cuda")
    binding.scan_fwd(dims, x, b, c, d["dt"], d["z"], d["a_log"], d["d"], d["bias"], d["first"], d["state"], d["y"], out, sv, ws)
    return d["y"], out, sv


def run_scan_bwd(dims, d, saved, dstate=True):
    torch = _torch()
    x, b, c = parts(d["xbc"], dims)
    dx, db, dc = parts(d["dxbc"], dims)
    H = dims.heads
    o = dict(a_log=torch.full((H,), 7.0, device="cuda"), d=torch.full((H,), 7.0, device="cuda"), bias=torch.full((H,), 7.0, device="cuda"),
             state=torch.full((dims.N, H, dims.head_dim, dims.state), 7.0, device="cuda"))
    ws = torch.full((binding.scan_workspace_bytes(dims, True),), 255, dtype=torch.uint8, device="cuda")
    binding.scan_bwd(dims, x, b, c, d["dt"], d["z"], d["a_log"], d["d"], d["bias"], d["first"], saved, d["dy"], d["dstate"] if dstate else None, dx, db, dc,
                     d["ddt"], d["dz"], o["a_log"], o["d"], o["bias"], o["state"], ws)
    return dict(o, xbc=d["dxbc"], dt=d["ddt"], z=d["dz"])


def scan_truth(dims, h, grads=False, dstate=True):
    torch = _torch()
    T, N, H, P, G, S = (getattr(dims, k) for k in ("T", "N", "heads", "head_dim", "groups", "state"))
    names = [k for k in ("xbc", "dt", "z", "a_log", "d", "bias", "state") if h[k] is not None]
    ins = {k: h[k].double().requires_grad_(grads) for k in names}
    x, b, c = parts(ins["xbc"], dims)
    z = ins["z"].reshape(T, N, H, P) if h["z"] is not None else None
    h0 = ins["state"] if h["state"] is not None else torch.zeros(N, H, P, S, dtype=torch.float64)
    y, last = scan_definition(x.reshape(T, N, H, P), b.reshape(T, N, G, S), c.reshape(T, N, G, S), ins["dt"], z, ins["a_log"], ins.get("d"),
                              ins.get("bias"), h["first"], h0)
    y = y.reshape(T, N, H * P)
    if not grads:
        return y, last, None
    loss = (y * h["dy"].double()).sum() + ((last * h["dstate"].double()).sum() if dstate else 0)
    got = torch.autograd.grad(loss, [ins[k] for k in names], allow_unused=True)
    return y, last, {k: v if v is not None else torch.zeros_like(ins[k]) for k, v in zip(names, got)}


# T, N, heads, head_dim, groups, state, p_first, gate, pad, order
SCAN = [(1, 1, 1, 1, 1, 1, 0.0, False, 0, "tn"), (1, 3, 4, 64, 1, 64, 0.5, True, 0, "tn"), (31, 2, 2, 32, 2, 16, 0.0, True, 0, "tn"),
        (32, 1, 5, 64, 1, 64, 0.1, False, 0, "nt"), (33, 2, 3, 8, 1, 40, 0.05, True, 1, "tn"), (100, 3, 4, 37, 2, 5, 0.03, True, 3, "nt"),
        (129, 1, 1, 64, 1, 16, 0.0, False, 8, "tn"), (257, 1, 2, 64, 1, 64, 0.005, True, 0, "tn"), (610, 2, 3, 9, 1, 21, 0.0, False, 0, "nt"),
        (333, 1, 8, 40, 2, 16, 0.3, True, 0, "tn"), (64, 5, 9, 24, 3, 64, 1.0, True, 0, "tn"), (70, 2, 6, 33, 1, 33, 0.2, False, 0, "tn")]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,N,H,P,G,S,p,gate,pad,order", SCAN)
def test_scan(T, N, H, P, G, S, p, gate, pad, order, dtype):
    dims, h, d = scan_problem(T, N, H, P, G, S, dtype, p, gate, seed=T + S, pad=pad, order=order, state=H != 5)
    y, last, _ = scan_truth(dims, h)
    got, out, _ = run_scan(dims, d)
    close(got, y, S + P + 32, dtype == BF16, "y")
    close(out, last, S + P + 32, False, "state")
    if pad:
        D = H * P
        assert (got.as_strided((T, N, pad), (got.stride(0), got.stride(1), 1), D) == 7.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,N,H,P,G,S,p,gate,pad,order", SCAN)
def test_scan_gradients(T, N, H, P, G, S, p, gate, pad, order, dtype):
    torch = _torch()
    dims, h, d = scan_problem(T, N, H, P, G, S, dtype, p, gate, seed=T + P, pad=pad, order=order, state=H != 5)
    dstate = H != 6
    _, _, want = scan_truth(dims, h, True, dstate)
    _, _, saved = run_scan(dims, d, saved=True)
    got = {k: v.clone() if v is not None else None for k, v in run_scan_bwd(dims, d, saved, dstate).items()}
    again = run_scan_bwd(dims, d, saved, dstate)
    chain = S + P + 32
    # the steps' gradients are sums of C . dC - dt B . dB, which cancel: against the largest such term times the largest decay rate
    _, b, c = parts(h["xbc"].double(), dims)
    _, db, dc = parts(want["xbc"], dims)
    term = max(float((b * db).reshape(T, N, G, S).abs().sum(-1).max()), float((c * dc).reshape(T, N, G, S).abs().sum(-1).max()))
    rate = float(torch.exp(h["a_log"]).max())
    for k in want:
        if k in ("xbc", "z", "dt"):
            close(got[k], want[k], chain, dtype == BF16, k, term * rate if k == "dt" else None)
        elif k == "state":
            close(got[k], want[k], chain, False, k)
        else:
            close(got[k], want[k], chain + T * N, False, k, term * rate if k != "d" else None)
    for k in got:
        assert got[k] is None or torch.equal(got[k], again[k]), k  # bit for bit
    if pad:
        v = d["dxbc"]
        assert (v.as_strided((T, N, pad), (v.stride(0), v.stride(1), 1), H * P + 2 * G * S) == 7.0).all()


def test_scan_gradients_of_the_definition_against_differences():
    torch = _torch()
    dims, h, _ = scan_problem(5, 2, 2, 3, 1, 2, F32, 0.2, True, seed=4)
    _, _, want = scan_truth(dims, h, True)

    def loss(v):
        y, last, _ = scan_truth(dims, v)
        return float((y * h["dy"].double()).sum() + (last * h["dstate"].double()).sum())

    for k in want:
        flat = want[k].reshape(-1)
        for i in range(0, flat.numel(), max(1, flat.numel() // 6)):
            vals = []
            for s in (1e-6, -1e-6):
                v = dict(h)
                v[k] = h[k].double().clone()
                v[k].reshape(-1)[i] += s
                vals.append(loss(v))
            assert abs((vals[0] - vals[1]) / 2e-6 - float(flat[i])) < 1e-6 * max(1.0, float(flat.abs().max())), (k, i)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_carries_its_state(dtype):
    """Two calls, the second from the first one's state in place, against one."""
    torch = _torch()
    dims, h, d = scan_problem(90, 3, 4, 64, 1, 16, dtype, 0.02, True, seed=11)
    y, last, _ = scan_truth(dims, h)
    whole, out, _ = run_scan(dims, d)
    whole, out = whole.clone(), out.clone()
    state = d["state"].clone()
    for t0, t1 in ((0, 41), (41, 90)):
        part = binding.ScanDims(t1 - t0, *[getattr(dims, f[0]) for f in dims._fields_][1:7], *[getattr(dims, f[0]) for f in dims._fields_][7:])
        dd = {k: (v[t0:t1] if v is not None and k in ("xbc", "dt", "z", "y", "first") else v) for k, v in d.items()}
        dd["state"] = state
        run_scan(part, dd, state_out=state)
    close(state, last, 112, False, "state")
    close(d["y"], y, 112, dtype == BF16, "y")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [50, 400])   # one span of time, several
def test_scan_keeps_episodes_apart(T, dtype):
    """Infinite and undefined inputs reach nothing of another episode, nothing of an earlier step, no other head or environment."""
    torch = _torch()
    dims, h, d = scan_problem(T, 2, 3, 40, 1, 24, dtype, 0.0, True, seed=5)
    first = torch.zeros(T, 2, dtype=torch.uint8)
    first[20, 0] = first[45, 0] = 1
    h["first"], d["first"] = first, first.cuda()
    y0, out0, s0 = run_scan(dims, d, saved=True)
    y0, out0 = y0.clone(), out0.clone()
    g0 = {k: v.clone() for k, v in run_scan_bwd(dims, d, s0).items()}
    P = 40
    for name, where in (("x", (10, 0, P + 3)), ("b", (12, 0, 3 * P + 2)), ("c", (15, 0, 3 * P + 24 + 1))):
        for value in (float("nan"), float("inf")):
            keep = d["xbc"].clone()
            d["xbc"][where] = value
            y, out, sv = run_scan(dims, d, saved=True)
            heads = slice(P, 2 * P) if name == "x" else slice(0, 3 * P)
            ok = torch.ones_like(y0, dtype=torch.bool)
            ok[where[0]:20, 0, heads] = False
            # (the chunk's other steps are taken one by one: other roundings)
            assert torch.allclose(y[ok].float(), y0[ok].float(), rtol=2.0 ** -7 if dtype == BF16 else 1e-5, atol=1e-4), name
            assert not torch.isfinite(y[where[0], 0, heads]).all()
            assert torch.allclose(out, out0, rtol=1e-5, atol=1e-5)
            g = run_scan_bwd(dims, d, sv)
            for k in ("xbc", "dt", "z"):
                a, bb = g[k].float(), g0[k].float()
                tol = 2.0 ** -6 * float(bb.abs().max()) if dtype == BF16 else 1e-4 * float(bb.abs().max())
                assert torch.allclose(a[:, 1], bb[:, 1], rtol=0, atol=tol) and torch.allclose(a[20:, 0], bb[20:, 0], rtol=0, atol=tol), (name, k)
            d["xbc"].copy_(keep)
    # an undefined gradient reaches its own episode's earlier steps only
    d["dy"][47, 0, 5] = float("nan")
    g = run_scan_bwd(dims, d, s0)
    for k in ("xbc", "dt", "z"):
        a, bb = g[k].float(), g0[k].float()
        tol = 2.0 ** -6 * float(bb.abs().max()) if dtype == BF16 else 1e-4 * float(bb.abs().max())
        assert torch.allclose(a[:45, 0], bb[:45, 0], rtol=0, atol=tol) and torch.allclose(a[:, 1], bb[:, 1], rtol=0, atol=tol), k


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_with_steps_that_forget(dtype):
    """Decays that underflow, steps of length zero, and small steps behind large ones."""
    dims, h, d = scan_problem(60, 2, 2, 16, 1, 16, dtype, 0.0, False, seed=6)
    for k in (h, d):
        k["dt"][5], k["dt"][17:19], k["dt"][30:40], k["dt"][41] = 60.0, 300.0, -200.0, 25.0
    y, last, want = scan_truth(dims, h, True)
    got, out, saved = run_scan(dims, d, saved=True)
    close(got, y, 64, dtype == BF16, "y")
    close(out, last, 64, False, "state")
    g = run_scan_bwd(dims, d, saved)
    for k in ("xbc", "state"):
        close(g[k], want[k], 64, dtype == BF16 and k == "xbc", k)


# ---- one step ----
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,H,P,G,S,W,p,gate", [(1, 1, 1, 1, 1, 1, 0.0, False), (1, 8, 64, 1, 64, 4, 0.0, True), (5, 6, 37, 2, 9, 3, 0.5, True),
                                                (33, 4, 64, 2, 16, 4, 0.2, False), (3, 3, 8, 3, 62, 2, 1.0, True)])
def test_step(N, H, P, G, S, W, p, gate, dtype):
    torch = _torch()
    dims, h, d = scan_problem(1, N, H, P, G, S, dtype, p, gate, seed=N + S)
    C = H * P + 2 * G * S
    g = torch.Generator().manual_seed(1)
    w, b, cin = torch.randn(C, W, generator=g) * W ** -0.5, torch.randn(C, generator=g), torch.randn(N, W - 1, C, generator=g).to(_kind(dtype))
    conv, seen = conv_definition(h["xbc"].double(), w.double(), b.double(), h["first"], cin.double(), 1)
    x, bb, cc = parts(conv, dims)
    z = h["z"].double().reshape(1, N, H, P) if gate else None
    y, last = scan_definition(x.reshape(1, N, H, P), bb.reshape(1, N, G, S), cc.reshape(1, N, G, S), h["dt"].double(), z, h["a_log"].double(),
                              h["d"].double(), h["bias"].double(), h["first"], h["state"].double())
    out = torch.full((N, W - 1, C), 7.0, dtype=_kind(dtype), device="cuda")
    state = d["state"].clone()   # in place
    binding.memory_step(dims, W, d["xbc"], d["dt"], d["z"], w.cuda(), b.cuda(), d["a_log"], d["d"], d["bias"], d["first"], cin.cuda(), state, d["y"],
                        out if W > 1 else None, state)
    close(d["y"], y.reshape(1, N, H * P), S + 16, dtype == BF16, "y")
    close(state, last, 16, False, "state")
    if W > 1:
        assert torch.equal(out.double().cpu(), seen)


def test_steps_follow_the_sequence():
    """Step after step in fp32 gives what the calls on the whole segment give."""
    torch = _torch()
    T, N, H, P, G, S, W = 20, 3, 2, 32, 1, 16, 4
    dims, h, d = scan_problem(T, N, H, P, G, S, F32, 0.1, True, seed=21)
    C = H * P + 2 * G * S
    w, b = torch.randn(C, W, device="cuda") * 0.5, torch.randn(C, device="cuda")
    raw = d["xbc"].clone()
    cd = binding.ConvDims(T, N, C, W, 1, F32)
    binding.conv_fwd(cd, raw, w, b, d["first"], None, d["xbc"], None)
    y, out, _ = run_scan(dims, d)
    one = binding.ScanDims(1, N, H, P, G, S, F32)
    conv, state, ys = [torch.zeros(N, W - 1, C, device="cuda") for _ in range(2)], d["state"].clone(), torch.empty_like(y)
    for t in range(T):
        binding.memory_step(one, W, raw[t], d["dt"][t], d["z"][t], w, b, d["a_log"], d["d"], d["bias"], d["first"][t], conv[t % 2], state, ys[t],
                            conv[1 - t % 2], state)
    assert torch.allclose(ys, y, rtol=1e-4, atol=1e-4) and torch.allclose(state, out, rtol=1e-4, atol=1e-5)


def test_time_steps_far_apart():
    """Strides that take a segment beyond 32-bit offsets."""
    torch = _torch()
    T, N, H, P, G, S, far = 40, 2, 2, 32, 1, 16, (1 << 26) + 8
    _, h, d = scan_problem(T, N, H, P, G, S, BF16, 0.1, True, seed=31)
    D, C = H * P, H * P + 2 * G * S
    y, last, _ = scan_truth(binding.ScanDims(T, N, H, P, G, S, BF16), h)
    room = torch.empty(T * far, dtype=torch.bfloat16, device="cuda")
    place = lambda n, at: room.as_strided((T, N, n), (far, n, 1), at)  # noqa: E731
    tensors, at = {}, 0
    for k, n in (("xbc", C), ("z", D), ("dt", H), ("y", D)):
        tensors[k] = place(n, at)
        at += N * n
        if k != "y":
            tensors[k].copy_(h[k])
    dims = binding.ScanDims(T, N, H, P, G, S, BF16, far, C, far, D, far, H, far, D)
    got, out, _ = run_scan(dims, dict(d, **tensors))
    close(got, y, S + P + 32, True, "y")
    close(out, last, S + P + 32, False, "state")
    conv = binding.ConvDims(T, N, C, 4, 1, BF16, far, C, far, C)
    w, other = torch.randn(C, 4), place(C, at)
    want, _ = conv_definition(h["xbc"].double(), w.double(), None, h["first"], torch.zeros(N, 3, C).double(), 1)
    binding.conv_fwd(conv, tensors["xbc"], w.cuda(), None, d["first"], None, other, None)
    close(other, want, 8, True, "convolution")
