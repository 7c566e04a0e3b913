"""An undefined or infinite time step (dt) stays in its episode: what other episodes, heads and environments get is what they get without it,
bit for bit, since no arithmetic of theirs takes part of it."""
import pytest

pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1
H, P, G, S = 3, 40, 1, 24


def _torch():
    import torch
    return torch


def both(T, begins, where, value, dtype):
    """(y, state, gradients) of a scan of two environments without and with dt[where, environment 0, head 1] = value."""
    from test_gpu_memory import run_scan, run_scan_bwd, scan_problem
    torch = _torch()
    dims, h, d = scan_problem(T, 2, H, P, G, S, dtype, 0.0, True, seed=T + where)
    d["first"] = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    for t in begins:
        d["first"][t, 0] = 1
    res = []
    for v in (None, value):
        if v is not None:
            d["dt"][where, 0, 1] = v
        y, out, saved = run_scan(dims, d, saved=True)
        y, out = y.clone(), out.clone()
        res.append((y, out, {k: g.clone() for k, g in run_scan_bwd(dims, d, saved).items()}))
    return res


def episode(T, begins, where):
    """first step of the episode that `where` is in, and the first of the next one"""
    edges = [0, *begins, T]
    i = max(i for i, e in enumerate(edges) if e <= where)
    return edges[i], edges[i + 1]


def apart(T, begins, where, value, dtype):
    torch = _torch()
    (y0, out0, g0), (y, out, g) = both(T, begins, where, value, dtype)
    e0, e1 = episode(T, begins, where)
    heads = lambda v, n: v.reshape(*v.shape[:2], H, n)  # noqa: E731
    ok = torch.ones(T, 2, H, dtype=torch.bool, device="cuda")
    ok[where:e1, 0, 1] = False
    assert torch.equal(heads(y, P)[ok], heads(y0, P)[ok])
    assert not torch.isfinite(heads(y, P)[where, 0, 1]).all()
    ends = torch.ones(2, H, dtype=torch.bool, device="cuda")
    ends[0, 1] = e1 < T
    assert torch.equal(out[ends], out0[ends])
    ok[e0:e1, 0] = False        # (dB and dC are sums over the heads)
    for k in ("xbc", "z", "dt"):
        a, b = g[k][ok.all(-1)], g0[k][ok.all(-1)]
        assert torch.isfinite(b).all() and torch.equal(a, b), k
    mine = torch.ones(2, H, dtype=torch.bool, device="cuda")
    mine[0, 1] = e0 > 0
    assert torch.equal(g["state"][mine], g0["state"][mine])
    for k in ("a_log", "d", "bias"):
        assert torch.equal(g[k][[0, 2]], g0[k][[0, 2]]), k


# 400 steps are several spans of 96 steps; the begin in another chunk of 32 steps than the step, of the same span or not
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("T,begins,where", [(400, (45,), 25), (400, (45,), 70), (400, (10, 120), 70), (400, (110,), 170), (400, (5, 390), 200),
                                            (90, (45,), 25), (90, (45,), 70)])
def test_a_step_in_another_chunk(T, begins, where, value, dtype):
    apart(T, begins, where, value, dtype)


# begin and step within the same 32 steps, on either side, with other begins about them; the begin itself; one chunk, several, several spans
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("T,begins,where", [(20, (9,), 14), (20, (9,), 4), (20, (9,), 9), (32, (3, 16, 29), 20), (90, (40, 50), 45), (90, (40,), 35),
                                            (400, (110, 150), 98), (400, (110,), 98), (400, (105,), 111), (400, (200, 210, 220), 215)])
def test_a_step_in_the_same_chunk(T, begins, where, value, dtype):
    apart(T, begins, where, value, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,begin", [(20, 9), (90, 50), (400, 110)])
@pytest.mark.parametrize("scale", [2.0 ** 20, 2.0 ** 60, 2.0 ** 110])   # the last: sums within the later episode overflow
def test_gradients_of_a_later_episode_leave_nothing_behind(T, begin, scale, dtype):
    """Large gradients behind a begin change no bit of those before it."""
    from test_gpu_memory import run_scan, run_scan_bwd, scan_problem
    torch = _torch()
    dims, h, d = scan_problem(T, 2, H, P, G, S, dtype, 0.0, True, seed=T)
    d["first"] = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    d["first"][begin, 0] = 1
    _, _, saved = run_scan(dims, d, saved=True)
    want = {k: v.clone() for k, v in run_scan_bwd(dims, d, saved).items()}
    d["dy"][begin:, 0] *= scale
    got = run_scan_bwd(dims, d, saved)
    for k in ("xbc", "z", "dt"):
        assert torch.equal(got[k][:begin, 0], want[k][:begin, 0]), k
        assert torch.equal(got[k][:, 1], want[k][:, 1]), k
    assert torch.equal(got["state"], want["state"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("T,begin", [(20, 0), (20, 9), (90, 40), (400, 5), (400, 200), (400, 399)])
def test_states_at_either_end(T, begin, value, dtype):
    """What is undefined in the state before the segment ends with its first episode, and in the gradient of the state behind it with the last one."""
    from test_gpu_memory import run_scan, run_scan_bwd, scan_problem
    torch = _torch()
    dims, h, d = scan_problem(T, 2, H, P, G, S, dtype, 0.0, True, seed=T + begin)
    d["first"] = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    d["first"][begin, 0] = 1
    heads = lambda v, n: v.reshape(*v.shape[:2], H, n)  # noqa: E731

    def run():
        y, out, saved = run_scan(dims, d, saved=True)
        return y.clone(), out.clone(), {k: g.clone() for k, g in run_scan_bwd(dims, d, saved).items()}

    y0, out0, g0 = run()
    keep = d["state"][0, 1, 3, 5].clone()
    d["state"][0, 1, 3, 5] = value
    y, out, g = run()
    ok = torch.ones(T, 2, H, dtype=torch.bool, device="cuda")
    ok[:begin, 0, 1] = False
    assert torch.equal(heads(y, P)[ok], heads(y0, P)[ok]) and torch.equal(out, out0)
    assert begin == 0 or not torch.isfinite(heads(y, P)[0, 0, 1]).all()
    for k in ("xbc", "z", "dt"):
        assert torch.equal(g[k][begin:], g0[k][begin:]) and torch.equal(g[k][:, 1], g0[k][:, 1]), k
    d["state"][0, 1, 3, 5] = keep
    d["dstate"][0, 1, 3, 5] = value
    y, out, g = run()
    assert torch.equal(y, y0) and torch.equal(out, out0)
    for k in ("xbc", "z", "dt"):
        assert torch.equal(g[k][:begin], g0[k][:begin]) and torch.equal(g[k][:, 1], g0[k][:, 1]), k
    assert torch.equal(g["state"], g0["state"])
