"""The operators together, as a policy block uses them, against the same block written out in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def written_out(block, p, x, index, first, state):
    """The block in float64 on the CPU from its definition; p: parameters in float64."""
    from test_gpu_memory import conv_definition, scan_definition
    torch = _torch()
    T, N = x.shape[:2]
    idx = index.long().cpu()

    def project(name, v):
        w = p[name + ".w0"] + p[name + ".A"] @ p[name + ".B"]            # [P, out, in]
        return torch.matmul(w[idx], v[..., None])[..., 0] + p[name + ".bias"]

    proj = project("in", x)
    z, raw, dt = block._slices(proj)
    xc, seen = conv_definition(raw, p["conv.w"], p["conv.b"], first, state[0], 1)
    xs, b, c = block._xbc(xc)
    H, Pd, G, S = block.H, block.Pd, block.G, block.S
    y, h = scan_definition(xs.reshape(T, N, H, Pd), b.reshape(T, N, G, S), c.reshape(T, N, G, S), dt, z.reshape(T, N, H, Pd), p["a_log"], p["d_skip"],
                           p["dt_bias"], first, state[1])
    return project("out", y.reshape(T, N, block.D)), (seen, h)


def setup(dtype, T=40, N=6, P=5, width=24):
    from paper_2603_09237_amd.memory import MemoryBlock
    torch = _torch()
    block = MemoryBlock(P, width, heads=4, head_dim=16, groups=2, state=8, rank=3, dtype=dtype, seed=3)
    g = torch.Generator().manual_seed(4)
    x = torch.randn(T, N, width, generator=g).to(dtype)
    first = (torch.rand(T, N, generator=g) < 0.08).to(torch.uint8)
    index = torch.randint(0, P, (N,), generator=g).to(torch.int32)
    state = (torch.randn(N, block.W - 1, block.C, generator=g).to(dtype), 0.2 * torch.randn(N, block.H, block.Pd, block.S, generator=g))
    return block, x, first, index, state


# fp32: three chained operators of sums of up to some hundred terms, each within 1e-5 of its largest values; bf16: every tensor between the
# operators is rounded (2^-9), five roundings in a row on values of the outputs' size
@pytest.mark.parametrize("kind,tol", [("float32", 3e-5), ("bfloat16", 3e-2)])
def test_segment_gradients_and_single_steps(kind, tol):
    torch = _torch()
    block, x, first, index, state = setup(getattr(torch, kind))
    p = {k: v.double().cpu().requires_grad_() for k, v in block.p.items()}
    x64 = x.double().requires_grad_()
    y64, after64 = written_out(block, p, x64, index, first, tuple(s.double() for s in state))
    dev = lambda t: t.cuda()  # noqa: E731
    args = (dev(x), dev(index), dev(first), tuple(dev(s) for s in state))
    y, after = block.segment(*args, train=True)

    def near(got, want, what, factor=1.0):
        got, want = got.double().cpu(), want.detach()
        top = float(want.abs().max())
        assert float((got - want).abs().max()) <= factor * tol * max(top, 1e-6), (what, float((got - want).abs().max()), top)

    near(y, y64, "y")
    near(after[1], after64[1], "state")
    dy = torch.randn(y64.shape, generator=torch.Generator().manual_seed(5)).to(x.dtype)
    names = list(p)
    want = dict(zip(names, torch.autograd.grad((y64 * dy.double()).sum(), [p[k] for k in names], retain_graph=True)))
    (dx64,) = torch.autograd.grad((y64 * dy.double()).sum(), [x64])
    dx = block.backward(dev(dy))
    near(dx, dx64, "dx", 3)
    for k in names:
        near(block.g[k], want[k], k, 3)   # sums of products of such values over T x N rows
    # one step after the other gives what the segment gave
    now, nxt = tuple(dev(s) for s in state), block.new_state(x.shape[1])
    for t in range(x.shape[0]):
        yt = block.act(dev(x[t]), dev(index), dev(first[t]), now, nxt)
        near(yt, y64[t], f"step {t}", float(y64.detach().abs().max()) / max(float(y64.detach()[t].abs().max()), 1e-6))
        now, nxt = nxt, now if t else block.new_state(x.shape[1])
    near(now[1], after64[1], "state after the steps")


def test_segments_join():
    """Two segments, the second from the first one's state, are one."""
    torch = _torch()
    block, x, first, index, state = setup(torch.float32)
    dev = lambda t: t.cuda()  # noqa: E731
    st = tuple(dev(s) for s in state)
    whole, end = block.segment(dev(x), dev(index), dev(first), st)
    a, mid = block.segment(dev(x[:17]), dev(index), dev(first[:17]), st)
    b, end2 = block.segment(dev(x[17:]), dev(index), dev(first[17:]), mid)
    assert torch.allclose(torch.cat([a, b]), whole, rtol=0, atol=2e-5 * float(whole.abs().max()))
    assert torch.equal(end[0], end2[0]) and torch.allclose(end[1], end2[1], rtol=0, atol=2e-5 * float(end[1].abs().max()))


def test_captured_in_a_graph():
    """A segment and its gradients recorded once and replayed, with other work between, against the calls themselves."""
    torch = _torch()
    block, x, first, index, state = setup(torch.bfloat16, T=260, N=2)   # (few heads: several spans of time)
    x, first, index, state = x.cuda(), first.cuda(), index.cuda(), tuple(s.cuda() for s in state)
    dy = torch.randn(260, 2, block.width, device="cuda").to(torch.bfloat16)

    def work():
        y, after = block.segment(x, index, first, state, train=True)
        return y, after[1], block.backward(dy)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        work()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for i in range(4):
        x.normal_()
        want = [t.clone() for t in work()] + [g.clone() for g in block.g.values()]
        for g in block.g.values():
            g.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(list(got) + list(block.g.values()), want):
            assert torch.equal(a, b), i
