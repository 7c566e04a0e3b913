"""What the memory block keeps between its calls: graphs and other sizes, acting beside an update, a memory that moves on before the backward."""
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def ready(T=40, N=6):
    from test_gpu_memory_block import setup
    torch = _torch()
    block, x, first, index, state = setup(torch.bfloat16, T=T, N=N)
    dy = torch.randn(T, N, block.width, generator=torch.Generator().manual_seed(7)).to(torch.bfloat16)
    return block, x.cuda(), first.cuda(), index.cuda(), tuple(s.cuda() for s in state), dy.cuda()


def test_a_graph_outlives_calls_of_other_sizes():
    """Captured, then calls of larger and smaller segments whose buffers take the old ones' places, other tensors filled, and replays."""
    torch = _torch()
    block, x, first, index, state, dy = ready()

    def work():
        y, after = block.segment(x, index, first, state, train=True)
        return y, after[1], block.backward(dy)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        work()
    stream.synchronize()
    want = [t.clone() for t in work()] + [g.clone() for g in block.g.values()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for T, N in ((90, 6), (7, 3), (300, 2)):
        other = torch.randn(T, N, block.width, device="cuda").to(torch.bfloat16)
        block.segment(other, index[:N].contiguous(), None, block.new_state(N), train=True)
        block.backward(other)
        taken = [torch.full((n,), float("nan"), device="cuda") for n in (1 << 10, 1 << 14, 1 << 16, 1 << 18, 1 << 20) for _ in range(4)]
        for g in block.g.values():
            g.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(list(got) + list(block.g.values()), want):
            assert torch.equal(a, b)
        assert all(torch.isnan(t).all() for t in taken)   # nothing of others' was written


def test_acting_beside_an_update():
    """A rollout's steps on one stream while segments and gradients run on another, against each alone."""
    torch = _torch()
    block, x, first, index, state, dy = ready(T=64, N=64)
    wide = torch.randn(64, 64, block.width, device="cuda").to(torch.bfloat16)

    def update():
        y, _ = block.segment(x, index, first, state, train=True)
        return y, block.backward(dy).clone()

    def rollout():
        now, nxt, out = block.new_state(64), block.new_state(64), []
        for t in range(64):
            out.append(block.act(wide[t], index, None, now, nxt))
            now, nxt = nxt, now
        return torch.stack(out)

    want, steps = update(), rollout()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(a):
            got = update()
        with torch.cuda.stream(b):
            out = rollout()
        torch.cuda.synchronize()
        assert torch.equal(out, steps)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_the_memory_may_move_on_before_the_backward():
    """Acting writes the next memory into the tensors that the segment started from, as a rollout that swaps two does; the gradients stay."""
    torch = _torch()
    block, x, first, index, state, dy = ready(T=5)
    block.segment(x, index, first, state, train=True)
    want = [block.backward(dy).clone()] + [g.clone() for g in block.g.values()]
    _, now = block.segment(x, index, first, state, train=True)
    block.act(x[0], index, None, now, state)     # into the segment's first state
    state[0].fill_(float("nan"))
    got = [block.backward(dy)] + list(block.g.values())
    for a, b in zip(got, want):
        assert torch.equal(a, b)
