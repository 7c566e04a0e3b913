"""The paged cache: its bookkeeping against the same with lists, one environment after the other, and one new step's attention over it against the
definition in 64 bits (tolerances as of the segment's attention: dot products of n terms n 2^-24, exponentials 4 2^-24 and their argument's error,
roundings to bf16 2^-8)."""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _torch():
    import torch
    return torch


# ---- pages ----
def books(page, slots, pages, first, length, table, queue, state):
    """One step's bookkeeping on lists."""
    length, table, queue = list(length), [list(r) for r in table], list(queue)
    head, count = state
    has = lambda e: 0 <= e < pages  # noqa: E731
    slot, back, taken = [], [], 0
    for n in range(len(length)):
        if length[n] < 0:
            slot.append(-1)
            continue
        if first is not None and first[n]:
            back += [e for e in table[n][1:] if has(e)]
            table[n][1:] = [-1] * (slots - 1)
            length[n] = 0
        j = (length[n] // page) % slots
        if not has(table[n][j]) and taken < count:
            table[n][j] = queue[(head + taken) % pages]
            taken += 1
        slot.append(table[n][j] * page + length[n] % page if has(table[n][j]) else -1)
        length[n] += 1
    for i, e in enumerate(back):
        queue[(head + count + i) % pages] = e
    return length, table, queue, [(head + taken) % pages, count - taken + len(back)], slot


def ints(v):
    return _torch().tensor(v, dtype=_torch().int32, device="cuda")


def step_books(d, first, length, table, queue, state, in_place):
    from paper_2603_09237_amd import binding
    torch = _torch()
    ins = [ints(v) for v in (length, table, queue, state)]
    outs = ins if in_place else [torch.full_like(t, 77) for t in ins]
    slot = torch.full((d.N,), 77, dtype=torch.int32, device="cuda")
    ws = torch.full((binding.pages_workspace_bytes(d),), 0xff, dtype=torch.uint8, device="cuda")
    f = None if first is None else torch.tensor(first, dtype=torch.uint8, device="cuda")
    binding.cache_pages(d, f, *ins, *outs, slot, ws)
    return [t.cpu().tolist() for t in outs] + [slot.cpu().tolist()]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("N,page,slots,pages", [(1, 1, 1, 1), (1, 4, 3, 3), (5, 2, 1, 4), (63, 1, 4, 252), (256, 4, 5, 700), (257, 2, 3, 771), (300, 1, 70, 9000),
                                                (1000, 8, 2, 1100)])
def test_pages_over_many_steps(N, page, slots, pages, in_place):
    from paper_2603_09237_amd import binding
    import random
    rng = random.Random(N * 7 + page)
    d = binding.PagesDims(N, page, slots, pages)
    now = ([-1 if rng.random() < 0.05 else 0 for _ in range(N)], [[-1] * slots for _ in range(N)], rng.sample(range(pages), pages), [rng.randrange(pages), pages])
    for step in range(12):
        first = None if step == 3 else [int(rng.random() < 0.15) for _ in range(N)]
        want = books(page, slots, pages, first, *now)
        got = step_books(d, first, *now, in_place)
        for name, a, b in zip(("length", "table", "queue", "state", "slot"), got, want):
            assert a == b, (step, name)
        now = want[:4]
        held = [e for r in now[1] for e in r if e >= 0]
        assert len(held) + now[3][1] == pages and len(set(held)) == len(held)


def test_pages_of_tables_with_entries_that_are_none():
    """Entries outside the pages are none, wherever they stand; what is out of range is never followed."""
    from paper_2603_09237_amd import binding
    d = binding.PagesDims(4, 2, 3, 10)
    length, table = [3, 6, 0, 2 ** 31 - 3], [[5, 99, -7], [1, 2 ** 31 - 1, 10], [-(2 ** 31), 3, 4], [6, 7, 8]]
    for first in (None, [1, 1, 0, 0]):
        want = books(2, 3, 10, first, length, table, list(range(10)), [8, 3])
        got = step_books(d, first, length, table, list(range(10)), [8, 3], False)
        assert [list(map(list, v)) if i == 1 else list(v) for i, v in enumerate(want)] == got


# ---- one step ----
def setup(dtype, N, H, KV, D, B, window, page, lengths, seed=0, spare=3, pad=0):
    from paper_2603_09237_amd import binding
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    slots = -(-window // page)
    pages = N * slots + spare
    r = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    c = dict(N=N, H=H, KV=KV, D=D, B=B, window=window, page=page, slots=slots, pages=pages, dtype=dtype, pad=pad, q=r(N, H, D), k=r(N, KV, D), v=r(N, KV, D),
             kc=r(pages, page, KV, D), vc=r(pages, page, KV, D), bias=torch.randn(H, B, generator=g) if B else None,
             edges=torch.tensor([j * (j + 3) // 4 for j in range(B)], dtype=torch.int32) if B else None,
             table=torch.randperm(pages, generator=g)[:N * slots].reshape(N, slots).to(torch.int32), length=torch.tensor(lengths, dtype=torch.int32))
    c["dims"] = binding.CacheDims(N, H, KV, D, B, window, page, slots, pages, 1 if dtype == torch.bfloat16 else 0, q_n=H * D + pad, k_n=KV * D + pad,
                                  y_n=H * D + pad)
    return c


def define(c):
    torch = _torch()
    N, H, KV, D, B, W, page, slots, pages = (c[k] for k in ("N", "H", "KV", "D", "B", "window", "page", "slots", "pages"))
    kc, vc = c["kc"].double().clone(), c["vc"].double().clone()
    y, bound = torch.zeros(N, H, D, dtype=torch.float64), torch.zeros(N, H, D, dtype=torch.float64)
    for n in range(N):
        pos = int(c["length"][n]) - 1
        if pos < 0:
            continue
        ks, vs, gaps = [c["k"][n].double()], [c["v"][n].double()], [0]
        for s in range(max(0, pos - W + 1), pos):
            e = int(c["table"][n, (s // page) % slots])
            if 0 <= e < pages:
                ks.append(kc[e, s % page]); vs.append(vc[e, s % page]); gaps.append(pos - s)
        e = int(c["table"][n, (pos // page) % slots])
        if 0 <= e < pages:
            kc[e, pos % page], vc[e, pos % page] = ks[0], vs[0]
        ks, vs = (torch.stack(t, 1).repeat_interleave(H // KV, 0) for t in (ks, vs))
        q = c["q"][n].double()[:, None]
        a = (q * ks).sum(-1) * D ** -0.5
        if B:
            bucket = (torch.tensor(gaps)[:, None] >= c["edges"][1:]).sum(-1)
            a = a + c["bias"].double()[:, bucket]
        p = torch.softmax(a, -1)
        y[n] = (p[..., None] * vs).sum(1)
        e_a = (D + 4) * U * D ** -0.5 * float((q.abs() * ks.abs()).sum(-1).max()) + 4 * U * float(a[torch.isfinite(a)].abs().max())
        bound[n] = (2 * e_a + (2 * len(gaps) + 16) * U) * (p[..., None] * vs.abs()).sum(1)
    return y, bound, kc.to(c["dtype"]), vc.to(c["dtype"])


def launch(c, dev=None):
    from paper_2603_09237_amd import binding
    torch = _torch()
    if dev is None:
        dev = {k: None if c[k] is None else c[k].cuda() for k in ("bias", "edges", "table", "length", "kc", "vc")}
        for k, w in (("q", c["H"]), ("k", c["KV"]), ("v", c["KV"])):
            dev[k] = torch.full((c["N"], w * c["D"] + c["pad"]), 7.0, dtype=c["dtype"], device="cuda")
            dev[k][:, :w * c["D"]] = c[k].reshape(c["N"], -1).cuda()
        dev["y"] = torch.full((c["N"], c["H"] * c["D"] + c["pad"]), 7.0, dtype=c["dtype"], device="cuda")
        dev["ws"] = torch.full((binding.attn_step_workspace_bytes(c["dims"]),), 0xff, dtype=torch.uint8, device="cuda")
    binding.attn_step(c["dims"], dev["q"], dev["k"], dev["v"], dev["bias"], dev["edges"], dev["table"], dev["length"], dev["kc"], dev["vc"], dev["y"],
                      dev["ws"])
    return dev


def check(c):
    torch = _torch()
    y, bound, kc, vc = define(c)
    dev = launch(c)
    got = dev["y"].cpu()
    w = c["H"] * c["D"]
    assert bool((got[:, w:] == 7.0).all())
    got = got[:, :w].reshape(y.shape)
    half = 2.0 ** -8 if c["dtype"] == torch.bfloat16 else U
    err, tol = (got.double() - y).abs(), bound + half * (y.abs() + bound) + 1e-30
    assert bool((err <= tol).all()), (int((err > tol).sum()), float((err / tol).max()))
    assert torch.equal(dev["kc"].cpu(), kc) and torch.equal(dev["vc"].cpu(), vc)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_step_of_the_longest_episode_and_window(kind):
    """Counts whose rounding up passes 2^31: two pages of an episode of 2^31 - 2 steps are there, the newest and one from near its begin."""
    from paper_2603_09237_amd import binding
    torch = _torch()
    dtype, H, D, B, page, slots, window, length = getattr(torch, kind), 2, 8, 3, 4096, 1 << 19, 2 ** 31 - 1, 2 ** 31 - 2
    g = torch.Generator().manual_seed(11)
    r = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    table = torch.full((1, slots), -1, dtype=torch.int32)
    pos = length - 1
    table[0, pos // page % slots], table[0, 5] = 1, 0
    c = dict(N=1, H=H, KV=1, D=D, pad=0, dtype=dtype, q=r(1, H, D), k=r(1, 1, D), v=r(1, 1, D), kc=r(2, page, 1, D), vc=r(2, page, 1, D),
             bias=torch.randn(H, B, generator=g), edges=torch.tensor([0, 10, 5000], dtype=torch.int32), table=table,
             length=torch.tensor([length], dtype=torch.int32), dims=binding.CacheDims(1, H, 1, D, B, window, page, slots, 2, int(kind == "bfloat16")))
    here = pos % page
    gaps = torch.cat([pos - (5 * page + torch.arange(page)), here - torch.arange(here + 1)])
    ks, vs = (torch.cat([t[0], t[1, :here], n]).double()[:, 0] for t, n in ((c["kc"], c["k"]), (c["vc"], c["v"])))
    a = c["q"][0].double() @ ks.T * D ** -0.5 + c["bias"].double()[:, (gaps[:, None] >= c["edges"][1:]).sum(-1)]
    p = torch.softmax(a, -1)
    y, size = p @ vs, p @ vs.abs()
    bound = (2 * ((D + 4) * U * D ** -0.5 * float((c["q"][0].double().abs() @ ks.abs().T).max()) + 4 * U * float(a.abs().max())) + (2 * len(gaps) + 16) * U) * size
    dev = launch(c)
    half = 2.0 ** -8 if kind == "bfloat16" else U
    err = (dev["y"].cpu().double().reshape(H, D) - y).abs()
    assert bool((err <= bound + half * (y.abs() + bound) + 1e-30).all())
    assert torch.equal(dev["kc"].cpu()[1, here], c["k"][0]) and torch.equal(dev["vc"].cpu()[1, here], c["v"][0])


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("N,H,KV,D,B,window,page,lengths,pad", [
    (1, 1, 1, 1, 0, 1, 1, [1], 0), (1, 1, 1, 16, 3, 8, 4, [1], 0), (5, 2, 2, 8, 4, 9, 2, [0, 1, 9, 10, 400], 0),
    (4, 4, 1, 33, 6, 40, 8, [40, 41, 39, -5], 3), (3, 6, 2, 64, 32, 300, 16, [300, 1000, 17], 0), (2, 8, 1, 128, 0, 700, 64, [700, 699], 8),
    (2, 10, 2, 127, 64, 130, 1, [500, 129], 1), (1, 20, 1, 64, 5, 1500, 32, [1499], 0), (3, 3, 1, 40, 17, 97, 32, [97, 98, 5000], 5),
    (1, 8, 8, 64, 8, 4096, 128, [5000], 0)])
def test_step(kind, N, H, KV, D, B, window, page, lengths, pad):
    check(setup(getattr(_torch(), kind), N, H, KV, D, B, window, page, lengths, pad=pad))


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_pages_that_are_none(kind):
    """Steps whose slots hold no page are not seen (nor read), a step without one is not kept."""
    torch = _torch()
    c = setup(getattr(torch, kind), 4, 4, 2, 32, 6, 64, 8, [64, 70, 30, 9], spare=6)
    c["table"][0, 3], c["table"][1, 0], c["table"][2, 0] = -1, c["pages"], 2 ** 31 - 1
    c["table"][1, (69 // 8) % 8], c["table"][3] = -(2 ** 31), -1
    check(c)


def test_values_that_are_not_seen_never_count():
    """Rows of the step's pages behind its window, before its episode's begin or in pages of others may hold anything."""
    torch = _torch()
    for bad in (float("nan"), float("inf")):
        c = setup(torch.bfloat16, 3, 4, 2, 32, 6, 21, 8, [21, 5, 40])
        seen = torch.zeros(c["pages"], 8, dtype=torch.bool)
        for n in range(3):
            for s in range(max(0, int(c["length"][n]) - 21), int(c["length"][n]) - 1):
                seen[int(c["table"][n, (s // 8) % 3]), s % 8] = True
        c["kc"][~seen], c["vc"][~seen] = bad, bad
        y, bound, _, _ = define(c)
        assert bool(torch.isfinite(y).all())
        got = launch(c)["y"].cpu().double().reshape(y.shape)
        assert bool(((got - y).abs() <= bound + 2.0 ** -8 * (y.abs() + bound)).all())


def test_step_repeats_and_replays():
    """Bit for bit again, on another stream, and replayed from a graph with lengths that have moved on."""
    torch = _torch()
    c = setup(torch.bfloat16, 3, 8, 2, 64, 8, 600, 16, [100, 600, 3])
    dev = launch(c)
    want = dev["y"].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        assert torch.equal(launch(c)["y"], want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        launch(c, dev)
    for i in range(4):
        dev["length"] += 7
        dev["q"].normal_()
        launch(c, dev)
        want = dev["y"].clone()
        dev["y"].fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dev["y"], want), i


def test_a_long_cache():
    """Elements beyond 2^31 of the cache: the last pages of 4.3 GB each."""
    torch = _torch()
    N, page, slots = 1, 4096, 1
    pages, KV, D = 2 ** 31 // 4096 // 4 + 1, 4, 2
    from paper_2603_09237_amd import binding
    d = binding.CacheDims(N, 4, KV, D, 0, 4096, page, slots, pages, 0)
    assert pages * page * KV * D > 2 ** 31
    g = torch.Generator().manual_seed(1)
    kc = torch.zeros(pages, page, KV, D, device="cuda")
    vc = torch.zeros_like(kc)
    kc[-1], vc[-1] = torch.randn(page, KV, D, generator=g).cuda(), torch.randn(page, KV, D, generator=g).cuda()
    q, k, v = (torch.randn(1, 4, D, generator=g).cuda() for _ in range(3))
    y, ws = torch.empty_like(q), torch.empty(binding.attn_step_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    table, length = ints([[pages - 1]]), ints([50])
    binding.attn_step(d, q, k, v, None, None, table, length, kc, vc, y, ws)
    ks, vs = torch.cat([kc[-1, :49], k]).double(), torch.cat([vc[-1, :49], v]).double()
    p = torch.softmax((ks * q[0].double()).sum(-1) * D ** -0.5, 0)
    assert float((y[0].double() - (p[..., None] * vs).sum(0)).abs().max()) < 1e-5   # (50 terms of size one, 2^-24 each, some times over)
    assert torch.equal(kc[-1, 49], k[0]) and torch.equal(vc[-1, 49], v[0])
