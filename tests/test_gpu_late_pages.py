"""A cache whose queue of free pages runs dry: pages come late, in the middle of their rows or a round of the slots later, and the rows before hold
what others left.  Against lists that note whose step each row holds: a step sees the steps that were kept, and no row that holds anything else."""
import random

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _torch():
    import torch
    return torch


class Lists:
    """The books of N environments, one after the other, with the step from which on each slot's page is the episode's, and what each row holds."""

    def __init__(self, N, page, slots, pages, unused=()):
        self.N, self.page, self.slots, self.pages = N, page, slots, pages
        self.length, self.table, self.since = [-1 if n in unused else 0 for n in range(N)], [[-1] * slots for _ in range(N)], [[0] * slots for _ in range(N)]
        self.queue, self.state = list(range(pages)), [0, pages]
        self.rows, self.episode, self.slot = {}, [0] * N, [-1] * N

    def step(self, first):
        head, count = self.state
        back, taken = [], 0
        for n in range(self.N):
            if self.length[n] < 0:
                self.slot[n] = -1
                continue
            if first[n]:
                back += [e for e in self.table[n][1:] if e >= 0]
                self.table[n][1:] = [-1] * (self.slots - 1)
                self.length[n], self.episode[n] = 0, self.episode[n] + 1
            p = self.length[n]
            j = p // self.page % self.slots
            if first[n] or self.table[n][j] < 0 or self.since[n][j] > p:
                self.since[n][j] = p
            if self.table[n][j] < 0 and taken < count:
                self.table[n][j] = self.queue[(head + taken) % self.pages]
                taken += 1
            e = self.table[n][j]
            self.slot[n] = -1 if e < 0 else e * self.page + p % self.page
            if e >= 0:
                self.rows[self.slot[n]] = (n, self.episode[n], p)
            self.length[n] = p + 1
        for i, e in enumerate(back):
            self.queue[(head + count + i) % self.pages] = e
        self.state = [(head + taken) % self.pages, count - taken + len(back)]

    def row_of(self, n, s):
        e = self.table[n][s // self.page % self.slots]
        return -1 if e < 0 else e * self.page + s % self.page

    def seen(self, n, window):
        """the steps before the present one that are kept, and those that stand in a page without being kept"""
        p = self.length[n] - 1
        held = [s for s in range(max(0, p - window + 1), p) if self.row_of(n, s) >= 0]
        kept = [s for s in held if self.rows.get(self.row_of(n, s)) == (n, self.episode[n], s)]
        return kept, [s for s in held if s not in kept]


def ints(v):
    return _torch().tensor(v, dtype=_torch().int32, device="cuda")


def begins(rng, N, p):
    return [int(rng.random() < p) for _ in range(N)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("N,page,slots,pages", [(1, 1, 1, 1), (2, 4, 4, 5), (5, 2, 3, 4), (64, 4, 3, 70), (257, 2, 70, 300), (1000, 8, 2, 900)])
def test_books(N, page, slots, pages, in_place):
    from paper_2603_09237_amd import binding
    torch = _torch()
    rng = random.Random(N + pages)
    want, d = Lists(N, page, slots, pages, [n for n in range(N) if rng.random() < 0.05 and N > 2]), binding.PagesDims(N, page, slots, pages)
    names = ("length", "table", "queue", "state", "since")
    for t in range(30):
        now = {k: ints(getattr(want, k)) for k in names}
        out = now if in_place else {k: torch.full_like(v, 77) for k, v in now.items()}
        slot, ws = ints([77] * N), torch.full((binding.pages_workspace_bytes(d),), 0xff, dtype=torch.uint8, device="cuda")
        first = begins(rng, N, 0.1)
        want.step(first)
        binding.cache_pages(d, torch.tensor(first, dtype=torch.uint8, device="cuda"), *(now[k] for k in names[:4]), *(out[k] for k in names[:4]), slot, ws,
                            since_in=now["since"], since=out["since"])
        for k in names:
            assert out[k].cpu().tolist() == getattr(want, k), (t, k)
        assert slot.cpu().tolist() == want.slot, t


def test_since_of_a_step_that_is_still_to_come():
    """A row that a new episode takes over by its length alone: what the last one noted beyond the present step does not hide it."""
    from paper_2603_09237_amd import binding
    torch = _torch()
    d = binding.PagesDims(3, 4, 2, 6)
    length, table, queue, state, since, slot = ints([0, 5, 5]), ints([[0, 1], [2, 3], [4, 5]]), ints([0] * 6), ints([0, 0]), ints([[3, 6], [0, 7], [0, 4]]), ints([0] * 3)
    ws = torch.empty(binding.pages_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    binding.cache_pages(d, None, length, table, queue, state, length, table, queue, state, slot, ws, since_in=since, since=since)
    assert since.cpu().tolist() == [[0, 6], [0, 5], [0, 4]]


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("N,H,KV,D,B,window,page,pages,T,often", [
    (2, 2, 1, 8, 3, 16, 4, 5, 80, 0.03), (5, 4, 2, 33, 6, 24, 8, 7, 90, 0.06), (3, 12, 1, 64, 0, 10, 2, 7, 60, 0.2), (4, 3, 3, 128, 5, 300, 32, 14, 500, 0.015)])
def test_books_and_steps(kind, N, H, KV, D, B, window, page, pages, T, often):
    """Rows that hold no living episode's step are undefined (a row that was read all the same shows)."""
    from paper_2603_09237_amd import binding
    torch = _torch()
    dtype, slots, rng = getattr(torch, kind), -(-window // page), random.Random(N * window)
    two, half = (2.0 ** -17, 2.0 ** -8) if kind == "bfloat16" else (0.0, U)   # probabilities in two parts, the output's rounding
    g = torch.Generator().manual_seed(N)
    lists, d = Lists(N, page, slots, pages), binding.CacheDims(N, H, KV, D, B, window, page, slots, pages, int(kind == "bfloat16"))
    pd = binding.PagesDims(N, page, slots, pages)
    bias = torch.randn(H, B, generator=g) if B else None
    edges = torch.tensor([j * (j + 3) // 4 for j in range(B)], dtype=torch.int32) if B else None
    db, de = (None if t is None else t.cuda() for t in (bias, edges))
    names = ("length", "table", "queue", "state")
    books, since, slot = [ints(getattr(lists, k)) for k in names], torch.full((N, slots), 12345, dtype=torch.int32, device="cuda"), ints([0] * N)
    kc, vc = (torch.full((pages, page, KV, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    y = torch.empty(N, H, D, dtype=dtype, device="cuda")
    ws = torch.full((max(binding.pages_workspace_bytes(pd), binding.attn_step_workspace_bytes(d)),), 0xff, dtype=torch.uint8, device="cuda")
    past, late, look = {}, 0, max(1, T // 40)
    for t in range(T):
        first = [0] * N if t == 0 else begins(rng, N, often)
        q, k, v = (torch.randn(N, h, D, generator=g).to(dtype) for h in (H, KV, KV))
        lists.step(first)
        keep = torch.zeros(pages * page, dtype=torch.bool)
        unkept = []
        for n in range(N):
            past[n, lists.episode[n], lists.length[n] - 1] = (k[n].double(), v[n].double())
            kept, others = lists.seen(n, window)
            unkept += others
            keep[[lists.row_of(n, s) for s in kept]] = True
        late += bool(unkept)
        keep = keep.cuda().reshape(pages, page)
        kc[~keep], vc[~keep] = float("nan"), float("nan")
        binding.cache_pages(pd, torch.tensor(first, dtype=torch.uint8, device="cuda"), *books, *books, slot, ws, since_in=since, since=since)
        binding.attn_step(d, q.cuda(), k.cuda(), v.cuda(), db, de, books[1], books[0], kc, vc, y, ws, since=since)
        assert slot.cpu().tolist() == lists.slot
        if t % look and not unkept:
            continue
        got = y.cpu().double()
        for n in range(N):
            p = lists.length[n] - 1
            steps = [p] + lists.seen(n, window)[0]
            ks, vs = (torch.stack([past[n, lists.episode[n], s][i] for s in steps], 1).repeat_interleave(H // KV, 0) for i in (0, 1))
            qn = q[n].double()[:, None]
            a = (qn * ks).sum(-1) * D ** -0.5
            if B:
                a = a + bias.double()[:, (p - torch.tensor(steps)[:, None] >= edges[1:]).sum(-1)]
            w = torch.softmax(a, -1)
            want = (w[..., None] * vs).sum(1)
            e_a = (D + 4) * U * D ** -0.5 * float((qn.abs() * ks.abs()).sum(-1).max()) + 4 * U * float(a.abs().max())
            bound = (2 * e_a + two + (2 * len(steps) + 16) * U) * (w[..., None] * vs.abs()).sum(1)
            assert bool(((got[n] - want).abs() <= bound + half * (want.abs() + bound) + 1e-30).all()), (t, n)
    assert late >= 5   # (steps at which a page held rows that were not kept)


@pytest.mark.parametrize("kind,tol", [("float32", 3e-5), ("bfloat16", 3e-2)])   # as for the block's segments: chained operators, six roundings to bf16
def test_acting_with_few_pages(kind, tol):
    """The block over a cache of fewer pages than its environments could hold is the block written out in 64 bits, over the steps that were kept."""
    from paper_2603_09237_amd.attention import AttentionBlock
    torch = _torch()
    dtype, N, T, P, width, page, pages = getattr(torch, kind), 6, 90, 4, 24, 4, 13
    block = AttentionBlock(P, width, heads=4, kv_heads=2, head_dim=16, buckets=8, window=20, rank=3, dtype=dtype, seed=3)
    H, KV, hd, D, E = block.H, block.KV, block.hd, block.D, block.E
    g, rng = torch.Generator().manual_seed(4), random.Random(5)
    x, h = (torch.randn(T, N, width, generator=g).to(dtype) for _ in range(2))
    index = torch.randint(0, P, (N,), generator=g).to(torch.int32)
    lists, cache = Lists(N, page, 5, pages), block.new_cache(N, page=page, pages=pages)
    cache.k.fill_(float("nan")), cache.v.fill_(float("nan"))
    p, idx = {k: v.double().cpu() for k, v in block.p.items()}, index.long()

    def project(name, v):
        return torch.matmul((p[name + ".w0"] + p[name + ".A"] @ p[name + ".B"])[idx], v[..., None])[..., 0] + p[name + ".bias"]

    proj = project("in", h.double())
    q, gate = proj[..., :D].reshape(T, N, H, hd), proj[..., D + 2 * E:]
    k, v = (proj[..., D + i * E:D + (i + 1) * E].reshape(T, N, KV, hd).repeat_interleave(H // KV, 2) for i in (0, 1))
    begin, late = [0] * N, 0
    rms = lambda t: t * (t.square().mean(-1, keepdim=True) + block.eps) ** -0.5  # noqa: E731
    for t in range(T):
        first = [0] * N if t == 0 else begins(rng, N, 0.06)
        lists.step(first)
        yt, nt = block.act(x[t].cuda(), h[t].cuda(), index.cuda(), torch.tensor(first, dtype=torch.uint8, device="cuda"), cache)
        att = torch.zeros(N, H, hd, dtype=torch.float64)
        for n in range(N):
            begin[n] = t if first[n] else begin[n]
            kept, others = lists.seen(n, block.window)
            late += bool(others)
            at = torch.tensor([t] + [begin[n] + s for s in kept])
            a = (q[t, n] * k[at, n]).sum(-1) * hd ** -0.5 + p["bias"][:, (t - at[:, None] >= block.edges.cpu()[1:]).sum(-1)].T
            att[n] = (torch.softmax(a, 0)[..., None] * v[at, n]).sum(0)
        y = x[t].double() + p["scale"] * torch.sigmoid(gate[t]) * rms(project("out", att.reshape(N, D))) * p["w_post"]
        for got, want in ((yt, y), (nt, rms(y) * p["w_pre"])):
            assert float((got.double().cpu() - want).abs().max()) <= tol * float(want.abs().max()), t
        assert cache.table.cpu().tolist() == lists.table and cache.state.cpu().tolist() == lists.state
    assert late >= 5
