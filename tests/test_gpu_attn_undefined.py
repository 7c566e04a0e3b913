"""Which buckets of the bias an undefined key, query or gradient reaches in a backward pass of attention: those of the distances that the rows which
see it see, and no other."""
import pytest
from test_gpu_attn import _torch, make, run

pytestmark = pytest.mark.gpu

EDGES = [0, 1, 2, 5, 5, 9, 20, 21]   # (bucket 3 holds no distance)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("T,S,N,H,KV,D", [(50, 60, 2, 2, 2, 16), (50, 50, 1, 4, 1, 32), (50, 51, 1, 2, 1, 128), (1100, 1100, 1, 1, 1, 16)])
def test_undefined_key_reaches_the_buckets_of_its_rows(kind, what, T, S, N, H, KV, D):
    """Environment 0: episodes begin at 21 steps and at one from the end: the rows between see distances of up to 19, the last row itself."""
    torch = _torch()
    c = make(getattr(torch, kind), T, S, N, H, KV, D, len(EDGES), S, 0.0)
    c["edges"] = torch.tensor(EDGES, dtype=torch.int32)
    c["first"] = torch.zeros(S, N, dtype=torch.uint8)
    c["first"][S - 21, 0] = c["first"][S - 1, 0] = 1
    clean = run(c)
    assert bool(torch.isfinite(clean["bias"]).all())
    for at, head, reached in ((S - 12, 0, [0, 1, 2, 4, 5]), (S - 1, KV - 1, [0])):   # (the rows that see it see from their episode's begin on)
        d = dict(c, k=c["k"].clone())
        d["k"][at, 0, head, D // 2] = what
        got = run(d)["bias"]
        hit = torch.zeros(H, len(EDGES), dtype=torch.bool)
        hit[head * (H // KV):(head + 1) * (H // KV), reached] = True
        assert torch.equal(torch.isfinite(got), ~hit), at
        assert torch.equal(got[~hit], clean["bias"][~hit]), at


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("name", ["q", "dy"])
def test_undefined_row_reaches_its_own_buckets(kind, name):
    torch = _torch()
    c = make(getattr(torch, kind), 70, 90, 1, 4, 2, 24, len(EDGES), 6, 0.0)   # a window of six: distances of up to 5
    c["edges"] = torch.tensor(EDGES, dtype=torch.int32)
    clean = run(c)
    d = dict(c, **{name: c[name].clone()})
    d[name][33, 0, 2, 1] = float("nan")
    got = run(d)["bias"]
    hit = torch.zeros(4, len(EDGES), dtype=torch.bool)
    hit[2, [0, 1, 2, 4]] = True
    assert torch.equal(torch.isfinite(got), ~hit)
    assert torch.equal(got[~hit], clean["bias"][~hit])
