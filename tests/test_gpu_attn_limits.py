"""Attention of as many environments as are served: launches of almost 2^32 threads."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,heads,buckets", [("bfloat16", 1, 1), ("float32", 3, 5)])
def test_the_most_environments_with_the_gradient_of_the_bias(kind, heads, buckets):
    """2^24 - 1 rows of one step, each a workgroup, and the sums of the bias's gradient beside them.  A step that sees itself only is its value, and
    hands its gradient on to it; its score has no gradient.

    Tolerances of y and dv, to the last bit: the probability is exp(a - L) of two scores of which each is off by e_a = 5 2^-24 |q k| (one product of
    three parts each, five additions) and 4 2^-24 (|q k| + |bias|) (its scaling, the bias's, their sum, the difference), so it is off by 2 e_a of itself
    and by 14 2^-24 (exponential 4, logarithm 4, quotient and products 6); then the rounding to the output's type."""
    import torch
    from paper_2603_09237_amd import binding
    N, dtype = (2 ** 24 - 1) // heads, getattr(torch, kind)
    assert N * heads == 2 ** 24 - 1
    d = binding.AttnDims(1, 1, N, heads, heads, 1, buckets, 1, int(kind == "bfloat16"))
    q, k, v, dy = (torch.randn(N, heads, device="cuda").to(dtype) for _ in range(4))
    bias, edges = torch.randn(heads, buckets, device="cuda"), torch.arange(buckets, dtype=torch.int32, device="cuda")
    y, dq, dk, dv = (torch.full_like(q, float("nan")) for _ in range(4))
    dbias = torch.full_like(bias, float("nan"))
    saved = torch.empty(binding.attn_saved_bytes(d), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(binding.attn_workspace_bytes(d), binding.attn_workspace_bytes(d, True)), dtype=torch.uint8, device="cuda")
    binding.attn_fwd(d, q, k, v, bias, edges, None, y, saved, ws)
    binding.attn_bwd(d, q, k, v, bias, edges, None, y, saved, dy, dq, dk, dv, dbias, ws)
    torch.cuda.synchronize()
    u, half = 2.0 ** -24, 2.0 ** -8 if kind == "bfloat16" else 2.0 ** -24
    qk = (q.double() * k.double()).abs()
    off = 2 * (5 * u * qk + 4 * u * (qk + bias[:, 0].double().abs())) + 14 * u
    for got, want in ((y, v), (dv, dy)):
        assert bool(((got.double() - want.double()).abs() <= (off + half * (1 + off)) * want.double().abs()).all())
    for got in (dq, dk, dbias):
        assert bool((got == 0).all())
