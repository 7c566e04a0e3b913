"""Operators of a preference-conditioned policy whose memory is attention over its own past, as cases with sizes, inputs, least work and
plain forms.  Four families, each through the package's public entry points (`binding`):

  attn     attention of a rollout segment's steps over the past steps of their own episode, with a learned bias by buckets of the
           distance in time: forward, and a training pass (forward and backward to q, k, v and the bias).
  step     the same for one new step of every environment, over a paged cache of keys and values that the step is added to.
  pages    the cache's bookkeeping for one step: episodes that begin give their pages back, environments that need a page get one.
  norm     what stands between two blocks: norm of a block's output, gate, residual scale, sum, norm for the next block; forward, and a
           training pass.

Sizes: environments, rollout lengths and widths of `configs.CONFIGS` (widths 256 and 512, 32 to 64 steps, thousands of environments),
generic ones for longer histories.
"""
from __future__ import annotations

import math

import torch

own = False

_DEV = "cuda:0"
_EPS = 1e-6


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _esize(case):
    return 2 if case["dtype"] == "bf16" else 4


# ---------------------------------------------------------------------------------------------------- cases
def _case(defaults, kind, name, c):
    d = dict(defaults, kind=kind)
    d.update(c)
    if name:
        d["name"] = name
    return d


def _attn(kind, name=None, **c):
    return _case(dict(T=1, past=0, N=1, heads=1, kv_heads=1, head_dim=64, buckets=0, window=1, p_first=0.0, dtype="bf16"), kind, name, c)


def _step(name=None, **c):
    return _case(dict(N=1, heads=1, kv_heads=1, head_dim=64, buckets=0, window=1, page=32, ragged=True, dtype="bf16"), "step", name, c)


def _pages(name=None, **c):
    return _case(dict(N=1, page=32, slots=1, p_first=0.01, tight=False), "pages", name, c)


def _norm(kind, name=None, **c):
    return _case(dict(rows=1, width=1, gate=True, dtype="bf16"), kind, name, c)


def listed():
    return [
        # a rollout segment of 64 steps evaluated at once, with the 64 steps before it, four heads to a head of keys
        _attn("attn_fwd", "attend-segment-bf16", T=64, past=64, N=1024, heads=8, kv_heads=2, buckets=32, window=96, p_first=0.005),
        # two long recorded histories in single precision, small heads, no bias
        _attn("attn_fwd", "attend-history-fp32", T=4099, N=2, heads=4, kv_heads=4, head_dim=32, window=4099, dtype="fp32"),
        # update on a minibatch of rollout segments
        _attn("attn_train", "attend-update-bf16", T=64, past=64, N=512, heads=8, kv_heads=8, buckets=32, window=128, p_first=0.005),
        # update on long histories of a few environments, large heads
        _attn("attn_train", "attend-histories-bf16", T=2048, N=8, heads=8, kv_heads=2, head_dim=128, buckets=32, window=2048, p_first=0.0005),
        # update of a small policy in single precision, sizes that are multiples of nothing
        _attn("attn_train", "attend-ragged-fp32", T=67, past=34, N=129, heads=6, kv_heads=3, head_dim=40, buckets=17, window=80, p_first=0.01,
              dtype="fp32"),
        # one environment with a long episode behind it asks for its next action: latency counts
        _step("decide-one-bf16", N=1, heads=8, kv_heads=2, buckets=32, window=8192, ragged=False),
        # a time step of a rollout, episodes of all ages
        _step("decide-rollout-bf16", N=1024, heads=8, kv_heads=2, buckets=32, window=1024),
        # a few environments in single precision, sizes that are multiples of nothing
        _step("decide-few-fp32", N=33, heads=6, kv_heads=3, head_dim=40, buckets=17, window=384, page=16, dtype="fp32"),
        # bookkeeping of a rollout's step
        _pages("pages-rollout", N=4096, slots=32),
        # the largest rollout, short pages, few of them free
        _pages("pages-tight", N=16384, page=16, slots=64, p_first=0.005, tight=True),
        # an update's rows between two blocks of 512
        _norm("norm_train", "norm-update-bf16", rows=65536, width=512),
        # an acting call's rows between two blocks of a small policy, no gate
        _norm("norm_fwd", "norm-act-fp32", rows=257, width=584, gate=False, dtype="fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    kv = rng.choice([1, 1, 2, 2, 3, 4, 8])
    return dict(kv_heads=kv, heads=kv * rng.choice([1, 1, 2, 3, 4, 8] if kv < 4 else [1, 1, 2, 4]))


def draw(rng):
    kind = rng.choice(["attn_fwd", "attn_fwd", "attn_train", "attn_train", "attn_train", "step", "step", "step", "pages", "norm_fwd", "norm_train"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind == "pages":
        c = _pages(N=_log(rng, 1, 32768), page=1 << rng.randint(0, 7), slots=_log(rng, 1, 256), p_first=rng.choice([0.0, 0.005, 0.05]),
                   tight=rng.random() < 0.4)
        while c["N"] * c["slots"] > 16384 * 64:
            c["slots"] = max(1, c["slots"] // 2)
        return c
    if kind.startswith("norm"):
        c = _norm(kind, rows=_log(rng, 1, 65536), width=_log(rng, 8, 4096), gate=rng.random() < 0.6, dtype=dtype)
        if rng.random() < 0.5:
            c["width"] = max(8, c["width"] // 8 * 8)
        while c["rows"] * c["width"] * _esize(c) > 65536 * 512 * 2:
            c["rows"] //= 2
        return c
    head_dim = rng.choice([64, 64, 128, 32, 8 * rng.randint(1, 16), rng.randint(4, 127)])
    buckets = rng.choice([0, 32, 32, rng.randint(1, 64)])
    if kind == "step":
        c = _step(N=_log(rng, 1, 4096), **_heads(rng), head_dim=head_dim, buckets=buckets, window=_log(rng, 4, 16384), page=1 << rng.randint(2, 7),
                  ragged=rng.random() < 0.8, dtype=dtype)
        while c["N"] * c["window"] * c["kv_heads"] * head_dim * _esize(c) > 1024 * 1024 * 2 * 64 * 2:
            c["N" if c["N"] > 1 and rng.random() < 0.5 or c["window"] < 8 else "window"] //= 2
        return c
    c = _attn(kind, T=_log(rng, 1, 4096), past=rng.choice([0, 0, _log(rng, 1, 512)]), N=_log(rng, 1, 2048), **_heads(rng), head_dim=head_dim,
              buckets=buckets, p_first=rng.choice([0.0, 0.0, 0.005, 0.05]), dtype=dtype)
    most = 8 * 8 * 2048 * 2048 * 128 // (8 if dtype == "fp32" else 2)
    while c["N"] * c["heads"] * c["T"] * (c["T"] + c["past"]) * max(head_dim, 32) > most:
        c["N" if c["N"] > 1 and rng.random() < 0.6 or c["T"] < 64 else "T"] //= 2
        c["N"], c["T"] = max(1, c["N"]), max(1, c["T"])
    S = c["T"] + c["past"]
    c["window"] = S if rng.random() < 0.5 else _log(rng, 1, S)
    return c


# ---------------------------------------------------------------------------------------------------- least work
def _pairs(case):
    """Pairs of a query and a key that it sees, of one environment and head: the key at a distance of d where no episode begins between."""
    T, past, W, stay = case["T"], case["past"], case["window"], 1.0 - case["p_first"]
    total = 0.0
    for t in range(T):
        n = min(past + t + 1, W)
        total += n if stay == 1.0 else (1.0 - stay ** n) / (1.0 - stay)
    return total


def work(case):
    k = case["kind"]
    if k == "pages":  # lengths and flags, the entry in use of every table, and the tables as they go into other buffers
        return {"bytes": case["N"] * (17 + 8 * case["slots"]) + 8 * case["N"] * case["slots"], "flops": 0.0}
    e = _esize(case)
    if k.startswith("norm"):
        M, D = case["rows"], case["width"]
        g = 1 if case["gate"] else 0
        fwd = e * M * D * (4 + g)
        if k == "norm_fwd":
            return {"bytes": fwd + 12 * D, "flops": 12.0 * M * D}
        return {"bytes": fwd + e * M * D * (4 + g) + 24 * D, "flops": 40.0 * M * D}
    N, H, KV, D = (case[n] for n in ("N", "heads", "kv_heads", "head_dim"))
    if k == "step":
        keys = N * (case["window"] / 2.0 if case["ragged"] else case["window"])
        return {"bytes": 2 * e * keys * KV * D + 2 * e * N * (H + 2 * KV) * D, "flops": 4.0 * keys * H * D}
    T, S = case["T"], case["T"] + case["past"]
    fwd = {"bytes": e * N * D * (2 * T * H + 2 * S * KV), "flops": 4.0 * D * N * H * _pairs(case)}
    if k == "attn_fwd":
        return fwd
    return {"bytes": fwd["bytes"] + e * N * D * (2 * T * H + 2 * S * KV), "flops": 3.5 * fwd["flops"]}


# ---------------------------------------------------------------------------------------------------- inputs
def _edges(buckets, reach):
    """Distances at which buckets begin: one by one for the first half, then ever wider up to `reach`."""
    half = max(1, buckets // 2)
    edges = list(range(half))
    for j in range(half, buckets):
        edges.append(max(edges[-1] + 1, int(half * (max(reach, half + 1) / half) ** ((j - half) / (buckets - half)))))
    return edges


def prepare(case, seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(int(seed))

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, device=_DEV, generator=g) * scale).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, device=_DEV, generator=g)

    s = {"case": dict(case)}
    k = case["kind"]
    if k == "pages":
        return _prepare_pages(s, uniform, g)
    dt = _dt(case)
    if k.startswith("norm"):
        M, D = case["rows"], case["width"]
        s.update(x=normal(M, D, scale=2.0, dtype=dt), u=normal(M, D, dtype=dt), gate=normal(M, D, dtype=dt) if case["gate"] else None,
                 scale=0.1 + 0.1 * uniform(D), w_post=1.0 + normal(D, scale=0.2), w_pre=1.0 + normal(D, scale=0.2))
        s.update(y=torch.empty(M, D, dtype=dt, device=_DEV), h=torch.empty(M, D, dtype=dt, device=_DEV))
        if k == "norm_train":
            s.update(dy=normal(M, D, dtype=dt), dh=normal(M, D, dtype=dt), dx=torch.empty(M, D, dtype=dt, device=_DEV),
                     du=torch.empty(M, D, dtype=dt, device=_DEV), dgate=torch.empty(M, D, dtype=dt, device=_DEV) if case["gate"] else None,
                     dscale=torch.empty(D, device=_DEV), dw_post=torch.empty(D, device=_DEV), dw_pre=torch.empty(D, device=_DEV))
        return s
    N, H, KV, D, B, W = (case[n] for n in ("N", "heads", "kv_heads", "head_dim", "buckets", "window"))
    s["bias"] = normal(H, B, scale=0.5) if B else None
    s["edges"] = torch.tensor(_edges(B, min(W, 256)), dtype=torch.int32, device=_DEV) if B else None
    if k == "step":
        page = case["page"]
        slots = -(-W // page)
        pages = N * slots
        # how many steps of its episode an environment holds, this one among them; beyond the window the oldest pages are used again
        length = torch.full((N,), W, dtype=torch.int32, device=_DEV)
        if case["ragged"]:
            length = (1 + uniform(N) * (W - 1)).round().to(torch.int32)
            length[uniform(N) < 0.03] += 2 * W
            length[uniform(N) < 0.03] = 0  # (rows of a batch that no environment uses)
        s.update(length=length, table=torch.randperm(pages, device=_DEV, generator=g).to(torch.int32).reshape(N, slots))
        s.update(q=normal(N, H, D, dtype=dt), k=normal(N, KV, D, dtype=dt), v=normal(N, KV, D, dtype=dt), y=torch.empty(N, H, D, dtype=dt, device=_DEV))
        s.update(k_cache=normal(pages, page, KV, D, dtype=dt), v_cache=normal(pages, page, KV, D, dtype=dt))
        return s
    T, S = case["T"], case["T"] + case["past"]
    s.update(q=normal(T, N, H, D, dtype=dt), k=normal(S, N, KV, D, dtype=dt), v=normal(S, N, KV, D, dtype=dt), y=torch.empty(T, N, H, D, dtype=dt, device=_DEV))
    s["first"] = (uniform(S, N) < case["p_first"]).to(torch.uint8) if case["p_first"] > 0 else None
    if k == "attn_train":
        s.update(dy=normal(T, N, H, D, dtype=dt), dbias=torch.empty(H, B, device=_DEV) if B else None)
        s.update({"d" + n: torch.empty_like(s[n]) for n in ("q", "k", "v")})
    return s


def _prepare_pages(s, uniform, g):
    c = s["case"]
    N, page, slots = c["N"], c["page"], c["slots"]
    pages = N * slots + 7
    length = (uniform(N) * (1.25 * page * slots)).to(torch.int32)  # some have gone round their pages already
    length[uniform(N) < 0.01] = -1                                  # rows of the batch that no environment uses
    used = ((length.clamp(min=0) + page - 1) // page).clamp(max=slots)
    held = torch.arange(slots, device=_DEV)[None, :] < used[:, None]
    order = torch.randperm(pages, device=_DEV, generator=g).to(torch.int32)
    table = torch.full((N, slots), -1, dtype=torch.int32, device=_DEV)
    n = int(held.sum())
    table[held] = order[:n]
    head, count = int(uniform(1) * pages), pages - n
    queue = torch.full((pages,), -1, dtype=torch.int32, device=_DEV)
    if c["tight"]:
        count = min(count, N // 64)
    queue[(head + torch.arange(count, device=_DEV)) % pages] = order[n:n + count]
    s.update(first=(uniform(N) < c["p_first"]).to(torch.uint8), length_in=length, table_in=table, queue_in=queue,
             state_in=torch.tensor([head, count], dtype=torch.int32, device=_DEV))
    s.update({o: torch.empty_like(s[o + "_in"]) for o in ("length", "table", "queue", "state")})
    s["slot"] = torch.empty(N, dtype=torch.int32, device=_DEV)
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


_PAGES_OUT = ("length", "table", "queue", "state", "slot")


def _run_own(s):
    from paper_2603_09237_amd import binding
    c = s["case"]
    k = c["kind"]
    plan = s.get("plan")  # dimensions, workspace and what the backward needs, which a program makes once

    def buffer(n):
        return torch.empty(n, dtype=torch.uint8, device=_DEV)

    if k == "pages":
        if plan is None:
            d = binding.PagesDims(N=c["N"], page=c["page"], slots=c["slots"], pages=s["queue"].numel())
            plan = s["plan"] = (d, buffer(binding.pages_workspace_bytes(d)))
        d, ws = plan
        binding.cache_pages(d, s["first"], s["length_in"], s["table_in"], s["queue_in"], s["state_in"], s["length"], s["table"], s["queue"],
                            s["state"], s["slot"], ws)
        return {n: s[n] for n in _PAGES_OUT}
    e = 1 if c["dtype"] == "bf16" else 0
    if k.startswith("norm"):
        if plan is None:
            d = binding.NormDims(rows=c["rows"], width=c["width"], dtype=e, eps=_EPS)
            plan = s["plan"] = (d, buffer(binding.norm_workspace_bytes(d) if k == "norm_train" else 0))
        d, ws = plan
        binding.norm_fwd(d, s["x"], s["u"], s["gate"], s["scale"], s["w_post"], s["w_pre"], s["y"], s["h"])
        if k == "norm_fwd":
            return {"y": s["y"], "h": s["h"]}
        binding.norm_bwd(d, s["x"], s["u"], s["gate"], s["scale"], s["w_post"], s["w_pre"], s["dy"], s["dh"], s["dx"], s["du"], s["dgate"],
                         s["dscale"], s["dw_post"], s["dw_pre"], ws)
        return {n: s[n] for n in ("y", "h", "dx", "du", "dscale", "dw_post", "dw_pre") + (("dgate",) if c["gate"] else ())}
    sizes = dict(N=c["N"], heads=c["heads"], kv_heads=c["kv_heads"], head_dim=c["head_dim"], buckets=c["buckets"], window=c["window"], dtype=e)
    if k == "step":
        if plan is None:
            d = binding.CacheDims(page=c["page"], slots=s["table"].shape[1], pages=s["k_cache"].shape[0], **sizes)
            plan = s["plan"] = (d, buffer(binding.attn_step_workspace_bytes(d)))
        d, ws = plan
        binding.attn_step(d, s["q"], s["k"], s["v"], s["bias"], s["edges"], s["table"], s["length"], s["k_cache"], s["v_cache"], s["y"], ws)
        return {n: s[n] for n in ("y", "k_cache", "v_cache")}
    train = k == "attn_train"
    if plan is None:
        d = binding.AttnDims(T=c["T"], S=c["T"] + c["past"], **sizes)
        n = max(binding.attn_workspace_bytes(d), binding.attn_workspace_bytes(d, True) if train else 0)
        plan = s["plan"] = (d, buffer(n), buffer(binding.attn_saved_bytes(d)) if train else None)
    d, ws, saved = plan
    binding.attn_fwd(d, s["q"], s["k"], s["v"], s["bias"], s["edges"], s["first"], s["y"], saved, ws)
    if not train:
        return s["y"]
    binding.attn_bwd(d, s["q"], s["k"], s["v"], s["bias"], s["edges"], s["first"], s["y"], saved, s["dy"], s["dq"], s["dk"], s["dv"], s["dbias"], ws)
    return {n: s[n] for n in ("y", "dq", "dk", "dv") + (("dbias",) if c["buckets"] else ())}


def _run_plain(s):
    c = s["case"]
    k = c["kind"]
    if k == "pages":
        return _plain_pages(s)
    dt = _dt(c)
    if k == "norm_fwd":
        y, h = _plain_norm(s["x"].float(), s["u"].float(), s["gate"].float() if c["gate"] else None, s["scale"], s["w_post"], s["w_pre"])
        return {"y": y.to(dt), "h": h.to(dt)}
    if k == "norm_train":
        names = ["x", "u", "scale", "w_post", "w_pre"] + (["gate"] if c["gate"] else [])
        ins = {n: s[n].float().detach().requires_grad_() for n in names}
        y, h = _plain_norm(ins["x"], ins["u"], ins.get("gate"), ins["scale"], ins["w_post"], ins["w_pre"])
        got = torch.autograd.grad([y, h], list(ins.values()), [s["dy"].float(), s["dh"].float()])
        out = {"y": y.detach().to(dt), "h": h.detach().to(dt)}
        out.update({"d" + n: v.to(s[n].dtype) for n, v in zip(names, got)})
        return out
    if k == "step":
        return _plain_step(s, dt)
    if k == "attn_fwd":
        return _plain_attn(c, s["q"].float(), s["k"].float(), s["v"].float(), s["bias"], s["edges"], s["first"]).to(dt)
    names = ["q", "k", "v"] + (["bias"] if c["buckets"] else [])
    ins = [s[n].float().detach().requires_grad_() for n in names]
    y = _plain_attn(c, *ins[:3], ins[3] if c["buckets"] else None, s["edges"], s["first"])
    got = torch.autograd.grad(y, ins, s["dy"].float())
    return dict({"y": y.detach().to(dt)}, **{"d" + n: v.to(s[n].dtype) for n, v in zip(names, got)})


def _plain_norm(x, u, gate, scale, w_post, w_pre):
    n = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + _EPS) * w_post
    if gate is not None:
        n = n / (1 + torch.exp(-gate))
    y = x + scale * n
    return y, y * torch.rsqrt((y * y).mean(-1, keepdim=True) + _EPS) * w_pre


def _plain_attn(c, q, k, v, bias, edges, first):
    """Scores of all steps with all steps, the ones that are not seen taken out, a softmax, a product."""
    T, N, H, D = q.shape
    S, KV = k.shape[0], k.shape[2]
    q, k, v = (t.permute(1, 2, 0, 3) for t in (q, k, v))  # [N, heads, time, D]
    if H > KV:
        k, v = (t[:, :, None].expand(N, KV, H // KV, S, D).reshape(N, H, S, D) for t in (k, v))
    at = torch.arange(S - T, S, device=_DEV)
    gap = at[:, None] - torch.arange(S, device=_DEV)[None, :]
    seen = (gap >= 0) & (gap < c["window"])
    if first is not None:
        episode = first.t().to(torch.int32).cumsum(1, dtype=torch.int32)  # [N, S]
        seen = (seen & (episode[:, at, None] == episode[:, None, :]))[:, None]
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * D ** -0.5
    if bias is not None:
        bucket = (torch.bucketize(gap.clamp(min=0), edges.long(), right=True) - 1).clamp(min=0)
        score = score + bias[:, bucket]
    score = torch.where(seen, score, float("-inf"))
    p = torch.exp(score - score.amax(-1, keepdim=True).detach())
    y = torch.matmul(p, v.contiguous()) / p.sum(-1, keepdim=True)
    return y.permute(2, 0, 1, 3).contiguous()


def _plain_step(s, dt):
    c = s["case"]
    N, H, KV, D, W, page = (c[n] for n in ("N", "heads", "kv_heads", "head_dim", "window", "page"))
    slots = s["table"].shape[1]
    at = s["length"].long() - 1
    live = at >= 0
    env = torch.arange(N, device=_DEV)
    now = s["table"].long()[env, (at.clamp(min=0) // page) % slots]
    keep = env[live]
    s["k_cache"][now[keep], at[keep] % page] = s["k"][keep]
    s["v_cache"][now[keep], at[keep] % page] = s["v"][keep]
    gap = torch.arange(W, device=_DEV)
    where = at[:, None] - gap  # [N, W] steps, newest first
    seen = where >= 0
    where = where.clamp(min=0)
    rows = s["table"].long()[env[:, None], (where // page) % slots] * page + where % page
    k, v = (s[n].reshape(-1, KV, D)[rows].float().permute(0, 2, 1, 3) for n in ("k_cache", "v_cache"))  # [N, KV, W, D]
    score = torch.matmul(s["q"].float().reshape(N, KV, H // KV, D), k.transpose(2, 3).contiguous()) * D ** -0.5
    if s["bias"] is not None:
        bucket = (torch.bucketize(gap, s["edges"].long(), right=True) - 1).clamp(min=0)
        score = score + s["bias"][:, bucket].reshape(KV, H // KV, W)
    score = torch.where((seen | ~live[:, None])[:, None, None, :], score, float("-inf"))
    p = torch.exp(score - score.amax(-1, keepdim=True))
    y = torch.matmul(p, v.contiguous()) / p.sum(-1, keepdim=True)
    y = torch.where(live[:, None, None, None], y, 0.0)
    return {"y": y.reshape(N, H, D).to(dt), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_pages(s):
    c = s["case"]
    N, page, slots = c["N"], c["page"], c["slots"]
    pages = s["queue"].numel()
    live = s["length_in"] >= 0
    begins = live & (s["first"] != 0)
    at = torch.where(begins, 0, s["length_in"]).long()
    table, env = s["table_in"].clone(), torch.arange(N, device=_DEV)
    # pages that go back: those of episodes that begin, but for the first, which serves again
    gives = begins[:, None] & (table >= 0) & (torch.arange(slots, device=_DEV) > 0)
    given = table[gives]
    table[gives] = -1
    column = (at.clamp(min=0) // page) % slots
    needs = live & (table[env, column] < 0)
    rank = needs.to(torch.int64).cumsum(0) - 1
    head, count = s["state_in"][0].long(), s["state_in"][1].long()
    gets = needs & (rank < count)
    entry = torch.where(gets, s["queue_in"][(head + rank.clamp(min=0)) % pages], table[env, column])
    table[env, column] = entry
    taken = gets.sum()
    queue = s["queue_in"].clone()
    queue[(head + count + torch.arange(given.numel(), device=_DEV)) % pages] = given
    slot = torch.where(live & (entry >= 0), entry * page + (at % page).to(torch.int32), -1)
    length = torch.where(live, at + 1, s["length_in"].long()).to(torch.int32)
    state = torch.stack([(head + taken) % pages, count - taken + given.numel()]).to(torch.int32)
    return {"length": length, "table": table, "queue": queue, "state": state, "slot": slot}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    k = case["kind"]
    if k == "pages":
        return _exact_pages(s)
    if k.startswith("norm"):
        return _exact_norm(s)
    if k == "step":
        return _exact_step(s)
    return _exact_attn(s)


def _exact_norm(s):
    c = s["case"]
    x, u, a, wo, wi = (s[n].double() for n in ("x", "u", "scale", "w_post", "w_pre"))
    sig = torch.sigmoid(s["gate"].double()) if c["gate"] else torch.ones_like(x)
    D = c["width"]
    p = (u.square().sum(1, keepdim=True) / D + _EPS) ** -0.5
    n = u * p * wo
    y = x + a * sig * n
    r = (y.square().sum(1, keepdim=True) / D + _EPS) ** -0.5
    out = {"y": y, "h": y * r * wi}
    if c["kind"] == "norm_fwd":
        return out
    dh = s["dh"].double()
    out["dw_pre"] = (dh * y * r).sum(0)
    dh = dh * wi
    dy = s["dy"].double() + r * dh - y * r ** 3 * (dh * y).sum(1, keepdim=True) / D
    out["dx"] = dy
    out["dscale"] = (dy * sig * n).sum(0)
    if c["gate"]:
        out["dgate"] = dy * a * n * sig * (1 - sig)
    dn = dy * a * sig
    out["dw_post"] = (dn * u * p).sum(0)
    dn = dn * wo
    out["du"] = p * dn - u * p ** 3 * (dn * u).sum(1, keepdim=True) / D
    order = ("y", "h", "dx", "du", "dscale", "dw_post", "dw_pre") + (("dgate",) if c["gate"] else ())
    return {n: out[n] for n in order}


def _exact_attn(s):
    """Environment by environment; gradients from the formulas."""
    c = s["case"]
    T, N, H, KV, D, B = (c[n] for n in ("T", "N", "heads", "kv_heads", "head_dim", "buckets"))
    S = T + c["past"]
    train = c["kind"] == "attn_train"
    gap = (torch.arange(T, device=_DEV) + c["past"])[:, None] - torch.arange(S, device=_DEV)
    near = (gap >= 0) & (gap < c["window"])
    if B:
        bucket = torch.zeros_like(gap)
        for j, e in enumerate(s["edges"].tolist()):
            bucket[gap >= e] = j
        shift = s["bias"].double()[:, bucket]  # [H, T, S]
        dbias = torch.zeros(H, B, dtype=torch.float64, device=_DEV)
    y = torch.empty(T, N, H, D, dtype=torch.float64, device=_DEV)
    grads = {n: torch.zeros(*s[n].shape, dtype=torch.float64, device=_DEV) for n in ("q", "k", "v")} if train else {}
    share = H // KV
    for n in range(N):
        q = s["q"][:, n].double().transpose(0, 1)  # [H, T, D]
        k, v = (s[m][:, n].double().transpose(0, 1).repeat_interleave(share, 0) for m in ("k", "v"))
        see = near
        if s["first"] is not None:
            number = s["first"][:, n].long().cumsum(0)
            see = near & (number[S - T:, None] == number[None])
        a = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
        if B:
            a = a + shift
        a = a.masked_fill(~see, -math.inf)
        p = torch.softmax(a, -1)
        o = torch.bmm(p, v)
        y[:, n] = o.transpose(0, 1)
        if not train:
            continue
        do = s["dy"][:, n].double().transpose(0, 1).contiguous()
        da = p * (torch.bmm(do, v.transpose(1, 2).contiguous()) - (do * o).sum(-1, keepdim=True))
        if B:
            dbias.index_add_(1, bucket.reshape(-1), da.reshape(H, -1))
        grads["q"][:, n] = (torch.bmm(da, k) / math.sqrt(D)).transpose(0, 1)
        dk = torch.bmm(da.transpose(1, 2).contiguous(), q.contiguous()) / math.sqrt(D)
        dv = torch.bmm(p.transpose(1, 2).contiguous(), do)
        for m, t in (("k", dk), ("v", dv)):
            grads[m][:, n] = t.reshape(KV, share, S, D).sum(1).transpose(0, 1)
    if not train:
        return y
    out = {"y": y, "dq": grads["q"], "dk": grads["k"], "dv": grads["v"]}
    if B:
        out["dbias"] = dbias
    return out


def _exact_step(s):
    c = s["case"]
    N, H, KV, D, W, page = (c[n] for n in ("N", "heads", "kv_heads", "head_dim", "window", "page"))
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    y = torch.zeros(N, H, D, dtype=torch.float64, device=_DEV)
    lengths, slots = s["length"].tolist(), s["table"].shape[1]
    for n in range(N):
        if lengths[n] <= 0:
            continue
        last = lengths[n] - 1
        steps = torch.arange(max(0, last - W + 1), last + 1, device=_DEV)
        ids = s["table"][n].long()[torch.div(steps, page, rounding_mode="floor") % slots]
        k_cache[ids[-1], last % page] = s["k"][n].double()
        v_cache[ids[-1], last % page] = s["v"][n].double()
        k, v = (t[ids, steps % page].repeat_interleave(H // KV, 1).transpose(0, 1) for t in (k_cache, v_cache))  # [H, steps, D]
        a = (k * s["q"][n].double()[:, None]).sum(-1) / math.sqrt(D)
        if s["bias"] is not None:
            bucket = torch.zeros_like(steps)
            for j, e in enumerate(s["edges"].tolist()):
                bucket[last - steps >= e] = j
            a = a + s["bias"].double()[:, bucket]
        y[n] = (torch.softmax(a, -1)[..., None] * v).sum(1)
    return {"y": y, "k_cache": k_cache, "v_cache": v_cache}


def _exact_pages(s):
    """One environment after the other, with lists."""
    page, slots = s["case"]["page"], s["case"]["slots"]
    first, length, table, queue = (s[n].tolist() for n in ("first", "length_in", "table_in", "queue_in"))
    head, count = s["state_in"].tolist()
    pages, slot, back, taken = len(queue), [], [], 0
    for n in range(len(length)):
        if length[n] < 0:
            slot.append(-1)
            continue
        if first[n]:
            back += [e for e in table[n][1:] if e >= 0]
            table[n][1:] = [-1] * (slots - 1)
            length[n] = 0
        j = (length[n] // page) % slots
        if table[n][j] < 0 and taken < count:
            table[n][j] = queue[(head + taken) % pages]
            taken += 1
        slot.append(table[n][j] * page + length[n] % page if table[n][j] >= 0 else -1)
        length[n] += 1
    for i, e in enumerate(back):
        queue[(head + count + i) % pages] = e
    out = (length, table, queue, [(head + taken) % pages, count - taken + len(back)], slot)
    return {n: torch.tensor(v, dtype=torch.int32, device=_DEV) for n, v in zip(_PAGES_OUT, out)}
