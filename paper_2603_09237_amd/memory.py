"""A block of a policy with memory, conditioned on preferences: projection in, causal convolution, selective scan, projection out, both
projections with a low-rank adapter per preference (Sec. III-B's W_l(p) = W0_l + A_l(p) B_l(p)), so that any mix of preferences runs
together, environment n with the adapter index[n] names.

  segment   a rollout segment [T, N, width] at once (an update's forward), from the state that the last call left
  backward  its gradients
  act       one time step of all environments (a rollout, serving)

Argument marshalling only: buffers and call order; every step runs in the library's kernels.  `python -m paper_2603_09237_amd.memory`
runs a rollout step by step, the same segment at once, and a few updates.
"""
from __future__ import annotations

import math

import torch

from . import binding


def _versions(*tensors):
    """How often each has been written to by torch (None: not known, as of inference tensors)."""
    return tuple(None if t is None or t.is_inference() else t._version for t in tensors)


def _check(name, t, shape, dtype):
    """The calls take addresses: a tensor of another shape, type or order would be read as what it is not."""
    if t.shape == shape and t.dtype is dtype and t.is_contiguous():
        return
    raise ValueError(f"{name} must be a contiguous {dtype} tensor {list(shape)}, not {t.dtype} {list(t.shape)} with strides {list(t.stride())}")


def _check_first(first, shape):
    if first is not None:
        _check("first", first, shape, torch.bool if first.dtype is torch.bool else torch.uint8)


class Block:
    """What blocks have in common: buffers by name, the two projections, parameters in `p`, gradients in `g`."""

    def _projections(self, preferences, width, inner, outer, rank, dtype, gen):
        """Parameters of the projections width -> inner and outer -> width."""
        def normal(*shape, scale, t=torch.float32):
            return (torch.randn(*shape, generator=gen) * scale).to(t).to(self.dev)

        p = {}
        for name, i, o in (("in", width, inner), ("out", outer, width)):
            p[name + ".w0"] = normal(o, i, scale=i ** -0.5, t=dtype)
            p[name + ".bias"] = torch.zeros(o, device=self.dev)
            p[name + ".A"] = normal(preferences, o, rank, scale=0.36 * rank ** -0.5, t=dtype)
            p[name + ".B"] = normal(preferences, rank, i, scale=0.36 * i ** -0.5, t=dtype)
        return p, normal

    def _ready(self):
        self.g = {k: torch.zeros(v.shape, device=self.dev) for k, v in self.p.items()}
        self.b, self.saved_for = {}, None
        self.captured, self.recording = {}, False   # buffers that graphs use; whether the present call is being captured

    def _capturing(self):
        return self.dev.type == "cuda" and torch.cuda.is_current_stream_capturing()

    def _replace(self, name, t):
        """The buffer of this name from now on.  The one before it may be in use on this stream still."""
        old = self.b.get(name)
        if old is not None and old.is_cuda and not self.recording:
            old.record_stream(torch.cuda.current_stream(self.dev))
        self.b[name] = t
        return t

    def _used(self, t):
        """A buffer that is about to be used: one that a graph will use on replays is kept."""
        if self.recording:
            self.captured[t.data_ptr()] = t
        return t

    def _buf(self, name, *shape, dtype=None):
        """A buffer of the block, kept while its size does not change."""
        t = self.b.get(name)
        if t is None or t.shape != shape:
            t = self._replace(name, torch.empty(*shape, dtype=dtype or self.dtype, device=self.dev))
        return self._used(t)

    def _scratch(self, n, name="ws"):
        t = self.b.get(name)
        if t is None or t.numel() < n:
            t = self._replace(name, torch.empty(n, dtype=torch.uint8, device=self.dev))
        return self._used(t)

    def _rows(self, name, rows):
        i, o = (self.width, self.L) if name == "in" else (self.D, self.width)
        return binding.AdapterDims(rows, i, o, self.r, self.P, self.kind)

    def _project(self, name, rows, x, index, y, ws="ws"):
        d = self._rows(name, rows)
        q = self.p
        binding.adapter_fwd(d, x, q[name + ".w0"], q[name + ".bias"], q[name + ".A"], q[name + ".B"], index, y,
                            self._scratch(binding.adapter_workspace_bytes(d), ws))


class MemoryBlock(Block):
    """Parameters are in `p`, gradients after `backward` in `g` under the same names (the projections' matrices and factors in the
    block's type, everything else and all gradients fp32).  Acting has buffers of its own: it may run on one stream while segments and
    their gradients run on another.  What a call that is captured in a graph uses stays for as long as the block, also when later calls
    of other sizes take other buffers."""

    def __init__(self, preferences, width, heads, head_dim=64, groups=1, state=64, conv=4, rank=16, dtype=torch.bfloat16, device="cuda", seed=0):
        self.P, self.width, self.H, self.Pd, self.G, self.S, self.W, self.r = preferences, width, heads, head_dim, groups, state, conv, rank
        self.D = heads * head_dim
        self.C = self.D + 2 * groups * state           # channels of the convolution: x, B, C
        self.L = self.D + self.C + heads               # a projected row: gate, x, B, C, dt
        self.dtype, self.kind, self.dev = dtype, 1 if dtype == torch.bfloat16 else 0, torch.device(device)
        gen = torch.Generator().manual_seed(seed)

        self.p, normal = self._projections(preferences, width, self.L, self.D, rank, dtype, gen)
        step = torch.exp(torch.rand(heads, generator=gen) * math.log(100.0) + math.log(1e-3))
        self.p.update({"conv.w": normal(self.C, conv, scale=conv ** -0.5), "conv.b": torch.zeros(self.C, device=self.dev),
                       "a_log": torch.log(1 + 15 * torch.rand(heads, generator=gen)).to(self.dev), "d_skip": torch.ones(heads, device=self.dev),
                       "dt_bias": (step + torch.log(-torch.expm1(-step))).to(self.dev)})
        self._ready()

    def _dims(self, T, N):
        conv = binding.ConvDims(T, N, self.C, self.W, 1, self.kind, N * self.L, self.L, N * self.C, self.C)
        scan = binding.ScanDims(T, N, self.H, self.Pd, self.G, self.S, self.kind, N * self.C, self.C, N * self.L, self.L, N * self.L, self.L,
                                N * self.D, self.D)
        return conv, scan

    def _slices(self, rows):
        """gate, x with B and C, dt of projected rows"""
        return rows[..., :self.D], rows[..., self.D:self.D + self.C], rows[..., self.D + self.C:]

    def _xbc(self, rows):
        GS = self.G * self.S
        return rows[..., :self.D], rows[..., self.D:self.D + GS], rows[..., self.D + GS:]

    def new_state(self, N):
        """An empty memory of N environments: (the convolution's last inputs, the scan's state)."""
        return (torch.zeros(N, self.W - 1, self.C, dtype=self.dtype, device=self.dev),
                torch.zeros(N, self.H, self.Pd, self.S, device=self.dev))

    def _check_memory(self, name, state, N):
        _check(name + "[0]", state[0], (N, self.W - 1, self.C), self.dtype)
        _check(name + "[1]", state[1], (N, self.H, self.Pd, self.S), torch.float32)

    def segment(self, x, index, first, state, train=False):
        """x [T, N, width], index [N] int32, first [T, N] u8 or None -> y [T, N, width] and the state behind the segment."""
        T, N = x.shape[:2]
        self.recording = self._capturing()
        _check("x", x, (T, N, self.width), self.dtype)
        _check_first(first, (T, N))
        self._check_memory("state", state, N)
        q = self.p
        self.saved_for = None  # (from here on buffers change)
        rows = self._buf("index", T * N, dtype=torch.int32)
        rows.view(T, N).copy_(index)
        proj, xc, yc = self._buf("proj", T, N, self.L), self._buf("xc", T, N, self.C), self._buf("yc", T, N, self.D)
        y, after = torch.empty(T, N, self.width, dtype=self.dtype, device=self.dev), self.new_state(N)
        self._project("in", T * N, x, rows, proj)
        z, raw, dt = self._slices(proj)
        conv, scan = self._dims(T, N)
        binding.conv_fwd(conv, raw, q["conv.w"], q["conv.b"], first, state[0], xc, after[0])
        saved = self._buf("saved", binding.scan_saved_bytes(scan), dtype=torch.uint8) if train else None
        xs, b, c = self._xbc(xc)
        binding.scan_fwd(scan, xs, b, c, dt, z, q["a_log"], q["d_skip"], q["dt_bias"], first, state[1], yc, after[1], saved,
                         self._scratch(binding.scan_workspace_bytes(scan)))
        self._project("out", T * N, yc, rows, y)
        if train:  # (the state may move on before the backward; x and first are the caller's to leave alone until then)
            kept = self._buf("state", *state[0].shape)
            kept.copy_(state[0])
            self.saved_for = (x, first, kept, _versions(x, first))
        return y, after

    def backward(self, dy):
        """Gradients of the last segment(train=True) from dy [T, N, width]: parameters into `g`, that of x returned (the state's is
        cut there, as truncated back-propagation through time does).  That segment's x and first have to be as they were."""
        if self.saved_for is None:
            raise RuntimeError("backward() needs the last segment() to have been one with train=True")
        x, first, state, versions = self.saved_for
        if versions != _versions(x, first):
            raise RuntimeError("backward() needs the segment's x and first, which have been written to since")
        T, N = x.shape[:2]
        self.recording = self._capturing()
        _check("dy", dy, (T, N, self.width), self.dtype)
        q, g = self.p, self.g
        rows, proj, xc, yc, saved = (self._used(self.b[n]) for n in ("index", "proj", "xc", "yc", "saved"))
        dproj, dxc, dyc, dx = (self._buf(n, T, N, w) for n, w in (("dproj", self.L), ("dxc", self.C), ("dyc", self.D), ("dx", self.width)))

        def back(name, xin, grad, dxin):
            d = self._rows(name, T * N)
            binding.adapter_bwd(d, xin, q[name + ".w0"], q[name + ".A"], q[name + ".B"], rows, grad, dxin, g[name + ".w0"], g[name + ".bias"],
                                g[name + ".A"], g[name + ".B"], self._scratch(binding.adapter_workspace_bytes(d, True)))

        back("out", yc, dy, dyc)
        conv, scan = self._dims(T, N)
        (z, raw, dt), (dz, draw, ddt) = self._slices(proj), self._slices(dproj)
        xs, b, c = self._xbc(xc)
        dxs, db, dc = self._xbc(dxc)
        binding.scan_bwd(scan, xs, b, c, dt, z, q["a_log"], q["d_skip"], q["dt_bias"], first, saved, dyc, None, dxs, db, dc, ddt, dz,
                         g["a_log"], g["d_skip"], g["dt_bias"], None, self._scratch(binding.scan_workspace_bytes(scan, True)))
        binding.conv_bwd(conv, raw, q["conv.w"], q["conv.b"], first, state, dxc, None, draw, g["conv.w"], g["conv.b"], None,
                         self._scratch(binding.conv_workspace_bytes(conv)))
        back("in", x, dproj, dx)
        return dx

    def act(self, x, index, first, state, after):
        """One time step: x [N, width], index [N] int32, first [N] u8 or None -> y [N, width]; the memory goes from `state` into `after`
        (its convolution part may not be the same tensor, its scan part may)."""
        N = x.shape[0]
        self.recording = self._capturing()
        _check("x", x, (N, self.width), self.dtype)
        _check("index", index, (N,), torch.int32)
        _check_first(first, (N,))
        self._check_memory("state", state, N)
        self._check_memory("after", after, N)
        q = self.p
        proj, yc = self._buf("act.proj", N, self.L), self._buf("act.yc", N, self.D)
        y = torch.empty(N, self.width, dtype=self.dtype, device=self.dev)
        self._project("in", N, x, index, proj, "act.ws")
        z, raw, dt = self._slices(proj)
        d = binding.ScanDims(1, N, self.H, self.Pd, self.G, self.S, self.kind, x_n=self.L, z_n=self.L, dt_n=self.L, y_n=self.D)
        binding.memory_step(d, self.W, raw, dt, z, q["conv.w"], q["conv.b"], q["a_log"], q["d_skip"], q["dt_bias"], first, state[0], state[1], yc,
                            after[0], after[1])
        self._project("out", N, yc, index, y, "act.ws")
        return y


def main():
    """A rollout step by step, the same segment at once, and updates towards a target that only a memory can meet: the sum of an
    environment's last four inputs, weighed by its preference."""
    torch.manual_seed(0)
    P, N, T, width = 8, 256, 32, 64
    block = MemoryBlock(P, width, heads=4, head_dim=32, state=16, rank=4)
    index = torch.randint(0, P, (N,), device="cuda").to(torch.int32)     # requests in any order
    x = torch.randn(T, N, width, device="cuda").to(torch.bfloat16)
    first = (torch.rand(T, N, device="cuda") < 0.03).to(torch.uint8)
    y, _ = block.segment(x, index, first, block.new_state(N))
    now, nxt = block.new_state(N), block.new_state(N)
    worst = 0.0
    for t in range(T):
        worst = max(worst, float((block.act(x[t], index, first[t], now, nxt).float() - y[t].float()).abs().max()))
        now, nxt = nxt, now
    print(f"acting step by step and the segment at once differ by at most {worst:.4f} (outputs up to {float(y.abs().max()):.2f}, bf16)")
    weight = torch.randn(P, width, device="cuda")[index.long()]
    past = torch.cat([torch.zeros(3, N, width, device="cuda"), x.float()]).unfold(0, 4, 1).sum(-1)
    target = past * weight * 0.2
    moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in block.g.items()}
    master = {k: v.float().clone() for k, v in block.p.items()}
    for it in range(1, 61):
        y, _ = block.segment(x, index, None, block.new_state(N), train=True)
        err = y.float() - target
        block.backward((err * (2.0 / err.numel())).to(torch.bfloat16))
        for k, g in block.g.items():  # Adam on fp32 copies
            m, v = moments[k]
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            master[k].sub_(3e-3 * (m / (1 - 0.9 ** it)) / ((v / (1 - 0.99 ** it)).sqrt() + 1e-8))
            block.p[k].copy_(master[k])
        if it % 20 == 1 or it == 60:
            print(f"update {it:3d}: mean squared error {float(err.square().mean()):.4f}")


if __name__ == "__main__":
    main()
