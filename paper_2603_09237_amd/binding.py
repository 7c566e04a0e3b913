"""ctypes binding of libmorlax.so: the same entry points as include/morlax.h.

Argument marshalling only.  Tensors are torch CUDA tensors used as device memory (data_ptr) and the
current torch stream is passed as the hipStream_t; every computation runs in the library's kernels.
Loading fails loudly when the library has not been built (`python -m paper_2603_09237_amd.build`).
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmorlax.so")

ACTOR, CRITIC = 0, 1
OK, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = 0, -1, -2, -3, -4, -5


class Dims(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("K", "P", "N", "T", "obs_dim", "act_dim", "n_hidden", "width",
                                         "act", "rank", "hyper_width", "wdtype", "mean_tanh", "sigma_state")]


class Rows(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("t0", "t_cnt", "j0", "j_cnt")]


class AdapterDims(C.Structure):
    """morlax_adapter_dims: `adapters` is n_adapters; row strides in elements, those of contiguous rows where they are not given."""
    _fields_ = [(n, C.c_int32) for n in ("rows", "d_in", "d_out", "rank", "n_adapters", "dtype")] + \
               [(n, C.c_int64) for n in ("ld_x", "ld_y")]

    def __init__(self, rows, d_in, d_out, rank, adapters, dtype, ld_x=None, ld_y=None):
        super().__init__(rows, d_in, d_out, rank, adapters, dtype, d_in if ld_x is None else ld_x, d_out if ld_y is None else ld_y)


class ConvDims(C.Structure):
    """morlax_conv_dims: strides in elements, those of a contiguous [T, N, channels] where they are not given."""
    _fields_ = [(n, C.c_int32) for n in ("T", "N", "channels", "width", "act", "dtype")] + \
               [(n, C.c_int64) for n in ("x_t", "x_n", "y_t", "y_n")]

    def __init__(self, T, N, channels, width, act, dtype, x_t=None, x_n=None, y_t=None, y_n=None):
        full = [N * channels, channels] * 2
        super().__init__(T, N, channels, width, act, dtype, *[f if v is None else v for v, f in zip((x_t, x_n, y_t, y_n), full)])


class ScanDims(C.Structure):
    """morlax_scan_dims: strides in elements; where they are not given, those of contiguous rows, x, B and C one after the other."""
    _fields_ = [(n, C.c_int32) for n in ("T", "N", "heads", "head_dim", "groups", "state", "dtype")] + \
               [(n, C.c_int64) for n in ("x_t", "x_n", "z_t", "z_n", "dt_t", "dt_n", "y_t", "y_n")]

    def __init__(self, T, N, heads, head_dim, groups, state, dtype, x_t=None, x_n=None, z_t=None, z_n=None, dt_t=None, dt_n=None,
                 y_t=None, y_n=None):
        D = heads * head_dim
        full = [k for w in (D + 2 * groups * state, D, heads, D) for k in (N * w, w)]
        super().__init__(T, N, heads, head_dim, groups, state, dtype,
                         *[f if v is None else v for v, f in zip((x_t, x_n, z_t, z_n, dt_t, dt_n, y_t, y_n), full)])


class MorlaxError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"morlax error {code}: {msg}")
        self.code = code


_lib = None

EXPORTS = ("morlax_create", "morlax_destroy", "morlax_last_error", "morlax_hparam_count",
           "morlax_theta_mat_len", "morlax_theta_vec_len", "morlax_saved_bytes", "morlax_workspace_bytes",
           "morlax_env_pref_index", "morlax_hypernet_fwd", "morlax_hypernet_bwd", "morlax_hypernet_bwd_kept",
           "morlax_policy_fwd",
           "morlax_policy_bwd", "morlax_vec_gae", "morlax_vec_gae_trunc", "morlax_adam_step",
           "morlax_sample_preferences", "morlax_scalarize_normalized", "morlax_ppo_loss_grad",
           "morlax_ppo_loss_grad_static", "morlax_eval_returns",
           "morlax_hypervolume_workspace_bytes", "morlax_pareto_hypervolume", "morlax_profile_begin",
           "morlax_profile_end", "morlax_adapter_workspace_bytes", "morlax_adapter_fwd", "morlax_adapter_bwd",
           "morlax_conv_workspace_bytes", "morlax_conv_fwd", "morlax_conv_bwd", "morlax_scan_saved_bytes",
           "morlax_scan_workspace_bytes", "morlax_scan_fwd", "morlax_scan_bwd", "morlax_memory_step")

GEMM_KINDS = ("fwd_first", "fwd_hidden", "dx_hidden", "dw_hidden", "dw_first", "fwd_fused")


def load():
    """dlopen the library (once) and declare the prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2603_09237_amd.build` "
                          "(there is no CPU fallback)")
    # torch provides the device memory and the streams, so the library must bind to the HIP runtime
    # torch has loaded (two runtimes in one process do not share devices): import torch first.
    import torch  # noqa: F401
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    lib.morlax_create.argtypes = [C.POINTER(Dims), C.POINTER(vp)]
    lib.morlax_create.restype = C.c_int
    lib.morlax_destroy.argtypes = [vp]
    lib.morlax_destroy.restype = None
    lib.morlax_last_error.argtypes = []
    lib.morlax_last_error.restype = C.c_char_p
    for name in ("morlax_hparam_count", "morlax_theta_mat_len", "morlax_theta_vec_len"):
        getattr(lib, name).argtypes = [vp, C.c_int]
        getattr(lib, name).restype = i64
    lib.morlax_saved_bytes.argtypes = [vp, C.c_int, C.POINTER(Rows)]
    lib.morlax_saved_bytes.restype = i64
    lib.morlax_workspace_bytes.argtypes = [vp, C.POINTER(Rows)]
    lib.morlax_workspace_bytes.restype = i64
    lib.morlax_env_pref_index.argtypes = [vp, vp, vp]
    lib.morlax_hypernet_fwd.argtypes = [vp, C.c_int, vp, vp, vp, vp, vp, i64, vp]
    lib.morlax_hypernet_bwd.argtypes = [vp, C.c_int, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.morlax_hypernet_bwd_kept.argtypes = [vp, C.c_int, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.morlax_policy_fwd.argtypes = [vp, C.c_int, vp, vp, vp, C.POINTER(Rows), vp, vp, vp, vp, vp, vp, i64, vp]
    lib.morlax_policy_bwd.argtypes = [vp, C.c_int, vp, vp, vp, C.POINTER(Rows), vp, vp, vp, vp, vp, vp, i64, vp]
    lib.morlax_vec_gae.argtypes = [vp, vp, vp, vp, vp, f32, f32, vp, vp, vp, vp]
    lib.morlax_vec_gae_trunc.argtypes = [vp, vp, vp, vp, vp, vp, f32, f32, vp, vp, vp, vp]
    lib.morlax_adam_step.argtypes = [vp, C.c_int, vp, vp, vp, vp, f32, f32, f32, f32, i32, vp]
    lib.morlax_sample_preferences.argtypes = [vp, vp, i32, vp, vp]
    lib.morlax_scalarize_normalized.argtypes = [vp, C.POINTER(Rows), vp, vp, vp, vp, i64, vp]
    lib.morlax_ppo_loss_grad.argtypes = [vp, C.POINTER(Rows), vp, vp, i32, vp, vp, vp, vp, vp, f32, i32,
                                         vp, vp, vp, vp, vp, i64, vp]
    lib.morlax_ppo_loss_grad_static.argtypes = [vp, C.POINTER(Rows), vp, vp, i32, vp, vp, vp, vp, vp, f32, i32,
                                                vp, vp, vp, vp, vp]
    lib.morlax_ppo_loss_grad_static.restype = C.c_int
    lib.morlax_eval_returns.argtypes = [vp, vp, vp, f32, vp, vp]
    lib.morlax_eval_returns.restype = C.c_int
    lib.morlax_hypervolume_workspace_bytes.argtypes = [i32, i32]
    lib.morlax_hypervolume_workspace_bytes.restype = i64
    lib.morlax_pareto_hypervolume.argtypes = [vp, vp, i32, i32, vp, vp, vp, i64, vp]
    lib.morlax_pareto_hypervolume.restype = C.c_int
    dp = C.POINTER(AdapterDims)
    lib.morlax_adapter_workspace_bytes.argtypes = [dp, i32]
    lib.morlax_adapter_workspace_bytes.restype = i64
    lib.morlax_adapter_fwd.argtypes = [dp] + [vp] * 8 + [i64, vp]
    lib.morlax_adapter_bwd.argtypes = [dp] + [vp] * 12 + [i64, vp]
    cp, sp = C.POINTER(ConvDims), C.POINTER(ScanDims)
    lib.morlax_conv_workspace_bytes.argtypes = [cp]
    lib.morlax_scan_saved_bytes.argtypes = [sp]
    lib.morlax_scan_workspace_bytes.argtypes = [sp, i32]
    for name in ("morlax_conv_workspace_bytes", "morlax_scan_saved_bytes", "morlax_scan_workspace_bytes"):
        getattr(lib, name).restype = i64
    lib.morlax_conv_fwd.argtypes = [cp] + [vp] * 8
    lib.morlax_conv_bwd.argtypes = [cp] + [vp] * 12 + [i64, vp]
    lib.morlax_scan_fwd.argtypes = [sp] + [vp] * 14 + [i64, vp]
    lib.morlax_scan_bwd.argtypes = [sp] + [vp] * 22 + [i64, vp]
    lib.morlax_memory_step.argtypes = [sp, i32] + [vp] * 15
    for name in ("morlax_conv_fwd", "morlax_conv_bwd", "morlax_scan_fwd", "morlax_scan_bwd", "morlax_memory_step"):
        getattr(lib, name).restype = C.c_int
    for name in ("morlax_adapter_fwd", "morlax_adapter_bwd"):
        getattr(lib, name).restype = C.c_int
    lib.morlax_profile_begin.argtypes = [vp]
    lib.morlax_profile_begin.restype = C.c_int
    lib.morlax_profile_end.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i64), C.POINTER(C.c_double)]
    lib.morlax_profile_end.restype = C.c_int
    for name in ("morlax_env_pref_index", "morlax_hypernet_fwd", "morlax_hypernet_bwd", "morlax_hypernet_bwd_kept",
           "morlax_policy_fwd",
                 "morlax_policy_bwd", "morlax_vec_gae", "morlax_vec_gae_trunc", "morlax_adam_step",
                 "morlax_sample_preferences", "morlax_scalarize_normalized", "morlax_ppo_loss_grad"):
        getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, tuple):      # (address, bytes): a workspace given as a raw address
        return t[0]
    return t.data_ptr()


def _nbytes(t):
    """Size of a workspace: a tensor's own, or -- for a raw address -- whatever the caller vouches for."""
    if t is None:
        return 0
    if isinstance(t, int):
        return 1 << 62
    if isinstance(t, tuple):
        return int(t[1])
    return t.numel() * t.element_size()


def _stream():
    """The current stream of the current device as a hipStream_t.  Asked for by its handle where this torch has a function for that:
    making the stream object takes the host 3 us, a third of a call of one launch, which bounds the smallest steps (7.7 and 4.9 us a
    call of `vec_gae`)."""
    import torch
    handle = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    device = getattr(torch._C, "_cuda_getDevice", None)
    if handle is None or device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return handle(device())


def _rows(rows):
    if rows is None:
        return None
    if isinstance(rows, Rows):
        return C.byref(rows)
    return C.byref(Rows(*[int(v) for v in rows]))


class Context:
    """Owns a morlax_ctx.  Methods mirror the C entry points and raise MorlaxError on failure."""

    def __init__(self, **dims):
        self.lib = load()
        self.dims = Dims(**{k: int(v) for k, v in dims.items()})
        h = C.c_void_p()
        rc = self.lib.morlax_create(C.byref(self.dims), C.byref(h))
        if rc != OK:
            raise MorlaxError(rc, self.lib.morlax_last_error().decode())
        self.h = h
        self.profiling = False   # between profile_begin and profile_end

    @classmethod
    def from_config(cls, cfg):
        return cls(**cfg.dims_dict())

    def close(self):
        if getattr(self, "h", None):
            self.lib.morlax_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc != OK:
            raise MorlaxError(rc, self.lib.morlax_last_error().decode())

    # ---- queries
    def hparam_count(self, net):
        return self.lib.morlax_hparam_count(self.h, net)

    def theta_mat_len(self, net):
        return self.lib.morlax_theta_mat_len(self.h, net)

    def theta_vec_len(self, net):
        return self.lib.morlax_theta_vec_len(self.h, net)

    def saved_bytes(self, net, rows=None):
        return self.lib.morlax_saved_bytes(self.h, net, _rows(rows))

    def workspace_bytes(self, rows=None):
        return self.lib.morlax_workspace_bytes(self.h, _rows(rows))

    def profile_begin(self):
        self._check(self.lib.morlax_profile_begin(self.h))
        self.profiling = True

    def profile_end(self):
        """-> {kind: (total_ms, launches, total_flops)} for the grouped-GEMM launches since profile_begin."""
        n = len(GEMM_KINDS)
        ms, cnt, fl = (C.c_double * n)(), (C.c_int64 * n)(), (C.c_double * n)()
        self.profiling = False
        self._check(self.lib.morlax_profile_end(self.h, ms, cnt, fl))
        return {k: (ms[i], cnt[i], fl[i]) for i, k in enumerate(GEMM_KINDS)}

    # ---- ops
    def env_pref_index(self, out, stream=None):
        self._check(self.lib.morlax_env_pref_index(self.h, _ptr(out), stream if stream is not None else _stream()))

    def hypernet_fwd(self, net, hparams, w, theta_mat, theta_vec, ws, stream=None):
        self._check(self.lib.morlax_hypernet_fwd(self.h, net, _ptr(hparams), _ptr(w), _ptr(theta_mat),
                                                 _ptr(theta_vec), _ptr(ws), _nbytes(ws),
                                                 stream if stream is not None else _stream()))

    def hypernet_bwd_kept(self, net, hparams, w, dtheta_mat, dtheta_vec, dhparams, ws_fwd, stream=None):
        self._check(self.lib.morlax_hypernet_bwd_kept(self.h, net, _ptr(hparams), _ptr(w), _ptr(dtheta_mat),
                                                      _ptr(dtheta_vec), _ptr(dhparams), _ptr(ws_fwd), _nbytes(ws_fwd),
                                                      stream if stream is not None else _stream()))

    def hypernet_bwd(self, net, hparams, w, dtheta_mat, dtheta_vec, dhparams, ws, stream=None):
        self._check(self.lib.morlax_hypernet_bwd(self.h, net, _ptr(hparams), _ptr(w), _ptr(dtheta_mat),
                                                 _ptr(dtheta_vec), _ptr(dhparams), _ptr(ws), _nbytes(ws),
                                                 stream if stream is not None else _stream()))

    def policy_fwd(self, net, theta_mat, theta_vec, x, rows, out, eps=None, act=None, logp=None, saved=None,
                   ws=None, stream=None):
        self._check(self.lib.morlax_policy_fwd(self.h, net, _ptr(theta_mat), _ptr(theta_vec), _ptr(x), _rows(rows),
                                               _ptr(out), _ptr(eps), _ptr(act), _ptr(logp), _ptr(saved), _ptr(ws),
                                               _nbytes(ws), stream if stream is not None else _stream()))

    def policy_bwd(self, net, theta_mat, theta_vec, x, rows, saved, dout, dlogsig, dtheta_mat, dtheta_vec, ws,
                   stream=None):
        self._check(self.lib.morlax_policy_bwd(self.h, net, _ptr(theta_mat), _ptr(theta_vec), _ptr(x), _rows(rows),
                                               _ptr(saved), _ptr(dout), _ptr(dlogsig), _ptr(dtheta_mat),
                                               _ptr(dtheta_vec), _ptr(ws), _nbytes(ws),
                                               stream if stream is not None else _stream()))

    def vec_gae(self, r, v, done, w, gamma, lam, adv_vec, vtarg, adv_s, stream=None):
        self._check(self.lib.morlax_vec_gae(self.h, _ptr(r), _ptr(v), _ptr(done), _ptr(w), float(gamma), float(lam),
                                            _ptr(adv_vec), _ptr(vtarg), _ptr(adv_s),
                                            stream if stream is not None else _stream()))

    def vec_gae_trunc(self, r, v, done, trunc, w, gamma, lam, adv_vec, vtarg, adv_s, stream=None):
        self._check(self.lib.morlax_vec_gae_trunc(self.h, _ptr(r), _ptr(v), _ptr(done), _ptr(trunc), _ptr(w),
                                                  float(gamma), float(lam), _ptr(adv_vec), _ptr(vtarg), _ptr(adv_s),
                                                  stream if stream is not None else _stream()))

    def sample_preferences(self, u, kappa, w, stream=None):
        self._check(self.lib.morlax_sample_preferences(self.h, _ptr(u), int(kappa), _ptr(w),
                                                       stream if stream is not None else _stream()))

    def eval_returns(self, r, done, gamma, J, stream=None):
        self._check(self.lib.morlax_eval_returns(self.h, _ptr(r), _ptr(done), float(gamma), _ptr(J),
                                                 stream if stream is not None else _stream()))

    def adam_step(self, net, hparams, dhparams, m, v, lr, beta1, beta2, eps, step, stream=None):
        self._check(self.lib.morlax_adam_step(self.h, net, _ptr(hparams), _ptr(dhparams), _ptr(m), _ptr(v),
                                              float(lr), float(beta1), float(beta2), float(eps), int(step),
                                              stream if stream is not None else _stream()))

    def scalarize_normalized(self, rows, adv_vec, w, adv_out, ws, stream=None):
        self._check(self.lib.morlax_scalarize_normalized(self.h, _rows(rows), _ptr(adv_vec), _ptr(w), _ptr(adv_out),
                                                         _ptr(ws), _nbytes(ws),
                                                         stream if stream is not None else _stream()))

    def ppo_loss_grad_static(self, rows, mu, logsig, logsig_stride, act, logp_old, adv_s, v, vtarg, clip_eps, norm_adv,
                             dmu, dlogsig, dv, stats, stream=None):
        """The loss call on the library's static scratch array (no workspace argument, nothing allocated)."""
        self._check(self.lib.morlax_ppo_loss_grad_static(self.h, _rows(rows), _ptr(mu), _ptr(logsig), int(logsig_stride),
                                                         _ptr(act), _ptr(logp_old), _ptr(adv_s), _ptr(v), _ptr(vtarg),
                                                         float(clip_eps), int(norm_adv), _ptr(dmu), _ptr(dlogsig),
                                                         _ptr(dv), _ptr(stats),
                                                         stream if stream is not None else _stream()))

    def ppo_loss_grad(self, rows, mu, logsig, logsig_stride, act, logp_old, adv_s, v, vtarg, clip_eps, norm_adv,
                      dmu, dlogsig, dv, stats, ws, stream=None):
        self._check(self.lib.morlax_ppo_loss_grad(self.h, _rows(rows), _ptr(mu), _ptr(logsig), int(logsig_stride),
                                                  _ptr(act), _ptr(logp_old), _ptr(adv_s), _ptr(v), _ptr(vtarg),
                                                  float(clip_eps), int(norm_adv), _ptr(dmu), _ptr(dlogsig),
                                                  _ptr(dv), _ptr(stats), _ptr(ws), _nbytes(ws),
                                                  stream if stream is not None else _stream()))


STATIC_SCRATCH_BYTES = 2 * 1024 * 1024


def hypervolume_workspace_bytes(n, K):
    """Bytes of device scratch morlax_pareto_hypervolume needs for n points in K objectives (-1: sizes not served)."""
    return int(load().morlax_hypervolume_workspace_bytes(int(n), int(K)))


def pareto_hypervolume(J, ref, n, K, front, hv, ws, stream=None):
    """morlax_pareto_hypervolume: needs no context; raises MorlaxError on failure."""
    lib = load()
    rc = lib.morlax_pareto_hypervolume(_ptr(J), _ptr(ref), int(n), int(K), _ptr(front), _ptr(hv), _ptr(ws),
                                       _nbytes(ws), stream if stream is not None else _stream())
    if rc != OK:
        raise MorlaxError(rc, lib.morlax_last_error().decode())


def _call(fn, *args):
    rc = fn(*args)
    if rc != OK:
        raise MorlaxError(rc, _lib.morlax_last_error().decode())


def _size(n):
    """What a workspace query answers; dimensions that are not served raise."""
    if n < 0:
        raise MorlaxError(ERR_SHAPE, _lib.morlax_last_error().decode())
    return int(n)


def adapter_workspace_bytes(dims, backward=False):
    """Bytes of device scratch that adapter_fwd (adapter_bwd) needs for these dimensions."""
    return _size(load().morlax_adapter_workspace_bytes(C.byref(dims), int(bool(backward))))


def adapter_fwd(dims, x, w0, bias, A, B, index, y, ws, stream=None):
    """morlax_adapter_fwd: y[m] = W0 x[m] + bias + A[p] (B[p] x[m]) with p = index[m]."""
    _call(load().morlax_adapter_fwd, C.byref(dims), _ptr(x), _ptr(w0), _ptr(bias), _ptr(A), _ptr(B), _ptr(index), _ptr(y), _ptr(ws),
          _nbytes(ws), stream if stream is not None else _stream())


def adapter_bwd(dims, x, w0, A, B, index, dy, dx, dw0, dbias, dA, dB, ws, stream=None):
    """morlax_adapter_bwd: gradients of adapter_fwd; outputs that are None are left out."""
    _call(load().morlax_adapter_bwd, C.byref(dims), _ptr(x), _ptr(w0), _ptr(A), _ptr(B), _ptr(index), _ptr(dy), _ptr(dx), _ptr(dw0),
          _ptr(dbias), _ptr(dA), _ptr(dB), _ptr(ws), _nbytes(ws), stream if stream is not None else _stream())


def conv_workspace_bytes(dims):
    """Bytes of device scratch that conv_bwd needs."""
    return _size(load().morlax_conv_workspace_bytes(C.byref(dims)))


def conv_fwd(dims, x, w, b, first, state_in, y, state_out, stream=None):
    """morlax_conv_fwd: the short causal convolution over the steps of each episode."""
    _call(load().morlax_conv_fwd, C.byref(dims), _ptr(x), _ptr(w), _ptr(b), _ptr(first), _ptr(state_in), _ptr(y), _ptr(state_out),
          stream if stream is not None else _stream())


def conv_bwd(dims, x, w, b, first, state_in, dy, dstate_out, dx, dw, db, dstate_in, ws, stream=None):
    """morlax_conv_bwd: gradients of conv_fwd."""
    _call(load().morlax_conv_bwd, C.byref(dims), _ptr(x), _ptr(w), _ptr(b), _ptr(first), _ptr(state_in), _ptr(dy), _ptr(dstate_out),
          _ptr(dx), _ptr(dw), _ptr(db), _ptr(dstate_in), _ptr(ws), _nbytes(ws), stream if stream is not None else _stream())


def scan_saved_bytes(dims):
    """Bytes of the `saved` buffer that scan_fwd fills for scan_bwd."""
    return _size(load().morlax_scan_saved_bytes(C.byref(dims)))


def scan_workspace_bytes(dims, backward=False):
    """Bytes of device scratch that scan_fwd (scan_bwd) needs."""
    return _size(load().morlax_scan_workspace_bytes(C.byref(dims), int(bool(backward))))


def scan_fwd(dims, x, b, c, dt, z, a_log, d_skip, dt_bias, first, state_in, y, state_out, saved, ws, stream=None):
    """morlax_scan_fwd: the selective state space scan of all environments and heads."""
    _call(load().morlax_scan_fwd, C.byref(dims), _ptr(x), _ptr(b), _ptr(c), _ptr(dt), _ptr(z), _ptr(a_log), _ptr(d_skip), _ptr(dt_bias),
          _ptr(first), _ptr(state_in), _ptr(y), _ptr(state_out), _ptr(saved), _ptr(ws), _nbytes(ws),
          stream if stream is not None else _stream())


def scan_bwd(dims, x, b, c, dt, z, a_log, d_skip, dt_bias, first, saved, dy, dstate_out, dx, db, dc, ddt, dz, da_log, dd_skip, ddt_bias,
             dstate_in, ws, stream=None):
    """morlax_scan_bwd: gradients of scan_fwd from what it saved."""
    _call(load().morlax_scan_bwd, C.byref(dims), _ptr(x), _ptr(b), _ptr(c), _ptr(dt), _ptr(z), _ptr(a_log), _ptr(d_skip), _ptr(dt_bias),
          _ptr(first), _ptr(saved), _ptr(dy), _ptr(dstate_out), _ptr(dx), _ptr(db), _ptr(dc), _ptr(ddt), _ptr(dz), _ptr(da_log),
          _ptr(dd_skip), _ptr(ddt_bias), _ptr(dstate_in), _ptr(ws), _nbytes(ws), stream if stream is not None else _stream())


def memory_step(dims, width, xbc, dt, z, conv_w, conv_b, a_log, d_skip, dt_bias, first, conv_in, state_in, y, conv_out, state_out,
                stream=None):
    """morlax_memory_step: one time step of the convolution and the scan in one launch."""
    _call(load().morlax_memory_step, C.byref(dims), int(width), _ptr(xbc), _ptr(dt), _ptr(z), _ptr(conv_w), _ptr(conv_b), _ptr(a_log),
          _ptr(d_skip), _ptr(dt_bias), _ptr(first), _ptr(conv_in), _ptr(state_in), _ptr(y), _ptr(conv_out), _ptr(state_out),
          stream if stream is not None else _stream())
