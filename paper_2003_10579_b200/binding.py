"""Thin ctypes binding of the C-ABI library (``include/straggler_sim.h``): argument marshalling
only.  torch supplies device memory and streams; every step of the simulation runs in the
library's CUDA kernels.  Importing this module loads ``libstraggler_sim.so`` and raises if it
has not been built - there is no CPU path behind these calls."""
from __future__ import annotations

import collections
import contextlib
import ctypes as C
import os
import struct

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libstraggler_sim.so")

VARIANTS = {"ksync": 0, "kbatchsync": 1, "kasync": 2, "kbatchasync": 3}
MODELS = {"none": 0, "lsq": 1, "logistic": 2, "softmax": 3, "mlp2": 4}
DELAYS = {"exp": 0, "shifted_exp": 1, "pareto2": 2}
STATUS = {0: "SIM_OK", 1: "SIM_ERR_ARG", 2: "SIM_ERR_ALLOC", 3: "SIM_ERR_CUDA", 4: "SIM_ERR_TIMEOUT",
          5: "SIM_ERR_STATE", 6: "SIM_ERR_INTERNAL"}

EXPORTS = ["sim_create", "sim_set_params", "sim_set_adasync", "sim_set_adasync_loss", "sim_set_tuning", "sim_reserve", "sim_run",
           "sim_trace_size", "sim_get_trace", "sim_get_params", "sim_eval_loss", "sim_error_curve", "sim_set_eval_every", "sim_risk_trace_size",
           "sim_get_risk_trace", "sim_risk_curve", "sim_risk_envelope", "sim_selftest_wait_timeout", "sim_n_params", "sim_last_error",
           "sim_destroy", "sim_draw_delays", "sim_draw_indices", "sim_simulate_host", "sim_sweep_host", "sim_schedule_noalloc",
           "sim_noalloc_last_error", "sim_adamw_create", "sim_adamw_step", "sim_adamw_step_device", "sim_adamw_destroy",
           "sim_mx_codes_bytes", "sim_mx_scales_bytes", "sim_mx_quantize", "sim_mx_dequantize", "sim_mx_matmul", "sim_set_adamw", "sim_eval_loss_mxfp4",
           "sim_ckpt_codes_bytes", "sim_ckpt_scales_bytes", "sim_ckpt_write", "sim_ckpt_read", "sim_act_backward_workspace", "sim_act_backward",
           "sim_matmul_workspace", "sim_matmul", "sim_log_probs", "sim_eval_log_probs"]
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}     # SIM_F32, SIM_BF16, SIM_F16
MXFP4 = 3
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


class SimProblem(C.Structure):
    _fields_ = [("model", C.c_int), ("n", C.c_int64), ("d", C.c_int32), ("n_classes", C.c_int32),
                ("hidden", C.c_int32), ("X", C.c_void_p), ("y", C.c_void_p), ("label", C.c_void_p),
                ("w_ref", C.c_void_p)]


class SimDelay(C.Structure):
    _fields_ = [("kind", C.c_int), ("mu", C.c_double), ("shift", C.c_double)]


class SimAdamwTensor(C.Structure):
    _fields_ = [("n", C.c_int64), ("p_type", C.c_int), ("g_type", C.c_int), ("p", C.c_void_p), ("g", C.POINTER(C.c_void_p)),
                ("g_scale", C.POINTER(C.c_void_p)), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("shadow", C.c_void_p), ("weight_decay", C.c_float)]


class SimProduct(C.Structure):
    _fields_ = [("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64), ("type", C.c_int), ("a", C.c_void_p), ("lda", C.c_int64), ("a_t", C.c_int32),
                ("b", C.c_void_p), ("ldb", C.c_int64), ("b_t", C.c_int32), ("bias", C.c_void_p), ("bias_type", C.c_int), ("act", C.c_int),
                ("act_grad", C.c_int32), ("z_codes", C.c_void_p), ("z_scales", C.c_void_p), ("residual", C.c_void_p), ("ldr", C.c_int64),
                ("c", C.c_void_p), ("c_type", C.c_int), ("ldc", C.c_int64)]


class SimError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("%s: %s" % (STATUS.get(status, status), message))
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError("%s is missing: build it with `python -m paper_2003_10579_b200.build` "
                          "(there is no CPU fallback)" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, u64, dbl = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_double
    L.sim_create.argtypes = [C.POINTER(SimProblem), i32, i32, C.c_int, SimDelay, C.c_float, i32, u64, i32,
                             i64, vp, C.POINTER(vp)]
    L.sim_set_params.argtypes = [vp, vp]
    L.sim_set_adasync.argtypes = [vp, i32, dbl]
    L.sim_set_adasync_loss.argtypes = [vp, i32, dbl]
    L.sim_set_tuning.argtypes = [vp, i32, i32, i32]
    L.sim_reserve.argtypes = [vp, i64]
    L.sim_run.argtypes = [vp, i64]
    L.sim_trace_size.argtypes = [vp, C.POINTER(i64), C.POINTER(i32)]
    L.sim_get_trace.argtypes = [vp] * 8
    L.sim_get_params.argtypes = [vp, vp]
    L.sim_eval_loss.argtypes = [vp, vp]
    L.sim_error_curve.argtypes = [vp, vp, i32, vp, vp]
    L.sim_selftest_wait_timeout.argtypes = [vp]
    L.sim_set_eval_every.argtypes = [vp, i64]
    L.sim_risk_trace_size.argtypes = [vp, C.POINTER(i64)]
    L.sim_get_risk_trace.argtypes = [vp, vp, vp]
    L.sim_risk_curve.argtypes = [vp, vp, i32, C.c_float, vp, vp]
    L.sim_risk_envelope.argtypes = [C.POINTER(vp), i32, vp, i32, C.c_float, vp, vp]
    L.sim_n_params.argtypes = [vp]
    L.sim_n_params.restype = i64
    L.sim_last_error.argtypes = [vp]
    L.sim_last_error.restype = C.c_char_p
    L.sim_destroy.argtypes = [vp]
    L.sim_destroy.restype = None
    L.sim_draw_delays.argtypes = [SimDelay, u64, i64, i32, i32, i32, vp, vp]
    L.sim_draw_indices.argtypes = [u64, i64, i32, i32, i32, i64, i32, vp, vp]
    L.sim_simulate_host.argtypes = [C.POINTER(SimProblem), i32, i32, C.c_int, SimDelay, C.c_float, i32, u64,
                                    i32, i64, vp, i32, dbl, i64] + [vp] * 8
    L.sim_sweep_host.argtypes = [C.POINTER(SimProblem), i32, i32, vp, vp, SimDelay, C.c_float, i32, u64, i32, i64, vp, i64,
                                 vp, vp, vp]
    L.sim_schedule_noalloc.argtypes = [i32, i32, C.c_int, SimDelay, u64, i64, i32, i32, dbl, i64] + [vp] * 6
    L.sim_noalloc_last_error.argtypes = []
    L.sim_noalloc_last_error.restype = C.c_char_p
    L.sim_adamw_create.argtypes = [C.POINTER(SimAdamwTensor), i32, i32, i32, dbl, dbl, dbl, u64, C.POINTER(vp)]
    L.sim_adamw_step.argtypes = [vp, i64, C.c_float, C.c_float, i32, vp]
    L.sim_adamw_step_device.argtypes = [vp, vp, vp, C.c_float, i32, vp]
    L.sim_adamw_destroy.argtypes = [vp]
    L.sim_adamw_destroy.restype = None
    L.sim_set_adamw.argtypes = [vp, dbl, dbl, dbl, C.c_float]
    L.sim_eval_loss_mxfp4.argtypes = [vp, vp]
    L.sim_mx_codes_bytes.argtypes = [i64, i64]
    L.sim_mx_scales_bytes.argtypes = [i64, i64, i32]
    L.sim_mx_quantize.argtypes = [vp, C.c_int, i64, i64, i64, i32, i32, u64, vp, vp, vp, vp, vp]
    L.sim_mx_dequantize.argtypes = [vp, vp, i64, i64, i32, C.c_int, vp, i64, vp]
    L.sim_mx_matmul.argtypes = [vp, vp, vp, vp, i64, i64, i64, C.c_int, vp, i64, vp]
    L.sim_ckpt_codes_bytes.argtypes = [i64, i64]
    L.sim_ckpt_scales_bytes.argtypes = [i64, i64]
    L.sim_ckpt_write.argtypes = [vp, C.c_int, i64, i64, i64, vp, vp, vp]
    L.sim_ckpt_read.argtypes = [vp, vp, i64, i64, C.c_int, C.c_int, vp, i64, vp]
    L.sim_act_backward_workspace.argtypes = [i64, i64]
    L.sim_act_backward.argtypes = [vp, C.c_int, i64, i64, i64, vp, vp, C.c_int, vp, i64, vp, C.c_int, vp, i64, vp]
    L.sim_matmul_workspace.argtypes = [vp]           # a sim_product
    L.sim_matmul.argtypes = [vp, vp, i64, vp]
    L.sim_log_probs.argtypes = [vp, C.c_int, i64, i64, i64, vp, i32, C.c_float, i32] + [vp] * 8 + [i64, vp]
    L.sim_eval_log_probs.argtypes = [vp, i32, i64, i64, i32, vp, vp, vp, vp]
    sizes = ("sim_mx_codes_bytes", "sim_mx_scales_bytes", "sim_ckpt_codes_bytes", "sim_ckpt_scales_bytes", "sim_act_backward_workspace", "sim_matmul_workspace")
    for name in EXPORTS:
        if name not in ("sim_n_params", "sim_last_error", "sim_destroy", "sim_noalloc_last_error", "sim_adamw_destroy") + sizes:
            getattr(L, name).restype = C.c_int
    for name in sizes:
        getattr(L, name).restype = i64
    return L


lib = _load()


def _check(status, handle=None):
    if status != 0:
        msg = lib.sim_last_error(handle)
        raise SimError(status, msg.decode() if msg else "")


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream_ptr(stream):
    return None if stream is None else C.c_void_p(stream.cuda_stream)


_U16 = getattr(torch, "uint16")
_U32 = getattr(torch, "uint32")


class Simulation:
    """One handle of the library: n_replicas independent parameter servers on the current device.

    data: dict with model, X [n,d] float32 cuda, y (float32 targets or int32 labels) cuda,
    n_classes, hidden; w_ref optional cuda float32.  The tensors are borrowed by the library and
    kept alive by this object."""

    def __init__(self, data, *, P, K, variant, delay_kind, mu, shift=0.0, eta, m, seed, n_replicas,
                 replica_base=0, w_ref=None, stream=None):
        self._h = C.c_void_p()
        model = data["model"] if data is not None else "none"
        prob = SimProblem(MODELS[model], 0, 0, 0, 0, None, None, None, None)
        self._keep = []
        if model != "none":
            X, y = data["X"], data["y"]
            assert X.is_cuda and X.dtype == torch.float32 and X.is_contiguous()
            prob.n, prob.d = X.shape
            prob.n_classes, prob.hidden = int(data.get("n_classes", 1)), int(data.get("hidden", 0))
            prob.X = X.data_ptr()
            if model == "lsq":
                assert y.dtype == torch.float32 and y.is_cuda
                prob.y = y.data_ptr()
            else:
                assert y.dtype == torch.int32 and y.is_cuda
                prob.label = y.data_ptr()
            if w_ref is not None:
                assert w_ref.is_cuda and w_ref.dtype == torch.float32
                prob.w_ref = w_ref.data_ptr()
            self._keep = [X, y, w_ref]
        self.R, self.stream = n_replicas, stream
        self.device = torch.device("cuda", torch.cuda.current_device())
        _check(lib.sim_create(C.byref(prob), P, K, VARIANTS[variant], SimDelay(DELAYS[delay_kind], mu, shift),
                              eta, m, seed, n_replicas, replica_base, _stream_ptr(stream), C.byref(self._h)))

    def _new(self, shape, dtype):
        """Room for a result.  The handle's stream waits for the current one, which may still be reading that memory as a tensor that was let go."""
        t = torch.empty(shape, dtype=dtype, device=self.device)
        current, own = torch.cuda.current_stream(self.device), self.stream if self.stream is not None else torch.cuda.default_stream(self.device)
        if own != current:
            own.wait_stream(current)
        return t

    def set_params(self, w0):
        assert w0.is_cuda and w0.dtype == torch.float32 and w0.numel() == self.n_params
        _check(lib.sim_set_params(self._h, _ptr(w0)), self._h)

    def set_adasync(self, K0, t_interval):
        _check(lib.sim_set_adasync(self._h, K0, t_interval), self._h)

    def set_adasync_loss(self, K0, t_interval):
        """Algorithm 1 as printed: K follows the full-data risk at interval boundaries."""
        _check(lib.sim_set_adasync_loss(self._h, K0, t_interval), self._h)

    def set_adamw(self, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0):
        """AdamW with step size eta instead of the plain step as the server's update (least squares and logistic)."""
        _check(lib.sim_set_adamw(self._h, betas[0], betas[1], eps, weight_decay), self._h)

    def set_tuning(self, stages=0, tile_rows=0, threads=0):
        _check(lib.sim_set_tuning(self._h, stages, tile_rows, threads), self._h)

    def reserve(self, total_updates):
        _check(lib.sim_reserve(self._h, total_updates), self._h)

    def run(self, iters):
        _check(lib.sim_run(self._h, iters), self._h)

    @property
    def n_params(self):
        return int(lib.sim_n_params(self._h))

    def trace_size(self):
        J, Km = C.c_int64(), C.c_int32()
        _check(lib.sim_trace_size(self._h, C.byref(J), C.byref(Km)), self._h)
        return J.value, Km.value

    def trace(self, to_numpy=True):
        J, Km = self.trace_size()
        R = self.R
        out = {"t": self._new((R, J), torch.float64),
               "loss": self._new((R, J), torch.float32),
               "dist2": self._new((R, J), torch.float32),
               "K": self._new((R, J), _U16),
               "worker": self._new((R, J, Km), _U16),
               "stale": self._new((R, J, Km), _U32),
               "seq": self._new((R, J, Km), _U32)}
        _check(lib.sim_get_trace(self._h, *[_ptr(out[k]) for k in ("t", "loss", "dist2", "K", "worker", "stale", "seq")]),
               self._h)
        return {k: v.cpu().numpy() for k, v in out.items()} if to_numpy else out

    def params(self, to_numpy=True):
        w = self._new((self.R, self.n_params), torch.float32)
        _check(lib.sim_get_params(self._h, _ptr(w)), self._h)
        return w.cpu().numpy() if to_numpy else w

    def eval_loss(self, to_numpy=True, mxfp4=False):
        """Full-data risk F(w_j) of every replica's current parameters; mxfp4: with data and parameters in 4 bits."""
        out = self._new((self.R,), torch.float32)
        _check((lib.sim_eval_loss_mxfp4 if mxfp4 else lib.sim_eval_loss)(self._h, _ptr(out)), self._h)
        if self.stream is not None:
            self.stream.synchronize()
        else:
            torch.cuda.synchronize()
        return out.cpu().numpy() if to_numpy else out

    def log_probs(self, replica=0, first=0, rows=None, top=0, to_numpy=True):
        """What a replica's current parameters make of samples [first, first + rows) (default: all behind first) of the data set, softmax and MLP models: dict of
        logp (of the labels) and entropy [rows], and for top > 0 top_ids and top_logp [rows, top]."""
        rows = (self._keep[0].shape[0] if self._keep else 0) - first if rows is None else rows
        n = max(rows, 0)
        out = {"logp": self._new((n,), torch.float32), "entropy": self._new((n,), torch.float32)}
        if top > 0:
            out["top_ids"] = self._new((n, top), torch.int32)
            out["top_logp"] = self._new((n, top), torch.float32)
        _check(lib.sim_eval_log_probs(self._h, replica, first, rows, top, *[_ptr(out.get(k)) for k in ("logp", "entropy", "top_ids", "top_logp")]), self._h)
        if self.stream is not None:
            self.stream.synchronize()
        else:
            torch.cuda.synchronize()
        return {k: v.cpu().numpy() for k, v in out.items()} if to_numpy else out

    def error_curve(self, grid):
        """Mean minibatch loss over replicas against simulated wall clock at the times in `grid`."""
        g = torch.as_tensor(np.asarray(grid, np.float64)).to(self.device)
        mean = self._new((g.numel(),), torch.float32)
        cnt = self._new((g.numel(),), torch.int32)
        _check(lib.sim_error_curve(self._h, _ptr(g), g.numel(), _ptr(mean), _ptr(cnt)), self._h)
        return mean.cpu().numpy(), cnt.cpu().numpy()

    def set_eval_every(self, every):
        """Record the full-data risk of every replica before the first and after every `every`-th update."""
        _check(lib.sim_set_eval_every(self._h, every), self._h)

    def risk_trace(self, to_numpy=True):
        """(risk [R, E], t [R, E]): entry 0 is F(w_0) at time 0, entry i the risk after i * every updates."""
        E = C.c_int64()
        _check(lib.sim_risk_trace_size(self._h, C.byref(E)), self._h)
        risk = self._new((self.R, E.value), torch.float32)
        t = self._new((self.R, E.value), torch.float64)
        _check(lib.sim_get_risk_trace(self._h, _ptr(risk), _ptr(t)), self._h)
        return (risk.cpu().numpy(), t.cpu().numpy()) if to_numpy else (risk, t)

    def risk_curve(self, grid, f_star=0.0):
        """Mean over replicas of F(w) - f_star against simulated wall clock at the times in `grid`."""
        g = torch.as_tensor(np.asarray(grid, np.float64)).to(self.device)
        mean = self._new((g.numel(),), torch.float32)
        cnt = self._new((g.numel(),), torch.int32)
        _check(lib.sim_risk_curve(self._h, _ptr(g), g.numel(), f_star, _ptr(mean), _ptr(cnt)), self._h)
        return mean.cpu().numpy(), cnt.cpu().numpy()

    def selftest_wait_timeout(self):
        """Diagnostic: makes a bounded device-side wait run out on this handle (it is unusable afterwards)."""
        _check(lib.sim_selftest_wait_timeout(self._h), self._h)

    def close(self):
        if self._h:
            lib.sim_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def risk_envelope(sims, grid, f_star=0.0):
    """Lower envelope over several simulations' risk curves on a common grid: (env [G], best [G])."""
    dev = sims[0].device
    g = torch.as_tensor(np.asarray(grid, np.float64)).to(dev)
    env, best = sims[0]._new((g.numel(),), torch.float32), sims[0]._new((g.numel(),), torch.int32)
    hs = (C.c_void_p * len(sims))(*[s._h for s in sims])
    st = lib.sim_risk_envelope(hs, len(sims), _ptr(g), g.numel(), f_star, _ptr(env), _ptr(best))
    _check(st)
    return env.cpu().numpy(), best.cpu().numpy()


def draw_delays(delay_kind, mu, shift, seed, replica_base, n_replicas, P, n_seq):
    out = torch.empty((n_replicas, P, n_seq), dtype=torch.float64, device="cuda")
    _check(lib.sim_draw_delays(SimDelay(DELAYS[delay_kind], mu, shift), seed, replica_base, n_replicas, P, n_seq,
                               _ptr(out), _stream_ptr(torch.cuda.current_stream())))
    return out.cpu().numpy()


def draw_indices(seed, replica_base, n_replicas, P, n_seq, n, m):
    out = torch.empty((n_replicas, P, n_seq, m), dtype=_U32, device="cuda")
    _check(lib.sim_draw_indices(seed, replica_base, n_replicas, P, n_seq, n, m, _ptr(out),
                                _stream_ptr(torch.cuda.current_stream())))
    return out.cpu().numpy()


def schedule_noalloc(out, *, P, K, variant, delay_kind, mu, shift=0.0, seed, n_replicas, iters, replica_base=0,
                     K0=0, t_interval=0.0, stream=None):
    """Clock-only simulation through the entry point that allocates nothing: the caller brings
    the five output tensors (`out`: t, K, worker, stale, seq on the device, shaped as in
    Simulation.trace) because the library may not create them.  For callers that cannot call
    cudaMalloc; the worker state sits in a fixed array inside the library, so sizes are capped and
    calls on one device must not overlap."""
    Ks = P if t_interval > 0 else K
    need = {"t": (torch.float64, n_replicas * iters), "K": (_U16, n_replicas * iters),
            "worker": (_U16, n_replicas * iters * Ks), "stale": (_U32, n_replicas * iters * Ks),
            "seq": (_U32, n_replicas * iters * Ks)}
    for k, (dt, count) in need.items():     # the library writes through raw pointers: a wrong buffer would be an out-of-bounds write
        t = out[k]
        if not (t.is_cuda and t.is_contiguous() and t.dtype == dt and t.numel() >= count):
            raise ValueError("schedule_noalloc: out[%r] must be a contiguous CUDA tensor of %s with at least %d elements" % (k, dt, count))
    st = lib.sim_schedule_noalloc(P, K, VARIANTS[variant], SimDelay(DELAYS[delay_kind], mu, shift), seed,
                                  replica_base, n_replicas, K0, t_interval, iters,
                                  *[_ptr(out[k]) for k in ("t", "K", "worker", "stale", "seq")],
                                  _stream_ptr(stream))
    if st != 0:
        raise SimError(st, lib.sim_noalloc_last_error().decode())


def simulate_host(data, *, P, K, variant, delay_kind, mu, shift=0.0, eta, m, seed, n_replicas, iters,
                  replica_base=0, w0=None, w_ref=None, K0=0, t_interval=0.0, want=("t", "loss")):
    """The one-shot call on HOST numpy arrays (copies in, runs, copies the trace back)."""
    model = data["model"] if data is not None else "none"
    prob = SimProblem(MODELS[model], 0, 0, 0, 0, None, None, None, None)
    keep = []

    def hp(a, dt):
        if a is None:
            return None
        a = np.ascontiguousarray(a, dtype=dt)
        keep.append(a)
        return a.ctypes.data

    npar = 0
    if model != "none":
        prob.n, prob.d = data["X"].shape
        prob.n_classes, prob.hidden = int(data.get("n_classes", 1)), int(data.get("hidden", 0))
        prob.X = hp(data["X"], np.float32)
        if model == "lsq":
            prob.y = hp(data["y"], np.float32)
        else:
            prob.label = hp(data["y"], np.int32)
        prob.w_ref = hp(w_ref, np.float32)
        d, Cc, H = prob.d, prob.n_classes, prob.hidden
        npar = {"lsq": d, "logistic": d, "softmax": Cc * d, "mlp2": d * H + H + H * Cc + Cc}[model]
    Ks = P if t_interval > 0 else K
    R, J = n_replicas, iters
    shapes = {"t": ((R, J), np.float64), "loss": ((R, J), np.float32), "dist2": ((R, J), np.float32),
              "K": ((R, J), np.uint16), "worker": ((R, J, Ks), np.uint16), "stale": ((R, J, Ks), np.uint32),
              "seq": ((R, J, Ks), np.uint32), "w": ((R, npar), np.float32)}
    out = {k: np.empty(*shapes[k]) for k in want}
    ptrs = [C.c_void_p(out[k].ctypes.data) if k in out else None
            for k in ("t", "loss", "dist2", "K", "worker", "stale", "seq", "w")]
    w0p = hp(w0, np.float32)
    _check(lib.sim_simulate_host(C.byref(prob), P, K, VARIANTS[variant], SimDelay(DELAYS[delay_kind], mu, shift),
                                 eta, m, seed, n_replicas, replica_base, w0p, K0, t_interval, iters, *ptrs))
    return out


def sweep_host(data, runs, *, P, delay_kind, mu, shift=0.0, eta, m, seed, n_replicas, iters, replica_base=0, w0=None,
               w_ref=None, want=("t", "loss"), out=None):
    """All (variant, K) pairs of `runs` on one HOST data set in one call: the data is copied in once,
    the runs overlap on the device, the traces come back as [n_runs, R, iters] numpy arrays.  `out` may hold
    arrays to write into (for instance views of pinned memory): C-contiguous, of that shape, float64 for "t" and
    float32 for "loss" and "dist2"; missing ones are made here."""
    model = data["model"]
    prob = SimProblem(MODELS[model], 0, 0, 0, 0, None, None, None, None)
    keep = []

    def hp(a, dt):
        if a is None:
            return None
        a = np.ascontiguousarray(a, dtype=dt)
        keep.append(a)
        return a.ctypes.data

    prob.n, prob.d = data["X"].shape
    prob.n_classes, prob.hidden = int(data.get("n_classes", 1)), int(data.get("hidden", 0))
    prob.X = hp(data["X"], np.float32)
    if model == "lsq":
        prob.y = hp(data["y"], np.float32)
    else:
        prob.label = hp(data["y"], np.int32)
    prob.w_ref = hp(w_ref, np.float32)
    variants = np.array([VARIANTS[v] for v, _ in runs], np.int32)
    Ks = np.array([k for _, k in runs], np.int32)
    shape = (len(runs), n_replicas, iters)
    dtypes = {"t": np.float64, "loss": np.float32, "dist2": np.float32}
    given, out = out or {}, {}
    for k in want:
        a = given.get(k)
        if a is None:
            a = np.empty(shape, dtypes[k])
        elif a.shape != shape or a.dtype != dtypes[k] or not a.flags["C_CONTIGUOUS"] or not a.flags["WRITEABLE"]:
            raise ValueError("out[%r] must be a writeable C-contiguous %s array of shape %r" % (k, np.dtype(dtypes[k]).name, shape))
        out[k] = a
    ptrs = [C.c_void_p(out[k].ctypes.data) if k in out else None for k in ("t", "loss", "dist2")]
    _check(lib.sim_sweep_host(C.byref(prob), P, len(runs), C.c_void_p(variants.ctypes.data), C.c_void_p(Ks.ctypes.data),
                              SimDelay(DELAYS[delay_kind], mu, shift), eta, m, seed, n_replicas, replica_base,
                              hp(w0, np.float32), iters, *ptrs))
    return out


# ---- operators of a parameter server for models of language-model size ---------------------------------------------------
# A call with stream=None works on the device's current stream.  With a stream given, results belong to it, and what other streams
# have to do before the call, or with its results, the caller orders (wait_stream, events).
class MxTensor:
    """A matrix [rows, cols] in MXFP4: E2M1 codes (two a byte, even element in the low half, rows padded to 128 elements) and
    a power-of-two scale byte per block of 32 elements of a row.  layout "linear": scale bytes [rows, ceil(cols / 32)]; a
    single row is also the form of a pushed gradient.  layout "tiles": the order the products read, 512 bytes per 128 rows x
    4 blocks (row r of a tile at byte 16 (r % 32) + 4 (r / 32)); the bytes of blocks behind a row's last may be anything but 0xFF.
    codes and scales are flat uint8 tensors."""

    __slots__ = ("rows", "cols", "layout", "device", "codes_ptr", "scales_ptr", "_codes", "_scales", "_buffer")

    def __init__(self, codes, scales, rows, cols, layout):
        if layout not in ("linear", "tiles"):
            raise ValueError("layout must be 'linear' or 'tiles'")
        need_c, need_s = _mx_bytes(rows, cols, layout)
        if rows == 1 and layout == "linear":
            need_c = -(-cols // 2)
        for name, t, need in (("codes", codes, need_c), ("scales", scales, need_s)):
            if t.dtype != torch.uint8 or not t.is_cuda or not t.is_contiguous() or t.numel() < need or t.device != codes.device:
                raise ValueError("%s must be a contiguous CUDA uint8 tensor of at least %d bytes, on one device" % (name, need))
        self._codes, self._scales, self._buffer = codes, scales, None
        self.rows, self.cols, self.layout, self.device = rows, cols, layout, codes.device
        self.codes_ptr, self.scales_ptr = codes.data_ptr(), scales.data_ptr()

    @classmethod
    def empty(cls, rows, cols, layout, device):
        """Uninitialised, codes and scales in one buffer that belongs to the device's current stream."""
        self = cls.__new__(cls)
        nc, ns = _mx_bytes(rows, cols, layout)
        self._buffer = buf = torch.empty_strided((nc + ns,), (1,), dtype=torch.uint8, device=device)
        self._codes = self._scales = None
        self.rows, self.cols, self.layout, self.device = rows, cols, layout, buf.device
        self.codes_ptr = buf.data_ptr()
        self.scales_ptr = self.codes_ptr + nc
        return self

    def record_stream(self, stream):
        """As of a tensor: the memory is not given to others before what `stream` has been given so far is done."""
        for t in (self._buffer,) if self._buffer is not None else (self._codes, self._scales):
            t.record_stream(stream)

    @property
    def codes(self):
        if self._codes is None:
            self._codes = self._buffer[:self.scales_ptr - self.codes_ptr]
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            self._scales = self._buffer[self.scales_ptr - self.codes_ptr:]
        return self._scales


def _mx_bytes(rows, cols, layout):
    """Bytes of codes (a multiple of 64) and of scales, as sim_mx_codes_bytes and sim_mx_scales_bytes give them."""
    kb = (cols + 127) // 128
    return rows * 64 * kb, (rows + 127) // 128 * kb * 512 if layout == "tiles" else rows * ((cols + 31) // 32)


# the raw stream of a device without a Stream object around it, where torch offers that (2 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_NO_STREAM = contextlib.nullcontext()


def _given(stream, device, *used):
    """A context in which new buffers belong to `stream`, which works on `used` too: memory that the caller gives back right after a call is
    not handed on before `stream` is done with it."""
    if stream.device != device:
        raise ValueError("the stream is one of %s, the buffers are on %s" % (stream.device, device))
    for t in used:
        t.record_stream(stream)
    return torch.cuda.stream(stream)


def _empty(rows, cols, dtype, device, stream):
    """A new matrix (with strides given torch takes 0.8 us less than torch.empty does)."""
    if stream is None:
        return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)


def _on(device, stream, call, *args):
    """call(*args, stream) with `device` current; stream None: the device's current one."""
    index = device.index
    st = _raw_stream(index) if stream is None else stream.cuda_stream
    if _current_device() == index:
        return call(*args, st)
    with torch.cuda.device(index):
        return call(*args, st)


def _ptr_array(pointers):
    return (C.c_void_p * len(pointers))(*pointers)


class AdamW:
    """AdamW over a list of tensors, stepped by the library in one launch per combination of types.

    params: CUDA tensors (float32 or bfloat16), updated in place.  grads: one list per push, each with a gradient per
    parameter - tensors (float32, bfloat16, float16) or MxTensor of one row in the linear layout; a step averages the first K
    pushes.  weight_decay: a number, or one per parameter.  state_bits 32 keeps fp32 moments, 8 keeps E4M3 codes of m and
    sqrt(v) with a scale per 32 elements.  state: dict of lists ("m", "v"; 8 bits also "m_scale", "v_scale") to work on
    instead of fresh zeros.  shadow: optional bfloat16 copies written each step.  All tensors are borrowed, contiguous and on
    one device, must not overlap, and must stay at their addresses; this object keeps them alive."""

    def __init__(self, params, grads, *, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, state=None, shadow=None,
                 seed=0):
        self._h = C.c_void_p()
        params, grads = list(params), [list(g) for g in grads]
        if not params or not grads or any(len(g) != len(params) for g in grads):
            raise ValueError("params and at least one push with a gradient per parameter are required")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 32 or 8")
        self.device, self.n_grads, self.state_bits = params[0].device, len(grads), state_bits
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(params)
        kinds = ("m", "v") if state_bits == 32 else ("m", "v", "m_scale", "v_scale")
        if state is None:
            dt = torch.float32 if state_bits == 32 else torch.uint8
            fresh = torch.cuda.current_stream(self.device) if self.device.type == "cuda" else None
            state = {k: [torch.zeros(-(-p.numel() // 32) if k.endswith("scale") else p.numel(), dtype=dt, device=self.device) for p in params] for k in kinds}
            if fresh is not None:
                fresh.synchronize()          # the first step may run on any stream
        if len(decay) != len(params) or (shadow is not None and len(shadow) != len(params)) or any(k not in state or len(state[k]) != len(params) for k in kinds):
            raise ValueError("weight_decay, shadow and every list of state need one entry per parameter")

        def check(t, dtypes, n, what, i):
            if not t.is_cuda or t.device != self.device or not t.is_contiguous() or t.dtype not in dtypes or t.numel() != n:
                raise ValueError("%s of parameter %d must be a contiguous tensor of %d elements on %s, of type %s" % (
                    what, i, n, self.device, " or ".join(str(d) for d in dtypes)))
            return t.data_ptr()

        recs, keep = (SimAdamwTensor * len(params))(), []
        for i, p in enumerate(params):
            n = p.numel()
            check(p, (torch.float32, torch.bfloat16), n, "the data", i)
            r = recs[i]
            r.n, r.p_type, r.p, r.weight_decay = n, DTYPES[p.dtype], p.data_ptr(), float(decay[i])
            mine = [g[i] for g in grads]
            if isinstance(mine[0], MxTensor):
                for q in mine:
                    if not isinstance(q, MxTensor) or q.rows != 1 or q.cols != n or q.layout != "linear" or q.device != self.device:
                        raise ValueError("the gradients of parameter %d must all be MxTensor of one row of %d elements, linear layout, on %s" % (i, n, self.device))
                r.g_type = MXFP4
                arrays = _ptr_array([q.codes_ptr for q in mine]), _ptr_array([q.scales_ptr for q in mine])
                r.g_scale = C.cast(arrays[1], C.POINTER(C.c_void_p))
            else:
                if any(isinstance(g, MxTensor) or g.dtype != mine[0].dtype for g in mine):
                    raise ValueError("the gradients of parameter %d must have one type" % i)
                arrays = (_ptr_array([check(g, tuple(DTYPES), n, "a gradient", i) for g in mine]),)
                r.g_type = DTYPES[mine[0].dtype]
            r.g = C.cast(arrays[0], C.POINTER(C.c_void_p))
            keep.append(arrays)
            codes = (torch.float32,) if state_bits == 32 else (torch.uint8, torch.float8_e4m3fn)
            r.m, r.v = check(state["m"][i], codes, n, "m", i), check(state["v"][i], codes, n, "v", i)
            if state_bits == 8:
                r.m_scale = check(state["m_scale"][i], (torch.uint8,), -(-n // 32), "m_scale", i)
                r.v_scale = check(state["v_scale"][i], (torch.uint8,), -(-n // 32), "v_scale", i)
            if shadow is not None and shadow[i] is not None:
                r.shadow = check(shadow[i], (torch.bfloat16,), n, "shadow", i)
        self.params, self.grads, self.state, self.shadow = params, grads, state, shadow
        with torch.cuda.device(self.device):
            _check(lib.sim_adamw_create(recs, len(params), len(grads), state_bits, betas[0], betas[1], eps, seed, C.byref(self._h)))

    def step(self, step, lr, *, K=None, grad_scale=1.0, stream=None):
        """Step number `step` (1, 2, ...) with learning rate lr and the average of the first K pushes (default: all), on
        `stream` (default: the device's current one).  step and lr may both be CUDA tensors of one element (int64, float32):
        they are read when the step runs, for steps captured in a graph."""
        if stream is not None:
            _given(stream, self.device, *(t for t in (step, lr) if torch.is_tensor(t) and t.is_cuda))
        st = _raw_stream(self.device.index) if stream is None else stream.cuda_stream
        K = self.n_grads if K is None else K
        if torch.is_tensor(step) or torch.is_tensor(lr):
            for t, dt in ((step, torch.int64), (lr, torch.float32)):
                if not torch.is_tensor(t) or t.device != self.device or t.dtype != dt or t.numel() != 1:
                    raise ValueError("step and lr must both be numbers, or CUDA tensors of one int64 and one float32 on %s" % self.device)
            _check(lib.sim_adamw_step_device(self._h, step.data_ptr(), lr.data_ptr(), grad_scale, K, st))
        else:
            _check(lib.sim_adamw_step(self._h, step, lr, grad_scale, K, st))

    def close(self):
        """Frees the tables; a graph that holds steps of this object must not be replayed after it."""
        if self._h:
            lib.sim_adamw_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _matrix(x, what):
    """A CUDA tensor of one or two dimensions with neighbouring elements along the last -> (rows, cols, elements between rows)."""
    if not x.is_cuda or x.dtype not in DTYPES or x.dim() not in (1, 2) or x.numel() == 0:
        raise ValueError("%s must be a CUDA tensor of float32, bfloat16 or float16 with one or two dimensions and at least one element" % what)
    rows, cols = (1, x.shape[0]) if x.dim() == 1 else x.shape
    if (cols > 1 and x.stride(-1) != 1) or (rows > 1 and x.stride(0) < cols):
        raise ValueError("%s must have neighbouring elements along its last dimension and rows that do not overlap" % what)
    return rows, cols, x.stride(0) if rows > 1 else cols


def mx_quantize(x, *, along="rows", rounding="nearest", seed=0, layout="tiles", stream=None):
    """MXFP4 form of a matrix (or vector: one row).  along "rows" -> MxTensor [rows, cols]; "cols" -> MxTensor [cols, rows] with
    blocks along x's columns; "both" -> the two from one read.  rounding "nearest" (even) or "stochastic" (from `seed`)."""
    if along not in ("rows", "cols", "both") or rounding not in ("nearest", "stochastic") or layout not in ("linear", "tiles"):
        raise ValueError("along: rows, cols or both; rounding: nearest or stochastic; layout: linear or tiles")
    rows, cols, ld = _matrix(x, "x")
    device = x.device
    with _NO_STREAM if stream is None else _given(stream, device, x):
        q = MxTensor.empty(rows, cols, layout, device) if along != "cols" else None
        qt = MxTensor.empty(cols, rows, layout, device) if along != "rows" else None
    _check(_on(device, stream, lib.sim_mx_quantize, x.data_ptr(), DTYPES[x.dtype], rows, cols, ld, layout == "tiles", rounding == "stochastic", seed,
               q and q.codes_ptr, q and q.scales_ptr, qt and qt.codes_ptr, qt and qt.scales_ptr))
    return (q, qt) if along == "both" else q if qt is None else qt


def mx_dequantize(q, dtype=torch.float32, *, out=None, stream=None):
    """The values of an MxTensor as a matrix [rows, cols] of dtype (float32, bfloat16, float16), or into `out`."""
    if stream is not None:
        _given(stream, q.device, q)
    if out is None:
        if dtype not in DTYPES:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        out, rows, cols, ld = _empty(q.rows, q.cols, dtype, q.device, stream), q.rows, q.cols, q.cols
    else:
        rows, cols, ld = _matrix(out, "out")
        if (rows, cols) != (q.rows, q.cols) or out.device != q.device:
            raise ValueError("out must be [%d, %d] on %s" % (q.rows, q.cols, q.device))
        if stream is not None:
            _given(stream, q.device, out)
    _check(_on(q.device, stream, lib.sim_mx_dequantize, q.codes_ptr, q.scales_ptr, rows, cols, q.layout == "tiles", DTYPES[out.dtype], out.data_ptr(), ld))
    return out


def mx_matmul(a, b, dtype=torch.bfloat16, *, out=None, stream=None):
    """a b^T [a.rows, b.rows] of two MxTensors with as many columns, layout "tiles", as bfloat16 or float32, or into `out`."""
    if a.cols != b.cols or a.layout != "tiles" or b.layout != "tiles" or a.device != b.device:
        raise ValueError("both operands need the same number of columns, the layout 'tiles' and one device")
    if stream is not None:
        _given(stream, a.device, a, b)
    if out is None:
        if dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("dtype must be bfloat16 or float32")
        out, ld = _empty(a.rows, b.rows, dtype, a.device, stream), b.rows
    else:
        rows, cols, ld = _matrix(out, "out")
        if (rows, cols) != (a.rows, b.rows) or out.device != a.device or out.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("out must be [%d, %d] of bfloat16 or float32 on %s" % (a.rows, b.rows, a.device))
        if stream is not None:
            _given(stream, a.device, out)
    _check(_on(a.device, stream, lib.sim_mx_matmul, a.codes_ptr, a.scales_ptr, b.codes_ptr, b.scales_ptr, a.rows, b.rows, a.cols, DTYPES[out.dtype], out.data_ptr(), ld))
    return out


# ---- operators of a worker for models of language-model size --------------------------------------------------------------
# Results stand outside torch's graph, whether or not an operand requires a gradient: the backward passes are calls of their own (linear_backward, act_backward,
# log_probs_backward).
class Checkpoint:
    """A matrix [rows, cols] kept in 8 bits: E4M3 codes in rows of 32 ceil(cols / 32) bytes and a power-of-two scale byte per block of 32
    elements of a row, [rows, ceil(cols / 32)].  codes (16-byte aligned) and scales are flat uint8 tensors."""

    __slots__ = ("rows", "cols", "device", "codes_ptr", "scales_ptr", "_codes", "_scales", "_buffer")

    def __init__(self, codes, scales, rows, cols):
        need_c, need_s = _ckpt_bytes(rows, cols)
        for name, t, need in (("codes", codes, need_c), ("scales", scales, need_s)):
            if t.dtype != torch.uint8 or not t.is_cuda or not t.is_contiguous() or t.numel() < need or t.device != codes.device:
                raise ValueError("%s must be a contiguous CUDA uint8 tensor of at least %d bytes, on one device" % (name, need))
        self._codes, self._scales, self._buffer = codes, scales, None
        self.rows, self.cols, self.device = rows, cols, codes.device
        self.codes_ptr, self.scales_ptr = codes.data_ptr(), scales.data_ptr()

    @classmethod
    def empty(cls, rows, cols, device):
        """Uninitialised, codes and scales in one buffer that belongs to the device's current stream."""
        self = cls.__new__(cls)
        nc, ns = _ckpt_bytes(rows, cols)
        self._buffer = buf = torch.empty_strided((nc + ns,), (1,), dtype=torch.uint8, device=device)
        self._codes = self._scales = None
        self.rows, self.cols, self.device = rows, cols, buf.device
        self.codes_ptr = buf.data_ptr()
        self.scales_ptr = self.codes_ptr + nc
        return self

    def record_stream(self, stream):
        """As of a tensor: the memory is not given to others before what `stream` has been given so far is done."""
        for t in (self._buffer,) if self._buffer is not None else (self._codes, self._scales):
            t.record_stream(stream)

    @property
    def codes(self):
        return self._buffer[:self.scales_ptr - self.codes_ptr] if self._codes is None else self._codes[:self.rows * (-(-self.cols // 32) * 32)]

    @property
    def scales(self):
        return self._buffer[self.scales_ptr - self.codes_ptr:] if self._scales is None else self._scales[:self.rows * -(-self.cols // 32)]


def _ckpt_bytes(rows, cols):
    """Bytes of codes and of scales, as sim_ckpt_codes_bytes and sim_ckpt_scales_bytes give them."""
    blocks = -(-cols // 32)
    return rows * 32 * blocks, rows * blocks


def _act_code(name):
    if name not in ACTS:
        raise ValueError("an activation is one of %s" % ", ".join(ACTS))
    return ACTS[name]


_ALL, _HALF = tuple(DTYPES), (torch.bfloat16, torch.float16)


def _plain(x, what, dtypes=_ALL):
    """A CUDA matrix (or vector: one row), possibly without elements, neighbours along the last dimension -> (rows, cols, elements between rows)."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in dtypes or x.dim() not in (1, 2):
        raise ValueError("%s must be a CUDA tensor of %s with one or two dimensions" % (what, " or ".join(str(d)[6:] for d in dtypes)))
    if x.dim() == 2:
        rows, cols = x.shape
        ld, step = x.stride()
    else:
        (cols,), (step,), rows, ld = x.shape, x.stride(), 1, 0
    if rows <= 1 or cols == 0:
        ld = cols
    if (step != 1 and cols > 1 and rows) or ld < cols:
        raise ValueError("%s must have neighbouring elements along its last dimension and rows that do not overlap" % what)
    return rows, cols, ld


def _same(device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError("all tensors must be on %s" % device)


def _result(out, rows, cols, dtypes, device, stream, what="out"):
    """(out or a new matrix of the first of dtypes, its row distance)"""
    if out is None:
        return _empty(rows, cols, dtypes[0], device, stream), cols
    r, c, ld = _plain(out, what, dtypes)
    if (r, c) != (rows, cols) or out.device != device:
        raise ValueError("%s must be [%d, %d] on %s" % (what, rows, cols, device))
    if stream is not None:
        _given(stream, device, out)
    return out, ld


def checkpoint(x, *, stream=None):
    """The 8-bit form of a matrix (or vector: one row) of float32, bfloat16 or float16."""
    rows, cols, ld = _plain(x, "x")
    device = x.device
    if stream is None:
        q = Checkpoint.empty(rows, cols, device)
    else:
        with _given(stream, device, x):
            q = Checkpoint.empty(rows, cols, device)
    _check(_on(device, stream, lib.sim_ckpt_write, x.data_ptr(), DTYPES[x.dtype], rows, cols, ld, q.codes_ptr, q.scales_ptr))
    return q


def checkpoint_read(q, dtype=torch.bfloat16, *, act="none", out=None, stream=None):
    """act of the values of a Checkpoint as a matrix [rows, cols] of dtype (float32, bfloat16, float16), or into `out`."""
    code = _act_code(act)
    if out is None and dtype not in DTYPES:
        raise ValueError("dtype must be float32, bfloat16 or float16")
    if stream is not None:
        _given(stream, q.device, q)
    out, ld = _result(out, q.rows, q.cols, (dtype,) if out is None else tuple(DTYPES), q.device, stream)
    _check(_on(q.device, stream, lib.sim_ckpt_read, q.codes_ptr, q.scales_ptr, q.rows, q.cols, code, DTYPES[out.dtype], out.data_ptr(), ld))
    return out


def _scratch(nbytes, device, stream):
    """Room that a call uses until it is done (None for none)."""
    if nbytes == 0:
        return None
    if stream is None:
        return torch.empty_strided((nbytes,), (1,), dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty_strided((nbytes,), (1,), dtype=torch.uint8, device=device)


def _pitch(cols):
    return -(-cols // 8) * 8 if cols <= 64 else -(-cols // 64) * 64


def _padded(rows, cols, dtype, device, stream):
    """(a matrix whose rows start on 16-byte boundaries, and on lines where they are longer than one, the elements between them)"""
    ld = _pitch(cols)
    with _NO_STREAM if stream is None else torch.cuda.stream(stream):
        return torch.empty_strided((rows, cols), (ld, 1), dtype=dtype, device=device), ld


def _sums(dy, rows, cols, ld, z, code, dz, lddz, db, device, stream):
    room = lib.sim_act_backward_workspace(rows, cols) if db is not None and rows > 256 else 0      # few rows need none
    ws = _scratch(room, device, stream)
    _check(_on(device, stream, lib.sim_act_backward, dy.data_ptr(), DTYPES[dy.dtype], rows, cols, ld, z and z.codes_ptr, z and z.scales_ptr, code,
               None if dz is None else dz.data_ptr(), lddz, None if db is None else db.data_ptr(), 0 if db is None else DTYPES[db.dtype],
               None if ws is None else ws.data_ptr(), room))


def _vector(out, n, dtypes, device, stream, what):
    if out is None:
        with _NO_STREAM if stream is None else torch.cuda.stream(stream):
            return torch.empty_strided((n,), (1,), dtype=dtypes[0], device=device)
    if not out.is_cuda or out.device != device or out.dtype not in dtypes or out.dim() != 1 or out.numel() != n or not out.is_contiguous():
        raise ValueError("%s must be a contiguous vector of %d on %s" % (what, n, device))
    if stream is not None:
        _given(stream, device, out)
    return out


def act_backward(dy, z, act, *, bias=True, dtype=torch.float32, out=None, stream=None):
    """(dz, db): dz = dy act'(z) in dy's type for a Checkpoint z of an activation's argument, db its sums over the rows (of dz before it is
    rounded) as a vector of dtype, or None without `bias`.  out: (dz, db) to write into, either may be None; dz may be dy."""
    code = _act_code(act)
    rows, cols, ld = _plain(dy, "dy")
    device = dy.device
    if not isinstance(z, Checkpoint) or (z.rows, z.cols) != (rows, cols) or z.device != device:
        raise ValueError("z must be a Checkpoint [%d, %d] on %s" % (rows, cols, device))
    if dtype not in DTYPES:
        raise ValueError("dtype must be float32, bfloat16 or float16")
    if stream is not None:
        _given(stream, device, dy, z)
    dz, db = out or (None, None)
    dz, lddz = _result(dz, rows, cols, (dy.dtype,), device, stream, "dz")
    db = _vector(db, cols, (dtype,) if db is None else tuple(DTYPES), device, stream, "db") if bias else None
    _sums(dy, rows, cols, ld, z, code, dz, lddz, db, device, stream)
    return dz, db


def _side(x, what, dtypes=_HALF):
    """An operand of a product, its rows along either dimension -> (rows, cols, elements between its rows in memory, whether those lie along the
    first dimension's neighbours)."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in dtypes or x.dim() not in (1, 2):
        raise ValueError("%s must be a CUDA tensor of %s with one or two dimensions" % (what, " or ".join(str(d)[6:] for d in dtypes)))
    if x.dim() == 2:
        rows, cols = x.shape
        ld, step = x.stride()
    else:
        (cols,), (step,), rows, ld = x.shape, x.stride(), 1, 0
    if rows == 0 or cols == 0:
        return rows, cols, cols, False
    if step == 1 or cols == 1:
        if rows == 1:
            return rows, cols, cols, False
        if ld >= cols:
            return rows, cols, ld, False
    if (ld == 1 or rows == 1) and step >= rows:
        return rows, cols, step, True
    raise ValueError("%s must have neighbouring elements along one dimension, and the others must not overlap" % what)


_PRODUCT = struct.Struct("@qqqiPqiPqiPiiiPPPqPiq")          # a sim_product; made in half the time of SimProduct
assert _PRODUCT.size == C.sizeof(SimProduct)


def _room(p, ld, t, along, k):
    """What sim_matmul_workspace counts for an operand: nothing where its rows in memory start on 16-byte boundaries, else their copy."""
    rows, cols = (k, along) if t else (along, k)
    return 0 if p & 15 == 0 and (rows <= 1 or ld & 7 == 0) else (rows * _pitch(cols) * 2 + 255) // 256 * 256


def _product(device, stream, M, N, K, dtype, a, lda, a_t, b, ldb, b_t, c, ldc, bias=None, act=0, act_grad=False, z=None, residual=None, ldr=0):
    p = _PRODUCT.pack(M, N, K, DTYPES[dtype], a, lda, a_t, b, ldb, b_t, *((0, 0) if bias is None else (bias.data_ptr(), DTYPES[bias.dtype])), act, act_grad,
                      *((0, 0) if z is None else (z.codes_ptr, z.scales_ptr)), 0 if residual is None else residual.data_ptr(), ldr, c.data_ptr(), DTYPES[c.dtype], ldc)
    room = 0 if (a | b | (lda | ldb) * 2) & 15 == 0 else _room(a, lda, a_t, M, K) + _room(b, ldb, b_t, N, K)
    ws = _scratch(room, device, stream)
    _check(_on(device, stream, lib.sim_matmul, p, None if ws is None else ws.data_ptr(), room))


def linear(x, w, bias=None, *, act="none", residual=None, keep=False, dtype=None, out=None, stream=None):
    """act(x w^T + bias) + residual as [tokens, out] for x [tokens, in] (or one token: [in]) and w [out, in], both bfloat16 or both float16, with
    either of their dimensions in memory's order.  bias [out]: float32 or the operands' type.  The result (dtype, or `out`) has the
    operands' type or float32, and so has the residual.  keep: (result, Checkpoint of x w^T + bias), for the backward pass."""
    code = _act_code(act)
    M, K, lda, a_t = _side(x, "x")
    kind = x.dtype
    N, Kw, ldb, b_t = _side(w, "w", (kind,))
    device = x.device
    if K != Kw:
        raise ValueError("x and w must have as many columns")
    kinds = (kind, torch.float32)
    if (out.dtype if out is not None else dtype or kind) not in kinds:
        raise ValueError("the result is float32 or of the operands' type")
    _same(device, w, bias, residual)
    if bias is not None and (bias.dtype not in kinds or bias.dim() != 1 or bias.numel() != N or (N > 1 and bias.stride(0) != 1)):
        raise ValueError("bias must be a contiguous vector of %d of float32 or the operands' type" % N)
    if stream is not None:
        _given(stream, device, *(t for t in (x, w, bias, residual) if t is not None))
    if out is None:
        out, ldc = _empty(M, N, dtype or kind, device, stream), N
    else:
        out, ldc = _result(out, M, N, kinds, device, stream)
    ldr = 0
    if residual is not None:
        r, c, ldr = _plain(residual, "residual", (out.dtype,))
        if (r, c) != (M, N):
            raise ValueError("residual must be [%d, %d]" % (M, N))
    z = None
    if keep:
        with _NO_STREAM if stream is None else torch.cuda.stream(stream):
            z = Checkpoint.empty(M, N, device)
    _product(device, stream, M, N, K, kind, x.data_ptr(), lda, a_t, w.data_ptr(), ldb, b_t, out, ldc, bias, code, False, z, residual, ldr)
    return (out, z) if keep else out


def _span(t):
    """(first byte, behind the last, bytes between rows, bytes of a row) of a matrix or vector that has neighbours along its last dimension or its first."""
    eb = t.element_size()
    (ld, cols), last = max(zip(t.stride(), reversed(t.shape))) if t.dim() == 2 else (0, 0), sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1
    return t.data_ptr(), t.data_ptr() + last * eb, ld * eb, cols * eb


def _apart(written, others, what):
    if written is None or written.numel() == 0:
        return
    lo, hi, pitch, width = _span(written)
    for t in others:
        if t is not None and t.numel() and t.device == written.device:
            a, b, p, w = _span(t)
            between = p == pitch > 0 and width <= (a - lo) % p <= p - w           # column slices of one buffer
            if a < hi and lo < b and not between:
                raise ValueError("%s overlaps a tensor that is still to be read, or another result" % what)


def _results_apart(need, dy, x, w, residual, grad, dx, dw, db):
    """Refuses results of linear_backward that lie over what is still to be read: db, dx, dw are written in this order.  A Checkpoint's buffers count as the tensor that it
    stands for; dx takes them too where the activation's slope is in it (grad)."""
    kept = isinstance(x, Checkpoint)
    values = [x.codes, x.scales] if kept else [x]
    for_dw = values if "w" in need else []
    left = ([dy] if "x" in need or "w" in need else []) + ([w, residual] if "x" in need else []) + (for_dw or (values if grad and "x" in need else []))
    _apart(db if "b" in need else None, left, "db")
    _apart(dx if "x" in need else None, for_dw + ([db] if "b" in need else []), "dx")
    _apart(dw if "w" in need else None, [t for n, t in (("x", dx), ("b", db)) if n in need], "dw")


def linear_backward(dy, x, w, *, x_act="none", residual=None, need="xwb", dtype=torch.float32, out=None, stream=None):
    """(dx, dw, db) of linear(x, w, bias) from dy [tokens, out], w [out, in] and x: the tensor [tokens, in] itself, or a Checkpoint.  With a
    Checkpoint v the layer's input was x_act(v) and is taken as x_act of the kept values, rounded to dy's type; dx is then the gradient by v,
    (dy w) x_act'(v).  residual [tokens, in]: added to dx (the gradient that reached the input another way).  dx has dy's type, dw [out, in]
    and db [out] have dtype (float32 or dy's).  dx and dw take dy and w with either dimension in memory's order, db dy with its last.  need: which of them ("x", "w", "b"); the others are None.  out: (dx, dw, db) to write
    into, each may be None; none may lie over a tensor, or a Checkpoint's buffers, that another of the three still needs."""
    code = _act_code(x_act)
    M, N, lda, a_t = _side(dy, "dy")
    Nw, K, ldb, b_t = _side(w, "w", (dy.dtype,))
    device = dy.device
    kept = isinstance(x, Checkpoint)
    if kept:
        Mx, Kx = x.rows, x.cols
    else:
        Mx, Kx, ldx, x_t = _side(x, "x", (dy.dtype,))
        if code:
            raise ValueError("x_act belongs to a Checkpoint: a tensor x is the layer's input itself")
    if Nw != N or Mx != M or Kx != K or x.device != device:
        raise ValueError("dy [%d, %d], w [%d, %d] and x [%d, %d] do not belong together, or are on several devices" % (M, N, Nw, K, Mx, Kx))
    _same(device, w, residual)
    kinds = (dy.dtype, torch.float32)
    if dtype not in kinds or not need or any(n not in "xwb" for n in need):
        raise ValueError("dtype is float32 or dy's, need is made of x, w and b")
    if stream is not None:
        _given(stream, device, *(t for t in (dy, x, w, residual) if t is not None))
    dx, dw, db = out or (None, None, None)
    if out:
        _results_apart(need, dy, x, w, residual, kept and code != 0, dx, dw, db)
    if "b" in need:
        if a_t:
            raise ValueError("db needs dy with neighbouring elements along its last dimension")
        db = _vector(db, N, (dtype,) if db is None else tuple(DTYPES), device, stream, "db")
        copy = None
        if (dy.data_ptr() | lda * 2) & 15 and len(need) > 1:       # the products want rows on 16-byte boundaries: copied on the way
            copy, ldd = _padded(M, N, dy.dtype, device, stream)
        _sums(dy, M, N, lda, None, 0, copy, 0 if copy is None else ldd, db, device, stream)
        if copy is not None:
            dy, lda = copy, ldd
    if "x" in need:
        dx, ldc = _result(dx, M, K, (dy.dtype,), device, stream, "dx")
        ldr = 0
        if residual is not None:
            r, c, ldr = _plain(residual, "residual", (dy.dtype,))
            if (r, c) != (M, K):
                raise ValueError("residual must be [%d, %d]" % (M, K))
        grad = kept and code != 0
        _product(device, stream, M, K, N, dy.dtype, dy.data_ptr(), lda, a_t, w.data_ptr(), ldb, not b_t, dx, ldc, act=code if grad else 0, act_grad=grad,
                 z=x if grad else None, residual=residual, ldr=ldr)
    if "w" in need:
        dw, ldc = _result(dw, N, K, (dtype,) if dw is None else kinds, device, stream, "dw")
        if kept:
            h, ldx = _padded(M, K, dy.dtype, device, stream)
            x_t = False
            _check(_on(device, stream, lib.sim_ckpt_read, x.codes_ptr, x.scales_ptr, M, K, code, DTYPES[dy.dtype], h.data_ptr(), ldx))
        else:
            h = x
        _product(device, stream, N, K, M, dy.dtype, dy.data_ptr(), lda, not a_t, h.data_ptr(), ldx, not x_t, dw, ldc)
    return dx if "x" in need else None, dw if "w" in need else None, db if "b" in need else None


LogProbs = collections.namedtuple("LogProbs", "logp entropy lse top_ids top_logp dlogits")


def log_probs(logits, tokens=None, *, top=0, temperature=1.0, d_logp=None, d_entropy=None, out=None, stream=None):
    """Of logits [rows, vocab] (float32, bfloat16, float16; one row: [vocab]) divided by temperature: a LogProbs with float32 vectors logp (of tokens
    [rows], int64 or int32; 0 where a token is negative; None without tokens), entropy and lse, and for top > 0 the `top` likeliest
    alternatives of each row: top_ids int32 and top_logp float32 [rows, top], the lower index first among equals.  With d_logp or
    d_entropy (float32 [rows]: the derivatives of a loss by logp and entropy) also dlogits, the loss' gradient by the logits in their type,
    in `out` where given (which may be logits itself)."""
    rows, vocab, ld, device, tb = _logits(logits, tokens, d_logp, d_entropy)
    grad = d_logp is not None or d_entropy is not None
    if out is not None and not grad:
        raise ValueError("out takes the gradient, which needs d_logp or d_entropy")
    if stream is not None:
        _given(stream, device, *(t for t in (logits, tokens, d_logp, d_entropy) if t is not None))
    if vocab == 0 or not 0 <= top <= min(32, vocab):
        raise ValueError("vocab must be at least 1 and top in [0, min(32, vocab)]")
    d, ldd = _result(out, rows, vocab, (logits.dtype,), device, stream) if grad else (None, 0)
    # one buffer for the vectors: logp, entropy, lse
    buf = _empty(3, rows, torch.float32, device, stream)
    at, size = buf.data_ptr(), 4 * rows
    ids = _empty(rows, top, torch.int32, device, stream) if top else None
    logs = _empty(rows, top, torch.float32, device, stream) if top else None
    _check(_on(device, stream, lib.sim_log_probs, logits.data_ptr(), DTYPES[logits.dtype], rows, vocab, ld, None if tokens is None else tokens.data_ptr(), tb,
               temperature, top, None if tokens is None else at, at + size, at + 2 * size, ids.data_ptr() if top else None, logs.data_ptr() if top else None,
               None if d_logp is None else d_logp.data_ptr(), None if d_entropy is None else d_entropy.data_ptr(), None if d is None else d.data_ptr(), ldd))
    if d is not None and logits.dim() == 1 and out is None:
        d = d[0]
    logp, entropy, lse = buf.unbind()
    return LogProbs(None if tokens is None else logp, entropy, lse, ids, logs, d)


def log_probs_backward(logits, tokens, d_logp=None, d_entropy=None, *, temperature=1.0, out=None, stream=None):
    """The gradient by the logits of a loss whose derivatives by logp and entropy are only known after the forward pass (log_probs)."""
    if d_logp is None and d_entropy is None:
        raise ValueError("d_logp or d_entropy is required")
    rows, vocab, ld, device, tb = _logits(logits, tokens, d_logp, d_entropy)
    if stream is not None:
        _given(stream, device, *(t for t in (logits, tokens, d_logp, d_entropy) if t is not None))
    d, ldd = _result(out, rows, vocab, (logits.dtype,), device, stream)
    _check(_on(device, stream, lib.sim_log_probs, logits.data_ptr(), DTYPES[logits.dtype], rows, vocab, ld, None if tokens is None else tokens.data_ptr(), tb,
               temperature, 0, None, None, None, None, None, None if d_logp is None else d_logp.data_ptr(), None if d_entropy is None else d_entropy.data_ptr(), d.data_ptr(), ldd))
    return d[0] if logits.dim() == 1 and out is None else d


def _logits(logits, tokens, d_logp, d_entropy):
    rows, vocab, ld = _plain(logits, "logits")
    device = logits.device
    if tokens is not None and (not torch.is_tensor(tokens) or tokens.device != device or tokens.dtype not in (torch.int64, torch.int32) or tokens.numel() != rows or
                               not tokens.is_contiguous()):
        raise ValueError("tokens must be a contiguous int64 or int32 tensor of %d elements on %s" % (rows, device))
    for name, t in (("d_logp", d_logp), ("d_entropy", d_entropy)):
        if t is not None and (not torch.is_tensor(t) or t.device != device or t.dtype != torch.float32 or t.numel() != rows or not t.is_contiguous()):
            raise ValueError("%s must be a contiguous float32 tensor of %d elements on %s" % (name, rows, device))
    if d_logp is not None and tokens is None:
        raise ValueError("d_logp needs tokens")
    return rows, vocab, ld, device, 0 if tokens is None else tokens.element_size()
