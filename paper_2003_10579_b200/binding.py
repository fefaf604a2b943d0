"""Thin ctypes binding of the C-ABI library (``include/straggler_sim.h``): argument marshalling
only.  torch supplies device memory and streams; every step of the simulation runs in the
library's CUDA kernels.  Importing this module loads ``libstraggler_sim.so`` and raises if it
has not been built - there is no CPU path behind these calls."""
from __future__ import annotations

import contextlib
import ctypes as C
import os

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
           "sim_mx_codes_bytes", "sim_mx_scales_bytes", "sim_mx_quantize", "sim_mx_dequantize", "sim_mx_matmul", "sim_set_adamw", "sim_eval_loss_mxfp4"]
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}     # SIM_F32, SIM_BF16, SIM_F16
MXFP4 = 3


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
    for name in EXPORTS:
        if name not in ("sim_n_params", "sim_last_error", "sim_destroy", "sim_noalloc_last_error", "sim_adamw_destroy", "sim_mx_codes_bytes", "sim_mx_scales_bytes"):
            getattr(L, name).restype = C.c_int
    L.sim_mx_codes_bytes.restype = L.sim_mx_scales_bytes.restype = i64
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
        R, dev = self.R, self.device
        out = {"t": torch.empty((R, J), dtype=torch.float64, device=dev),
               "loss": torch.empty((R, J), dtype=torch.float32, device=dev),
               "dist2": torch.empty((R, J), dtype=torch.float32, device=dev),
               "K": torch.empty((R, J), dtype=_U16, device=dev),
               "worker": torch.empty((R, J, Km), dtype=_U16, device=dev),
               "stale": torch.empty((R, J, Km), dtype=_U32, device=dev),
               "seq": torch.empty((R, J, Km), dtype=_U32, device=dev)}
        _check(lib.sim_get_trace(self._h, *[_ptr(out[k]) for k in ("t", "loss", "dist2", "K", "worker", "stale", "seq")]),
               self._h)
        return {k: v.cpu().numpy() for k, v in out.items()} if to_numpy else out

    def params(self, to_numpy=True):
        w = torch.empty((self.R, self.n_params), dtype=torch.float32, device=self.device)
        _check(lib.sim_get_params(self._h, _ptr(w)), self._h)
        return w.cpu().numpy() if to_numpy else w

    def eval_loss(self, to_numpy=True, mxfp4=False):
        """Full-data risk F(w_j) of every replica's current parameters; mxfp4: with data and parameters in 4 bits."""
        out = torch.empty((self.R,), dtype=torch.float32, device=self.device)
        _check((lib.sim_eval_loss_mxfp4 if mxfp4 else lib.sim_eval_loss)(self._h, _ptr(out)), self._h)
        if self.stream is not None:
            self.stream.synchronize()
        else:
            torch.cuda.synchronize()
        return out.cpu().numpy() if to_numpy else out

    def error_curve(self, grid):
        """Mean minibatch loss over replicas against simulated wall clock at the times in `grid`."""
        g = torch.as_tensor(np.asarray(grid, np.float64)).to(self.device)
        mean = torch.empty((g.numel(),), dtype=torch.float32, device=self.device)
        cnt = torch.empty((g.numel(),), dtype=torch.int32, device=self.device)
        _check(lib.sim_error_curve(self._h, _ptr(g), g.numel(), _ptr(mean), _ptr(cnt)), self._h)
        return mean.cpu().numpy(), cnt.cpu().numpy()

    def set_eval_every(self, every):
        """Record the full-data risk of every replica before the first and after every `every`-th update."""
        _check(lib.sim_set_eval_every(self._h, every), self._h)

    def risk_trace(self, to_numpy=True):
        """(risk [R, E], t [R, E]): entry 0 is F(w_0) at time 0, entry i the risk after i * every updates."""
        E = C.c_int64()
        _check(lib.sim_risk_trace_size(self._h, C.byref(E)), self._h)
        risk = torch.empty((self.R, E.value), dtype=torch.float32, device=self.device)
        t = torch.empty((self.R, E.value), dtype=torch.float64, device=self.device)
        _check(lib.sim_get_risk_trace(self._h, _ptr(risk), _ptr(t)), self._h)
        return (risk.cpu().numpy(), t.cpu().numpy()) if to_numpy else (risk, t)

    def risk_curve(self, grid, f_star=0.0):
        """Mean over replicas of F(w) - f_star against simulated wall clock at the times in `grid`."""
        g = torch.as_tensor(np.asarray(grid, np.float64)).to(self.device)
        mean = torch.empty((g.numel(),), dtype=torch.float32, device=self.device)
        cnt = torch.empty((g.numel(),), dtype=torch.int32, device=self.device)
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
    env = torch.empty((g.numel(),), dtype=torch.float32, device=dev)
    best = torch.empty((g.numel(),), dtype=torch.int32, device=dev)
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
    with _NO_STREAM if stream is None else torch.cuda.stream(stream):
        return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)


def _on(device, stream, call, *args):
    """call(*args, stream) with `device` current; stream None: the device's current one."""
    index = device.index
    st = _raw_stream(index) if stream is None else stream.cuda_stream
    if torch.cuda.current_device() == index:
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
