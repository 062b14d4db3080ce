"""ctypes binding of libvcas.so: one Python function per C entry point of include/vcas.h and include/vcas_train.h.

Argument marshalling only: torch tensors provide device memory and the current CUDA stream,
every step of the method runs in the library's kernels.  If the compiled library is missing
this module raises on first use; there is no other implementation to fall back to.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import ClassVar

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvcas.so")

VCAS_OK = 0
ERRORS = {-1: "VCAS_ERR_BAD_ARG", -2: "VCAS_ERR_SHAPE", -3: "VCAS_ERR_DTYPE", -4: "VCAS_ERR_WORKSPACE",
          -5: "VCAS_ERR_CUDA", -6: "VCAS_ERR_TIMEOUT", -7: "VCAS_ERR_INTERNAL"}
DTYPE_F32, DTYPE_BF16 = 0, 1
GEMM_AUTO, GEMM_FMA, GEMM_TENSOR = 0, 1, 2

EXPORTS = ["vcas_default_config", "vcas_create", "vcas_destroy", "vcas_workspace_bytes", "vcas_linear_bwd",
           "vcas_linear_bwd_ex", "vcas_linear_bwd_chain", "vcas_chain_parts", "vcas_layernorm_bwd", "vcas_join", "vcas_dense_bwd", "vcas_dense_bwd_ex", "vcas_score", "vcas_last_sampling", "vcas_mask_from_probs",
           "vcas_variance_probe", "vcas_update_ratios", "vcas_last_device_status", "vcas_launch_count",
           "vcas_set_profiling", "vcas_stage_times", "vcas_set_wait_limit",
           "vcas_set_probe_subsample", "vcas_get_probe_subsample", "vcas_score_static", "vcas_set_tuning",
           "vcas_last_plan", "vcas_version",
           "vcas_loss_create", "vcas_loss_destroy", "vcas_loss_fwd", "vcas_loss_bwd", "vcas_loss_status",
           "vcas_adamw_step", "vcas_adamw_rates",
           "vcas_attn_create", "vcas_attn_destroy", "vcas_attn_workspace_bytes", "vcas_attn_fwd", "vcas_attn_bwd",
           "vcas_attn_status", "vcas_attn_set_wait_limit"]


class VcasError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where} failed: {ERRORS.get(code, code)}")
        self.code = code


class LayerDesc(C.Structure):
    _fields_ = [("N", C.c_int32), ("T", C.c_int32), ("d_in", C.c_int32), ("d_out", C.c_int32),
                ("dtype", C.c_int32), ("gemm_path", C.c_int32)]


class Config(C.Structure):
    _fields_ = [("F", C.c_int32), ("M", C.c_int32), ("tau_act", C.c_float), ("tau_w", C.c_float),
                ("alpha", C.c_float), ("beta", C.c_float), ("rho_min", C.c_float), ("nu_min", C.c_float)]


class State(C.Structure):
    _fields_ = [("s", C.c_float), ("t", C.c_int32), ("L", C.c_int32),
                ("rho", C.POINTER(C.c_float)), ("nu", C.POINTER(C.c_float))]


class ChainArgs(C.Structure):
    _fields_ = [("H", C.c_void_p), ("a_in", C.c_void_p), ("a_in_parts", C.c_int32), ("alive_in", C.c_void_p),
                ("alive_cnt_in", C.c_void_p), ("a_out", C.c_void_p), ("kept_out", C.c_void_p),
                ("kept_cnt_out", C.c_void_p), ("skip_dropped_rows", C.c_int32), ("defer_join", C.c_int32)]


class AttnDesc(C.Structure):
    _fields_ = [("max_tokens", C.c_int32), ("max_seqs", C.c_int32), ("heads_q", C.c_int32), ("heads_kv", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float)]


class AttnTensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("token", C.c_int64), ("head", C.c_int64)]


class LossDesc(C.Structure):
    _fields_ = [("max_rows", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("top", C.c_int32)]


class AdamWEntry(C.Structure):
    _fields_ = [("p", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("copy", C.c_void_p), ("n", C.c_int64), ("weight_decay", C.c_float),
                ("p_dtype", C.c_int32), ("g_dtype", C.c_int32), ("state_bits", C.c_int32)]


class AdamWArgs(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_int64),
                ("seed", C.c_uint64), ("grad_scale", C.c_void_p), ("rates", C.c_void_p), ("seed_dev", C.c_void_p)]


_P, _I, _F, _U64 = C.c_void_p, C.c_int32, C.c_float, C.c_uint64
_I64, _D = C.c_int64, C.c_double
# argument types, so that plain numbers and addresses can be passed (void pointers take an int or None)
_SAMPLING_OUT = [_P] * 8
ARGTYPES = {
    "vcas_default_config": [_P], "vcas_create": [_P] * 3, "vcas_destroy": [_P], "vcas_workspace_bytes": [_P] * 2,
    "vcas_linear_bwd": [_P] * 4 + [_F, _F, _U64] + [_P] * 3,
    "vcas_linear_bwd_ex": [_P] * 4 + [_F, _F, _U64] + [_P] * 6,
    "vcas_linear_bwd_chain": [_P] * 4 + [_F, _F, _U64] + [_P] * 4,
    "vcas_chain_parts": [_P] * 2,
    "vcas_layernorm_bwd": [_P] * 4 + [_F, _F, _U64] + [_P] * 5,
    "vcas_join": [_P] * 2, "vcas_dense_bwd": [_P] * 7, "vcas_dense_bwd_ex": [_P] * 8,
    "vcas_score": [_P] * 3 + [_F, _F, _U64] + _SAMPLING_OUT + [_P],
    "vcas_last_sampling": [_P] + _SAMPLING_OUT + [_P],
    "vcas_mask_from_probs": [_P, _P, _I, _U64, _I] + [_P] * 4,
    "vcas_variance_probe": [_P, _I] + [_P] * 3 + [_F, _F, _F, _U64] + [_P] * 6,
    "vcas_update_ratios": [_P, _I] + [_P] * 6,
    "vcas_last_device_status": [_P] * 2, "vcas_launch_count": [_P] * 2,
    "vcas_set_profiling": [_P, _I], "vcas_stage_times": [_P] * 3, "vcas_set_wait_limit": [_P, _U64, _I],
    "vcas_set_probe_subsample": [_P, _I, _U64], "vcas_get_probe_subsample": [_P] * 3,
    "vcas_score_static": [_I] * 5 + [_P, _P, _F, _F, _U64] + _SAMPLING_OUT + [_P],
    "vcas_set_tuning": [_P] + [_I] * 6, "vcas_last_plan": [_P] * 2, "vcas_version": [],
    "vcas_loss_create": [_P] * 2, "vcas_loss_destroy": [_P], "vcas_loss_status": [_P] * 2,
    "vcas_loss_fwd": [_P, _P, _I64, _P, _I, _I] + [_P] * 6,
    "vcas_loss_bwd": [_P, _P, _I64, _P, _I, _I] + [_P] * 5 + [_I64] + [_P] * 2,
    "vcas_attn_create": [_P] * 2, "vcas_attn_destroy": [_P], "vcas_attn_workspace_bytes": [_P] * 2, "vcas_attn_status": [_P] * 2,
    "vcas_attn_fwd": [_P] * 5 + [_I, _I] + [_P] * 3, "vcas_attn_set_wait_limit": [_P, _U64, _I],
    "vcas_attn_bwd": [_P] * 8 + [_I, _I, _P, _P, _I] + [_P] * 4,
    "vcas_adamw_step": [_P, _I, _P, _P], "vcas_adamw_rates": [_D, _D, _D, _I64, _P],
}

_lib = None


def lib() -> C.CDLL:
    """Loads libvcas.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2402_17227_b200.build` (needs nvcc); "
                               "there is no CPU implementation")
        l = C.CDLL(LIB_PATH)
        for name in EXPORTS:
            fn = getattr(l, name)
            fn.restype, fn.argtypes = C.c_int, ARGTYPES[name]
        _lib = l
    return _lib


def _check(code: int, where: str) -> None:
    if code != VCAS_OK:
        raise VcasError(code, where)


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors only"
    return t.data_ptr()


# the current stream's handle without the Python stream object around it (0.3 us instead of 3)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def default_config() -> Config:
    cfg = Config()
    _check(lib().vcas_default_config(C.byref(cfg)), "vcas_default_config")
    return cfg


@dataclass
class Sampling:
    g: torch.Tensor
    p: torch.Tensor
    w: torch.Tensor
    q: torch.Tensor
    idxA: torch.Tensor
    cntA: int
    idxW: torch.Tensor
    cntW: int


def _sampling_buffers(N: int, R: int, dev):
    """g, p, w, q, idxA, idxW and the two counts: the outputs of a scoring call, which writes all of them."""
    f, i = torch.float32, torch.int32
    return (torch.empty(N, dtype=f, device=dev), torch.empty(N, dtype=f, device=dev), torch.empty(R, dtype=f, device=dev),
            torch.empty(R, dtype=f, device=dev), torch.empty(N, dtype=i, device=dev), torch.empty(R, dtype=i, device=dev),
            torch.empty(2, dtype=i, device=dev))


def _sampling_ptrs(b):
    g, p, w, q, idxA, idxW, cnt = [t.data_ptr() for t in b]
    return g, p, w, q, idxA, cnt, idxW, cnt + 4


class Layer:
    """A handle for one layer shape (vcas_create / vcas_destroy) on the current CUDA device."""

    def __init__(self, N: int, T: int, d_in: int, d_out: int, dtype: torch.dtype = torch.bfloat16,
                 gemm_path: int = GEMM_AUTO, config: Config | None = None):
        if not torch.cuda.is_available():
            raise RuntimeError("libvcas needs a CUDA device (sm_100a); there is no CPU path")
        self.N, self.T, self.d_in, self.d_out, self.dtype = N, T, d_in, d_out, dtype
        self.R = N * T
        self.config = config if config is not None else default_config()
        desc = LayerDesc(N, T, d_in, d_out, {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}[dtype], gemm_path)
        self._h = C.c_void_p(None)
        _check(lib().vcas_create(C.byref(self._h), C.byref(desc), C.byref(self.config)), "vcas_create")

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().vcas_destroy(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------ products
    def _outs(self, dX, dW, dev):
        if dX is None:
            dX = torch.empty(self.R, self.d_in, dtype=self.dtype, device=dev)
        if dW is None:
            dW = torch.empty(self.d_out, self.d_in, dtype=torch.float32, device=dev)
        return dX, dW

    def linear_bwd(self, X, dY, W, rho: float, nu: float, seed: int, *, p_in=None, q_in=None, H=None,
                   dX=None, dW=None):
        dX, dW = self._outs(dX, dW, X.device)
        rc = lib().vcas_linear_bwd_ex(self._h, _ptr(X), _ptr(dY), _ptr(W), rho, nu,
                                      seed, _ptr(p_in), _ptr(q_in), _ptr(H), _ptr(dX), _ptr(dW),
                                      _stream())
        _check(rc, "vcas_linear_bwd_ex")
        return dX, dW

    def linear_bwd_chain(self, X, dY, W, rho: float, nu: float, seed: int, dX, dW, *, H=None, a_in=None,
                         a_in_parts: int = 1, alive_in=None, alive_cnt_in=None, a_out=None, kept_out=None,
                         kept_cnt_out=None, skip_dropped_rows: bool = False, defer_join: bool = False):
        """vcas_linear_bwd_chain: scores handed down from the layer above (a_in, alive_in) and to the layer
        below (a_out, kept_out); every extra is an optional device tensor."""
        dp = lambda t: None if t is None else t.data_ptr()
        args = ChainArgs(dp(H), dp(a_in), a_in_parts, dp(alive_in), dp(alive_cnt_in), dp(a_out), dp(kept_out),
                         dp(kept_cnt_out), 1 if skip_dropped_rows else 0, 1 if defer_join else 0)
        _check(lib().vcas_linear_bwd_chain(self._h, _ptr(X), _ptr(dY), _ptr(W), rho, nu,
                                           seed, C.byref(args), _ptr(dX), _ptr(dW), _stream()),
               "vcas_linear_bwd_chain")

    def layernorm_bwd(self, X, gamma, dY, rho: float, seed: int, eps: float = 1e-5, *, dX=None, a_in=None,
                      a_in_parts: int = 1, alive_in=None, alive_cnt_in=None, a_out=None, kept_out=None,
                      kept_cnt_out=None, skip_dropped_rows: bool = False):
        """vcas_layernorm_bwd on a handle made with d_in = d_out = the normalised width.  Returns (dX, dgamma, dbeta)."""
        dev = X.device
        if dX is None:
            dX = torch.empty(self.R, self.d_in, dtype=self.dtype, device=dev)
        dg = torch.empty(self.d_in, dtype=torch.float32, device=dev)
        db = torch.empty(self.d_in, dtype=torch.float32, device=dev)
        dp = lambda t: None if t is None else t.data_ptr()
        args = ChainArgs(None, dp(a_in), a_in_parts, dp(alive_in), dp(alive_cnt_in), dp(a_out), dp(kept_out),
                         dp(kept_cnt_out), 1 if skip_dropped_rows else 0, 0)
        _check(lib().vcas_layernorm_bwd(self._h, _ptr(X), _ptr(gamma), _ptr(dY), eps, rho,
                                        seed, C.byref(args), _ptr(dX), _ptr(dg), _ptr(db), _stream()),
               "vcas_layernorm_bwd")
        return dX, dg, db

    def join(self) -> None:
        _check(lib().vcas_join(self._h, _stream()), "vcas_join")

    def chain_parts(self) -> int:
        n = C.c_int32(0)
        _check(lib().vcas_chain_parts(self._h, C.byref(n)), "vcas_chain_parts")
        return n.value

    def linear_bwd_plain(self, X, dY, W, rho: float, nu: float, seed: int, dX, dW):
        """vcas_linear_bwd with caller-provided outputs (the call a training loop makes)."""
        _check(lib().vcas_linear_bwd(self._h, _ptr(X), _ptr(dY), _ptr(W), rho, nu,
                                     seed, _ptr(dX), _ptr(dW), _stream()), "vcas_linear_bwd")

    def dense_bwd(self, X, dY, W, *, H=None, dX=None, dW=None):
        dX, dW = self._outs(dX, dW, X.device)
        _check(lib().vcas_dense_bwd_ex(self._h, _ptr(X), _ptr(dY), _ptr(W), _ptr(H), _ptr(dX), _ptr(dW), _stream()),
               "vcas_dense_bwd_ex")
        return dX, dW

    # ------------------------------------------------------------------ sampling
    def _sampling_buffers(self, dev):
        return _sampling_buffers(self.N, self.R, dev)

    @staticmethod
    def _pack_sampling(b) -> Sampling:
        g, p, w, q, idxA, idxW, cnt = b
        ca, cw = cnt.tolist()           # one wait for both counts
        return Sampling(g, p, w, q, idxA[:ca], ca, idxW[:cw], cw)

    def score(self, X, dY, rho: float, nu: float, seed: int) -> Sampling:
        b = self._sampling_buffers(X.device)
        _check(lib().vcas_score(self._h, _ptr(X), _ptr(dY), rho, nu, seed,
                                *_sampling_ptrs(b), _stream()), "vcas_score")
        return self._pack_sampling(b)

    def last_sampling(self, device=None) -> Sampling:
        b = self._sampling_buffers(device or torch.device("cuda", torch.cuda.current_device()))
        _check(lib().vcas_last_sampling(self._h, *_sampling_ptrs(b), _stream()), "vcas_last_sampling")
        return self._pack_sampling(b)

    def mask_from_probs(self, p, seed: int, sampler_id: int):
        n = p.numel()
        keep = torch.empty(n, dtype=torch.uint8, device=p.device)
        idx = torch.empty(n, dtype=torch.int32, device=p.device)
        cnt = torch.zeros(1, dtype=torch.int32, device=p.device)
        _check(lib().vcas_mask_from_probs(self._h, _ptr(p), n, seed, sampler_id,
                                          _ptr(keep), _ptr(idx), _ptr(cnt), _stream()), "vcas_mask_from_probs")
        c = int(cnt.item())
        return keep, idx[:c], c

    # --------------------------------------------------------------------- probe
    def variance_probe(self, Xs, dYs, W, rho: float, nu: float, s: float, seed: int, out=None):
        """Returns a device tensor [V_s, V_act, V_w, p_lo, p_hi] (fp32), filled asynchronously."""
        M = len(Xs)
        if out is None:
            out = torch.zeros(5, dtype=torch.float32, device=W.device)
        xa = (C.c_void_p * M)(*[x.data_ptr() for x in Xs])
        ya = (C.c_void_p * M)(*[y.data_ptr() for y in dYs])
        base, st = out.data_ptr(), 4
        rc = lib().vcas_variance_probe(self._h, M, xa, ya, _ptr(W), rho, nu,
                                       s, seed, *[base + st * k for k in range(5)],
                                       _stream())
        _check(rc, "vcas_variance_probe")
        return out

    # ---------------------------------------------------------------------- misc
    def device_status(self) -> int:
        st = C.c_int32(0)
        _check(lib().vcas_last_device_status(self._h, C.byref(st)), "vcas_last_device_status")
        return st.value

    def set_tuning(self, dx_tile_n: int = 0, dw_tile_n: int = 0, dx_split_k: int = 0, dw_split_k: int = 0,
                   tile_m: int = 0, dw_tile_m: int | None = None) -> None:
        """tile_m: tile height of the dX product, and of the dW product too unless dw_tile_m is given."""
        _check(lib().vcas_set_tuning(self._h, dx_tile_n, dw_tile_n, dx_split_k,
                                     dw_split_k, tile_m,
                                     tile_m if dw_tile_m is None else dw_tile_m), "vcas_set_tuning")

    def last_plan(self):
        """((width, slices, height code) of the dX product, the same of the dW product) of the last call."""
        a = (C.c_int32 * 6)()
        _check(lib().vcas_last_plan(self._h, a), "vcas_last_plan")
        return tuple(a[0:3]), tuple(a[3:6])

    def set_probe_subsample(self, rows: int, seed: int = 0) -> None:
        _check(lib().vcas_set_probe_subsample(self._h, rows, seed), "vcas_set_probe_subsample")

    def probe_subsample(self):
        """The rows of the parameter gradient the probe samples (host list; empty when it uses all rows)."""
        n = C.c_int32(0)
        _check(lib().vcas_get_probe_subsample(self._h, None, C.byref(n)), "vcas_get_probe_subsample")
        rows = (C.c_int32 * max(1, n.value))()
        _check(lib().vcas_get_probe_subsample(self._h, rows, C.byref(n)), "vcas_get_probe_subsample")
        return list(rows)[:n.value]

    def set_wait_limit(self, limit_ns: int, stall_once: bool = False) -> None:
        _check(lib().vcas_set_wait_limit(self._h, limit_ns, 1 if stall_once else 0),
               "vcas_set_wait_limit")

    def set_profiling(self, enable: bool) -> None:
        _check(lib().vcas_set_profiling(self._h, 1 if enable else 0), "vcas_set_profiling")

    def stage_times(self):
        """(ms[8], calls[2]) summed over the calls recorded since profiling was enabled or last read."""
        ms = (C.c_float * 8)()
        calls = (C.c_int32 * 2)()
        _check(lib().vcas_stage_times(self._h, ms, calls), "vcas_stage_times")
        return list(ms), list(calls)

    def launch_count(self) -> int:
        n = C.c_uint64(0)
        _check(lib().vcas_launch_count(self._h, C.byref(n)), "vcas_launch_count")
        return n.value

    def workspace_bytes(self) -> int:
        n = C.c_size_t(0)
        _check(lib().vcas_workspace_bytes(self._h, C.byref(n)), "vcas_workspace_bytes")
        return n.value


def update_ratios(s: float, rho, nu, V_s, V_act, V_w, p_lo, p_hi, config: Config, t: int = 0):
    """vcas_update_ratios on host lists of length L; returns (s, rho, nu)."""
    L = len(rho)
    arr = lambda v: (C.c_float * L)(*[float(x) for x in v])
    rho_a, nu_a = arr(rho), arr(nu)
    st = State(float(s), int(t), L, C.cast(rho_a, C.POINTER(C.c_float)), C.cast(nu_a, C.POINTER(C.c_float)))
    rc = lib().vcas_update_ratios(C.byref(st), L, arr(V_s), arr(V_act), arr(V_w), arr(p_lo), arr(p_hi),
                                  C.byref(config))
    _check(rc, "vcas_update_ratios")
    return st.s, list(rho_a), list(nu_a)


def score_static(X, dY, N: int, T: int, rho: float, nu: float, seed: int) -> Sampling:
    """vcas_score_static: scores, probabilities and index lists without a handle or any device
    allocation by the library (the output tensors below are the caller's, made by torch).
    Limits: N <= 4096, N*T <= 16384.  Calls sharing a device must not overlap on the GPU."""
    b = _sampling_buffers(N, N * T, X.device)
    dt = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}[X.dtype]
    rc = lib().vcas_score_static(N, T, X.shape[1], dY.shape[1],
                                 dt, _ptr(X), _ptr(dY), rho, nu, seed,
                                 *_sampling_ptrs(b), _stream())
    _check(rc, "vcas_score_static")
    return Layer._pack_sampling(b)


# --------------------------------------------------------------------- around the sampled backward (vcas_train.h)
_DTYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _stream_at(index: int):
    """The current stream of a device."""
    return _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream(index).cuda_stream


def _on(device, what: str, *tensors) -> None:
    for t in tensors:
        _need(t is None or t.device == device, f"{what} on {device} only")


def _current_device() -> torch.device:
    if not torch.cuda.is_available():
        raise RuntimeError("libvcas needs a CUDA device (sm_100a); there is no CPU path")
    return torch.device("cuda", torch.cuda.current_device())


class _Handle:
    """Creates a handle on the current device and destroys it with the object.  Calls are enqueued on that device's current
    stream, whichever device is current."""
    _kind = ""

    def _create(self, desc) -> None:
        self.device = _current_device()
        self._index = self.device.index
        self._h = C.c_void_p(None)
        _check(getattr(lib(), f"vcas_{self._kind}_create")(C.byref(self._h), C.byref(desc)), f"vcas_{self._kind}_create")

    def device_status(self) -> int:
        st = C.c_int32(0)
        _check(getattr(lib(), f"vcas_{self._kind}_status")(self._h, C.byref(st)), f"vcas_{self._kind}_status")
        return st.value

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            getattr(lib(), f"vcas_{self._kind}_destroy")(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Attention(_Handle):
    """Self-attention over packed sequences of up to max_tokens tokens in up to max_seqs sequences (vcas_attn_*).  Tensors are
    [total, heads, head_dim] with any strides that keep a head's values side by side; starts: int32 [N + 1] on the device."""
    _kind = "attn"

    def __init__(self, max_tokens: int, max_seqs: int, heads_q: int, heads_kv: int, head_dim: int,
                 dtype: torch.dtype = torch.bfloat16, causal: bool = False, scale: float = 0.0):
        _need(dtype in _DTYPES, "attention is in bfloat16 or float32")
        self.heads_q, self.heads_kv, self.head_dim, self.dtype, self.causal = heads_q, heads_kv, head_dim, dtype, bool(causal)
        self._create(AttnDesc(max_tokens, max_seqs, heads_q, heads_kv, head_dim, _DTYPES[dtype], 1 if causal else 0, scale))
        # the tensors of a call as the library takes them: filled anew by every call (d_o, q, k, v, o, dq, dk, dv)
        self._args = [AttnTensor() for _ in range(8)]
        self._refs = [C.byref(a) for a in self._args]

    def _tensor(self, place: int, t, total: int, heads: int, written: bool = False):
        if t.shape != (total, heads, self.head_dim) or t.dtype is not self.dtype:
            raise ValueError(f"expected [{total}, {heads}, {self.head_dim}] of {self.dtype}, got {tuple(t.shape)} of {t.dtype}")
        if t.get_device() != self._index:
            raise ValueError(f"tensors of a call on {self.device} only")
        token, head, inner = t.stride()
        if inner != 1 and self.head_dim != 1:
            raise ValueError("a head's values lie side by side")
        if written:      # no two elements in one place
            least = self.head_dim
            for stride, n in ((token, total), (head, heads)) if token < head else ((head, heads), (token, total)):
                if n > 1:
                    if stride < least:
                        raise ValueError("rows of an output overlap")
                    least = stride * n
        a = self._args[place]
        a.ptr, a.token, a.head = t.data_ptr(), token, head
        return self._refs[place]

    def _sequences(self, starts):
        if starts.dim() != 1 or starts.dtype is not torch.int32 or not starts.is_contiguous() or starts.get_device() != self._index:
            raise ValueError(f"starts is int32 [N + 1] on {self.device}")
        n = starts.shape[0] - 1
        _need(n >= 0, "starts is int32 [N + 1]")
        return n

    def _lse(self, lse, total):
        if lse.shape != (self.heads_q, total) or lse.dtype is not torch.float32 or not lse.is_contiguous() or \
                lse.get_device() != self._index:
            raise ValueError(f"lse is float32 [heads_q, total] on {self.device}")
        return lse.data_ptr()

    def fwd(self, q, k, v, starts, *, o=None, lse=None):
        """Returns (o, lse)."""
        total, N, Hq, Hk, T = q.shape[0], self._sequences(starts), self.heads_q, self.heads_kv, self._tensor
        if o is None:
            o = torch.empty(total, Hq, self.head_dim, dtype=self.dtype, device=self.device)
        if lse is None:
            lse = torch.empty(Hq, total, dtype=torch.float32, device=self.device)
        _check(lib().vcas_attn_fwd(self._h, T(1, q, total, Hq), T(2, k, total, Hk), T(3, v, total, Hk), starts.data_ptr(), N, total,
                                   T(4, o, total, Hq, True), self._lse(lse, total), _stream_at(self._index)), "vcas_attn_fwd")
        return o, lse

    def bwd(self, d_o, q, k, v, o, lse, starts, *, dq=None, dk=None, dv=None, alive_in=None, alive_cnt_in=None,
            skip_dropped_rows: bool = False):
        """Returns (dq, dk, dv).  alive_in, alive_cnt_in: the kept_out, kept_cnt_out of the layer above."""
        total, N, Hq, Hk, T = q.shape[0], self._sequences(starts), self.heads_q, self.heads_kv, self._tensor
        new = lambda h: torch.empty(total, h, self.head_dim, dtype=self.dtype, device=self.device)
        dq, dk, dv = new(Hq) if dq is None else dq, new(Hk) if dk is None else dk, new(Hk) if dv is None else dv
        alive = cnt = None
        if alive_in is not None or alive_cnt_in is not None:
            if alive_in is None or alive_cnt_in is None or alive_in.dtype is not torch.int32 or alive_cnt_in.dtype is not torch.int32 \
                    or alive_in.numel() < N or alive_cnt_in.numel() < 1 or not alive_in.is_contiguous():
                raise ValueError("alive_in is int32 [N], alive_cnt_in int32 [1], and they come together")
            _on(self.device, "alive_in", alive_in, alive_cnt_in)
            alive, cnt = alive_in.data_ptr(), alive_cnt_in.data_ptr()
        _check(lib().vcas_attn_bwd(self._h, T(0, d_o, total, Hq), T(1, q, total, Hq), T(2, k, total, Hk), T(3, v, total, Hk),
                                   T(4, o, total, Hq), self._lse(lse, total), starts.data_ptr(), N, total, alive, cnt,
                                   1 if skip_dropped_rows else 0, T(5, dq, total, Hq, True), T(6, dk, total, Hk, True),
                                   T(7, dv, total, Hk, True), _stream_at(self._index)), "vcas_attn_bwd")
        return dq, dk, dv

    def set_wait_limit(self, limit_ns: int, stall_once: bool = False) -> None:
        _check(lib().vcas_attn_set_wait_limit(self._h, limit_ns, 1 if stall_once else 0), "vcas_attn_set_wait_limit")

    def workspace_bytes(self) -> int:
        n = C.c_size_t(0)
        _check(lib().vcas_attn_workspace_bytes(self._h, C.byref(n)), "vcas_attn_workspace_bytes")
        return n.value


@dataclass
class LogProbs:
    logp: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor
    top_logp: torch.Tensor | None
    top_ids: torch.Tensor | None


class TokenLoss(_Handle):
    """Log probabilities of given tokens, entropy and top alternatives of up to max_rows rows of `vocab` logits, and their
    gradient (vcas_loss_*)."""
    _kind = "loss"

    def __init__(self, max_rows: int, vocab: int, dtype: torch.dtype = torch.bfloat16, top: int = 0):
        _need(dtype in _DTYPES, "logits are bfloat16 or float32")
        self.max_rows, self.vocab, self.dtype, self.top = max_rows, vocab, dtype, top
        self._create(LossDesc(max_rows, vocab, _DTYPES[dtype], top))
        # what a call's outputs look like, for as many rows as the last one had (empty_like takes 1.3 us, empty 2.3)
        self._like = (-1, None, None, None)

    def _rows(self, logits, tokens):
        """Rows and the elements between them."""
        V = self.vocab
        if logits.dim() != 2 or logits.shape[1] != V or logits.dtype is not self.dtype or logits.get_device() != self._index:
            raise ValueError(f"logits are [rows, {V}] of {self.dtype} on {self.device}")
        rows = logits.shape[0]
        ld, inner = logits.stride()
        if inner != 1 and V != 1:
            raise ValueError("a row's logits lie side by side")
        if ld < V:
            if rows > 1:
                raise ValueError("rows that overlap")
            ld = V
        if tokens.shape != (rows,) or tokens.dtype not in (torch.int64, torch.int32) or not tokens.is_contiguous() or \
                tokens.get_device() != self._index:
            raise ValueError(f"tokens are [rows], int32 or int64, on {self.device}")
        return rows, ld

    def fwd(self, logits, tokens) -> LogProbs:
        """tokens: [rows], negative where there is none."""
        rows, ld = self._rows(logits, tokens)
        if self._like[0] != rows:
            new = lambda shape, dt: torch.empty(shape, dtype=dt, device=self.device)
            self._like = (rows, new((3, rows), torch.float32), new((rows, self.top), torch.float32), new((rows, self.top), torch.int32))
        _, like, tl_like, ti_like = self._like
        f = torch.empty_like(like)
        base = f.data_ptr()
        lse, logp, entropy = f.unbind(0)
        tl = torch.empty_like(tl_like) if self.top else None
        ti = torch.empty_like(ti_like) if self.top else None
        _check(lib().vcas_loss_fwd(self._h, logits.data_ptr(), ld, tokens.data_ptr(), tokens.element_size(), rows, base + 4 * rows,
                                   base + 8 * rows, base, tl.data_ptr() if self.top else None, ti.data_ptr() if self.top else None,
                                   _stream_at(self._index)), "vcas_loss_fwd")
        return LogProbs(logp, entropy, lse, tl, ti)

    def bwd(self, logits, tokens, lse, g_logp, *, entropy=None, g_entropy=None, dlogits=None, a_out=None):
        """Returns (dlogits, a_out); dlogits may be logits itself.  a_out: the rows' square-norms for linear_bwd_chain(a_in=)."""
        rows, ld = self._rows(logits, tokens)
        if dlogits is None:
            dlogits = torch.empty((rows, self.vocab), dtype=self.dtype, device=self.device)
        if a_out is None:
            a_out = torch.empty(rows, dtype=torch.float32, device=self.device)
        ld_d = ld if dlogits is logits else self._rows(dlogits, tokens)[1]
        at = []
        for t in (lse, entropy, g_logp, g_entropy, a_out):
            if t is None:
                at.append(None)
                continue
            if t.shape != (rows,) or t.dtype is not torch.float32 or not t.is_contiguous() or t.get_device() != self._index:
                raise ValueError(f"lse, entropy, the derivatives and a_out are [rows] of float32 on {self.device}")
            at.append(t.data_ptr())
        _check(lib().vcas_loss_bwd(self._h, logits.data_ptr(), ld, tokens.data_ptr(), tokens.element_size(), rows, at[0], at[1], at[2],
                                   at[3], dlogits.data_ptr(), ld_d, at[4], _stream_at(self._index)), "vcas_loss_bwd")
        return dlogits, a_out


@dataclass
class AdamWTensor:
    """One tensor of an AdamW step.  m, v: float32, or float8_e4m3fn (v then holds sqrt(v)) with m_scale and v_scale, one float32
    for each 256 elements.  copy: bfloat16 copy of p to be written (float32 p).  A field may be set at any time: the next step of every
    AdamW that has this tensor follows it."""
    changes: ClassVar[int] = 0       # fields set since their tensors were made, of all tensors
    p: torch.Tensor
    g: torch.Tensor
    m: torch.Tensor
    v: torch.Tensor
    m_scale: torch.Tensor | None = None
    v_scale: torch.Tensor | None = None
    copy: torch.Tensor | None = None
    weight_decay: float = 0.0

    def __post_init__(self):
        self.__dict__["_version"] = 0

    def __setattr__(self, name, value):
        d = self.__dict__
        d[name] = value
        if "_version" in d:
            d["_version"] += 1
            AdamWTensor.changes += 1

    @staticmethod
    def make(p, g, bits: int = 32, copy=None, weight_decay: float = 0.0) -> "AdamWTensor":
        """With fresh states of 32 or 8 bits."""
        z = lambda n, dt: torch.zeros(n, dtype=dt, device=p.device)
        if bits == 32:
            return AdamWTensor(p, g, z(p.shape, torch.float32), z(p.shape, torch.float32), copy=copy, weight_decay=weight_decay)
        n = (p.numel() + 255) // 256
        e4m3 = lambda: torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
        return AdamWTensor(p, g, e4m3(), e4m3(), z(n, torch.float32), z(n, torch.float32), copy, weight_decay)


class AdamW:
    """AdamW over a list of tensors in one launch for each combination of types (vcas_adamw_step).  Its table of addresses is made once
    and follows the tensors' fields where these are set.  It holds the memory that the fields had then: a tensor that moves its
    data by itself (`x.data = ...`) is followed once the field is set again."""

    def __init__(self, tensors: list[AdamWTensor]):
        self.device = tensors[0].p.device if tensors else _current_device()
        self.tensors = tuple(tensors)
        self._table = (AdamWEntry * max(1, len(tensors)))()
        self._args = AdamWArgs()         # filled anew by every step
        self._ref = C.byref(self._args)
        # of each tensor: the version that the table has, and the memory that it points to
        self._versions, self._held, self._seen = [None] * len(tensors), [None] * len(tensors), None
        self._follow()

    def _follow(self) -> None:
        """Brings the table up to date with the tensors' fields."""
        seen = AdamWTensor.changes
        for i, t in enumerate(self.tensors):
            if self._versions[i] != t._version:
                self._fill(i, t)
        self._seen = seen

    def _fill(self, i: int, t: AdamWTensor) -> None:
        version = t._version
        _need(all(x is not None for x in (t.p, t.g, t.m, t.v)), "a tensor of a step has p, g, m and v")
        bits = 8 if t.m.dtype == torch.float8_e4m3fn else 32
        n = t.p.numel()
        _need(t.p.dtype in _DTYPES, "p is float32 or bfloat16")
        _need(t.m.dtype == t.v.dtype and t.m.dtype in (torch.float32, torch.float8_e4m3fn), "states are float32 or float8_e4m3fn")
        _need(t.m.numel() == n and t.v.numel() == n, "states have an element for each of p")
        scales = [t.m_scale, t.v_scale]
        if bits == 8:
            _need(all(s is not None and s.dtype == torch.float32 and s.numel() == (n + 255) // 256 for s in scales),
                  "8-bit states have a float32 scale for each 256 elements")
        else:
            _need(scales == [None, None], "float32 states have no scales")
        _need(t.copy is None or (t.copy.dtype == torch.bfloat16 and t.copy.numel() == n and t.p.dtype == torch.float32),
              "copy is bfloat16, of a float32 p")
        self._check_grad(t, t.g)
        every = [x for x in (t.g, t.p, t.m, t.v, t.m_scale, t.v_scale, t.copy) if x is not None]
        _need(all(x.is_cuda and x.is_contiguous() for x in every), "device-resident contiguous tensors only")
        _on(self.device, "tensors of a step", *every)
        dp = lambda x: None if x is None else x.data_ptr()
        self._table[i] = AdamWEntry(dp(t.p), dp(t.g), dp(t.m), dp(t.v), dp(t.m_scale), dp(t.v_scale), dp(t.copy), n, t.weight_decay,
                                    _DTYPES[t.p.dtype], _DTYPES[t.g.dtype], bits)
        self._held[i] = [x.untyped_storage() for x in every]
        self._versions[i] = version

    def _check_grad(self, t: AdamWTensor, g) -> None:
        _need(g is not None and g.dtype in _DTYPES and g.numel() == t.p.numel() and g.is_contiguous(),
              "g is contiguous, float32 or bfloat16, as large as p")
        _on(self.device, "gradients of a step", g)

    def set_grad(self, i: int, g: torch.Tensor) -> None:
        """The gradient of tensor i: `tensors[i].g = g`, checked at once, and cheaper than the next step's look at all fields."""
        t = self.tensors[i]
        self._check_grad(t, g)
        rest, all_seen = self._versions[i] == t._version, self._seen == AdamWTensor.changes
        t.g = g
        if rest:                         # the other fields are those of the table
            self._table[i].g, self._table[i].g_dtype = g.data_ptr(), _DTYPES[g.dtype]
            self._held[i][0] = g.untyped_storage()
            self._versions[i] = t._version
            if all_seen:
                self._seen = AdamWTensor.changes

    def step(self, step: int, *, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, seed: int = 0,
             grad_scale=None, rates=None, seed_dev=None) -> None:
        """step: 1 for the first.  seed: another one each step (8-bit states).  grad_scale: float32 [1] on the device.
        rates (adamw_rates, float32 [3]) and seed_dev (int64 [1]) on the device are read in place of lr and step, and of seed:
        a captured step then follows them."""
        if self._seen != AdamWTensor.changes:
            self._follow()
        a = self._args
        a.lr, a.beta1, a.beta2, a.eps, a.step, a.seed = lr, beta1, beta2, eps, step, seed & 0xFFFFFFFFFFFFFFFF
        a.grad_scale = a.rates = a.seed_dev = None
        if grad_scale is not None or rates is not None or seed_dev is not None:
            at = []
            for t, n, dt in ((grad_scale, 1, torch.float32), (rates, 3, torch.float32), (seed_dev, 1, torch.int64)):
                if t is not None and (t.dtype is not dt or t.numel() != n or not t.is_contiguous() or t.device != self.device):
                    raise ValueError(f"grad_scale is float32 [1], rates float32 [3], seed_dev int64 [1], on {self.device}")
                at.append(None if t is None else t.data_ptr())
            a.grad_scale, a.rates, a.seed_dev = at
        call = lambda: lib().vcas_adamw_step(self._table, len(self.tensors), self._ref, _stream_at(self.device.index))
        if torch.cuda.current_device() == self.device.index:
            rc = call()
        else:
            with torch.cuda.device(self.device):
                rc = call()
        _check(rc, "vcas_adamw_step")


def adamw_rates(lr: float, beta1: float, beta2: float, step: int) -> torch.Tensor:
    """float32 [3] on the host: what AdamW.step(rates=) reads, once copied to the device."""
    r = (C.c_float * 3)()
    _check(lib().vcas_adamw_rates(lr, beta1, beta2, step, r), "vcas_adamw_rates")
    return torch.tensor(list(r), dtype=torch.float32)


def version() -> int:
    return lib().vcas_version()
