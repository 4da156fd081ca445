"""ctypes binding of libsaf_b200.so: the same names as the C ABI, argument marshalling only.

Tensors are passed as torch CUDA tensors (device memory and streams are torch's); every step of
the computation runs in the library's kernels.  There is no fallback: if the shared library is
missing or the device is not sm_100-class the calls raise.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsaf_b200.so")

SAF_OK = 0
SAF_ERR_INVALID_ARG, SAF_ERR_UNSUPPORTED, SAF_ERR_CUDA, SAF_ERR_DEVICE_TIMEOUT, SAF_ERR_ARCH, SAF_ERR_NOMEM = range(1, 7)
SAF_BF16, SAF_F32 = 0, 1
SAF_KERNEL_FWD, SAF_KERNEL_BWD, SAF_KERNEL_BWD_PREP, SAF_KERNEL_BWD_FINALIZE, SAF_KERNEL_LOGZ, SAF_KERNEL_SCALE = range(6)
SAF_KERNEL_PGRAD, SAF_KERNEL_FIT, SAF_KERNEL_FIT_MARGINALS, SAF_KERNEL_CALIB, SAF_KERNEL_CALIB_FINALIZE = 6, 7, 8, 9, 10
SAF_KERNEL_ROTARY, SAF_KERNEL_CACHE_PLAN, SAF_KERNEL_CACHE_APPEND, SAF_KERNEL_CACHE_ATTN = range(11, 15)
SAF_ROPE_PLAIN, SAF_ROPE_LINEAR, SAF_ROPE_BASE, SAF_ROPE_RAMP = range(4)


class SafProblem(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("T", C.c_int32), ("D", C.c_int32), ("Tp", C.c_int32),
                ("softmax_scale", C.c_float), ("grad_dtype", C.c_int32), ("kv_group", C.c_int32),
                ("packed_qk", C.c_int32), ("o_dtype", C.c_int32),
                ("q_strides", C.c_int64 * 3), ("k_strides", C.c_int64 * 3), ("v_strides", C.c_int64 * 3),
                ("o_strides", C.c_int64 * 3)]


class SafRotary(C.Structure):
    _fields_ = [("B", C.c_int32), ("T", C.c_int32), ("Hq", C.c_int32), ("Hk", C.c_int32), ("D", C.c_int32), ("rot_dim", C.c_int32),
                ("interleaved", C.c_int32), ("in_dtype", C.c_int32), ("out_dtype", C.c_int32), ("mscale", C.c_float),
                ("q_strides", C.c_int64 * 3), ("k_strides", C.c_int64 * 3), ("qo_strides", C.c_int64 * 3), ("ko_strides", C.c_int64 * 3)]


class SafCache(C.Structure):
    _fields_ = [("R", C.c_int32), ("N", C.c_int32), ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32),
                ("H", C.c_int32), ("kv_group", C.c_int32), ("D", C.c_int32), ("Tp", C.c_int32), ("max_len", C.c_int32),
                ("max_new", C.c_int32), ("o_dtype", C.c_int32), ("softmax_scale", C.c_float), ("reserved", C.c_int32),
                ("q_strides", C.c_int64 * 2), ("o_strides", C.c_int64 * 2), ("vn_strides", C.c_int64 * 2),
                ("k_strides", C.c_int64 * 3), ("v_strides", C.c_int64 * 3)]


class SafError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: status {code} ({status_string(code)})")


_lib = None


def load_library() -> C.CDLL:
    """dlopen the shared library and declare the prototypes.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} not built; run `python -m paper_2609_34650_b200.build`")
    lib = C.CDLL(LIB_PATH)
    vp, i32, u8p, f32p = C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p
    pp = C.POINTER(SafProblem)
    lib.saf_version.restype = C.c_int
    lib.saf_status_string.restype = C.c_char_p
    lib.saf_status_string.argtypes = [C.c_int]
    lib.saf_create.argtypes = [C.POINTER(vp), C.c_int]
    lib.saf_destroy.argtypes = [vp]
    lib.saf_pattern_prepare.argtypes = [vp, i32, i32, u8p, f32p, f32p, f32p, vp]
    lib.saf_hybrid_attn_fwd.argtypes = [vp, pp, vp, vp, vp, u8p, f32p, f32p, f32p, vp, f32p, vp]
    lib.saf_hybrid_attn_bwd.argtypes = [vp, pp, vp, vp, vp, vp, vp, f32p, u8p, f32p, f32p, f32p, vp, vp, vp, vp]
    lib.saf_hybrid_attn_step_host.argtypes = [vp, pp, vp, vp, vp, vp, u8p, f32p, f32p, i32, vp, f32p, vp, vp, vp]
    lib.saf_pattern_grad.argtypes = [vp, pp, vp, vp, vp, u8p, f32p, f32p, f32p, f32p, f32p, vp]
    lib.saf_fit_marginals.argtypes = [vp, i32, i32, vp, C.c_float, vp, vp, vp, vp]
    lib.saf_fit_compact.argtypes = [vp, i32, i32, vp, vp, vp, i32, C.c_double, vp, vp, vp, C.c_int64, vp, vp, vp]
    lib.saf_calib_accumulate.argtypes = [vp, pp, vp, vp, vp, vp, vp, vp, i32, vp]
    lib.saf_calib_finalize.argtypes = [vp, i32, i32, C.c_int64, vp, vp, vp, vp, vp, vp]
    lib.saf_last_device_status.argtypes = [vp, C.POINTER(C.c_int32)]
    lib.saf_set_profiling.argtypes = [vp, i32]
    lib.saf_get_kernel_time.argtypes = [vp, i32, C.POINTER(C.c_float), C.POINTER(C.c_int32)]
    lib.saf_pattern_logz_static.argtypes = [i32, i32, i32, u8p, f32p, f32p, f32p, vp]
    lib.saf_pattern_logz_static.restype = C.c_int
    lib.saf_fit_handover.argtypes = [vp, i32, C.POINTER(i32)]
    lib.saf_fit_math.argtypes = [i32, i32, i32, vp, vp, vp]
    pr, pc, dp = C.POINTER(SafRotary), C.POINTER(SafCache), C.POINTER(C.c_double)
    lib.saf_rotary_freqs.argtypes = [i32, C.c_double, i32, C.c_double, i32, dp, C.POINTER(C.c_float)]
    lib.saf_rotary_fwd.argtypes = [vp, pr, vp, vp, vp, vp, vp, vp, vp]
    lib.saf_rotary_bwd.argtypes = [vp, pr, vp, vp, vp, vp, vp, vp, vp]
    lib.saf_cache_plan.argtypes = [vp, pc] + [vp] * 16
    lib.saf_cache_append.argtypes = [vp, pc, pr] + [vp] * 10
    lib.saf_cache_attn.argtypes = [vp, pc] + [vp] * 8 + [u8p] + [vp] * 5
    lib.saf_build_worklist.argtypes = [i32, i32, i32, u8p, i32, i32, i32, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    for name in ("saf_create", "saf_destroy", "saf_pattern_prepare", "saf_hybrid_attn_fwd", "saf_hybrid_attn_bwd",
                 "saf_hybrid_attn_step_host", "saf_last_device_status", "saf_build_worklist", "saf_set_profiling",
                 "saf_get_kernel_time", "saf_pattern_grad", "saf_fit_marginals", "saf_fit_compact", "saf_calib_accumulate", "saf_calib_finalize", "saf_fit_handover",
                 "saf_fit_math", "saf_rotary_freqs", "saf_rotary_fwd", "saf_rotary_bwd", "saf_cache_plan", "saf_cache_append",
                 "saf_cache_attn"):
        getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load_library().saf_status_string(code).decode()


def saf_version() -> int:
    return load_library().saf_version()


def _check(code: int, what: str):
    if code != SAF_OK:
        raise SafError(code, what)


# Marshalling is most of a short call's host time, which bounds short calls one after another (forward + backward of 1 x 4 x 256 x
# 64: 32 us on the host against 27 of the GPU's): masks go as bytes, addresses and the stream as plain integers (a stream
# object, its wrapper and a ctypes array pointer cost 3.5, 0.3 and 1.7 us; these 0.3, 0.1 and 0.4).
def _mask(mask):
    if type(mask) is list:
        try:
            return bytes(mask)                             # (0.6 us less than by way of an array)
        except (TypeError, ValueError):
            pass
    return np.asarray(mask, dtype=np.uint8).tobytes()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _ptrs(*tensors):
    # (one Python call for all of a call's tensors: 0.5 us less than _ptr for each of sixteen)
    return [None if t is None else t.data_ptr() for t in tensors]


_raw_stream = None


def _stream():
    global _raw_stream
    if _raw_stream is None:
        import torch
        # (the queries behind the public ones, which other torch releases need not have)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw:
            torch.cuda.current_device()                    # CUDA is set up, which the private query does not see to
        current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _raw_stream = (lambda: raw(current_device())) if raw else (lambda: torch.cuda.current_stream().cuda_stream)
    return _raw_stream()


def saf_build_worklist(B, H, T, mask, backward, n_ctas, frozen_weight_pct=60):
    """Host-only: returns (items [n,4] int32 = (b,h,block,kind), offsets [n_ctas+1] int32)."""
    lib = load_library()
    nblk = (T + 127) // 128
    items = np.zeros((B * H * nblk, 4), dtype=np.int32)
    offsets = np.zeros(n_ctas + 1, dtype=np.int32)
    _check(lib.saf_build_worklist(B, H, T, _mask(mask), int(backward), n_ctas, frozen_weight_pct,
                                  items.ctypes.data_as(C.POINTER(C.c_int32)),
                                  offsets.ctypes.data_as(C.POINTER(C.c_int32))), "saf_build_worklist")
    return items, offsets


def saf_pattern_logz_static(device, mask, alpha, rho, logZ_out):
    """Row normalisers through the entry point that allocates nothing (no context; at most 1024 heads)."""
    H, Tp = alpha.shape
    _check(load_library().saf_pattern_logz_static(device, H, Tp, _mask(mask), _ptr(alpha), _ptr(rho), _ptr(logZ_out), _stream()),
           "saf_pattern_logz_static")


def make_problem(q_like, Tp, softmax_scale=0.0, grad_dtype=SAF_F32, k_like=None, v_like=None, o_like=None,
                 kv_group=1, packed_qk=False, H=None, o_dtype=SAF_BF16):
    """saf_problem from [B,H,T,D] torch tensors (any strides with a unit feature stride); with kv_group > 1
    k_like / v_like are the [B,H/kv_group,T,D] shared key/value tensors."""
    B, Hq, T, D = q_like.shape
    H = Hq if H is None else H              # packed_qk: q_like has only the ordinary heads, pass H
    p = SafProblem()
    p.B, p.H, p.T, p.D, p.Tp = B, H, T, D, Tp
    p.softmax_scale = softmax_scale
    p.grad_dtype = grad_dtype
    p.kv_group = kv_group
    p.packed_qk = int(packed_qk)
    p.o_dtype = o_dtype
    for name, t in (("q_strides", q_like), ("k_strides", k_like if k_like is not None else q_like),
                    ("v_strides", v_like if v_like is not None else q_like),
                    ("o_strides", o_like if o_like is not None else q_like)):
        assert t.stride(3) == 1, "feature stride must be 1"
        arr = getattr(p, name)
        arr[0], arr[1], arr[2] = t.stride(0), t.stride(1), t.stride(2)
    return p


def _dtype(t):
    import torch
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise SafError(SAF_ERR_UNSUPPORTED, f"dtype {t.dtype}")
    return SAF_F32 if t.dtype == torch.float32 else SAF_BF16


def make_rotary(q, k, q_out, k_out, rot_dim, interleaved=False, mscale=1.0):
    """saf_rotary from [B,H,T,D] tensors (any strides with a unit feature stride), or [N,H,D] ones: packed rows, one batch entry.
    q or k (with its output) may be None, and k_out where the keys go into a cache; for saf_rotary_bwd pass the gradients."""
    first = q if q is not None else k
    r = SafRotary()
    packed = first.dim() == 3
    r.B, r.T, r.D = (1, first.shape[0], first.shape[2]) if packed else (first.shape[0], first.shape[2], first.shape[3])
    r.Hq, r.Hk = (0 if t is None else t.shape[1] for t in (q, k))
    r.rot_dim, r.interleaved, r.mscale = rot_dim, int(interleaved), mscale
    r.in_dtype = _dtype(first)
    out = q_out if q_out is not None else k_out
    r.out_dtype = r.in_dtype if out is None else _dtype(out)
    for name, t, like in (("q_strides", q, q), ("k_strides", k, k), ("qo_strides", q_out, q), ("ko_strides", k_out, k)):
        if t is None:
            continue
        assert t.stride(-1) == 1, "feature stride must be 1"
        assert t.shape == like.shape and t.shape[-1] == r.D and t.dim() == first.dim(), "outputs have their inputs' shapes"
        assert t.shape[0] == first.shape[0] and (packed or t.shape[2] == r.T), "queries and keys have the same tokens"
        assert _dtype(t) == (r.in_dtype if name[1] == "_" else r.out_dtype), "one dtype for both inputs, one for both outputs"
        arr = getattr(r, name)
        arr[0], arr[1], arr[2] = (t.shape[0] * t.stride(0), t.stride(1), t.stride(0)) if packed else (t.stride(0), t.stride(1), t.stride(2))
    return r


def make_cache(R, N, page_size, n_pages, max_pages, k_cache=None, v_cache=None, q_like=None, o_like=None, v_like=None, Tp=0,
               max_len=0, max_new=1, softmax_scale=0.0):
    """saf_cache from its sizes and, as far as a call uses them, the pools [n_pages,heads,page_size,D], queries and outputs [N,H,D]
    and new values [N,heads,D] (any strides with a unit feature stride)."""
    c = SafCache()
    c.R, c.N, c.page_size, c.n_pages, c.max_pages = R, N, page_size, n_pages, max_pages
    c.Tp, c.max_len, c.max_new, c.softmax_scale = Tp, max_len, max_new, softmax_scale
    c.kv_group = 1
    for name, t in (("k_strides", k_cache), ("v_strides", v_cache)):
        if t is not None:
            assert t.stride(3) == 1 and t.shape[0] == n_pages and t.shape[2] == page_size, "pools are [n_pages,heads,page_size,D]"
            c.H, c.D = t.shape[1], t.shape[3]
            getattr(c, name)[:] = [t.stride(0), t.stride(1), t.stride(2)]
    for name, t in (("q_strides", q_like), ("o_strides", o_like), ("vn_strides", v_like)):
        if t is not None:
            assert t.stride(2) == 1 and t.shape[0] == N and t.shape[2] == c.D, "packed rows are [N,heads,D]"
            getattr(c, name)[:] = [t.stride(0), t.stride(1)]
    if k_cache is not None and v_cache is not None:
        assert k_cache.shape == v_cache.shape, "one shape of both pools"
    if v_like is not None:
        assert v_like.shape[1] == c.H, "new values have the pools' heads"
    if q_like is not None:
        assert q_like.shape[1] % c.H == 0, "query heads are a multiple of the pools' heads"
        c.kv_group = q_like.shape[1] // c.H
        c.H = q_like.shape[1]
    if o_like is not None:
        assert o_like.shape[1] == c.H, "outputs have the query heads"
        c.o_dtype = _dtype(o_like)
    return c


def saf_rotary_freqs(rot_dim, base=10000.0, scaling=SAF_ROPE_PLAIN, factor=1.0, trained_len=0):
    """Host only: (radians per position, float64 [rot_dim/2]; factor for make_rotary's mscale)."""
    freqs, mscale = np.zeros(max(rot_dim // 2, 1), dtype=np.float64), C.c_float(1.0)
    _check(load_library().saf_rotary_freqs(rot_dim, float(base), int(scaling), float(factor), int(trained_len),
                                           freqs.ctypes.data_as(C.POINTER(C.c_double)), C.byref(mscale)), "saf_rotary_freqs")
    return freqs, mscale.value


def saf_fit_math(device, which, x, y):
    """y = 1 / x (which = 0), sqrt(x) (1) or exp(x) (2) by the fitter's own fp64 functions."""
    _check(load_library().saf_fit_math(device, which, x.numel(), _ptr(x), _ptr(y), _stream()), "saf_fit_math")


class Context:
    """Owns a saf_ctx on one CUDA device."""

    def __init__(self, device: int = 0):
        self._lib = load_library()
        self._h = C.c_void_p()
        _check(self._lib.saf_create(C.byref(self._h), device), "saf_create")

    def close(self):
        if self._h:
            self._lib.saf_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def saf_pattern_prepare(self, mask, alpha, rho, logZ_out):
        H, Tp = alpha.shape
        _check(self._lib.saf_pattern_prepare(self._h, H, Tp, _mask(mask), _ptr(alpha), _ptr(rho), _ptr(logZ_out), _stream()),
               "saf_pattern_prepare")

    def saf_hybrid_attn_fwd(self, prob, Q, K, V, mask, alpha, rho, logZ, O, LSE):
        _check(self._lib.saf_hybrid_attn_fwd(self._h, C.byref(prob), _ptr(Q), _ptr(K), _ptr(V), _mask(mask), _ptr(alpha),
                                             _ptr(rho), _ptr(logZ), _ptr(O), _ptr(LSE), _stream()),
               "saf_hybrid_attn_fwd")

    def saf_hybrid_attn_bwd(self, prob, Q, K, V, O, dO, LSE, mask, alpha, rho, logZ, dQ, dK, dV):
        _check(self._lib.saf_hybrid_attn_bwd(self._h, C.byref(prob), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO),
                                             _ptr(LSE), _mask(mask), _ptr(alpha), _ptr(rho), _ptr(logZ), _ptr(dQ), _ptr(dK),
                                             _ptr(dV), _stream()), "saf_hybrid_attn_bwd")

    def saf_pattern_grad(self, prob, V, O, dO, mask, alpha, rho, logZ, dalpha, drho):
        _check(self._lib.saf_pattern_grad(self._h, C.byref(prob), _ptr(V), _ptr(O), _ptr(dO), _mask(mask), _ptr(alpha),
                                          _ptr(rho), _ptr(logZ), _ptr(dalpha), _ptr(drho), _stream()),
               "saf_pattern_grad")

    def saf_fit_marginals(self, Hf, T, mean_attn, floor_value, eta_abs, eta_rel, plogp):
        _check(self._lib.saf_fit_marginals(self._h, int(Hf), int(T), _ptr(mean_attn), float(floor_value), _ptr(eta_abs),
                                           _ptr(eta_rel), _ptr(plogp), _stream()), "saf_fit_marginals")

    def saf_fit_compact(self, Hf, T, eta_abs, eta_rel, plogp, steps, lr, alpha, rho, logZ, out_stride, loss, kl):
        _check(self._lib.saf_fit_compact(self._h, int(Hf), int(T), _ptr(eta_abs), _ptr(eta_rel), _ptr(plogp),
                                         int(steps), float(lr), _ptr(alpha), _ptr(rho), _ptr(logZ), int(out_stride),
                                         _ptr(loss), _ptr(kl), _stream()), "saf_fit_compact")

    def saf_fit_handover(self, Hf):
        """Per head of the last fit: -1 transforms throughout, k >= 1 direct sums from step k on, 0 direct sums throughout."""
        steps = np.zeros(Hf, dtype=np.int32)
        _check(self._lib.saf_fit_handover(self._h, Hf, steps.ctypes.data_as(C.POINTER(C.c_int32))), "saf_fit_handover")
        return steps

    def saf_calib_accumulate(self, prob, Q, K, LSE, mean_sum, sumsq, sum_plogp, accumulate):
        _check(self._lib.saf_calib_accumulate(self._h, C.byref(prob), _ptr(Q), _ptr(K), _ptr(LSE), _ptr(mean_sum),
                                              _ptr(sumsq), _ptr(sum_plogp), int(bool(accumulate)), _stream()),
               "saf_calib_accumulate")

    def saf_calib_finalize(self, H, T, n_total, mean, sumsq, sum_plogp, s_var, s_kl):
        _check(self._lib.saf_calib_finalize(self._h, int(H), int(T), int(n_total), _ptr(mean), _ptr(sumsq),
                                            _ptr(sum_plogp), _ptr(s_var), _ptr(s_kl), _stream()), "saf_calib_finalize")

    def saf_hybrid_attn_step_host(self, prob, Q, K, V, dO, mask, alpha, rho, prepare, O, LSE, dQ, dK, dV):
        """All tensor arguments are HOST tensors (torch CPU tensors, ideally pinned) or None."""
        _check(self._lib.saf_hybrid_attn_step_host(self._h, C.byref(prob), _ptr(Q), _ptr(K), _ptr(V), _ptr(dO), _mask(mask),
                                                   _ptr(alpha), _ptr(rho), int(prepare), _ptr(O), _ptr(LSE), _ptr(dQ),
                                                   _ptr(dK), _ptr(dV)), "saf_hybrid_attn_step_host")

    def saf_rotary_fwd(self, rot, q, k, positions, freqs, q_out, k_out):
        _check(self._lib.saf_rotary_fwd(self._h, C.byref(rot), *_ptrs(q, k, positions, freqs, q_out, k_out), _stream()),
               "saf_rotary_fwd")

    def saf_rotary_bwd(self, rot, dq_out, dk_out, positions, freqs, dq, dk):
        _check(self._lib.saf_rotary_bwd(self._h, C.byref(rot), *_ptrs(dq_out, dk_out, positions, freqs, dq, dk), _stream()),
               "saf_rotary_bwd")

    def saf_cache_plan(self, cache, ctx_lens, new_lens, parents, held_in, held_out, free_count_in, free_count_out, free_list,
                       block_table, new_offsets, kv_lens, slots, positions, tree_masks, missing):
        _check(self._lib.saf_cache_plan(self._h, C.byref(cache),
                                        *_ptrs(ctx_lens, new_lens, parents, held_in, held_out, free_count_in, free_count_out,
                                               free_list, block_table, new_offsets, kv_lens, slots, positions, tree_masks,
                                               missing), _stream()), "saf_cache_plan")

    def saf_cache_append(self, cache, rot, q, k, v, slots, positions, freqs, q_out, k_cache, v_cache):
        _check(self._lib.saf_cache_append(self._h, C.byref(cache), C.byref(rot),
                                          *_ptrs(q, k, v, slots, positions, freqs, q_out, k_cache, v_cache), _stream()),
               "saf_cache_append")

    def saf_cache_attn(self, cache, Q, k_cache, v_cache, block_table, new_offsets, kv_lens, positions, tree_masks, mask, alpha, rho,
                       O, LSE):
        _check(self._lib.saf_cache_attn(self._h, C.byref(cache),
                                        *_ptrs(Q, k_cache, v_cache, block_table, new_offsets, kv_lens, positions, tree_masks),
                                        _mask(mask), *_ptrs(alpha, rho, O, LSE), _stream()), "saf_cache_attn")

    def saf_set_profiling(self, enable: bool):
        _check(self._lib.saf_set_profiling(self._h, int(enable)), "saf_set_profiling")

    def saf_get_kernel_time(self, which: int):
        """(total milliseconds, launches) of kernel `which` since the previous query."""
        ms, n = C.c_float(0.0), C.c_int32(0)
        _check(self._lib.saf_get_kernel_time(self._h, which, C.byref(ms), C.byref(n)), "saf_get_kernel_time")
        return ms.value, n.value

    def saf_last_device_status(self):
        detail = C.c_int32(0)
        code = self._lib.saf_last_device_status(self._h, C.byref(detail))
        return code, detail.value
