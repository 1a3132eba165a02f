"""Python binding of libecasq (include/ecasq.h): argument marshalling only.

Every step of the computation runs in the library's HIP kernels; PyTorch
provides device memory and the current stream.  The functions carry the C
names.  If libecasq.so is missing or cannot be loaded, the first call raises:
there is no fallback.
"""
import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libecasq.so")

ECASQ_OK = 0
ECASQ_EINVAL = -1
ECASQ_ENONFINITE = -2
ECASQ_EINFEASIBLE = -3
ECASQ_ENOMEM = -4
ECASQ_EHIP = -5
ECASQ_EWORKSPACE = -6

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


class ecasq_options(ctypes.Structure):
    _fields_ = [
        ("refine_rounds", ctypes.c_int32),
        ("refine_exhaustive", ctypes.c_int32),
        ("exact_s", ctypes.c_int32),
        ("max_search_passes", ctypes.c_int32),
        ("recovery", ctypes.c_int32),
        ("search_width", ctypes.c_int32),
        ("dp_schedule", ctypes.c_int32),
        ("alphabet", ctypes.c_int32),
        ("alphabet_size", ctypes.c_int32),
        ("optimal_scan", ctypes.c_int32),
        ("dp_objective", ctypes.c_int32),
    ]


class ecasq_info(ctypes.Structure):
    _fields_ = [
        ("t", ctypes.c_int32),
        ("p", ctypes.c_int32),
        ("lambda_", ctypes.c_double),
        ("mse", ctypes.c_double),
        ("vnmse", ctypes.c_double),
        ("entropy", ctypes.c_double),
        ("entropy_surrogate", ctypes.c_double),
        ("objective", ctypes.c_double),
        ("rate_total", ctypes.c_double),
        ("dp_solves", ctypes.c_int32),
        ("refine_rounds_run", ctypes.c_int32),
        ("cells", ctypes.c_int64),
        ("status", ctypes.c_int32),
        ("search_passes", ctypes.c_int32),
    ]

    def as_dict(self):
        d = {k: getattr(self, k) for k, _ in self._fields_}
        d["lambda"] = d.pop("lambda_")
        return d


class _kv_struct(ctypes.Structure):
    _fields_ = [
        ("dt", ctypes.c_int32),
        ("coded", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("batch", ctypes.c_int32),
        ("max_pages", ctypes.c_int32),
        ("n_pages", ctypes.c_int32),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_books", ctypes.c_void_p),
        ("v_books", ctypes.c_void_p),
        ("table", ctypes.c_void_p),
        ("lens", ctypes.c_void_p),
        ("mass", ctypes.c_void_p),
        ("pos", ctypes.c_void_p),
    ]


class EcasqError(RuntimeError):
    def __init__(self, status):
        self.status = status
        super().__init__(f"ecasq status {status}: {ecasq_status_string(status)}")


_lib = None
EXPORTS = (
    "ecasq_default_options", "ecasq_solve", "ecasq_solve_ex", "ecasq_solve_lagrangian",
    "ecasq_quantize", "ecasq_solve_batched", "ecasq_workspace_size", "ecasq_status_string",
    "ecasq_histogram", "ecasq_dp_trace", "ecasq_timing_enable", "ecasq_timing_read",
    "ecasq_solve_budgets", "ecasq_solve_optimal", "ecasq_opt_trace",
    "ecasq_solve_timeshare", "ecasq_quantize_timeshare", "ecasq_encode_bound", "ecasq_encode",
    "ecasq_decode", "ecasq_quantize_noalloc", "ecasq_inspect_enable", "ecasq_inspect_points",
    "ecasq_inspect_results", "ecasq_trim",
    "ecasq_weights_size", "ecasq_weights_pack", "ecasq_matvec", "ecasq_kv_write",
    "ecasq_kv_attention_workspace", "ecasq_kv_attention", "ecasq_kv_evict_workspace",
    "ecasq_kv_evict",
)


def lib():
    """Load libecasq.so (built in place by build.py); raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with python -m "
                           "paper_2608_18147_amd.build")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, dbl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double
    P = ctypes.POINTER
    L.ecasq_default_options.argtypes = [P(ecasq_options)]
    L.ecasq_default_options.restype = None
    L.ecasq_solve.argtypes = [vp, i32, i64, i32, dbl, vp, vp, vp, P(ecasq_info)]
    L.ecasq_solve_ex.argtypes = [vp, i32, i64, i32, dbl, P(ecasq_options), vp, vp, vp,
                                 P(ecasq_info), vp, ctypes.c_size_t]
    L.ecasq_solve_lagrangian.argtypes = [vp, i32, i64, i32, dbl, P(ecasq_options), vp, vp, vp,
                                         P(ecasq_info)]
    L.ecasq_solve_budgets.argtypes = [vp, i32, i64, i32, i32, P(dbl), P(ecasq_options), vp, vp,
                                      vp, P(ecasq_info)]
    L.ecasq_quantize.argtypes = [vp, i32, i64, vp, i32, ctypes.c_uint64, vp, vp, vp, vp]
    L.ecasq_quantize_noalloc.argtypes = [vp, i32, i64, vp, i32, ctypes.c_uint64, vp, vp, vp, vp]
    L.ecasq_solve_optimal.argtypes = [vp, i32, i64, i32, dbl, P(ecasq_options), vp, vp, vp,
                                      P(ecasq_info)]
    L.ecasq_opt_trace.argtypes = [vp, i32, i64, i32, dbl, P(ecasq_options), vp, i64, vp, vp,
                                  P(i32), P(dbl)]
    L.ecasq_solve_timeshare.argtypes = [vp, i32, i64, i32, dbl, P(ecasq_options), vp, vp, vp,
                                        P(dbl), P(ecasq_info)]
    L.ecasq_quantize_timeshare.argtypes = [vp, i32, i64, vp, i32, vp, i32, dbl,
                                           ctypes.c_uint64, vp, vp, vp, vp, vp]
    L.ecasq_encode_bound.argtypes = [i64, i32]
    L.ecasq_encode_bound.restype = ctypes.c_size_t
    L.ecasq_encode.argtypes = [vp, i64, i32, vp, vp, ctypes.c_size_t, P(i64)]
    L.ecasq_decode.argtypes = [vp, i64, i64, i32, vp, vp]
    L.ecasq_solve_batched.argtypes = [vp, i32, i64, i64, i32, dbl, P(ecasq_options), vp, vp,
                                      vp, vp]
    L.ecasq_workspace_size.argtypes = [i64, i32, i32]
    L.ecasq_workspace_size.restype = ctypes.c_size_t
    L.ecasq_trim.argtypes = []
    L.ecasq_status_string.argtypes = [i32]
    L.ecasq_status_string.restype = ctypes.c_char_p
    L.ecasq_histogram.argtypes = [vp, i32, i64, vp, vp, vp, vp, vp, P(i64)]
    L.ecasq_dp_trace.argtypes = [vp, i32, i64, i32, i32, P(dbl), i32, vp, vp, vp, vp, vp,
                                 P(dbl)]
    L.ecasq_inspect_enable.argtypes = [i32]
    L.ecasq_inspect_enable.restype = None
    L.ecasq_inspect_points.argtypes = [vp, i32]
    L.ecasq_inspect_points.restype = i32
    L.ecasq_inspect_results.argtypes = [vp, vp, i32]
    L.ecasq_inspect_results.restype = i32
    L.ecasq_timing_enable.argtypes = [i32]
    L.ecasq_timing_enable.restype = None
    L.ecasq_timing_read.argtypes = [i32, P(dbl), P(i64), P(i64), i32]
    L.ecasq_timing_read.restype = None
    L.ecasq_weights_size.argtypes = [i64, i64, i64]
    L.ecasq_weights_size.restype = ctypes.c_size_t
    L.ecasq_weights_pack.argtypes = [vp, vp, i32, vp, i32, i64, i64, i64, vp, vp,
                                     ctypes.c_size_t]
    L.ecasq_matvec.argtypes = [vp, i32, i64, i64, i64, vp, i64, i64, vp, vp]
    L.ecasq_kv_write.argtypes = [P(_kv_struct), vp, i64, vp, i64, i64, vp, vp, vp, vp, vp, vp, vp,
                                 i32, ctypes.c_uint64, vp, vp]
    L.ecasq_kv_attention_workspace.argtypes = [P(_kv_struct), i32, i32]
    L.ecasq_kv_attention_workspace.restype = ctypes.c_size_t
    L.ecasq_kv_attention.argtypes = [P(_kv_struct), vp, i64, i32, dbl, vp, vp, vp, vp,
                                     ctypes.c_size_t]
    L.ecasq_kv_evict_workspace.argtypes = [P(_kv_struct), i32]
    L.ecasq_kv_evict_workspace.restype = ctypes.c_size_t
    L.ecasq_kv_evict.argtypes = [P(_kv_struct), i32, i32, vp, vp, vp, vp, vp, ctypes.c_size_t]
    for name in ("ecasq_weights_pack", "ecasq_matvec", "ecasq_kv_write", "ecasq_kv_attention",
                 "ecasq_kv_evict"):
        getattr(L, name).restype = i32
    for name in ("ecasq_solve", "ecasq_solve_ex", "ecasq_solve_lagrangian", "ecasq_quantize",
                 "ecasq_solve_batched", "ecasq_histogram", "ecasq_dp_trace",
                 "ecasq_solve_budgets", "ecasq_solve_optimal", "ecasq_opt_trace",
                 "ecasq_solve_timeshare", "ecasq_quantize_timeshare", "ecasq_encode",
                 "ecasq_decode", "ecasq_quantize_noalloc", "ecasq_trim"):
        getattr(L, name).restype = i32
    _lib = L
    return L


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _check_x(x):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("x must be a CUDA (HIP) tensor")
    if x.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {x.dtype}")
    return x.contiguous().reshape(-1)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _raise(st, allow=(ECASQ_OK,)):
    if st not in allow:
        raise EcasqError(st)


def ecasq_default_options(**overrides):
    o = ecasq_options()
    lib().ecasq_default_options(ctypes.byref(o))
    for k, v in overrides.items():
        setattr(o, k, int(v))
    return o


def ecasq_status_string(status):
    return lib().ecasq_status_string(int(status)).decode()


def ecasq_workspace_size(d, s, flags=0):
    return int(lib().ecasq_workspace_size(int(d), int(s), int(flags)))


def ecasq_trim():
    """Give back the device memory and pinned blocks that the library keeps between calls."""
    _raise(lib().ecasq_trim())


def ecasq_solve(x, s, bits_per_entry, options=None, stream=None, workspace=None):
    """Budget mode.  Returns (codebook fp64 [t], rank int32 [t], info dict)."""
    x = _check_x(x)
    cb = torch.empty(int(s), dtype=torch.float64, device=x.device)
    rk = torch.empty(int(s), dtype=torch.int32, device=x.device)
    info = ecasq_info()
    if options is None and workspace is None:
        st = lib().ecasq_solve(_ptr(x), _DTYPES[x.dtype], x.numel(), int(s),
                               float(bits_per_entry), _stream(stream), _ptr(cb), _ptr(rk),
                               ctypes.byref(info))
    else:
        o = options if options is not None else ecasq_default_options()
        ws = _ptr(workspace)
        nb = workspace.numel() * workspace.element_size() if workspace is not None else 0
        st = lib().ecasq_solve_ex(_ptr(x), _DTYPES[x.dtype], x.numel(), int(s),
                                  float(bits_per_entry), ctypes.byref(o), _stream(stream),
                                  _ptr(cb), _ptr(rk), ctypes.byref(info), ws, nb)
    _raise(st, (ECASQ_OK, ECASQ_EINFEASIBLE))
    t = info.t
    return cb[:t], rk[:t], info.as_dict()


ecasq_solve_ex = ecasq_solve


def ecasq_solve_budgets(x, s, budgets, options=None, stream=None):
    """Several budgets on one input with shared DP solves.  Returns a list of
    (codebook fp64 [t], rank int32 [t], info dict), one per budget."""
    x = _check_x(x)
    nb = len(budgets)
    cb = torch.empty((nb, int(s)), dtype=torch.float64, device=x.device)
    rk = torch.empty((nb, int(s)), dtype=torch.int32, device=x.device)
    infos = (ecasq_info * nb)()
    o = options if options is not None else ecasq_default_options()
    bs = (ctypes.c_double * nb)(*[float(b) for b in budgets])
    st = lib().ecasq_solve_budgets(_ptr(x), _DTYPES[x.dtype], x.numel(), int(s), nb, bs,
                                   ctypes.byref(o), _stream(stream), _ptr(cb), _ptr(rk), infos)
    _raise(st, (ECASQ_OK, ECASQ_EINFEASIBLE))
    return [(cb[k, :infos[k].t], rk[k, :infos[k].t], infos[k].as_dict()) for k in range(nb)]


def ecasq_solve_lagrangian(x, s, lam, options=None, stream=None):
    """Fixed multiplier (vNMSE units).  Returns (codebook, rank, info dict)."""
    x = _check_x(x)
    cb = torch.empty(int(s), dtype=torch.float64, device=x.device)
    rk = torch.empty(int(s), dtype=torch.int32, device=x.device)
    info = ecasq_info()
    o = options if options is not None else ecasq_default_options()
    st = lib().ecasq_solve_lagrangian(_ptr(x), _DTYPES[x.dtype], x.numel(), int(s), float(lam),
                                      ctypes.byref(o), _stream(stream), _ptr(cb), _ptr(rk),
                                      ctypes.byref(info))
    _raise(st)
    t = info.t
    return cb[:t], rk[:t], info.as_dict()


def ecasq_solve_optimal(x, s, lam, options=None, stream=None):
    """Optimal lambda-ECASQ (Sec. 4) at lam (vNMSE units).  Returns (codebook,
    rank, info dict)."""
    x = _check_x(x)
    cb = torch.empty(int(s), dtype=torch.float64, device=x.device)
    rk = torch.empty(int(s), dtype=torch.int32, device=x.device)
    info = ecasq_info()
    o = options if options is not None else ecasq_default_options()
    st = lib().ecasq_solve_optimal(_ptr(x), _DTYPES[x.dtype], x.numel(), int(s), float(lam),
                                   ctypes.byref(o), _stream(stream), _ptr(cb), _ptr(rk),
                                   ctypes.byref(info))
    _raise(st)
    t = info.t
    return cb[:t], rk[:t], info.as_dict()


def ecasq_opt_trace(x, s, lam, p, options=None, stream=None):
    """Every layer of the optimal DP for an input with p permissible values.
    Returns (F [imax+1, p, p] with F[i, j, l] = dp(i, l, j), K [imax+1, p, p]
    with K[i, l, j] the minimising k, chain list, DP value, cells); entries
    outside a layer's valid (l, j) are unspecified."""
    x = _check_x(x)
    imax = min(int(s), int(p))
    cap = (imax + 1) * p * p
    F = torch.empty(cap, dtype=torch.float64, device=x.device)
    K = torch.empty(cap, dtype=torch.int32, device=x.device)
    chain = (ctypes.c_int32 * int(s))()
    out = (ctypes.c_double * 4)()
    o = options if options is not None else ecasq_default_options()
    st = lib().ecasq_opt_trace(_ptr(x), _DTYPES[x.dtype], x.numel(), int(s), float(lam),
                               ctypes.byref(o), _stream(stream), cap, _ptr(F), _ptr(K), chain,
                               out)
    _raise(st)
    if int(out[2]) != p:
        raise ValueError(f"input has {int(out[2])} permissible values, not {p}")
    t = int(out[1])
    return (F.view(imax + 1, p, p), K.view(imax + 1, p, p), list(chain[:t]), out[0],
            int(out[3]))


def ecasq_solve_timeshare(x, s, bits_per_entry, options=None, stream=None):
    """Two-way time-sharing (Sec. 7).  Returns (minus, plus, alpha): minus
    and plus are (codebook, rank, info dict) of B (H <= b) and A (H > b);
    alpha is the share of entries quantized with plus."""
    x = _check_x(x)
    cb = torch.empty((2, int(s)), dtype=torch.float64, device=x.device)
    rk = torch.empty((2, int(s)), dtype=torch.int32, device=x.device)
    infos = (ecasq_info * 2)()
    alpha = ctypes.c_double(0.0)
    o = options if options is not None else ecasq_default_options()
    st = lib().ecasq_solve_timeshare(_ptr(x), _DTYPES[x.dtype], x.numel(), int(s),
                                     float(bits_per_entry), ctypes.byref(o), _stream(stream),
                                     _ptr(cb), _ptr(rk), ctypes.byref(alpha), infos)
    _raise(st, (ECASQ_OK, ECASQ_EINFEASIBLE))
    out = [(cb[k, :infos[k].t], rk[k, :infos[k].t], infos[k].as_dict()) for k in range(2)]
    return out[0], out[1], alpha.value


def ecasq_quantize_timeshare(x, codebook0, codebook1, alpha, seed, stream=None):
    """Returns (symbols uint8 [d], part uint8 [d] (1 = codebook1), entropy
    (0-d fp64 tensor), hist int64 [t0 + t1])."""
    x = _check_x(x)
    c0 = codebook0.to(device=x.device, dtype=torch.float64).contiguous()
    c1 = codebook1.to(device=x.device, dtype=torch.float64).contiguous()
    t0, t1 = c0.numel(), c1.numel()
    sym = torch.empty(x.numel(), dtype=torch.uint8, device=x.device)
    part = torch.empty(x.numel(), dtype=torch.uint8, device=x.device)
    ent = torch.empty((), dtype=torch.float64, device=x.device)
    hist = torch.empty(t0 + t1, dtype=torch.int64, device=x.device)
    st = lib().ecasq_quantize_timeshare(_ptr(x), _DTYPES[x.dtype], x.numel(), _ptr(c0), t0,
                                        _ptr(c1), t1, float(alpha),
                                        ctypes.c_uint64(int(seed) & (2 ** 64 - 1)),
                                        _stream(stream), _ptr(sym), _ptr(part), _ptr(ent),
                                        _ptr(hist))
    _raise(st)
    return sym, part, ent, hist


def ecasq_encode(symbols, t, stream=None):
    """rANS-code uint8 symbols (device) over t values.  Returns the stream as
    a uint8 device tensor."""
    if not isinstance(symbols, torch.Tensor) or not symbols.is_cuda or symbols.dtype != torch.uint8:
        raise TypeError("symbols must be a uint8 CUDA (HIP) tensor")
    sym = symbols.contiguous()
    d = sym.numel()
    cap = lib().ecasq_encode_bound(d, int(t))
    if cap == 0:
        raise ValueError("d or t out of range")
    out = torch.empty(cap, dtype=torch.uint8, device=sym.device)
    n = ctypes.c_int64(0)
    st = lib().ecasq_encode(_ptr(sym), d, int(t), _stream(stream), _ptr(out), cap,
                            ctypes.byref(n))
    _raise(st)
    return out[: n.value]


def ecasq_decode(data, d, t, stream=None):
    """Decode a stream of ecasq_encode back to d uint8 symbols (device)."""
    data = data.contiguous()
    sym = torch.empty(int(d), dtype=torch.uint8, device=data.device)
    st = lib().ecasq_decode(_ptr(data), data.numel(), int(d), int(t), _stream(stream), _ptr(sym))
    _raise(st)
    return sym


def ecasq_quantize(x, codebook, seed, stream=None):
    """Returns (symbols uint8 [d], empirical entropy (0-d fp64 tensor), hist int64 [t])."""
    x = _check_x(x)
    cb = codebook.to(device=x.device, dtype=torch.float64).contiguous()
    t = cb.numel()
    sym = torch.empty(x.numel(), dtype=torch.uint8, device=x.device)
    ent = torch.empty((), dtype=torch.float64, device=x.device)
    hist = torch.empty(t, dtype=torch.int64, device=x.device)
    st = lib().ecasq_quantize(_ptr(x), _DTYPES[x.dtype], x.numel(), _ptr(cb), t,
                              ctypes.c_uint64(int(seed) & (2 ** 64 - 1)), _stream(stream),
                              _ptr(sym), _ptr(ent), _ptr(hist))
    _raise(st)
    return sym, ent, hist


def ecasq_quantize_noalloc(x, codebook, seed, symbols, entropy, hist=None, stream=None):
    """ecasq_quantize into caller-provided outputs, with no allocation inside
    the library: symbols uint8 [d], entropy 0-d fp64, hist int64 [t] or None
    (all on x's device).  codebook must be a contiguous fp64 tensor there."""
    x = _check_x(x)
    if (codebook.dtype != torch.float64 or not codebook.is_contiguous()
            or codebook.device != x.device):
        raise TypeError("codebook must be a contiguous fp64 tensor on x's device")
    t = codebook.numel()
    st = lib().ecasq_quantize_noalloc(_ptr(x), _DTYPES[x.dtype], x.numel(), _ptr(codebook), t,
                                      ctypes.c_uint64(int(seed) & (2 ** 64 - 1)),
                                      _stream(stream), _ptr(symbols), _ptr(entropy),
                                      _ptr(hist) if hist is not None else None)
    _raise(st)
    return symbols, entropy, hist


def ecasq_solve_batched(x, s, bits_per_entry, options=None, stream=None):
    """x: [n, d] rows.  Returns (codebooks fp64 [n, s], t int32 [n], infos uint8 view)."""
    if x.dim() != 2:
        raise ValueError("x must be [n, d]")
    n, d = x.shape
    xc = _check_x(x)
    cbs = torch.zeros((n, int(s)), dtype=torch.float64, device=x.device)
    tt = torch.zeros(n, dtype=torch.int32, device=x.device)
    infos = torch.zeros((n, ctypes.sizeof(ecasq_info)), dtype=torch.uint8, device=x.device)
    o = options if options is not None else ecasq_default_options()
    st = lib().ecasq_solve_batched(_ptr(xc), _DTYPES[x.dtype], n, d, int(s),
                                   float(bits_per_entry), ctypes.byref(o), _stream(stream),
                                   _ptr(cbs), _ptr(tt), _ptr(infos))
    _raise(st, (ECASQ_OK, ECASQ_EINFEASIBLE))
    return cbs, tt, infos


# ---------------------------------------------------------------------------
# Serving: products with 4-bit weights and the paged key/value cache.  These calls
# run on their tensors' device, on its current stream or on `stream`, and allocate
# what they return and their workspace there with torch's allocator.  They have no
# gradients, and refuse tensors that require one where torch records them.

_HALF = {torch.float16: 1, torch.bfloat16: 2}


class _on:
    """The device of a call's tensors as the current one, and the call's stream
    as torch's, so that what the call allocates belongs to that stream."""

    def __init__(self, device, stream):
        if stream is not None and stream.device != device:
            raise ValueError(f"the stream must be on {device}")
        self.device, self.stream = torch.cuda.device(device), stream

    def __enter__(self):
        self.device.__enter__()
        if self.stream is not None:
            self.stream = torch.cuda.stream(self.stream)
            self.stream.__enter__()

    def __exit__(self, *exc):
        if self.stream is not None:
            self.stream.__exit__(*exc)
        self.device.__exit__(*exc)


def _run(f, device, stream, *args):
    """f(stream, *args) with the device and the stream as torch's current ones,
    which most calls find that way (the contexts cost as much as a small kernel)."""
    index = device.index
    if stream is None and torch._C._cuda_getDevice() == index:
        return f(torch._C._cuda_getCurrentRawStream(index), *args)
    with _on(device, stream):
        return f(torch._C._cuda_getCurrentRawStream(index), *args)


def _tensor(x, name, dtype, device, shape=None):
    """x, once it is seen to be a contiguous tensor as the library needs it."""
    if not isinstance(x, torch.Tensor) or x.dtype != dtype or x.device != device:
        raise TypeError(f"{name} must be a {dtype} tensor on {device}")
    if shape is not None and x.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}")
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return x


def _no_gradient(x, name):
    """Refuses x where its gradient would be recorded.  (Calls of each step ask for
    x.requires_grad themselves.)"""
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, and there is none: detach it, or call "
                         "under torch.no_grad()")


def _half_tensor(x, name):
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in _HALF:
        raise TypeError(f"{name} must be a float16 or bfloat16 CUDA (HIP) tensor")
    return x


def _rows_apart(x, inner):
    """x [rows, ...] whose rows of `inner` entries are contiguous, and the entries
    between their starts; copied where they do not lie that way."""
    if x.is_contiguous():
        return x, inner
    want = 1
    for size, step in zip(reversed(x.shape[1:]), reversed(x.stride()[1:])):
        if size != 1 and step != want:
            return x.contiguous(), inner
        want *= size
    step = x.stride(0) if x.shape[0] > 1 else inner
    return (x, step) if step >= inner else (x.contiguous(), inner)


class ecasq_weights:
    """A packed 4-bit weight matrix (ecasq_weights_pack)."""

    __slots__ = ("packed", "dtype", "device", "n_out", "n_in", "group")

    def __init__(self, packed, dtype, n_out, n_in, group):
        self.packed, self.dtype, self.device = packed, dtype, packed.device
        self.n_out, self.n_in, self.group = n_out, n_in, group


def ecasq_weights_pack(symbols, codebook, scales, group, stream=None):
    """Lays out symbols uint8 [n_out, n_in] with a codebook of at most 16 values
    and scales (float16 or bfloat16, the products' type) [n_out, ceil(n_in /
    group)] for ecasq_matvec."""
    _half_tensor(scales, "scales")
    if not isinstance(symbols, torch.Tensor) or symbols.dim() != 2 or \
            symbols.dtype != torch.uint8 or symbols.device != scales.device:
        raise TypeError("symbols must be a uint8 tensor [n_out, n_in] on the scales' device")
    n_out, n_in = symbols.shape
    group = int(group)
    size = lib().ecasq_weights_size(n_out, n_in, group)
    if size == 0:
        raise ValueError("sizes or group out of range")
    if tuple(scales.shape) != (n_out, -(-n_in // group)):
        raise ValueError("scales must be [n_out, ceil(n_in / group)]")
    _no_gradient(scales, "scales")
    _no_gradient(codebook, "codebook")
    return _run(_pack, scales.device, stream, symbols, codebook, scales, group, size)


def _pack(st, symbols, codebook, scales, group, size):
    n_out, n_in = symbols.shape
    cb = codebook.to(device=scales.device, dtype=torch.float64).contiguous().reshape(-1)
    packed = torch.empty(size, dtype=torch.uint8, device=scales.device)
    symbols, scales = symbols.contiguous(), scales.contiguous()
    _raise(lib().ecasq_weights_pack(symbols.data_ptr(), cb.data_ptr(), cb.numel(),
                                    scales.data_ptr(), _HALF[scales.dtype], n_out, n_in, group,
                                    st, packed.data_ptr(), size))
    return ecasq_weights(packed, scales.dtype, n_out, n_in, group)


def ecasq_matvec(w, x, out=None, stream=None):
    """y = W x for every row of x [..., n_in]; returns y [..., n_out]."""
    if not isinstance(x, torch.Tensor) or x.dtype != w.dtype or x.device != w.device:
        raise TypeError(f"x must be a {w.dtype} tensor on {w.device}")
    shape = x.shape
    if not shape or shape[-1] != w.n_in:
        raise ValueError(f"x must end in {w.n_in} entries")
    if x.requires_grad:
        _no_gradient(x, "x")
    if out is not None:
        _tensor(out, "out", w.dtype, w.device, shape[:-1] + (w.n_out,))
    return _run(_matvec, w.device, stream, w, x, shape, out)


def _matvec(st, w, x, shape, out):
    n_in = w.n_in
    if len(shape) == 2 and (x.is_contiguous() or (x.stride(1) == 1 and x.stride(0) >= n_in)):
        m = shape[0]
        step = x.stride(0) if m > 1 else n_in
        if out is None:
            out = x.new_empty((m, w.n_out))
    else:
        x = x.reshape(-1, n_in).contiguous()
        m, step = x.shape[0], n_in
        if out is None:
            out = x.new_empty(shape[:-1] + (w.n_out,))
    if m:
        _raise(lib().ecasq_matvec(w.packed.data_ptr(), _HALF[w.dtype], w.n_out, n_in, w.group,
                                  x.data_ptr(), m, step, st, out.data_ptr()))
    return out


class ecasq_kv_cache:
    """A paged key/value cache over the caller's tensors, which it keeps and which
    are updated in place (another tensor cannot take an old one's name):
    k, v [n_pages, heads, page_size, head_dim] of float16 or bfloat16, or uint8
    [..., head_dim / 2] with k_books, v_books [n_pages, heads, page_size, 16];
    table int32 [batch, max_pages]; lens int32 [batch]; mass float32 and pos int32
    [batch, heads, max_pages * page_size], each where it is needed."""

    def __init__(self, k, v, table, lens, k_books=None, v_books=None, mass=None, pos=None):
        if not isinstance(k, torch.Tensor) or not k.is_cuda or k.dim() != 4:
            raise TypeError("k must be a CUDA (HIP) tensor [n_pages, heads, page_size, entries]")
        self.coded = k.dtype == torch.uint8
        if self.coded and (k_books is None or v_books is None):
            raise ValueError("a cache of symbols needs k_books and v_books")
        if not self.coded and (k_books is not None or v_books is not None):
            raise ValueError("a cache of rows has no codebooks")
        self.dtype = _half_tensor(k_books if self.coded else k, "k").dtype
        dev = self.device = k.device
        self.n_pages, self.heads, self.page_size, last = k.shape
        self.head_dim = 2 * last if self.coded else last
        if not isinstance(table, torch.Tensor) or table.dim() != 2:
            raise TypeError("table must be an int32 tensor [batch, max_pages]")
        self.batch, self.max_pages = table.shape
        self.slots = self.max_pages * self.page_size
        self.k, self.v = _tensor(k, "k", k.dtype, dev), _tensor(v, "v", k.dtype, dev, k.shape)
        self.k_books, self.v_books, self.mass, self.pos = k_books, v_books, mass, pos
        self.table = _tensor(table, "table", torch.int32, dev)
        self.lens = _tensor(lens, "lens", torch.int32, dev, (self.batch,))
        if self.coded:
            for name, x in (("k_books", k_books), ("v_books", v_books)):
                _tensor(x, name, self.dtype, dev, k.shape[:3] + (16,))
        for name, x in (("k", k), ("v", v), ("k_books", k_books), ("v_books", v_books)):
            if x is not None:
                _no_gradient(x, name)
        self._slots_shape = (self.batch, self.heads, self.slots)
        if mass is not None:
            _tensor(mass, "mass", torch.float32, dev, self._slots_shape)
        if pos is not None:
            _tensor(pos, "pos", torch.int32, dev, self._slots_shape)
        self._c = _kv_struct(_HALF[self.dtype], int(self.coded), self.heads, self.head_dim,
                             self.page_size, self.batch, self.max_pages, self.n_pages,
                             *[x.data_ptr() if x is not None else None for x in
                               (k, v, k_books, v_books, table, lens, mass, pos)])
        self._ref = ctypes.byref(self._c)
        self._unused = table.new_empty(256, dtype=torch.uint8)
        self._sizes = {}

    def __setattr__(self, name, value):
        if "_sizes" in self.__dict__ and self.__dict__.get(name) is not value:
            raise AttributeError(f"{name} is set once: update the cache's tensors in place")
        self.__dict__[name] = value

    def _workspace(self, name, *args):
        """A workspace of the size that the library's function `name` says (256 bytes:
        the call needs none, and any will do)."""
        key = (name,) + args
        size = self._sizes.get(key)
        if size is None:
            size = getattr(lib(), name)(self._ref, *args)
            if size == 0:
                raise EcasqError(ECASQ_EINVAL)
            self._sizes[key] = size
        if size <= 256:
            return self._unused, size
        return self.table.new_empty(size, dtype=torch.uint8), size


def ecasq_kv_write(kv, k, v, starts, positions=None, k_codebooks=None, k_counts=None,
                   v_codebooks=None, v_counts=None, seed=0, k_hat=None, v_hat=None, stream=None):
    """Writes new tokens' rows k, v [rows, heads, head_dim] into the cache, rows
    starts[b] .. starts[b+1]-1 (int32, device) at the end of sequence b, whose lens
    already counts them.  positions (int32 [rows], device) are the tokens' places in their
    sequences; without them the slots count as such, which holds until a sequence
    has been cut by ecasq_kv_evict.  A cache of symbols takes the rows' codebooks and counts
    as ecasq_solve_batched returns them for k.reshape(rows * heads, head_dim), and
    gives back the rounded rows in k_hat, v_hat where they are given.  Calls with one seed
    draw the same uniforms: every layer and step needs its own."""
    dev = kv.device
    for name, x in (("k", k), ("v", v)):
        if not isinstance(x, torch.Tensor) or x.dtype != kv.dtype or x.device != dev:
            raise TypeError(f"{name} must be a {kv.dtype} tensor on {dev}")
        if x.dim() != 3 or x.shape[1:] != (kv.heads, kv.head_dim) or x.shape[0] != k.shape[0]:
            raise ValueError(f"{name} must be [rows, {kv.heads}, {kv.head_dim}]")
        if x.requires_grad:
            _no_gradient(x, name)
    rows = k.shape[0]
    _tensor(starts, "starts", torch.int32, dev, (kv.batch + 1,))
    if positions is not None:
        _tensor(positions, "positions", torch.int32, dev, (rows,))
    s, books = 0, [None] * 4
    if kv.coded:
        if k_codebooks is None or v_codebooks is None or k_counts is None or v_counts is None:
            raise ValueError("a cache of symbols needs the rows' codebooks and counts")
        s = k_codebooks.shape[-1]
        for name, x in (("k_codebooks", k_codebooks), ("v_codebooks", v_codebooks)):
            _tensor(x, name, torch.float64, dev, (rows * kv.heads, s))
        for name, x in (("k_counts", k_counts), ("v_counts", v_counts)):
            _tensor(x, name, torch.int32, dev, (rows * kv.heads,))
        books = [x.data_ptr() for x in (k_codebooks, k_counts, v_codebooks, v_counts)]
        for name, x in (("k_hat", k_hat), ("v_hat", v_hat)):
            if x is not None:
                _tensor(x, name, kv.dtype, dev, (rows, kv.heads, kv.head_dim))
    elif k_codebooks is not None or v_codebooks is not None:
        raise ValueError("a cache of rows takes no codebooks")
    if rows:
        _run(_write, dev, stream, kv, k, v, starts, positions, books, s,
             int(seed) & (2 ** 64 - 1), k_hat, v_hat)


def _write(st, kv, k, v, starts, positions, books, s, seed, k_hat, v_hat):
    inner = kv.heads * kv.head_dim
    rows = k.shape[0]
    k, ks = _rows_apart(k, inner)
    v, vs = _rows_apart(v, inner)
    _raise(lib().ecasq_kv_write(kv._ref, k.data_ptr(), ks, v.data_ptr(), vs, rows,
                                starts.data_ptr(),
                                positions.data_ptr() if positions is not None else None, st,
                                *books, s, seed,
                                k_hat.data_ptr() if k_hat is not None else None,
                                v_hat.data_ptr() if v_hat is not None else None))


def ecasq_kv_attention(kv, q, scale=None, mass_out=None, out=None, stream=None):
    """Attention of one token per sequence, q [batch, q_heads, head_dim], over the
    cache; scale: 1 / sqrt(head_dim) if None.  With mass_out (float32, as
    kv.mass, which it may be) the weights of the slots are added to kv.mass there.
    Returns out [batch, q_heads, head_dim]."""
    if not isinstance(q, torch.Tensor) or q.dtype != kv.dtype or q.device != kv.device:
        raise TypeError(f"q must be a {kv.dtype} tensor on {kv.device}")
    if q.dim() != 3 or q.shape[0] != kv.batch or q.shape[2] != kv.head_dim:
        raise ValueError(f"q must be [{kv.batch}, q_heads, {kv.head_dim}]")
    if q.requires_grad:
        _no_gradient(q, "q")
    if mass_out is not None:
        _tensor(mass_out, "mass_out", torch.float32, kv.device, kv._slots_shape)
    if out is not None:
        _tensor(out, "out", kv.dtype, kv.device, q.shape)
    return _run(_attention, kv.device, stream, kv, q, scale, mass_out, out)


def _attention(st, kv, q, scale, mass_out, out):
    q_heads = q.shape[1]
    if out is None:
        out = q.new_empty(q.shape)
    q, step = _rows_apart(q, q_heads * kv.head_dim)
    ws, size = kv._workspace("ecasq_kv_attention_workspace", q_heads, int(mass_out is not None))
    _raise(lib().ecasq_kv_attention(kv._ref, q.data_ptr(), step, q_heads,
                                    kv.head_dim ** -0.5 if scale is None else float(scale),
                                    mass_out.data_ptr() if mass_out is not None else None, st,
                                    out.data_ptr(), ws.data_ptr(), size))
    return out


def ecasq_kv_evict(kv, keep, recent=0, mass_out=None, pos_out=None, lens_out=None, stream=None):
    """Every head of a sequence with more than `keep` slots gives up all but
    those of the `recent` newest positions and the largest mass; the kept rows
    are moved below slot `keep`.  kv.mass, kv.pos and kv.lens are updated, or the
    tensors given for them in their place."""
    keep, recent = int(keep), int(recent)
    if not -2 ** 31 <= keep < 2 ** 31 or not -2 ** 31 <= recent < 2 ** 31:
        raise ValueError("keep and recent must be 32-bit integers")
    if kv.mass is None or kv.pos is None:
        raise ValueError("the cache needs mass and pos")
    mass_out = kv.mass if mass_out is None else \
        _tensor(mass_out, "mass_out", torch.float32, kv.device, kv._slots_shape)
    pos_out = kv.pos if pos_out is None else \
        _tensor(pos_out, "pos_out", torch.int32, kv.device, kv._slots_shape)
    lens_out = kv.lens if lens_out is None else \
        _tensor(lens_out, "lens_out", torch.int32, kv.device, (kv.batch,))
    _run(_evict, kv.device, stream, kv, keep, recent, mass_out, pos_out, lens_out)


def _evict(st, kv, keep, recent, mass_out, pos_out, lens_out):
    ws, size = kv._workspace("ecasq_kv_evict_workspace", keep)
    _raise(lib().ecasq_kv_evict(kv._ref, keep, recent, mass_out.data_ptr(), pos_out.data_ptr(),
                                lens_out.data_ptr(), st, ws.data_ptr(), size))


def infos_to_dicts(infos):
    """Decode the device info array of ecasq_solve_batched."""
    raw = infos.cpu().numpy().tobytes()
    sz = ctypes.sizeof(ecasq_info)
    return [ecasq_info.from_buffer_copy(raw[i * sz:(i + 1) * sz]).as_dict()
            for i in range(len(raw) // sz)]


def ecasq_histogram(x, stream=None):
    """Sorted distinct values and exact prefix sums: (v, N, S, S2) fp64 [p]."""
    x = _check_x(x)
    d = x.numel()
    bufs = [torch.empty(d, dtype=torch.float64, device=x.device) for _ in range(4)]
    p = ctypes.c_int64(0)
    st = lib().ecasq_histogram(_ptr(x), _DTYPES[x.dtype], d, _stream(stream),
                               *[_ptr(b) for b in bufs], ctypes.byref(p))
    _raise(st)
    return tuple(b[: p.value] for b in bufs)


def ecasq_dp_trace(x, s, lam, stream=None, accumulators=False, schedule=0, argmins=True):
    """All layers of forward solves at one multiplier (lam a number) or at the
    8 multipliers of a search pass (lam a sequence of 8).  Returns F
    [nlam, s+1, d] fp64 (NaN where unset), kstar [nlam, s+1, d] int32 (-1
    where unset), the accumulators M and Ph like F (None unless asked for),
    and per multiplier (J, MSE, H(I,B), i*, cells).  With a scalar lam the
    leading nlam axis is dropped."""
    x = _check_x(x)
    d = x.numel()
    scalar = not hasattr(lam, "__len__")
    lams = [float(lam)] if scalar else [float(v) for v in lam]
    n = len(lams)
    shape = (n, int(s) + 1, d)
    F = torch.full(shape, float("nan"), dtype=torch.float64, device=x.device)
    K = torch.full(shape, -1, dtype=torch.int32, device=x.device) if argmins else None
    M = torch.full(shape, float("nan"), dtype=torch.float64, device=x.device) if accumulators else None
    Ph = torch.full(shape, float("nan"), dtype=torch.float64, device=x.device) if accumulators else None
    la = (ctypes.c_double * n)(*lams)
    out = (ctypes.c_double * (5 * n))()
    st = lib().ecasq_dp_trace(_ptr(x), _DTYPES[x.dtype], d, int(s), n, la, int(schedule),
                              _stream(stream), _ptr(F), _ptr(K), _ptr(M), _ptr(Ph), out)
    _raise(st)
    res = [tuple(out[5 * m:5 * m + 5]) for m in range(n)]
    if scalar:
        return (F[0], K[0] if K is not None else None, M[0] if M is not None else None,
                Ph[0] if Ph is not None else None, res[0])
    return F, K, M, Ph, res


def ecasq_inspect_enable(on=True):
    lib().ecasq_inspect_enable(1 if on else 0)


def ecasq_inspect_points():
    """The recorded search points as a float64 array [n, 4]: lambda, H, vNMSE,
    t (clears them)."""
    n = lib().ecasq_inspect_points(None, 0)
    out = np.zeros((max(n, 1), 4))
    lib().ecasq_inspect_points(out.ctypes.data_as(ctypes.c_void_p), n)
    return out[:n]


def ecasq_inspect_results():
    """The recorded budget results (clears them): dicts with lam_B (the
    multiplier the codebook was found at), lam_final (the refinement's), pre
    and post (value indices before and after refinement)."""
    n = lib().ecasq_inspect_results(None, None, 0)
    lams = np.zeros(2 * max(n, 1))
    ch = np.zeros(514 * max(n, 1), dtype=np.int32)
    lib().ecasq_inspect_results(lams.ctypes.data_as(ctypes.c_void_p),
                                ch.ctypes.data_as(ctypes.c_void_p), n)
    out = []
    for k in range(n):
        row = ch[514 * k: 514 * (k + 1)]
        out.append(dict(lam_B=float(lams[2 * k]), lam_final=float(lams[2 * k + 1]),
                        pre=row[1: 1 + row[0]].copy(), post=row[258: 258 + row[257]].copy()))
    return out


def ecasq_timing_enable(on=True, verbose=False):
    lib().ecasq_timing_enable((2 if verbose else 1) if on else 0)


TIMING_SINGLE = 0  # one multiplier per DP layer launch
TIMING_PASS = 1    # the 8 multipliers of a search pass per launch
TIMING_SWEEP = 2   # one whole solve of DP schedule 1
TIMING_OPT = 3     # one layer of the optimal DP
TIMING_BATCHED = 4  # one launch of ecasq_solve_batched


def ecasq_timing_read(variant=TIMING_PASS, reset=False):
    """(milliseconds, launches, cells) of the timed DP layer kernel launches of
    one variant; cells are (column, predecessor) pairs, each evaluated for
    every multiplier of its launch."""
    ms = ctypes.c_double(0)
    n = ctypes.c_int64(0)
    c = ctypes.c_int64(0)
    lib().ecasq_timing_read(int(variant), ctypes.byref(ms), ctypes.byref(n), ctypes.byref(c),
                            1 if reset else 0)
    return ms.value, n.value, c.value
