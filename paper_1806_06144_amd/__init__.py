"""Python binding of libeigenpro: argument marshalling over the C ABI only.

Every function has the name and meaning of its C counterpart in
``include/eigenpro.h``; device arguments may be torch tensors (checked for
dtype, device and contiguity, then passed by pointer) or raw integer device
addresses. All computation happens in the HIP library: if ``libeigenpro.so``
is missing this module raises at import, it never falls back.
"""

import ctypes
import os
import re

_HERE = os.path.dirname(os.path.abspath(__file__))
# EIGENPRO_LIB selects another build of the same library (e.g. to compare
# kernel variants); by default the in-tree build is loaded.
LIB_PATH = os.environ.get("EIGENPRO_LIB") or os.path.join(_HERE, "libeigenpro.so")
HEADER_PATH = os.path.join(os.path.dirname(_HERE), "include", "eigenpro.h")

EP_OK, EP_EINVAL, EP_ENOMEM, EP_EDEVICE, EP_ENUMERIC, EP_EINDEX = 0, -1, -2, -3, -4, -5
EP_GAUSSIAN, EP_LAPLACIAN = 0, 1
EP_SOLVER_AUTO, EP_SOLVER_DENSE, EP_SOLVER_SUBSPACE = 0, 1, 2
EP_CONTRACT_AUTO, EP_CONTRACT_FUSED, EP_CONTRACT_BLOCKED = 0, 1, 2
CONTRACTIONS = {"auto": EP_CONTRACT_AUTO, "fused": EP_CONTRACT_FUSED,
                "blocked": EP_CONTRACT_BLOCKED}
EP_BF16, EP_FP16, EP_E4M3 = 0, 1, 2
EP_PASS_FLOAT32, EP_PASS_SPLIT, EP_PASS_BLOCKED = 0, 1, 2
SOLVERS = {"auto": EP_SOLVER_AUTO, "dense": EP_SOLVER_DENSE, "subspace": EP_SOLVER_SUBSPACE}
KERNELS = {"gaussian": EP_GAUSSIAN, "laplacian": EP_LAPLACIAN}
_CODES = {EP_EINVAL: "EP_EINVAL", EP_ENOMEM: "EP_ENOMEM", EP_EDEVICE: "EP_EDEVICE",
          EP_ENUMERIC: "EP_ENUMERIC", EP_EINDEX: "EP_EINDEX"}


class EpInfo(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("d", ctypes.c_int64), ("l", ctypes.c_int64),
                ("s", ctypes.c_int64), ("k", ctypes.c_int64),
                ("sigma_1", ctypes.c_double), ("sigma_k1", ctypes.c_double),
                ("lambda_k1", ctypes.c_double), ("beta", ctypes.c_double),
                ("m_star", ctypes.c_double), ("m", ctypes.c_int64),
                ("eta", ctypes.c_double), ("setup_ms", ctypes.c_double),
                ("k_max", ctypes.c_int64), ("accel", ctypes.c_double),
                ("solver", ctypes.c_int64), ("solver_iters", ctypes.c_int64),
                ("solver_matvecs", ctypes.c_int64), ("eig_residual", ctypes.c_double)]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class EpSetupOpts(ctypes.Structure):
    _fields_ = [("solver", ctypes.c_int32), ("max_degree", ctypes.c_int32),
                ("max_iters", ctypes.c_int32), ("no_fallback", ctypes.c_int32),
                ("guard", ctypes.c_int64), ("tol", ctypes.c_double)]


class EpTiming(ctypes.Structure):
    _fields_ = [("kmv_ms", ctypes.c_double), ("kmv_launches", ctypes.c_int64),
                ("step_ms", ctypes.c_double), ("steps", ctypes.c_int64),
                ("kblock_ms", ctypes.c_double), ("kblock_launches", ctypes.c_int64),
                ("gemm_ms", ctypes.c_double), ("gemm_launches", ctypes.c_int64)]


class EpRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class EpAttn(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("causal", ctypes.c_int32), ("batch", ctypes.c_int64),
                ("heads", ctypes.c_int64), ("kv_heads", ctypes.c_int64), ("dim", ctypes.c_int64),
                ("tokens_q", ctypes.c_int64), ("tokens_k", ctypes.c_int64),
                ("window", ctypes.c_int64), ("start_q", ctypes.c_void_p),
                ("start_k", ctypes.c_void_p), ("scale", ctypes.c_float)]


class EpCacheDesc(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int64),
                ("kv_heads", ctypes.c_int64), ("dim", ctypes.c_int64), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p)]


class EpPages(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("table", ctypes.c_void_p), ("cols", ctypes.c_int64),
                ("lengths", ctypes.c_void_p), ("err", ctypes.c_void_p)]


class EigenProError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{_CODES.get(code, code)}: {msg}")
        self.code = code


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                          "or python paper_1806_06144_amd/build.py")
    # torch ships its own HIP runtime under the same soname; loading torch
    # first makes the library bind to that one, so the process holds a
    # single runtime (two copies would not see each other's devices).
    import torch  # noqa: F401
    lib = ctypes.CDLL(LIB_PATH)
    P, I64, I, F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    PA, PC, PP = (ctypes.POINTER(t) for t in (EpAttn, EpCacheDesc, EpPages))
    sig = {
        "ep_setup": (I, [ctypes.POINTER(P), P, I64, I64, I64, I, F, I64, I64, P,
                         ctypes.c_uint64, P, ctypes.POINTER(EpInfo)]),
        "ep_setup_ex": (I, [ctypes.POINTER(P), P, I64, I64, I64, I, F, I64, I64, P,
                            ctypes.c_uint64, P, ctypes.POINTER(EpSetupOpts),
                            ctypes.POINTER(EpInfo)]),
        "ep_restore": (I, [ctypes.POINTER(P), P, I64, I64, I64, I, F, I64, I64, P, P, P, P,
                           ctypes.POINTER(EpInfo)]),
        "ep_step": (I, [P, P, I64, P, P]),
        "ep_predict": (I, [P, P, I64, P]),
        "ep_predict_noalloc": (I, [P, P, I64, P]),
        "ep_get_alpha": (I, [P, P]),
        "ep_set_alpha": (I, [P, P]),
        "ep_get_preconditioner": (I, [P, P, P, P, P]),
        "ep_get_info": (I, [P, ctypes.POINTER(EpInfo)]),
        "ep_set_checks": (I, [P, I]),
        "ep_set_rank": (I, [P, I64]),
        "ep_set_contraction": (I, [P, I, I64]),
        "ep_step_pass": (I, [P, I64, ctypes.POINTER(I)]),
        "ep_adapt": (I, [P, I64, ctypes.POINTER(EpInfo)]),
        "ep_batch_sweep": (I, [P, P, I, I, P]),
        "ep_resource_batch": (I, [P, ctypes.c_double, ctypes.POINTER(I64), ctypes.POINTER(I64),
                                  ctypes.POINTER(I64)]),
        "ep_batch_knee": (I, [P, P, I, ctypes.c_double, ctypes.POINTER(I64),
                              ctypes.POINTER(ctypes.c_double)]),
        "ep_timing_enable": (I, [P, I]),
        "ep_timing_read": (I, [P, ctypes.POINTER(EpTiming)]),
        "ep_attention_bytes": (I64, [PA]),
        "ep_attention": (I, [PA, EpRows, EpRows, EpRows, EpRows, P, P, I64, P]),
        "ep_attention_backward_bytes": (I64, [PA]),
        "ep_attention_backward": (I, [PA, EpRows, EpRows, EpRows, EpRows, EpRows, P, EpRows,
                                      EpRows, EpRows, P, I64, P]),
        "ep_cache_write": (I, [PC, PP, I, EpRows, EpRows, I64, P, P]),
        "ep_cache_read": (I, [PC, PP, I, EpRows, EpRows, I64, P, P]),
        "ep_cache_attention_bytes": (I64, [PA, PC, PP]),
        "ep_cache_attention": (I, [PA, PC, PP, EpRows, EpRows, P, P, I64, P]),
        "ep_sync": (I, [P]),
        "ep_device_probe": (I, [P, P]),
        "ep_destroy": (None, [P]),
        "ep_last_error": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = _load()


def declared_symbols():
    """Names of the functions declared in include/eigenpro.h."""
    with open(HEADER_PATH) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(ep_[a-z_0-9]+)\s*\(", text)))


def _check(rc):
    if rc != EP_OK:
        raise EigenProError(rc, _lib.ep_last_error().decode())
    return rc


def _ptr(x, dtype=None, allow_none=False):
    """Device address of a tensor (validated) or an integer address."""
    if x is None:
        if allow_none:
            return None
        raise ValueError("a device buffer is required")
    if isinstance(x, int):
        return x
    if not x.is_cuda:
        raise ValueError("expected a device tensor")
    if dtype is not None and x.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {x.dtype}")
    if not x.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return x.data_ptr()


def _torch():
    import torch
    return torch


_int32, _float32 = _torch().int32, _torch().float32
# (a torch without devices has neither; what needs no tensors works there too)
_current_device = getattr(_torch()._C, "_cuda_getDevice", None)
_raw_stream = getattr(_torch()._C, "_cuda_getCurrentRawStream", None)
_ATTN_TYPES = {_torch().bfloat16: EP_BF16, _torch().float16: EP_FP16}
_CACHE_TYPES = {**_ATTN_TYPES, _torch().float8_e4m3fn: EP_E4M3, _torch().uint8: EP_E4M3}


def _stream_handle(stream):
    if stream is None:
        return _torch().cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def ep_last_error():
    return _lib.ep_last_error().decode()


def ep_setup(X, n, d, l, kernel, bandwidth, s, k, sub_idx=None, seed=0, stream=None):
    """Returns (ctx, EpInfo). X: device float32 n x d (borrowed: keep it
    alive until ep_destroy). sub_idx: host int64 sequence of s indices or
    None."""
    return ep_setup_ex(X, n, d, l, kernel, bandwidth, s, k, sub_idx, seed, stream, None)


def ep_setup_ex(X, n, d, l, kernel, bandwidth, s, k, sub_idx=None, seed=0, stream=None,
                opts=None):
    """ep_setup with setup options: ``opts`` is an EpSetupOpts, a dict of its
    fields (``solver`` may be "auto", "dense" or "subspace"), or None."""
    torch = _torch()
    if isinstance(kernel, str):
        kernel = KERNELS[kernel]
    xp = _ptr(X, torch.float32)
    sub_ptr = None
    keep = None
    if sub_idx is not None:
        import numpy as np
        keep = np.ascontiguousarray(np.asarray(sub_idx, dtype=np.int64))
        if keep.shape != (s,):
            raise ValueError("sub_idx must hold s indices")
        sub_ptr = keep.ctypes.data
    if isinstance(opts, dict):
        o = dict(opts)
        if isinstance(o.get("solver"), str):
            o["solver"] = SOLVERS[o["solver"]]
        opts = EpSetupOpts(**o)
    ctx = ctypes.c_void_p()
    info = EpInfo()
    if opts is None:
        _check(_lib.ep_setup(ctypes.byref(ctx), xp, n, d, l, kernel, bandwidth, s, k, sub_ptr,
                             seed, _stream_handle(stream), ctypes.byref(info)))
    else:
        _check(_lib.ep_setup_ex(ctypes.byref(ctx), xp, n, d, l, kernel, bandwidth, s, k,
                                sub_ptr, seed, _stream_handle(stream), ctypes.byref(opts),
                                ctypes.byref(info)))
    return ctx, info


def ep_restore(X, n, d, l, kernel, bandwidth, s, k, sub_idx, sigma, V, stream=None):
    """Rebuild a context from a saved setup (sub_idx, sigma[k+1], V[s, k] as
    returned by ep_get_preconditioner). Returns (ctx, EpInfo)."""
    import numpy as np
    torch = _torch()
    if isinstance(kernel, str):
        kernel = KERNELS[kernel]
    r = np.ascontiguousarray(np.asarray(sub_idx, dtype=np.int64))
    sg = np.ascontiguousarray(np.asarray(sigma, dtype=np.float64))
    if r.shape != (s,) or sg.shape != (k + 1,):
        raise ValueError("sub_idx must hold s entries and sigma k+1")
    Vh = np.ascontiguousarray(np.asarray(V, dtype=np.float32).reshape(s, k)) if k else None
    ctx = ctypes.c_void_p()
    info = EpInfo()
    _check(_lib.ep_restore(ctypes.byref(ctx), _ptr(X, torch.float32), n, d, l, kernel,
                           bandwidth, s, k, r.ctypes.data, sg.ctypes.data,
                           Vh.ctypes.data if Vh is not None else None,
                           _stream_handle(stream), ctypes.byref(info)))
    return ctx, info


def ep_step(ctx, t, m, y_b, f_out=None):
    torch = _torch()
    return _check(_lib.ep_step(ctx, _ptr(t, torch.int64), m, _ptr(y_b, torch.float32),
                               _ptr(f_out, torch.float32, allow_none=True)))


def ep_step_pass(ctx, m):
    """EP_PASS_FLOAT32, EP_PASS_SPLIT or EP_PASS_BLOCKED: how ep_step forms F
    for a batch of m rows."""
    p = ctypes.c_int()
    _check(_lib.ep_step_pass(ctx, m, ctypes.byref(p)))
    return p.value


def ep_predict(ctx, Z, n_z, out):
    torch = _torch()
    return _check(_lib.ep_predict(ctx, _ptr(Z, torch.float32), n_z, _ptr(out, torch.float32)))


def ep_predict_noalloc(ctx, Z, n_z, out):
    torch = _torch()
    return _check(_lib.ep_predict_noalloc(ctx, _ptr(Z, torch.float32), n_z,
                                          _ptr(out, torch.float32)))


def ep_get_alpha(ctx, out):
    return _check(_lib.ep_get_alpha(ctx, _ptr(out, _torch().float32)))


def ep_set_alpha(ctx, alpha):
    return _check(_lib.ep_set_alpha(ctx, _ptr(alpha, _torch().float32)))


def ep_get_preconditioner(ctx, info):
    """Returns numpy (sigma[k+1], D[k], V[s, k] float32, r[s])."""
    import numpy as np
    k, s = info.k, info.s
    sigma = np.zeros(k + 1, dtype=np.float64)
    D = np.zeros(max(k, 1), dtype=np.float64)
    V = np.zeros((s, max(k, 1)), dtype=np.float32)
    r = np.zeros(s, dtype=np.int64)
    _check(_lib.ep_get_preconditioner(ctx, sigma.ctypes.data, D.ctypes.data, V.ctypes.data,
                                      r.ctypes.data))
    return sigma, D[:k], V[:, :k], r


def ep_get_info(ctx):
    info = EpInfo()
    _check(_lib.ep_get_info(ctx, ctypes.byref(info)))
    return info


def ep_set_rank(ctx, k):
    return _check(_lib.ep_set_rank(ctx, k))


def ep_set_contraction(ctx, mode, block_bytes=0):
    """mode: EP_CONTRACT_* or "auto" / "fused" / "blocked"; block_bytes: cap
    of the blocked form's kernel-block buffer (0: 2 GiB)."""
    if isinstance(mode, str):
        mode = CONTRACTIONS[mode]
    return _check(_lib.ep_set_contraction(ctx, mode, block_bytes))


def ep_adapt(ctx, m_G):
    info = EpInfo()
    _check(_lib.ep_adapt(ctx, m_G, ctypes.byref(info)))
    return info


def ep_batch_sweep(ctx, ms, reps=3):
    """ms per fused step-2 pass for each batch size in ms."""
    import numpy as np
    arr = np.ascontiguousarray(np.asarray(ms, dtype=np.int64))
    out = np.zeros(arr.shape[0], dtype=np.float64)
    _check(_lib.ep_batch_sweep(ctx, arr.ctypes.data, arr.shape[0], reps, out.ctypes.data))
    return out


def ep_resource_batch(ctx, tol=0.1):
    """(m_C, m_S, m_G) of Section 3 Step 1."""
    mc, ms, mg = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    _check(_lib.ep_resource_batch(ctx, tol, ctypes.byref(mc), ctypes.byref(ms), ctypes.byref(mg)))
    return mc.value, ms.value, mg.value


def ep_batch_knee(ms, ms_per_pass, tol=0.1):
    """(m_C, knee) of a time-per-iteration curve (host only)."""
    import numpy as np
    m = np.ascontiguousarray(np.asarray(ms, dtype=np.int64))
    t = np.ascontiguousarray(np.asarray(ms_per_pass, dtype=np.float64))
    if m.shape != t.shape:
        raise ValueError("ms and ms_per_pass differ in length")
    mc, kn = ctypes.c_int64(), ctypes.c_double()
    _check(_lib.ep_batch_knee(m.ctypes.data, t.ctypes.data, m.shape[0], tol, ctypes.byref(mc),
                              ctypes.byref(kn)))
    return mc.value, kn.value


def ep_set_checks(ctx, on):
    return _check(_lib.ep_set_checks(ctx, 1 if on else 0))


def ep_timing_enable(ctx, on):
    return _check(_lib.ep_timing_enable(ctx, 1 if on else 0))


def ep_timing_read(ctx):
    t = EpTiming()
    _check(_lib.ep_timing_read(ctx, ctypes.byref(t)))
    return t


def ep_device_probe():
    """(sustained fp32 MFMA TFLOP/s, shader clock MHz) of the current device."""
    tf = ctypes.c_double()
    mhz = ctypes.c_double()
    _check(_lib.ep_device_probe(ctypes.byref(tf), ctypes.byref(mhz)))
    return tf.value, mhz.value


# ---- attention over packed sequences and over a paged cache ----
#
# These calls may take less time on the device than Python takes to marshal
# them, so every check is a single comparison.


def _mismatch(x, name, dtype, shape, device):
    if x.device != device:
        raise ValueError(f"{name}: expected a tensor on {device}")
    if x.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {x.dtype}")
    if x.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(x.shape)}")
    raise ValueError(f"{name}: expected a contiguous tensor")


def _device(x):
    if not x.is_cuda:
        raise ValueError("expected a device tensor")
    return x.device


def _rows(x, name, shape, dtype, device):
    """EpRows of a [tokens, heads, dim] tensor; its last axis is contiguous,
    the others may be strided (slices of a wider array)."""
    if x.dtype is not dtype or x.shape != shape or x.device != device:
        _mismatch(x, name, dtype, shape, device)
    row, head, one = x.stride()
    if one != 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    return EpRows(x.data_ptr(), row, head)


def _dense(x, name, dtype, shape, device):
    """Address of a contiguous tensor of that type, shape and device."""
    if (x.dtype is not dtype or x.shape != shape or x.device != device
            or not x.is_contiguous()):
        _mismatch(x, name, dtype, shape, device)
    return x.data_ptr()


def _attn_type(x):
    kind = _ATTN_TYPES.get(x.dtype)
    if kind is None:
        raise TypeError(f"expected bfloat16 or float16, got {x.dtype}")
    return kind


def _attn(q, kv_heads, tokens_k, start_q, start_k, scale, causal, window, device):
    kind = _attn_type(q)
    if len(q.shape) != 3:
        raise ValueError("q: expected [tokens, heads, dim]")
    tokens_q, heads, dim = q.shape
    starts = start_q.shape
    return EpAttn(kind, 1 if causal else 0, starts[0] - 1 if len(starts) == 1 else -1, heads,
                  kv_heads, dim, tokens_q, tokens_k, window,
                  _dense(start_q, "start_q", _int32, starts, device),
                  None if start_k is None else _dense(start_k, "start_k", _int32, starts, device),
                  max(dim, 1) ** -0.5 if scale is None else scale)


def _on_stream(device, stream, call):
    """call(stream handle, device) with the tensors' device current; memory
    that call allocates belongs to the stream that the work goes to."""
    torch = _torch()
    if stream is None and device.index == _current_device():
        return call(_raw_stream(device.index), device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    elif stream is not None and stream.device != device:
        raise ValueError(f"stream: expected one of {device}, got one of {stream.device}")
    with torch.cuda.device(device), torch.cuda.stream(stream):
        return call(torch.cuda.current_stream().cuda_stream, device)


def _work(device, n):
    """(address, bytes) of n bytes, and what holds them; n is a ..._bytes answer."""
    if n == 0:
        return None, 0, None
    if n < 0:
        _check(int(n))
    x = _torch().empty(n, dtype=_torch().uint8, device=device)
    return x.data_ptr(), n, x


def _lse(lse, q, device):
    return None if lse is None else _dense(lse, "lse", _float32, q.shape[:2], device)


def ep_attention(q, k, v, out, lse, start_q, start_k, scale=None, causal=True, window=0,
                 stream=None):
    """out = softmax(scale q k^T) v over packed sequences, lse its log-sums
    (float32 [tokens, heads], or None). q, out: [tokens, heads, dim] bfloat16
    or float16; k, v: [tokens_k, kv_heads, dim]; start_q, start_k: int32,
    batch + 1 values. scale: dim ** -0.5 by default; window: 0 for none."""
    dev, dt, qs, ks = _device(q), q.dtype, q.shape, k.shape
    if len(ks) != 3:
        raise ValueError("k: expected [tokens, kv_heads, dim]")
    a = _attn(q, ks[1], ks[0], start_q, start_k, scale, causal, window, dev)
    kv = (a.tokens_k, a.kv_heads, a.dim)
    args = (ctypes.byref(a), _rows(q, "q", qs, dt, dev), _rows(k, "k", kv, dt, dev),
            _rows(v, "v", kv, dt, dev), _rows(out, "out", qs, dt, dev), _lse(lse, q, dev))

    def call(s, device):
        work, n, _hold = _work(device, _lib.ep_attention_bytes(args[0]))
        return _check(_lib.ep_attention(*args, work, n, s))
    return _on_stream(dev, stream, call)


def ep_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, start_q, start_k, scale=None,
                          causal=True, window=0, stream=None):
    """Gradients dq, dk, dv of ep_attention for the gradient dout of out; out
    and lse are what it returned. Written, not added to."""
    dev, dt, qs, ks = _device(q), q.dtype, q.shape, k.shape
    if len(ks) != 3:
        raise ValueError("k: expected [tokens, kv_heads, dim]")
    a = _attn(q, ks[1], ks[0], start_q, start_k, scale, causal, window, dev)
    kv = (a.tokens_k, a.kv_heads, a.dim)
    args = (ctypes.byref(a), _rows(dout, "dout", qs, dt, dev), _rows(q, "q", qs, dt, dev),
            _rows(k, "k", kv, dt, dev), _rows(v, "v", kv, dt, dev),
            _rows(out, "out", qs, dt, dev), _dense(lse, "lse", _float32, qs[:2], dev),
            _rows(dq, "dq", qs, dt, dev), _rows(dk, "dk", kv, dt, dev),
            _rows(dv, "dv", kv, dt, dev))

    def call(s, device):
        work, n, _hold = _work(device, _lib.ep_attention_backward_bytes(args[0]))
        return _check(_lib.ep_attention_backward(*args, work, n, s))
    return _on_stream(dev, stream, call)


class EpCache:
    """A paged cache: k_pages and v_pages are [pages, page_size, kv_heads, dim]
    bfloat16, float16, or float8_e4m3fn (uint8 is taken as that) with float32
    k_scale and v_scale [pages, page_size, kv_heads]: a row is its values times
    its scale, a power of two where ep_cache_write wrote it. Holds the tensors."""

    def __init__(self, k_pages, v_pages, k_scale=None, v_scale=None):
        shape, dt, dev = k_pages.shape, k_pages.dtype, _device(k_pages)
        if len(shape) != 4:
            raise ValueError("k_pages: expected [pages, page_size, kv_heads, dim]")
        ks = vs = None
        kind = _CACHE_TYPES.get(dt)
        if kind is None:
            raise TypeError(f"expected bfloat16, float16 or float8_e4m3fn, got {dt}")
        if kind == EP_E4M3:
            if k_scale is None or v_scale is None:
                raise ValueError("an 8-bit cache needs k_scale and v_scale")
            ks = _dense(k_scale, "k_scale", _float32, shape[:3], dev)
            vs = _dense(v_scale, "v_scale", _float32, shape[:3], dev)
        self.tensors = (k_pages, v_pages, k_scale, v_scale)
        self.device = dev
        self.kv_heads, self.dim = shape[2], shape[3]
        self.desc = EpCacheDesc(kind, *shape, _dense(k_pages, "k_pages", dt, shape, dev),
                                _dense(v_pages, "v_pages", dt, shape, dev), ks, vs)


def _pages(cache, table, lengths, err):
    dev, shape = cache.device, table.shape
    if len(shape) != 2:
        raise ValueError("table: expected [batch, cols]")
    return EpPages(shape[0], _dense(table, "table", _int32, shape, dev), shape[1],
                   _dense(lengths, "lengths", _int32, shape[:1], dev),
                   None if err is None else _dense(err, "err", _int32, (1,), dev))


def _cache_move(fn, cache, k, v, table, lengths, start, err, stream):
    dev, dt = cache.device, k.dtype
    p = _pages(cache, table, lengths, err)
    shape = (k.shape[0], cache.kv_heads, cache.dim)
    args = (ctypes.byref(cache.desc), ctypes.byref(p), _attn_type(k),
            _rows(k, "k", shape, dt, dev), _rows(v, "v", shape, dt, dev), shape[0],
            _dense(start, "start", _int32, (p.batch + 1,), dev))
    return _on_stream(dev, stream, lambda s, _: _check(fn(*args, s)))


def ep_cache_write(cache, k, v, table, lengths, start, err=None, stream=None):
    """New tokens k, v [tokens, kv_heads, dim] into their pages; lengths
    [batch] count them already. err: int32 [1], set to 1 on a bad page."""
    return _cache_move(_lib.ep_cache_write, cache, k, v, table, lengths, start, err, stream)


def ep_cache_read(cache, k, v, table, lengths, start, err=None, stream=None):
    """Cached tokens back into packed rows k, v: row start[b] + j gets token j
    of sequence b."""
    return _cache_move(_lib.ep_cache_read, cache, k, v, table, lengths, start, err, stream)


def ep_cache_attention(q, cache, out, lse, table, lengths, start_q, scale=None, causal=True,
                       window=0, err=None, stream=None):
    """ep_attention of new tokens' queries over the cached keys and values
    (theirs included: write them first)."""
    dev, dt, qs = cache.device, q.dtype, q.shape
    a = _attn(q, cache.kv_heads, 0, start_q, None, scale, causal, window, dev)
    refs = (ctypes.byref(a), ctypes.byref(cache.desc),
            ctypes.byref(_pages(cache, table, lengths, err)))
    args = (_rows(q, "q", qs, dt, dev), _rows(out, "out", qs, dt, dev), _lse(lse, q, dev))

    def call(s, device):
        work, n, _hold = _work(device, _lib.ep_cache_attention_bytes(*refs))
        return _check(_lib.ep_cache_attention(*refs, *args, work, n, s))
    return _on_stream(dev, stream, call)


def ep_sync(ctx):
    return _check(_lib.ep_sync(ctx))


def ep_destroy(ctx):
    _lib.ep_destroy(ctx)


def raw_call(name, *args):
    """Call a C entry point with already-marshalled arguments and return its
    integer status (used to exercise error paths)."""
    return getattr(_lib, name)(*args)
