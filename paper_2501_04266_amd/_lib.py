"""ctypes binding of libzq.so (include/zq.h).

Argument marshalling only: every step runs in the HIP kernels.  Tensors are
torch tensors on the GPU (torch is used for device memory and streams); the
work is enqueued on torch's current stream unless `stream` is given.  There is
no CPU fallback: if the library is not built this module raises on use.
"""
import ctypes
import os

import torch  # noqa: F401  -- loads torch's HIP runtime first, so libzq binds to the same one

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("ZQ_LIBRARY") or os.path.join(_PKG, "libzq.so")

ZQ_F32, ZQ_F16, ZQ_BF16 = 0, 1, 2
ZQ_I32, ZQ_I64, ZQ_INT4, ZQ_INT8, ZQ_F8 = 3, 4, 5, 6, 7
STATUS = {0: "ZQ_OK", -1: "ZQ_E_NULL", -2: "ZQ_E_BLOCK", -3: "ZQ_E_DTYPE", -4: "ZQ_E_ALIGN",
          -5: "ZQ_E_SIZE", -6: "ZQ_E_P", -7: "ZQ_E_HIP", -8: "ZQ_E_ALIAS"}
EXPORTS = ["qwz_quantize", "qwz_dequantize", "qgz_quantize", "qgz_reduce_level", "qgz_dequantize",
           "qgz_reduce_dequantize", "qgz_reduce_level_gather", "qgz_reduce_level_gather_noalloc",
           "qwz_dequant_gemm", "zq_embedding", "qwz_embedding", "zq_embedding_grad", "zq_embedding_grad_bytes",
           "zq_grad_plan_make", "zq_grad_plan_table", "zq_grad_norm", "zq_grad_clip", "zq_int4_dequant_gemm",
           "zq_int4_dequant_gemm_bytes", "zq_adamw_plan_make", "zq_adamw_plan_table", "zq_adamw_step",
           "zq_rms_norm", "qwz_rms_norm", "zq_rms_norm_grad", "zq_rms_norm_grad_bytes",
           "zq_token_logp", "zq_policy_loss", "zq_policy_loss_bytes",
           "zq_num_scales", "zq_int4_bytes", "zq_status_string"]

_TORCH_DT = {torch.float32: ZQ_F32, torch.float16: ZQ_F16, torch.bfloat16: ZQ_BF16}
_DT_TORCH = {v: k for k, v in _TORCH_DT.items()}
_ID_DT = {torch.int32: ZQ_I32, torch.int64: ZQ_I64}
_lib = None


class _Grad(ctypes.Structure):  # zq_grad
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("block", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class _GradPlan(ctypes.Structure):  # zq_grad_plan
    _fields_ = [("bytes", ctypes.c_int64), ("norm_chunks", ctypes.c_int64), ("clip_chunks", ctypes.c_int64),
                ("count", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _AdamW(ctypes.Structure):  # zq_adamw
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("grad_scales", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("m_scales", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("out", ctypes.c_void_p), ("out_scales", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("weight_decay", ctypes.c_double), ("lr_scale", ctypes.c_double),
                ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("state_dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("grad_block", ctypes.c_int32), ("state_block", ctypes.c_int32),
                ("out_block", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _AdamWPlan(ctypes.Structure):  # zq_adamw_plan
    _fields_ = [("bytes", ctypes.c_int64), ("pieces", ctypes.c_int64), ("block_pieces", ctypes.c_int64),
                ("count", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _AdamWArgs(ctypes.Structure):  # zq_adamw_args
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64), ("max_norm", ctypes.c_float),
                ("scale", ctypes.c_float)]


class _Policy(ctypes.Structure):  # zq_policy
    _fields_ = [("old_logp", ctypes.c_void_p), ("advantages", ctypes.c_void_p), ("weights", ctypes.c_void_p),
                ("ref_logp", ctypes.c_void_p), ("clip_low", ctypes.c_float), ("clip_high", ctypes.c_float),
                ("kl", ctypes.c_float), ("scale", ctypes.c_float), ("grad_scale", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


class ZQError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: {STATUS.get(status, status)} ({lib().zq_status_string(status).decode()})")


def lib():
    """The loaded libzq.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2501_04266_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, ci, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int, ctypes.c_float
    f64 = ctypes.c_double
    sig = {
        "qwz_quantize": [vp, ci, i64, i32, vp, vp, vp],
        "qwz_dequantize": [vp, vp, i64, i32, vp, ci, vp],
        "qgz_quantize": [vp, ci, i64, i32, vp, vp, vp],
        "qgz_dequantize": [vp, vp, i64, i32, vp, ci, vp],
        "qgz_reduce_level": [vp, vp, i32, i64, i32, vp, vp, vp],
        "qgz_reduce_dequantize": [vp, vp, i32, i64, i32, vp, ci, vp, vp, vp],
        "qwz_dequant_gemm": [vp, ci, vp, vp, i64, i64, i64, i32, vp, vp],
        "qgz_reduce_level_gather": [vp, vp, i32, i64, i32, vp, vp, vp],
        "qgz_reduce_level_gather_noalloc": [vp, vp, i32, i64, i32, vp, vp, vp],
        "zq_embedding": [vp, ci, i64, vp, ci, i64, i64, f32, vp, ci, vp],
        "qwz_embedding": [vp, ci, i64, vp, vp, i64, i64, i32, f32, vp, ci, vp],
        "zq_embedding_grad": [vp, ci, i64, vp, ci, i64, i64, f32, ci, vp, ci, vp, i64, vp],
        "zq_grad_plan_make": [vp, i32, vp],
        "zq_grad_plan_table": [vp, vp, vp],
        "zq_grad_norm": [vp, vp, f32, vp, vp],
        "zq_grad_clip": [vp, vp, vp, f32, f32, vp],
        "zq_int4_dequant_gemm": [vp, ci, vp, vp, i64, i64, i64, i32, vp, vp, i64, vp],
        "zq_adamw_plan_make": [vp, i32, vp],
        "zq_adamw_plan_table": [vp, vp, vp],
        "zq_adamw_step": [vp, vp, vp, vp, vp, vp, vp],
        "zq_rms_norm": [vp, vp, ci, vp, ci, i64, i64, f64, vp, vp, ci, vp, vp],
        "qwz_rms_norm": [vp, vp, ci, vp, ci, i64, i64, f64, vp, vp, vp, i32, vp, vp],
        "zq_rms_norm_grad": [vp, ci, vp, ci, vp, ci, vp, vp, i64, i64, vp, ci, vp, ci, vp, i64, vp],
        "zq_token_logp": [vp, ci, i64, i64, i64, vp, ci, f32, vp, vp],
        "zq_policy_loss": [vp, ci, i64, i64, i64, vp, ci, vp, vp, vp, vp, ci, i64, vp, i64, vp],
    }
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes, fn.restype = args, ci
    L.zq_num_scales.argtypes, L.zq_num_scales.restype = [i64, i32], i64
    L.zq_int4_bytes.argtypes, L.zq_int4_bytes.restype = [i64], i64
    L.zq_embedding_grad_bytes.argtypes, L.zq_embedding_grad_bytes.restype = [i64, i64, i64], i64
    L.zq_int4_dequant_gemm_bytes.argtypes, L.zq_int4_dequant_gemm_bytes.restype = [i64, i64, i64], i64
    L.zq_rms_norm_grad_bytes.argtypes, L.zq_rms_norm_grad_bytes.restype = [i64, i64], i64
    L.zq_policy_loss_bytes.argtypes, L.zq_policy_loss_bytes.restype = [i64], i64
    L.zq_status_string.argtypes, L.zq_status_string.restype = [ci], ctypes.c_char_p
    _lib = L
    return L


def num_scales(n, block):
    return (n + block - 1) // block


def int4_bytes(n):
    return (n + 1) // 2


def _stream(stream):
    if stream is None:
        # the handle alone: torch.cuda.current_stream() builds a Stream object
        # around it, 2.8 us of a small call's 10.6
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _stream_object(stream, device):
    if hasattr(stream, "cuda_stream"):
        return stream
    # a tensor on the CPU is refused, as such, once the call looks at its address
    return torch.cuda.ExternalStream(int(stream), device=device if device.type == "cuda" else None)


def _output(stream, device, dtype, *shape):
    """A tensor for a call on `stream` to write and return, allocated on the current
    stream, where its user expects it.  Another `stream` waits for the work that is
    pending on the current one (the memory's last user may be part of it), and, given as
    an object, the allocator keeps the tensor until that stream has passed the call.  (A
    raw handle may be gone by the time the tensor is freed: its owner keeps the tensor
    until the call has run.)"""
    # plain sizes: 0.6 us less than a tuple
    t = torch.empty(*shape or (1,), dtype=dtype, device=device)
    if stream is not None and t.is_cuda:
        st, current = _stream_object(stream, device), torch.cuda.current_stream(device)
        if st.cuda_stream != current.cuda_stream:
            st.wait_stream(current)
            if st is stream:
                t.record_stream(st)
    return t if shape else t.view(())


def _dev(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _need(t, name, count, dtypes):
    """Host-side size and dtype check of a caller's buffer: the C ABI takes raw
    pointers and cannot tell an undersized buffer from a large one."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}; expected one of {[str(d) for d in dtypes]}")
    if t.numel() < count:
        raise ValueError(f"{name} holds {t.numel()} elements; {count} needed")


def _ptr(t, name, count, dtypes):
    """The address of a buffer that passes _need and _dev, checked in one go (0.3 us a
    buffer, 0.5 by the two); else what _need raises, or None: left to _dev, once the
    other buffers' sizes are checked."""
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.numel() >= count and t.is_contiguous()):
        return t.data_ptr()
    _need(t, name, count, dtypes)


def _nsc(n, block):
    """Scales needed for n elements; 0 for a block the library will reject
    itself (ZQ_E_BLOCK), so that error is reported as the library's."""
    if not isinstance(block, int) or block < 32 or block > 1024 or block & (block - 1):
        return 0
    return num_scales(n, block)


def _alloc_nsc(n, block):
    """Scales to allocate for n elements (one for a block the library rejects)."""
    return _nsc(n, block) if _nsc(n, block) or n == 0 else 1


_ELEM = (torch.float32, torch.float16, torch.bfloat16)
_I8 = (torch.int8,)
_U8 = (torch.uint8,)
_F32 = (torch.float32,)
_IDS = tuple(_ID_DT)
_HALF = (torch.bfloat16, torch.float16)
_I64 = (torch.int64,)
_F8 = {"exp_avg": torch.float8_e4m3fn, "exp_avg_sq": torch.float8_e5m2}


def _check(status, what):
    if status != 0:
        raise ZQError(status, what)


def qwz_quantize(x, block=256, codes=None, scales=None, stream=None):
    """INT8 block quantisation of x (f32/f16/bf16) -> (codes int8[n], scales f32[ceil(n/B)])."""
    n = x.numel()
    _need(x, "x", n, _ELEM)
    if codes is None:
        codes = _output(stream, x.device, torch.int8, n)
    if scales is None:
        scales = _output(stream, x.device, torch.float32, _alloc_nsc(n, block))
    _need(codes, "codes", n, _I8)
    _need(scales, "scales", _nsc(n, block), _F32)
    _check(lib().qwz_quantize(_dev(x, "x"), _TORCH_DT[x.dtype], n, block, _dev(codes, "codes"),
                              _dev(scales, "scales"), _stream(stream)), "qwz_quantize")
    return codes, scales


def qwz_dequantize(codes, scales, block=256, out_dtype=torch.bfloat16, y=None, n=None, stream=None):
    n = codes.numel() if n is None else n
    if y is None:
        y = _output(stream, codes.device, out_dtype, n)
    _need(codes, "codes", n, _I8)
    _need(scales, "scales", _nsc(n, block), _F32)
    _need(y, "y", n, _ELEM)
    _check(lib().qwz_dequantize(_dev(codes, "codes"), _dev(scales, "scales"), n, block, _dev(y, "y"),
                                _TORCH_DT[y.dtype], _stream(stream)), "qwz_dequantize")
    return y


def qgz_quantize(g, block=128, packed=None, scales=None, stream=None):
    """INT4 block quantisation -> (packed uint8[ceil(n/2)], scales f32[ceil(n/B)])."""
    n = g.numel()
    _need(g, "g", n, _ELEM)
    if packed is None:
        packed = _output(stream, g.device, torch.uint8, int4_bytes(n))
    if scales is None:
        scales = _output(stream, g.device, torch.float32, _alloc_nsc(n, block))
    _need(packed, "packed", int4_bytes(n), _U8)
    _need(scales, "scales", _nsc(n, block), _F32)
    _check(lib().qgz_quantize(_dev(g, "g"), _TORCH_DT[g.dtype], n, block, _dev(packed, "packed"),
                              _dev(scales, "scales"), _stream(stream)), "qgz_quantize")
    return packed, scales


def qgz_dequantize(packed, scales, n, block=128, out_dtype=torch.float32, y=None, stream=None):
    if y is None:
        y = _output(stream, packed.device, out_dtype, n)
    _need(packed, "packed", int4_bytes(n), _U8)
    _need(scales, "scales", _nsc(n, block), _F32)
    _need(y, "y", n, _ELEM)
    _check(lib().qgz_dequantize(_dev(packed, "packed"), _dev(scales, "scales"), n, block, _dev(y, "y"),
                                _TORCH_DT[y.dtype], _stream(stream)), "qgz_dequantize")
    return y


def qgz_reduce_level(packed_in, scales_in, P, m, block=128, packed_out=None, scales_out=None, stream=None):
    """Dequant -> sum over P slices (ascending) -> INT4 requant.  packed_in holds
    P slices of ceil(m/2) bytes back to back, scales_in P x ceil(m/B)."""
    dev = packed_in.device
    if packed_out is None:
        packed_out = _output(stream, dev, torch.uint8, int4_bytes(m))
    if scales_out is None:
        scales_out = _output(stream, dev, torch.float32, _alloc_nsc(m, block))
    _need(packed_in, "packed_in", P * int4_bytes(m), _U8)
    _need(scales_in, "scales_in", P * _nsc(m, block), _F32)
    _need(packed_out, "packed_out", int4_bytes(m), _U8)
    _need(scales_out, "scales_out", _nsc(m, block), _F32)
    _check(lib().qgz_reduce_level(_dev(packed_in, "packed_in"), _dev(scales_in, "scales_in"), P, m, block,
                                  _dev(packed_out, "packed_out"), _dev(scales_out, "scales_out"),
                                  _stream(stream)), "qgz_reduce_level")
    return packed_out, scales_out


def qgz_reduce_dequantize(packed_in, scales_in, P, m, block=128, out_dtype=torch.float32, y=None,
                          packed_out=None, scales_out=None, stream=None):
    """Last level fused with the final dequantisation: returns y (m elements of
    out_dtype) bit-identical to qgz_dequantize(qgz_reduce_level(...)).  Pass
    packed_out and scales_out to also receive the INT4 result."""
    if y is None:
        y = _output(stream, packed_in.device, out_dtype, m)
    if (packed_out is None) != (scales_out is None):
        raise ValueError("give both packed_out and scales_out, or neither")
    _need(packed_in, "packed_in", P * int4_bytes(m), _U8)
    _need(scales_in, "scales_in", P * _nsc(m, block), _F32)
    _need(y, "y", m, _ELEM)
    if packed_out is not None:
        _need(packed_out, "packed_out", int4_bytes(m), _U8)
        _need(scales_out, "scales_out", _nsc(m, block), _F32)
    _check(lib().qgz_reduce_dequantize(_dev(packed_in, "packed_in"), _dev(scales_in, "scales_in"), P, m, block,
                                       _dev(y, "y"), _TORCH_DT[y.dtype],
                                       None if packed_out is None else _dev(packed_out, "packed_out"),
                                       None if scales_out is None else _dev(scales_out, "scales_out"),
                                       _stream(stream)), "qgz_reduce_dequantize")
    return y


def gather_tables(packed_slices, scale_slices):
    """Device tables (int64 tensors) of the slices' addresses, for
    qgz_reduce_level_gather; build them once to reuse them, e.g. under graph
    capture, where the per-call host-to-device copy is not allowed."""
    dev = packed_slices[0].device
    tab = torch.tensor([_dev(t, "packed_slices[p]") for t in packed_slices], dtype=torch.int64).to(dev)
    stab = torch.tensor([_dev(t, "scale_slices[p]") for t in scale_slices], dtype=torch.int64).to(dev)
    return tab, stab


def qgz_reduce_level_gather(packed_slices, scale_slices, m, block=128, packed_out=None, scales_out=None,
                            stream=None, tables=None):
    """qgz_reduce_level over P slices held in separate tensors (lists of P
    uint8 tensors of ceil(m/2) bytes and P float32 tensors of ceil(m/B)
    scales), read in place through device tables of their addresses (built
    here, or passed as `tables` from gather_tables).  Bit-identical to
    qgz_reduce_level on the slices laid out back to back."""
    P = len(packed_slices)
    if P != len(scale_slices) or P == 0:
        raise ValueError("give P >= 1 byte slices and as many scale slices")
    for p, (a, b) in enumerate(zip(packed_slices, scale_slices)):
        _need(a, f"packed_slices[{p}]", int4_bytes(m), _U8)
        _need(b, f"scale_slices[{p}]", _nsc(m, block), _F32)
        # the library reads the slice addresses on the device and cannot check
        # them itself: its contract asks for 16-byte alignment where m % 32 == 0
        if m % 32 == 0 and _dev(a, f"packed_slices[{p}]") % 16:
            raise ValueError(f"packed_slices[{p}] must be 16-byte aligned when m % 32 == 0")
        if _dev(b, f"scale_slices[{p}]") % 4:
            raise ValueError(f"scale_slices[{p}] must be 4-byte aligned")
    dev = packed_slices[0].device
    if packed_out is None:
        packed_out = _output(stream, dev, torch.uint8, int4_bytes(m))
    if scales_out is None:
        scales_out = _output(stream, dev, torch.float32, _alloc_nsc(m, block))
    _need(packed_out, "packed_out", int4_bytes(m), _U8)
    _need(scales_out, "scales_out", _nsc(m, block), _F32)
    # the pointer tables live in device memory (the kernel reads them); built
    # here they are allocated on the current stream and, if the call runs on
    # another (a torch stream or a raw handle), recorded on it so the
    # allocator keeps them until the kernel has read them
    if tables is None:
        tab, stab = gather_tables(packed_slices, scale_slices)
        if stream is not None:
            st = _stream_object(stream, dev)
            tab.record_stream(st)
            stab.record_stream(st)
    else:
        tab, stab = tables
        _need(tab, "tables[0]", P, (torch.int64,))
        _need(stab, "tables[1]", P, (torch.int64,))
    _check(lib().qgz_reduce_level_gather(tab.data_ptr(), stab.data_ptr(), P, m, block,
                                         _dev(packed_out, "packed_out"), _dev(scales_out, "scales_out"),
                                         _stream(stream)), "qgz_reduce_level_gather")
    return packed_out, scales_out


def qgz_reduce_level_gather_noalloc(packed_slices, scale_slices, m, block, packed_out, scales_out, stream=None):
    """qgz_reduce_level_gather without any device allocation: the slice
    addresses go to the library in host arrays, and the caller passes the
    outputs.  Up to 64 slices the addresses travel as kernel arguments; beyond
    that through one device table per GPU that the library keeps, so calls of more
    than 64 slices that may overlap on one GPU must be ordered (one stream)."""
    import ctypes
    P = len(packed_slices)
    if P != len(scale_slices) or P == 0:
        raise ValueError("give P >= 1 byte slices and as many scale slices")
    for p, (a, b) in enumerate(zip(packed_slices, scale_slices)):
        _need(a, f"packed_slices[{p}]", int4_bytes(m), _U8)
        _need(b, f"scale_slices[{p}]", _nsc(m, block), _F32)
    _need(packed_out, "packed_out", int4_bytes(m), _U8)
    _need(scales_out, "scales_out", _nsc(m, block), _F32)
    tab = (ctypes.c_void_p * P)(*[_dev(t, f"packed_slices[{p}]") for p, t in enumerate(packed_slices)])
    stab = (ctypes.c_void_p * P)(*[_dev(t, f"scale_slices[{p}]") for p, t in enumerate(scale_slices)])
    _check(lib().qgz_reduce_level_gather_noalloc(ctypes.cast(tab, ctypes.c_void_p), ctypes.cast(stab, ctypes.c_void_p),
                                                 P, m, block, _dev(packed_out, "packed_out"),
                                                 _dev(scales_out, "scales_out"), _stream(stream)),
           "qgz_reduce_level_gather_noalloc")
    return packed_out, scales_out


def qwz_dequant_gemm(x, codes, scales, N, block=256, y=None, stream=None):
    """y[M, N] = x[M, K] @ deq(W)^T with W the N x K INT8 weight (codes int8
    [N*K] row-major, scales [ceil(N*K/block)]) dequantised to x's dtype
    (bf16 or fp16) on load; y is float32.  K must be a multiple of 64."""
    if x.dim() != 2:
        raise ValueError("x must be 2-D [M, K]")
    M, K = x.shape
    _need(x, "x", M * K, (torch.bfloat16, torch.float16))
    _need(codes, "codes", N * K, _I8)
    _need(scales, "scales", _nsc(N * K, block), _F32)
    if y is None:
        y = _output(stream, x.device, torch.float32, M, N)
    _need(y, "y", M * N, _F32)
    _check(lib().qwz_dequant_gemm(_dev(x, "x"), _TORCH_DT[x.dtype], _dev(codes, "codes"), _dev(scales, "scales"),
                                  M, N, K, block, _dev(y, "y"), _stream(stream)), "qwz_dequant_gemm")
    return y


def embedding(ids, table, scale=1.0, out_dtype=None, out=None, stream=None):
    """Rows of an embedding table by token id, times scale: out[..., :] =
    scale * table[ids[...], :], rounded once to out_dtype (the table's if not
    given).  ids int32 or int64 of any shape; an id outside [0, V) gives a row of
    zeros (padding).  table [V, D] f32 / f16 / bf16 -> out [*ids.shape, D]."""
    if table.dim() != 2:
        raise ValueError("table must be 2-D [V, D]")
    V, D = table.shape
    T = ids.numel()
    ids_at = _ptr(ids, "ids", T, _IDS)
    table_at = _ptr(table, "table", V * D, _ELEM)
    if out is None:
        out = _output(stream, ids.device, out_dtype or table.dtype, *ids.shape, D)
    out_at = _ptr(out, "out", T * D, _ELEM)
    _check(lib().zq_embedding(ids_at or _dev(ids, "ids"), _ID_DT[ids.dtype], T, table_at or _dev(table, "table"),
                              _TORCH_DT[table.dtype], V, D, scale, out_at or _dev(out, "out"), _TORCH_DT[out.dtype],
                              _stream(stream)), "embedding")
    return out


def qwz_embedding(ids, codes, scales, V, D, block=256, scale=1.0, out_dtype=torch.bfloat16, out=None, stream=None):
    """embedding from a table in the INT8 format (codes int8 [V*D], scales
    [ceil(V*D/block)], as gathered): only the rows that occur are read and
    dequantised.  With scale 1 they are the rows qwz_dequantize writes."""
    T = ids.numel()
    ids_at = _ptr(ids, "ids", T, _IDS)
    codes_at = _ptr(codes, "codes", V * D, _I8)
    scales_at = _ptr(scales, "scales", _nsc(V * D, block), _F32)
    if out is None:
        out = _output(stream, ids.device, out_dtype, *ids.shape, D)
    out_at = _ptr(out, "out", T * D, _ELEM)
    _check(lib().qwz_embedding(ids_at or _dev(ids, "ids"), _ID_DT[ids.dtype], T, codes_at or _dev(codes, "codes"),
                               scales_at or _dev(scales, "scales"), V, D, block, scale, out_at or _dev(out, "out"),
                               _TORCH_DT[out.dtype], _stream(stream)), "qwz_embedding")
    return out


def _workspace(nbytes, device, stream):
    """Memory for one call on `stream`, from that stream's own pool: its last user and
    its next one are ordered with the call."""
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(_stream_object(stream, device)):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _given_workspace(workspace, need, device, stream):
    """(address, bytes) of the caller's workspace, or of one for this call."""
    if workspace is None:
        if need <= 0:
            return 0, 0
        workspace = _workspace(need, device, stream)
    _need(workspace, "workspace", max(need, 0), _U8)
    return _dev(workspace, "workspace"), workspace.numel()


def embedding_grad_bytes(T, V, D):
    """Bytes of workspace embedding_grad takes for T tokens and a V x D table."""
    n = lib().zq_embedding_grad_bytes(T, V, D)
    if n < 0:
        raise ValueError(f"embedding_grad does not take T={T}, V={V}, D={D}")
    return n


def embedding_grad(ids, dy, V, scale=1.0, out_dtype=torch.float32, out=None, accumulate=False, workspace=None,
                   stream=None):
    """Gradient of the embedding table from dy [*ids.shape, D]: dense [V, D] of
    out_dtype, row v the scaled sum of the rows of dy whose id is v (binary32, in a
    fixed order), zeros where none is.  Ids outside [0, V) take no part.  With
    accumulate the sums are added to `out` (required) and other rows stay as they
    are.  workspace: uint8, embedding_grad_bytes(T, V, D) or more; allocated if not
    given."""
    T = ids.numel()
    ids_at = _ptr(ids, "ids", T, _IDS)
    if dy.dim() < 1 or dy.numel() != T * dy.shape[-1]:
        raise ValueError(f"dy has shape {tuple(dy.shape)}; expected {(*ids.shape, 'D')}")
    D = dy.shape[-1]
    dy_at = _ptr(dy, "dy", T * D, _ELEM)
    need = embedding_grad_bytes(T, V, D)
    if out is None:
        if accumulate:
            raise ValueError("accumulate adds to out: give it")
        out = _output(stream, dy.device, out_dtype, V, D)
    out_at = _ptr(out, "out", V * D, _ELEM)
    ws_at, ws_size = _given_workspace(workspace, need, dy.device, stream)
    _check(lib().zq_embedding_grad(ids_at or _dev(ids, "ids"), _ID_DT[ids.dtype], T, dy_at or _dev(dy, "dy"),
                                   _TORCH_DT[dy.dtype], V, D, scale, int(bool(accumulate)), out_at or _dev(out, "out"),
                                   _TORCH_DT[out.dtype], ws_at, ws_size, _stream(stream)), "embedding_grad")
    return out


class GradTable:
    """A rank's gradient tensors for grad_norm and grad_clip (grad_table makes it).
    Holds the tensors; they may change their values, not their places.  Calls with
    one table must be ordered (one stream, or events)."""

    def __init__(self, tensors, outs, plan, table):
        self.tensors, self.outs, self.plan, self.table = tensors, outs, plan, table


def grad_table(grads, outs=None):
    """GradTable of a list of gradients, built once for gradients that stay in
    place.  A gradient is a dense tensor (f32 / f16 / bf16) or an INT4 shard as a
    tuple (packed, scales, n, block).  outs: where grad_clip writes, an entry per
    gradient: a tensor of as many elements, or None for in place (an INT4 shard's
    scales; an INT4 shard with an out is dequantised into it)."""
    grads = list(grads)
    outs = [None] * len(grads) if outs is None else list(outs)
    if len(outs) != len(grads):
        raise ValueError(f"{len(outs)} outs for {len(grads)} gradients")
    entries = (_Grad * max(1, len(grads)))()
    dev = None
    for i, (g, o, e) in enumerate(zip(grads, outs, entries)):
        if isinstance(g, (tuple, list)):
            packed, scales, n, block = g
            _need(packed, f"grads[{i}] packed", int4_bytes(n), _U8)
            _need(scales, f"grads[{i}] scales", _nsc(n, block), _F32)
            e.data, e.scales = _dev(packed, f"grads[{i}] packed"), _dev(scales, f"grads[{i}] scales")
            e.n, e.dtype, e.block = n, ZQ_INT4, block
            at = packed.device
        else:
            _need(g, f"grads[{i}]", 0, _ELEM)
            e.data, e.n, e.dtype = _dev(g, f"grads[{i}]"), g.numel(), _TORCH_DT[g.dtype]
            at = g.device
        if o is not None:
            _need(o, f"outs[{i}]", e.n, _ELEM)
            e.out, e.out_dtype = _dev(o, f"outs[{i}]"), _TORCH_DT[o.dtype]
            if o.device != at:
                raise ValueError(f"outs[{i}] is on {o.device}, its gradient on {at}")
        if dev is not None and at != dev:
            raise ValueError(f"grads[{i}] is on {at}, those before it on {dev}")
        dev = at
    if dev is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    plan = _GradPlan()
    _check(lib().zq_grad_plan_make(entries, len(grads), ctypes.byref(plan)), "grad_table")
    host = torch.zeros(plan.bytes, dtype=torch.uint8)
    _check(lib().zq_grad_plan_table(entries, ctypes.byref(plan), host.data_ptr()), "grad_table")
    return GradTable(grads, outs, plan, host.to(dev))


def _table(grads, stream):
    """grads as a GradTable; one built here is kept until `stream` has passed."""
    if isinstance(grads, GradTable):
        return grads
    t = grad_table(grads)
    if stream is not None:
        t.table.record_stream(_stream_object(stream, t.table.device))
    return t


def grad_norm(grads, scale=1.0, out=None, stream=None):
    """The 2-norm of all gradients together, times |scale|: a float32 scalar tensor.
    grads: a GradTable, or a list that grad_table takes (built for this call: it
    copies a small table to the GPU).  Squares and sums are binary64, in a fixed
    order."""
    t = _table(grads, stream)
    if out is None:
        out = _output(stream, t.table.device, torch.float32, 1).view(())
    _need(out, "out", 1, _F32)
    _check(lib().zq_grad_norm(ctypes.byref(t.plan), t.table.data_ptr(), scale, _dev(out, "out"), _stream(stream)),
           "grad_norm")
    return out


def grad_clip(grads, norm, max_norm, scale=1.0, stream=None):
    """Scales every gradient by scale * min(1, max_norm / (norm + 1e-6)), read from
    `norm` (grad_norm's, called with the same scale) on the GPU.  Dense tensors and
    INT4 shards' scales in place, or into the table's outs.  Returns the tensors
    written: per gradient its out, itself, or an INT4 shard's scales."""
    t = _table(grads, stream)
    _need(norm, "norm", 1, _F32)
    _check(lib().zq_grad_clip(ctypes.byref(t.plan), t.table.data_ptr(), _dev(norm, "norm"), max_norm, scale,
                              _stream(stream)), "grad_clip")
    return [o if o is not None else g[1] if isinstance(g, (tuple, list)) else g for g, o in zip(t.tensors, t.outs)]


def int4_dequant_gemm_bytes(M, N, K):
    """Bytes of workspace int4_dequant_gemm takes for M rows and an N x K weight."""
    n = lib().zq_int4_dequant_gemm_bytes(M, N, K)
    if n < 0:
        raise ValueError(f"int4_dequant_gemm does not take M={M}, N={N}, K={K}")
    return n


def int4_dequant_gemm(x, packed, scales, N, block=128, y=None, workspace=None, stream=None):
    """y[M, N] = x[M, K] @ W^T with W the N x K weight in the INT4 format (packed
    uint8 [N*K/2] row-major, scales [ceil(N*K/block)]: qgz_quantize of the weight),
    read as it is; meant for few rows.  x bf16 or fp16, y float32.  K must be a
    multiple of 64.  Codes are summed before they are scaled: bf16 x of 2^122 and more
    may overflow, of less than 2^-110 lose bits.  workspace: uint8, int4_dequant_gemm_bytes(M, N, K) or more;
    allocated if not given."""
    if x.dim() != 2:
        raise ValueError("x must be 2-D [M, K]")
    M, K = x.shape
    x_at = _ptr(x, "x", M * K, _HALF)
    packed_at = _ptr(packed, "packed", int4_bytes(N * K), _U8)
    scales_at = _ptr(scales, "scales", _nsc(N * K, block), _F32)
    if y is None:
        y = _output(stream, x.device, torch.float32, M, N)
    y_at = _ptr(y, "y", M * N, _F32)
    at, size = _given_workspace(workspace, lib().zq_int4_dequant_gemm_bytes(M, N, K), x.device, stream)
    _check(lib().zq_int4_dequant_gemm(x_at or _dev(x, "x"), _TORCH_DT[x.dtype], packed_at or _dev(packed, "packed"),
                                      scales_at or _dev(scales, "scales"), M, N, K, block, y_at or _dev(y, "y"), at,
                                      size, _stream(stream)), "int4_dequant_gemm")
    return y


def adamw_states(params, bits=32, block=256):
    """Fresh moments for adamw_table: (exp_avg, exp_avg_sq), a list each with an entry per
    parameter: binary32 zeros, or with bits=8 tuples (codes, scales, block) of float8 zeros
    (e4m3 and e5m2) and a binary32 scale a block."""
    if bits not in (32, 8):
        raise ValueError(f"bits is {bits}; expected 32 or 8")
    lists = []
    for name in ("exp_avg", "exp_avg_sq"):
        if bits == 32:
            lists.append([torch.zeros(p.shape, dtype=torch.float32, device=p.device) for p in params])
        else:
            lists.append([(torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(_F8[name]),
                           torch.zeros(_alloc_nsc(p.numel(), block), dtype=torch.float32, device=p.device), block)
                          for p in params])
    return tuple(lists)


class AdamWTable:
    """The tensors of an optimizer's step (adamw_table makes it).  Holds them; they may
    change their values, not their places.  Calls with one table must be ordered (one
    stream, or events)."""

    def __init__(self, tensors, plan, table):
        self.tensors, self.plan, self.table = tensors, plan, table
        self.params = tensors[0]


def _per_tensor(v, n, name):
    v = list(v) if isinstance(v, (list, tuple)) else [v] * n
    if len(v) != n:
        raise ValueError(f"{len(v)} {name} for {n} parameters")
    return v


def adamw_table(params, grads, exp_avg, exp_avg_sq, outs=None, weight_decay=0.0, lr_scale=1.0):
    """AdamWTable of a list of parameters (f32 / f16 / bf16, updated in place) with their
    gradients and moments, built once for tensors that stay in place.
    grads: dense tensors (f32 / f16 / bf16) or INT4 shards (packed, scales, n, block).
    exp_avg, exp_avg_sq: float32 tensors, or (codes, scales, block) with codes
    float8_e4m3fn and float8_e5m2 and scales float32 [ceil(n/block)] (adamw_states makes
    either).  outs: None, or per parameter None, a dense tensor (f32 / f16 / bf16) that
    receives the new weight, or (codes int8, scales, block): what qwz_quantize of it
    writes.  weight_decay, lr_scale: numbers, or one per parameter."""
    lists = [list(params), list(grads), list(exp_avg), list(exp_avg_sq)]
    count = len(lists[0])
    lists.append([None] * count if outs is None else list(outs))
    for name, one in zip(("grads", "exp_avg", "exp_avg_sq", "outs"), lists[1:]):
        if len(one) != count:
            raise ValueError(f"{len(one)} {name} for {count} parameters")
    decays, rates = _per_tensor(weight_decay, count, "weight_decay"), _per_tensor(lr_scale, count, "lr_scale")
    entries = (_AdamW * max(1, count))()
    dev = lists[0][0].device if count else None
    for i, (p, g, m, v, o, e) in enumerate(zip(*lists, entries)):
        def at(t, name, need, dtypes):
            _need(t, f"{name}[{i}]", need, dtypes)
            if t.device != dev:
                raise ValueError(f"{name}[{i}] is on {t.device}, the parameters on {dev}")
            return _dev(t, f"{name}[{i}]")
        e.param, e.n = at(p, "params", 0, _ELEM), p.numel()
        e.param_dtype, n = _TORCH_DT[p.dtype], e.n
        if isinstance(g, (tuple, list)):
            packed, scales, of, block = g
            if of != n:
                raise ValueError(f"grads[{i}] has {of} elements, its parameter {n}")
            e.grad, e.grad_dtype, e.grad_block = at(packed, "grads", int4_bytes(n), _U8), ZQ_INT4, block
            e.grad_scales = at(scales, "grads", _nsc(n, block), _F32)
        else:
            e.grad = at(g, "grads", n, _ELEM)
            if g.numel() != n:
                raise ValueError(f"grads[{i}] has {g.numel()} elements, its parameter {n}")
            e.grad_dtype = _TORCH_DT[g.dtype]
        if isinstance(m, (tuple, list)) != isinstance(v, (tuple, list)):
            raise ValueError(f"exp_avg[{i}] and exp_avg_sq[{i}] are not held alike")
        if isinstance(m, (tuple, list)):
            if m[2] != v[2]:
                raise ValueError(f"exp_avg[{i}] has blocks of {m[2]}, exp_avg_sq[{i}] of {v[2]}")
            e.state_dtype, e.state_block = ZQ_F8, m[2]
            e.m, e.v = at(m[0], "exp_avg", n, (_F8["exp_avg"],)), at(v[0], "exp_avg_sq", n, (_F8["exp_avg_sq"],))
            e.m_scales = at(m[1], "exp_avg", _nsc(n, m[2]), _F32)
            e.v_scales = at(v[1], "exp_avg_sq", _nsc(n, m[2]), _F32)
        else:
            e.state_dtype = ZQ_F32
            e.m, e.v = at(m, "exp_avg", n, _F32), at(v, "exp_avg_sq", n, _F32)
        if isinstance(o, (tuple, list)):
            e.out, e.out_dtype, e.out_block = at(o[0], "outs", n, _I8), ZQ_INT8, o[2]
            e.out_scales = at(o[1], "outs", _nsc(n, o[2]), _F32)
        elif o is not None:
            e.out = at(o, "outs", n, _ELEM)
            e.out_dtype = _TORCH_DT[o.dtype]
        e.weight_decay, e.lr_scale = decays[i], rates[i]
    plan = _AdamWPlan()
    _check(lib().zq_adamw_plan_make(entries, count, ctypes.byref(plan)), "adamw_table")
    host = torch.zeros(plan.bytes, dtype=torch.uint8)
    _check(lib().zq_adamw_plan_table(entries, ctypes.byref(plan), host.data_ptr()), "adamw_table")
    return AdamWTable(lists, plan, host.to(dev or torch.device("cuda", torch.cuda.current_device())))


def adamw_step(table, step, lr, betas=(0.9, 0.999), eps=1e-8, norm=None, max_norm=None, scale=1.0, stream=None):
    """One AdamW step over an AdamWTable, in a launch or two; returns the parameters, updated
    in place.  step counts from 1.  With norm (grad_norm's, on the GPU, called with the
    same scale) gradients are clipped to max_norm on the way, as grad_clip does, and a
    norm that is not finite leaves everything as it is; scale multiplies the gradients.
    step (int64) and lr (float32) may be GPU tensors of one element, read when the work
    runs: what a captured step needs to go on.  8-bit moments are rounded up or down by
    bits that follow from the step, so the same step gives the same result."""
    if not isinstance(table, AdamWTable):
        raise TypeError("table must be an AdamWTable")
    a = _AdamWArgs(0.0, betas[0], betas[1], eps, 0, 0.0, scale)
    step_at = lr_at = norm_at = None
    if isinstance(step, torch.Tensor):
        _need(step, "step", 1, _I64)
        step_at = _dev(step, "step")
    else:
        a.step = step
    if isinstance(lr, torch.Tensor):
        _need(lr, "lr", 1, _F32)
        lr_at = _dev(lr, "lr")
    else:
        a.lr = lr
    if norm is not None:
        if max_norm is None:
            raise ValueError("norm clips to max_norm: give it")
        _need(norm, "norm", 1, _F32)
        norm_at, a.max_norm = _dev(norm, "norm"), max_norm
    _here(table=table.table, step=step if step_at else None, lr=lr if lr_at else None, norm=norm)
    _check(lib().zq_adamw_step(ctypes.byref(table.plan), table.table.data_ptr(), ctypes.byref(a), step_at, lr_at,
                               norm_at, _stream(stream)), "adamw_step")
    return table.params


def _here(**tensors):
    """The call runs on the current device, and its tensors (None: not given) are there."""
    now = torch._C._cuda_getDevice()
    for name, t in tensors.items():
        if t is not None and t.get_device() != now:
            raise ValueError(f"{name} is on {t.device}, the current device is cuda:{now}")


def _elements(dtype, name):
    """A type of elements that a call is to allocate."""
    if dtype not in _TORCH_DT:
        raise TypeError(f"{name} is {dtype}; expected one of {[str(d) for d in _ELEM]}")
    return dtype


def _rows(x, name="x"):
    """(rows, row length) of a tensor whose last dimension is normed."""
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"{name} has shape {tuple(x.shape)}; expected [..., D]")
    return x.numel() // x.shape[-1], x.shape[-1]


def _like(t, name, x, dtypes):
    """The address of a tensor of x's shape (None stays None)."""
    if t is None:
        return None
    at = _ptr(t, name, x.numel(), dtypes)
    if t.shape != x.shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}; expected {tuple(x.shape)}")
    return at or _dev(t, name)


def _weight(weight, D):
    """(address, dtype code) of a norm's weight, which may be None."""
    if weight is None:
        return None, ZQ_F32
    at = _ptr(weight, "weight", D, _ELEM)
    if weight.numel() != D:
        raise ValueError(f"weight holds {weight.numel()} elements; rows have {D}")
    return at or _dev(weight, "weight"), _TORCH_DT[weight.dtype]


def _rms_args(x, weight, residual, hidden, rstd, out, stream):
    """What both kinds of norm take, checked; what the call allocates itself is not."""
    T, D = _rows(x)
    x_at = _ptr(x, "x", T * D, _ELEM) or _dev(x, "x")
    w_at, wt = _weight(weight, D)
    _here(x=x, weight=weight, residual=residual, hidden=hidden, rstd=rstd, out=out)
    res_at = h_at = None
    if residual is None:
        if hidden is not None:
            raise ValueError("hidden receives x + residual: give the residual")
        hidden = x
    else:
        res_at = _like(residual, "residual", x, (x.dtype,))
        if hidden is None:
            hidden = _output(stream, x.device, x.dtype, *x.shape)
            h_at = hidden.data_ptr()
        else:
            h_at = _like(hidden, "hidden", x, (x.dtype,))
    if rstd is None:
        rstd = _output(stream, x.device, torch.float32, T)
        r_at = rstd.data_ptr()
    else:
        r_at = _ptr(rstd, "rstd", T, _F32) or _dev(rstd, "rstd")
    return T, D, x_at, w_at, wt, res_at, hidden, h_at, rstd, r_at


def rms_norm(x, weight, residual=None, eps=1e-6, out_dtype=None, out=None, hidden=None, rstd=None, stream=None):
    """Root-mean-square norm of x's last dimension after the residual's addition:
    (y, h, rstd) with h = x + residual (x itself without one), rstd = 1 / sqrt(mean(h^2)
    + eps) of each row (binary64, rounded once) and y = h * rstd * weight.  x f32 / f16 /
    bf16 [..., D], residual of its type and shape, weight f32 / f16 / bf16 [D] or None
    (ones); y of out_dtype (x's if not given).  out, hidden, rstd: where y, h and rstd go;
    hidden may be residual or x itself.  h and rstd are what rms_norm_grad takes."""
    T, D, x_at, w_at, wt, res_at, h, h_at, rstd, r_at = _rms_args(x, weight, residual, hidden, rstd, out, stream)
    if out is None:
        out = _output(stream, x.device, _elements(out_dtype or x.dtype, "out_dtype"), *x.shape)
        y_at = out.data_ptr()
    else:
        y_at = _like(out, "out", x, _ELEM)
    _check(lib().zq_rms_norm(x_at, res_at, _TORCH_DT[x.dtype], w_at, wt, T, D, eps, h_at, y_at, _TORCH_DT[out.dtype],
                             r_at, _stream(stream)), "rms_norm")
    return out, h, rstd


def qwz_rms_norm(x, weight, residual=None, eps=1e-6, block=256, codes=None, scales=None, hidden=None, rstd=None,
                 stream=None):
    """rms_norm with its output in the INT8 format: (codes, scales, h, rstd), codes int8 of
    x's shape and scales [numel / block], what qwz_quantize gives for the unrounded y.  D
    must be a multiple of block."""
    T, D, x_at, w_at, wt, res_at, h, h_at, rstd, r_at = _rms_args(x, weight, residual, hidden, rstd, codes, stream)
    if codes is None:
        codes = _output(stream, x.device, torch.int8, *x.shape)
        c_at = codes.data_ptr()
    else:
        c_at = _ptr(codes, "codes", T * D, _I8) or _dev(codes, "codes")
    if scales is None:
        scales = _output(stream, x.device, torch.float32, _alloc_nsc(T * D, block))
        s_at = scales.data_ptr()
    else:
        s_at = _ptr(scales, "scales", _nsc(T * D, block), _F32) or _dev(scales, "scales")
        _here(scales=scales)
    _check(lib().qwz_rms_norm(x_at, res_at, _TORCH_DT[x.dtype], w_at, wt, T, D, eps, h_at, c_at, s_at, block, r_at,
                              _stream(stream)), "qwz_rms_norm")
    return codes, scales, h, rstd


def rms_norm_grad_bytes(T, D):
    """Bytes of workspace rms_norm_grad takes for T rows of D elements."""
    n = lib().zq_rms_norm_grad_bytes(T, D)
    if n < 0:
        raise ValueError(f"rms_norm_grad does not take T={T}, D={D}")
    return n


def rms_norm_grad(dy, h, weight, rstd, dh=None, out=None, dweight=None, accumulate=False, workspace=None, stream=None):
    """Gradient of rms_norm: (dx, dweight).  dy is the gradient of y [..., D], h and rstd
    what rms_norm returned, dh (of h's type, or None) the gradient that reaches h by
    itself.  dx [..., D] of h's type is the gradient of x and of the residual; out may be
    dh.  dweight [D] is float32 if not given; with accumulate it is added to the given
    one.  Sums are binary32 in a fixed order.  workspace: uint8, rms_norm_grad_bytes(rows,
    D) or more; allocated if not given."""
    T, D = _rows(h, "h")
    h_at = _ptr(h, "h", T * D, _ELEM)
    dy_at = _like(dy, "dy", h, _ELEM)
    w_at, wt = _weight(weight, D)
    r_at = _ptr(rstd, "rstd", T, _F32)
    dh_at = _like(dh, "dh", h, (h.dtype,))
    h_at, r_at = h_at or _dev(h, "h"), r_at or _dev(rstd, "rstd")
    _here(h=h, dy=dy, weight=weight, rstd=rstd, dh=dh, out=out, dweight=dweight, workspace=workspace)
    if out is None:
        out = _output(stream, h.device, h.dtype, *h.shape)
        out_at = out.data_ptr()
    else:
        out_at = _like(out, "out", h, (h.dtype,))
    if dweight is None:
        if accumulate:
            raise ValueError("accumulate adds to dweight: give it")
        dweight = _output(stream, h.device, torch.float32, D)
        dw_at = dweight.data_ptr()
    else:
        dw_at = _ptr(dweight, "dweight", D, _ELEM) or _dev(dweight, "dweight")
        if dweight.numel() != D:
            raise ValueError(f"dweight holds {dweight.numel()} elements; rows have {D}")
    ws_at, ws_size = _given_workspace(workspace, rms_norm_grad_bytes(T, D), h.device, stream)
    _check(lib().zq_rms_norm_grad(dy_at, _TORCH_DT[dy.dtype], h_at, _TORCH_DT[h.dtype], w_at, wt, r_at, dh_at, T, D,
                                  out_at, int(bool(accumulate)), dw_at, _TORCH_DT[dweight.dtype], ws_at, ws_size,
                                  _stream(stream)), "rms_norm_grad")
    return out, dweight


def _logits(t, name, dtypes, rows=None):
    """(address, rows, V, distance of rows) of logits [..., V]: contiguous, or of two
    dimensions with rows further apart (a padded head's logits[:, :V])."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}; expected one of {[str(d) for d in dtypes]}")
    T, V = _rows(t, name)
    if rows is not None and T != rows:
        raise ValueError(f"{name} has {T} rows; expected {rows}")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.is_contiguous():
        return t.data_ptr(), T, V, V
    if t.dim() != 2 or (V > 1 and t.stride(1) != 1) or t.stride(0) < V:
        raise ValueError(f"{name} must be contiguous, or rows of contiguous elements")
    return t.data_ptr(), T, V, t.stride(0)


def _per_row(t, name, T):
    if t is None:
        return None
    at = _ptr(t, name, T, _F32)
    if t.numel() != T:
        raise ValueError(f"{name} holds {t.numel()} elements; {T} needed")
    return at or _dev(t, name)


def _token_ids(ids, T):
    at = _ptr(ids, "ids", T, _IDS)
    if ids.numel() != T:
        raise ValueError(f"{ids.numel()} ids for {T} rows of logits")
    return at or _dev(ids, "ids")


def token_logp(logits, ids, scale=1.0, out=None, stream=None):
    """Log-probability of one token a row: log_softmax(scale * logits)[..., ids], float32 of
    ids' shape.  logits f32 / f16 / bf16 [..., V], contiguous or a padded head's
    logits[:, :V]; ids int32 or int64, one a row; scale, above 0 and up to 2^127, is 1 /
    temperature.  An id outside [0, V) gives 0."""
    l_at, T, V, ld = _logits(logits, "logits", _ELEM)
    ids_at = _token_ids(ids, T)
    _here(logits=logits, ids=ids, out=out)
    if out is None:
        out = _output(stream, logits.device, torch.float32, *ids.shape)
        out_at = out.data_ptr()
    else:
        out_at = _per_row(out, "out", T)
    _check(lib().zq_token_logp(l_at, _TORCH_DT[logits.dtype], T, V, ld, ids_at, _ID_DT[ids.dtype], scale, out_at,
                               _stream(stream)), "token_logp")
    return out


def policy_loss_bytes(T):
    """Bytes of workspace policy_loss takes for T rows of logits."""
    n = lib().zq_policy_loss_bytes(T)
    if n < 0:
        raise ValueError(f"policy_loss does not take T={T}")
    return n


def policy_loss(logits, ids, old_logp, advantages, weights=None, ref_logp=None, clip=(0.2, 0.2), kl=0.0, scale=1.0,
                grad_scale=1.0, grad=True, grad_dtype=None, logp=None, workspace=None, stream=None):
    """The clipped policy loss with a KL term from logits [..., V], and the logits' gradient:
    (sums, logp, grad).  With logp = token_logp(logits, ids, scale), r = exp(logp -
    old_logp) and u = ref_logp - logp the loss of a token is -min(r * A, clip(r, 1 -
    clip[0], 1 + clip[1]) * A) + kl * (exp(u) - u - 1), A its advantage; sums (float32,
    4) holds the sums over tokens, by weight, of the loss, its first term, the KL, and of
    the tokens whose ratio is clipped.
    ids as token_logp takes them (outside [0, V): no loss, a gradient of zeros);
    a logit of -infinity masks its token: a gradient of 0; chosen all the same, a ratio of
    0 and an infinite KL term;
    old_logp, advantages, weights (None: 1 each; 0: masked), ref_logp (needed for kl)
    float32, one a row; scale, above 0 and up to 2^127, is 1 / temperature.
    grad: True (a tensor of logits' shape and of grad_dtype, logits' if not given), a
    tensor to write to (of logits' shape; logits itself for in place), or False (None is
    returned); times grad_scale.  workspace: uint8, policy_loss_bytes(rows) or more;
    allocated if not given."""
    l_at, T, V, ld = _logits(logits, "logits", _ELEM)
    ids_at = _token_ids(ids, T)
    p = _Policy(_per_row(old_logp, "old_logp", T), _per_row(advantages, "advantages", T),
                _per_row(weights, "weights", T), _per_row(ref_logp, "ref_logp", T), clip[0], clip[1], kl, scale,
                grad_scale, 0)
    g_at, gt, ldg = None, ZQ_F32, V
    given = grad if isinstance(grad, torch.Tensor) else None
    _here(logits=logits, ids=ids, old_logp=old_logp, advantages=advantages, weights=weights, ref_logp=ref_logp,
          grad=given, logp=logp, workspace=workspace)
    if given is not None:
        g_at, _, gV, ldg = _logits(grad, "grad", _ELEM, T)
        if gV != V:
            raise ValueError(f"grad has rows of {gV}; logits of {V}")
        gt = _TORCH_DT[grad.dtype]
    elif grad:
        grad = _output(stream, logits.device, _elements(grad_dtype or logits.dtype, "grad_dtype"), *logits.shape)
        g_at, gt = grad.data_ptr(), _TORCH_DT[grad.dtype]
    else:
        grad = None
    sums = _output(stream, logits.device, torch.float32, 4)
    if logp is None:
        logp = _output(stream, logits.device, torch.float32, *ids.shape)
        logp_at = logp.data_ptr()
    else:
        logp_at = _per_row(logp, "logp", T)
    ws_at, ws_size = _given_workspace(workspace, policy_loss_bytes(T), logits.device, stream)
    _check(lib().zq_policy_loss(l_at, _TORCH_DT[logits.dtype], T, V, ld, ids_at, _ID_DT[ids.dtype], ctypes.byref(p),
                                sums.data_ptr(), logp_at, g_at, gt, ldg, ws_at, ws_size,
                                _stream(stream)), "policy_loss")
    return sums, logp, grad
