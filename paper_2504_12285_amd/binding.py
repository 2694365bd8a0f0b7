"""ctypes binding of the BitLinear C-ABI (include/bitlinear.h); the small calls of a decode loop go through
the native form of the same marshalling (csrc/bl_torch.cpp) first.

Argument marshalling only: every step of the path runs in the HIP kernels of
libbitlinear_hip.so.  PyTorch supplies device memory and the current stream.
There is no CPU fallback: if the library is missing, load() raises.
"""
import ctypes
import math
import os
import warnings

from . import build as _build

BL_OK = 0
BL_LAYOUT_ROWMAJOR, BL_LAYOUT_K16, BL_LAYOUT_TRIT5, BL_LAYOUT_KMAJOR = 0, 1, 2, 3
BL_IN_FP32_LATENT, BL_IN_INT8_TERNARY = 0, 1
BL_OP_PACK, BL_OP_QUANT, BL_OP_GEMV, BL_OP_GEMM = 0, 1, 2, 3

_i64, _vp, _ci, _sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t

# name -> (restype, argtypes); mirrors include/bitlinear.h one to one
SIGNATURES = {
    "bl_version": (_ci, []),
    "bl_status_str": (ctypes.c_char_p, [_ci]),
    "bl_packed_bytes": (_sz, [_i64, _i64, _ci]),
    "bl_padded_k": (_i64, [_i64]),
    "bl_workspace_bytes": (_sz, [_ci, _i64, _i64, _i64]),
    "bl_pack_ternary": (_ci, [_vp, _ci, _i64, _i64, _ci, _vp, _vp, _vp, _vp]),
    "bl_unpack_ternary": (_ci, [_vp, _i64, _i64, _ci, _vp, _vp, _vp]),
    "bl_quant_act_int8": (_ci, [_vp, _i64, _i64, _vp, _vp, _vp, _vp]),
    "bl_gemv_w158a8": (_ci, [_vp, _vp, _ci, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "bl_gemm_w158a8": (_ci, [_vp, _vp, _ci, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "bl_bitlinear_decode": (_ci, [_vp, _vp, _ci, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp]),
    "bl_bitlinear_decode_group": (_ci, [_vp, _ci, _ci, _i64, _vp]),
    "bl_quant_act_ex": (_ci, [_vp, _i64, _i64, _vp, _vp, _vp, _vp]),
    "bl_gemm_w158a8_res": (_ci, [_vp, _vp, _ci, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp]),
    "bl_gemm_w158a8_fused": (_ci, [_vp, _vp, _ci, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "bl_quant_from_absmax": (_ci, [_vp, _vp, _i64, _i64, _vp, _vp, _vp, _vp]),
    "bl_stack_table_bytes": (_sz, [_vp, _ci]),
    "bl_stack_table_bytes_batched": (_sz, [_vp, _ci, _i64]),
    "bl_stack_build": (_ci, [_vp, _ci, _ci, _i64, _vp, _vp, _vp]),
    "bl_stack_run": (_ci, [_vp, _vp, _vp]),
    "bl_kv_tables": (_ci, [_vp, _vp]),
    "bl_kv_tables_limited": (_ci, [_vp, _vp]),
    "bl_kv_tables_held": (_ci, [_vp, _vp]),
    "bl_kv_append": (_ci, [_vp, _vp]),
    "bl_kv_append_norm": (_ci, [_vp, _vp]),
    "bl_attn_workspace_bytes": (_sz, [_vp]),
    "bl_attn_kv8": (_ci, [_vp, _vp]),
    "bl_attn_shared_workspace_bytes": (_sz, [_vp]),
    "bl_attn_kv8_shared": (_ci, [_vp, _vp]),
    "bl_f8_workspace_bytes": (_sz, [_vp]),
    "bl_f8_linear": (_ci, [_vp, _vp]),
    "bl_f8_embed": (_ci, [_vp, _vp]),
    "bl_debug_force_path": (_ci, [_ci]),
    "bl_probe_stream_read": (_ci, [_vp, _sz, _ci, _vp, _vp]),
    "bl_probe_stream_write": (_ci, [_vp, _i64, _i64, _ci, _vp]),
    "bl_probe_mfma_i8": (_ci, [_ci, _vp, _vp, _vp]),
    "bl_probe_mfma_i8_ex": (_ci, [_ci, _vp, _vp, _vp, _vp, _vp]),
    "bl_probe_wall_clock_khz": (_ci, []),
    "bl_debug_clock_stamps": (_ci, [_vp]),
    "bl_gemm_w158a8_noalloc": (_ci, [_vp, _vp, _ci, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp]),
}

BL_PROD_BF16, BL_PROD_F32, BL_PROD_ATTN_V, BL_PROD_RESIDUAL, BL_PROD_RELU2_GATE = 0, 1, 2, 3, 4


class Producer(ctypes.Structure):
    """Mirror of bl_producer."""
    _fields_ = [("kind", _ci), ("in0", _vp), ("in1", _vp), ("aux_out", _vp),
                ("n_q", _ci), ("n_kv", _ci), ("head_dim", _ci),
                ("norm", _ci), ("gain", _vp), ("eps", ctypes.c_float)]


def make_producer(kind, in0, in1=None, aux_out=None, n_q=0, n_kv=0, head_dim=0, norm=False, gain=None, eps=1e-5):
    """norm=True: RMS normalisation (optional fp32 gains [K]) in front of the quantiser.  The descriptor keeps its tensors alive: memory of a temporary
    would else be free again before the call that reads it, for an output of that call among others."""
    p = Producer()
    p.tensors = (in0, in1, aux_out, gain)
    p.kind, p.in0, p.in1, p.aux_out = int(kind), _ptr(in0), _ptr(in1), _ptr(aux_out)
    p.n_q, p.n_kv, p.head_dim = int(n_q), int(n_kv), int(head_dim)
    p.norm, p.gain, p.eps = int(bool(norm)), _ptr(gain), float(eps)
    return p


def _producer_width(p, K):
    """Values of a row of in0 where a producer's rows have K; None where the call itself refuses it."""
    kind = p.kind
    if kind == BL_PROD_ATTN_V:
        return (p.n_q + 2 * p.n_kv) * p.head_dim if p.n_q * p.head_dim == K else None
    return K if kind in (BL_PROD_BF16, BL_PROD_F32, BL_PROD_RESIDUAL) else 2 * K if kind == BL_PROD_RELU2_GATE else None


class DecodeDesc(ctypes.Structure):
    """Mirror of bl_decode_desc."""
    _fields_ = [("packed", _vp), ("beta", _vp), ("X", _vp), ("q", _vp), ("scale", _vp), ("rowsum", _vp),
                ("N", _i64), ("K", _i64), ("acc", _vp), ("y", _vp), ("q_out", _vp), ("scale_out", _vp),
                ("fixed_scale", ctypes.c_float), ("prod", Producer), ("residual", _vp)]


BL_EPI_RESIDUAL, BL_EPI_RELU2_GATE = 1, 2


class GemmEpilogue(ctypes.Structure):
    """Mirror of bl_gemm_epilogue."""
    _fields_ = [("kind", _ci), ("residual", _vp), ("y", _vp), ("x_bf16", _vp), ("absmax", _vp)]


class StackPlan(ctypes.Structure):
    """Mirror of bl_stack_plan."""
    _fields_ = [("count", ctypes.c_int32), ("blocks", ctypes.c_int32), ("prep_count", ctypes.c_int32),
                ("inline_count", ctypes.c_int32), ("norm", ctypes.c_int32), ("lds_bytes", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("red_ints", ctypes.c_int32),
                ("wg_offset", _i64), ("prep_offset", _i64),
                ("packed_bytes", _i64), ("table_bytes", _i64),
                ("tokens", ctypes.c_int32), ("entries", ctypes.c_int32)]


BL_KV_INT8, BL_KV_E4M3 = 0, 1
BL_KV_FROM_F32, BL_KV_FROM_BF16 = 0, 1


class KVCacheDesc(ctypes.Structure):
    """Mirror of bl_kv_cache."""
    _fields_ = [("kind", _ci), ("block", _ci), ("n_kv", _ci), ("head_dim", _ci), ("n_blocks", _i64),
                ("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp),
                ("k_stride", _i64), ("v_stride", _i64), ("scale_stride", _i64)]


class KVBatchDesc(ctypes.Structure):
    """Mirror of bl_kv_batch."""
    _fields_ = [("B", _i64), ("rows", _i64), ("table_stride", _i64), ("free_cap", _i64),
                ("block", ctypes.c_int32), ("max_blocks", ctypes.c_int32)] + \
               [(n, _vp) for n in ("seq_len", "new_len", "free_count", "table", "free_list", "seq_len_out", "free_count_out",
                                   "start", "q_start", "positions", "slots", "bad")]


class KVLimitedBatchDesc(ctypes.Structure):
    """Mirror of bl_kv_limited_batch."""
    _fields_ = [("batch", KVBatchDesc), ("max_new", _i64)]


class KVHeldBatchDesc(ctypes.Structure):
    """Mirror of bl_kv_held_batch."""
    _fields_ = [("batch", KVBatchDesc), ("max_new", _i64), ("held", _vp)]


class KVTokensDesc(ctypes.Structure):
    """Mirror of bl_kv_tokens."""
    _fields_ = [("cache", KVCacheDesc), ("qkv", _vp), ("qkv_stride", _i64), ("q_stride", _i64), ("T", _i64), ("n_pos", _i64),
                ("qkv_kind", ctypes.c_int32), ("n_q", ctypes.c_int32)] + \
               [(n, _vp) for n in ("positions", "slots", "cos", "sin", "q_out", "bad")]


class KVNormTokensDesc(ctypes.Structure):
    """Mirror of bl_kv_norm_tokens."""
    _fields_ = [("tokens", KVTokensDesc), ("q_gain", _vp), ("k_gain", _vp), ("eps", ctypes.c_float)]


class AttnDesc(ctypes.Structure):
    """Mirror of bl_attn_desc."""
    _fields_ = [("cache", KVCacheDesc), ("q", _vp), ("q_stride", _i64), ("out_stride", _i64), ("table_stride", _i64), ("B", _i64),
                ("T", _i64), ("q_start", _vp), ("seq_len", _vp), ("table", _vp)] + \
               [(n, ctypes.c_int32) for n in ("n_q", "max_blocks", "max_q", "max_len", "window")] + \
               [("softmax_scale", ctypes.c_float), ("out", _vp), ("workspace", _vp)]


class AttnSharedDesc(ctypes.Structure):
    """Mirror of bl_attn_shared_desc."""
    _fields_ = [("attn", AttnDesc), ("group", _vp), ("shared_blocks", _vp), ("shared_table", _vp), ("shared_stride", _i64), ("n_groups", _i64),
                ("max_shared", ctypes.c_int32), ("max_own", ctypes.c_int32)]


BL_F8_OUT_F32, BL_F8_OUT_BF16 = 0, 1


class F8MatrixDesc(ctypes.Structure):
    """Mirror of bl_f8_matrix."""
    _fields_ = [("codes", _vp), ("scale", _vp), ("N", _i64), ("K", _i64), ("stride", _i64), ("scale_stride", _i64)]


class F8ProductDesc(ctypes.Structure):
    """Mirror of bl_f8_product."""
    _fields_ = [("w", F8MatrixDesc), ("prod", Producer), ("M", _i64), ("y_stride", _i64), ("y", _vp), ("y_kind", ctypes.c_int32), ("workspace", _vp)]


class F8LookupDesc(ctypes.Structure):
    """Mirror of bl_f8_lookup."""
    _fields_ = [("w", F8MatrixDesc), ("ids", _vp), ("T", _i64), ("out_stride", _i64), ("out", _vp), ("out_kind", ctypes.c_int32),
                ("multiplier", ctypes.c_float), ("bad", _vp)]


class BitLinearError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__("%s failed: %s" % (where, status_str(status)))


_lib = None


def load():
    """Load the built library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.LIB_PATH):
            raise RuntimeError("libbitlinear_hip.so is not built (run __graft_entry__.build()); "
                               "this package has no fallback path")
        lib = ctypes.CDLL(_build.LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def status_str(status):
    return load().bl_status_str(int(status)).decode()


def _check(status, where):
    if status != BL_OK:
        raise BitLinearError(status, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


_torch = None


def _get_torch():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _first_stream():
    """Resolves how the current stream is read (once), and reads it.  The two raw getters are what
    torch.cuda.current_stream() ends in; the Stream object around them costs 2.8 us a call against 0.2."""
    global _stream
    torch = _get_torch()
    handle = torch.cuda.current_stream().cuda_stream        # initialises the device, raises without one
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None:
        _stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    else:
        _stream = lambda: raw(device())  # noqa: E731
    return handle


_stream = _first_stream


_native = None


class _PythonForm:
    """Stands for the native form where that is not built: every call is done in Python below."""

    @staticmethod
    def quant(*args):
        return NotImplemented

    product = decode = run = kv = holds = quant


def _first_native():
    """The small calls in native code (csrc/bl_torch.cpp), bound to the loaded library.  A call that it hands back
    (NotImplemented) is done in Python below; so are all of them, more slowly, where it is not built for this
    interpreter and torch."""
    global _native
    lib = load()
    _get_torch()
    try:
        from . import _bl_torch
        if _bl_torch.__doc__ != "built for torch %s" % _build.torch_version():
            raise ImportError("it is " + _bl_torch.__doc__)
    except ImportError as e:
        warnings.warn("the binding's small calls run in Python (7 - 11 us each, 3 - 4 in native code): _bl_torch is not "
                      "built for this interpreter and torch (%s)" % e, RuntimeWarning, stacklevel=3)
        _native = _PythonForm()
        return _native
    _bl_torch.bind(*(ctypes.cast(fn, _vp).value for fn in (lib.bl_quant_act_int8, lib.bl_gemv_w158a8,
                                                            lib.bl_gemm_w158a8, lib.bl_bitlinear_decode, lib.bl_stack_run)))
    _bl_torch.bind_kv(*(ctypes.cast(fn, _vp).value for fn in (lib.bl_kv_tables, lib.bl_kv_append, lib.bl_attn_kv8, lib.bl_kv_tables_limited, lib.bl_kv_tables_held,
                                                               lib.bl_kv_append_norm, lib.bl_attn_kv8_shared, lib.bl_f8_linear, lib.bl_f8_embed)))
    _native = _bl_torch
    return _native


def _result(out, where):
    if type(out) is int:
        raise BitLinearError(out, where)
    return out


def bl_version():
    return load().bl_version()


def bl_packed_bytes(N, K, layout=BL_LAYOUT_K16):
    return load().bl_packed_bytes(N, K, layout)


def bl_padded_k(K):
    """Mirror of bl_padded_k: the same arithmetic without a foreign call (it sits in front of every launch)."""
    return (K + 63) // 64 * 64 if 1 <= K <= 1 << 24 else 0


def bl_workspace_bytes(op, M, N, K):
    return load().bl_workspace_bytes(op, M, N, K)


def _workspace(nbytes, device):
    torch = _get_torch()
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def bl_pack_ternary(W, layout=BL_LAYOUT_K16, beta=None):
    """W: cuda fp32 [N][K] latent weights, or cuda int8 ternary with `beta` given.
    Returns (packed uint8 [N*K/4], beta fp32 [1])."""
    torch = _get_torch()
    N, K = W.shape
    assert W.is_cuda and W.is_contiguous()
    nbytes = bl_packed_bytes(N, K, layout)
    if nbytes == 0:
        raise BitLinearError(2 if layout in (0, 1, 2, 3) else 3, "bl_packed_bytes")
    packed = torch.empty(nbytes, dtype=torch.uint8, device=W.device)
    if W.dtype == torch.float32:
        kind = BL_IN_FP32_LATENT
        beta_t = torch.empty(1, dtype=torch.float32, device=W.device)
    elif W.dtype == torch.int8:
        kind = BL_IN_INT8_TERNARY
        beta_t = torch.as_tensor([float(beta)], dtype=torch.float32, device=W.device) \
            if not isinstance(beta, torch.Tensor) else beta
    else:
        raise TypeError("W must be float32 or int8")
    ws = _workspace(bl_workspace_bytes(BL_OP_PACK, 0, N, K), W.device)
    _check(load().bl_pack_ternary(_ptr(W), kind, N, K, layout, _ptr(packed), _ptr(beta_t), _ptr(ws), _stream()),
           "bl_pack_ternary")
    return packed, beta_t


def bl_unpack_ternary(packed, N, K, layout=BL_LAYOUT_K16):
    """Returns (Wt int8 [N][K], bad int32 [1])."""
    torch = _get_torch()
    Wt = torch.empty((N, K), dtype=torch.int8, device=packed.device)
    bad = torch.empty(1, dtype=torch.int32, device=packed.device)
    _check(load().bl_unpack_ternary(_ptr(packed), N, K, layout, _ptr(Wt), _ptr(bad), _stream()),
           "bl_unpack_ternary")
    return Wt, bad


def bl_quant_act_int8(X, want_rowsum=True):
    """X: cuda bfloat16 [M][K].  Returns (q int8 [M][Kp] with Kp = bl_padded_k(K) and zeros in the padding,
    scale fp32 [M], rowsum int32 [M] or None)."""
    out = (_native or _first_native()).quant(X, want_rowsum)
    if out is not NotImplemented:
        return _result(out, "bl_quant_act_int8")
    torch = _get_torch()
    assert X.is_cuda and X.is_contiguous() and X.dtype == torch.bfloat16
    M, K = X.shape
    q = torch.empty((M, bl_padded_k(K)), dtype=torch.int8, device=X.device)
    scale = torch.empty(M, dtype=torch.float32, device=X.device)
    rowsum = torch.empty(M, dtype=torch.int32, device=X.device) if want_rowsum else None
    _check(load().bl_quant_act_int8(_ptr(X), M, K, _ptr(q), _ptr(scale), _ptr(rowsum), _stream()),
           "bl_quant_act_int8")
    return q, scale, rowsum


def _matmul(fn_name, op, packed, beta, layout, q, scale, rowsum, N, want_acc, want_y, acc, y, workspace, K=None):
    out = (_native or _first_native()).product(0 if op == BL_OP_GEMV else 1, packed, beta, layout, q, scale, rowsum, N,
                                               want_acc, want_y, acc, y, workspace, K)
    if out is not NotImplemented:
        return _result(out, fn_name)
    torch = _get_torch()
    M = q.shape[0]
    K = q.shape[1] if K is None else K          # q is [M][Kp]: pass the true K of a ragged matrix explicitly
    assert q.shape[1] == bl_padded_k(K)
    assert q.is_cuda and q.is_contiguous() and q.dtype == torch.int8
    if want_acc and acc is None:
        acc = torch.empty((M, N), dtype=torch.int32, device=q.device)
    if want_y and y is None:
        y = torch.empty((M, N), dtype=torch.float32, device=q.device)
    if workspace is None and rowsum is None:
        workspace = _workspace(bl_workspace_bytes(op, M, N, K), q.device)
    fn = getattr(load(), fn_name)
    _check(fn(_ptr(packed), _ptr(beta), layout, _ptr(q), _ptr(scale), _ptr(rowsum), M, N, K,
              _ptr(acc), _ptr(y), _ptr(workspace), _stream()), fn_name)
    return acc, y


def bl_gemv_w158a8(packed, beta, layout, q, scale, rowsum, N, want_acc=True, want_y=True,
                   acc=None, y=None, workspace=None, K=None):
    """Decode product, 1 <= M <= 64.  Returns (acc int32 [M][N] or None, y fp32 [M][N] or None)."""
    return _matmul("bl_gemv_w158a8", BL_OP_GEMV, packed, beta, layout, q, scale, rowsum, N, want_acc, want_y,
                   acc, y, workspace, K)


def bl_gemm_w158a8(packed, beta, layout, q, scale, rowsum, N, want_acc=True, want_y=True,
                   acc=None, y=None, workspace=None, K=None):
    """Prefill product, any M.  Returns (acc, y) like bl_gemv_w158a8."""
    return _matmul("bl_gemm_w158a8", BL_OP_GEMM, packed, beta, layout, q, scale, rowsum, N, want_acc, want_y,
                   acc, y, workspace, K)


def bl_bitlinear_decode(packed, beta, layout, X, N, want_acc=False, want_y=True, want_q=False, acc=None, y=None):
    """Fused decode BitLinear, M <= 4: bf16 X [M][K] -> (acc, y, q, scale)."""
    out = (_native or _first_native()).decode(packed, beta, layout, X, N, want_acc, want_y, want_q, acc, y)
    if out is not NotImplemented:
        return _result(out, "bl_bitlinear_decode")
    torch = _get_torch()
    assert X.is_cuda and X.is_contiguous() and X.dtype == torch.bfloat16
    M, K = X.shape
    if want_acc and acc is None:
        acc = torch.empty((M, N), dtype=torch.int32, device=X.device)
    if want_y and y is None:
        y = torch.empty((M, N), dtype=torch.float32, device=X.device)
    q = torch.empty((M, K), dtype=torch.int8, device=X.device) if want_q else None
    scale = torch.empty(M, dtype=torch.float32, device=X.device) if want_q else None
    _check(load().bl_bitlinear_decode(_ptr(packed), _ptr(beta), layout, _ptr(X), M, N, K, _ptr(acc), _ptr(y),
                                      _ptr(q), _ptr(scale), _stream()), "bl_bitlinear_decode")
    return acc, y, q, scale


_QUANT_TENSORS = ("in0", "in1", "aux_out", "gain", "q", "scale", "rowsum")


def _hold(names, *pairs):
    """Each tensor (or None) has so many bytes of memory from its first value on: pairs of them, names for the errors."""
    short = (_native or _first_native()).holds(*pairs)
    if short is NotImplemented:
        short = next((i for i, (t, n) in enumerate(zip(pairs[::2], pairs[1::2])) if t is not None and n > _memory(t)), -1)
    if short >= 0:
        raise ValueError("%s has %d bytes, %d are needed" % (names[short], _memory(pairs[2 * short]), pairs[2 * short + 1]))


def _memory(t):
    return t.untyped_storage().nbytes() - t.storage_offset() * t.element_size()


def make_decode_descs(items):
    """items: list of dicts with tensor values for the bl_decode_desc fields
    (packed, beta, X or q/scale/rowsum, acc, y, q_out, scale_out) and int N, K.
    Returns a ctypes array usable with bl_bitlinear_decode_group."""
    arr = (DecodeDesc * len(items))()
    for d, it in zip(arr, items):
        for f in ("packed", "beta", "X", "q", "scale", "rowsum", "acc", "y", "q_out", "scale_out", "residual"):
            setattr(d, f, _ptr(it.get(f)))
        d.N, d.K = int(it["N"]), int(it["K"])
        d.fixed_scale = float(it.get("fixed_scale", 0.0))
        if it.get("prod") is not None:
            d.prod = it["prod"]
    return arr


def bl_bitlinear_decode_group(descs, layout, M):
    """descs: ctypes array from make_decode_descs (host memory)."""
    _check(load().bl_bitlinear_decode_group(descs, len(descs), layout, M, _stream()), "bl_bitlinear_decode_group")


def bl_quant_act_ex(prod, M, K, device, want_rowsum=True, q=None, scale=None, rowsum=None):
    """Producer + quantiser (prefill side).  prod: Producer from make_producer, whose tensors have memory for M rows.
    Returns (q int8 [M][K], scale fp32 [M], rowsum int32 [M] or None)."""
    torch = _get_torch()
    if q is None:
        q = torch.empty((M, K), dtype=torch.int8, device=device)
    if scale is None:
        scale = torch.empty(M, dtype=torch.float32, device=device)
    if rowsum is None and want_rowsum:
        rowsum = torch.empty(M, dtype=torch.int32, device=device)
    in0, in1, aux_out, gain = getattr(prod, "tensors", (None,) * 4)
    width, both = _producer_width(prod, K) or 0, M * K * 4 if prod.kind == BL_PROD_RESIDUAL else 0
    _hold(_QUANT_TENSORS, in0, M * width * (2 if prod.kind == BL_PROD_BF16 else 4), in1, both, aux_out, both, gain, K * 4 if prod.norm else 0,
          q, M * K, scale, M * 4, rowsum, M * 4)
    _check(load().bl_quant_act_ex(ctypes.byref(prod), M, K, _ptr(q), _ptr(scale), _ptr(rowsum), _stream()),
           "bl_quant_act_ex")
    return q, scale, rowsum


def bl_gemm_w158a8_res(packed, beta, layout, q, scale, rowsum, N, residual, want_acc=False, want_y=True,
                       acc=None, y=None, workspace=None):
    """Prefill product with a residual added in the epilogue.  Returns (acc, y)."""
    torch = _get_torch()
    M, K = q.shape
    if want_acc and acc is None:
        acc = torch.empty((M, N), dtype=torch.int32, device=q.device)
    if want_y and y is None:
        y = torch.empty((M, N), dtype=torch.float32, device=q.device)
    if workspace is None and rowsum is None:
        workspace = _workspace(bl_workspace_bytes(BL_OP_GEMM, M, N, K), q.device)
    _check(load().bl_gemm_w158a8_res(_ptr(packed), _ptr(beta), layout, _ptr(q), _ptr(scale), _ptr(rowsum), M, N, K,
                                     _ptr(residual), _ptr(acc), _ptr(y), _ptr(workspace), _stream()),
           "bl_gemm_w158a8_res")
    return acc, y


def bl_gemm_w158a8_noalloc(packed, beta, layout, q, scale, N, acc=None, y=None):
    """Prefill product through the entry point that allocates nothing (row sums in the
    library's static device scratch).  The caller passes the outputs; returns (acc, y)."""
    M, K = q.shape
    _check(load().bl_gemm_w158a8_noalloc(_ptr(packed), _ptr(beta), layout, _ptr(q), _ptr(scale), M, N, K,
                                         _ptr(acc), _ptr(y), _stream()), "bl_gemm_w158a8_noalloc")
    return acc, y


class Stack:
    """A product table of the persistent streaming decode kernel: bl_stack_build once,
    bl_stack_run per step.  Holds the device table and keeps the descriptors' tensors alive."""

    def __init__(self, items, layout, M, device):
        torch = _get_torch()
        self.items = items                      # keeps every tensor of the table alive
        self.descs = make_decode_descs(items)
        nbytes = load().bl_stack_table_bytes(self.descs, len(items)) if M == 1 else \
            load().bl_stack_table_bytes_batched(self.descs, len(items), M)
        if nbytes == 0:
            raise BitLinearError(2, "bl_stack_table_bytes")
        self.table = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.plan = StackPlan()
        _check(load().bl_stack_build(self.descs, len(items), layout, M, _ptr(self.table), ctypes.byref(self.plan),
                                     _stream()), "bl_stack_build")

    def run(self):
        out = (_native or _first_native()).run(self.table, ctypes.addressof(self.plan))
        if out is not NotImplemented:
            return _result(out, "bl_stack_run")
        _check(load().bl_stack_run(_ptr(self.table), ctypes.byref(self.plan), _stream()), "bl_stack_run")


def bl_gemm_w158a8_fused(packed, beta, layout, q, scale, rowsum, N, kind, x_bf16, absmax, residual=None, y=None,
                         acc=None):
    """Prefill product with a fused producer epilogue (bl_gemm_w158a8_fused).  x_bf16: bf16 [M][N_out]
    out; absmax: fp32 [M], zero before the call."""
    M, K = q.shape
    ep = GemmEpilogue()
    ep.kind, ep.residual, ep.y, ep.x_bf16, ep.absmax = int(kind), _ptr(residual), _ptr(y), _ptr(x_bf16), _ptr(absmax)
    _check(load().bl_gemm_w158a8_fused(_ptr(packed), _ptr(beta), layout, _ptr(q), _ptr(scale), _ptr(rowsum), M, N, K,
                                       ctypes.byref(ep), _ptr(acc), _stream()), "bl_gemm_w158a8_fused")


def bl_quant_from_absmax(X, absmax, q=None, scale=None, rowsum=None):
    """One-pass quantiser of bf16 rows X [M][K] with known row maxima (cleared by the call)."""
    torch = _get_torch()
    M, K = X.shape
    if q is None:
        q = torch.empty((M, K), dtype=torch.int8, device=X.device)
    if scale is None:
        scale = torch.empty(M, dtype=torch.float32, device=X.device)
    if rowsum is None:
        rowsum = torch.empty(M, dtype=torch.int32, device=X.device)
    _check(load().bl_quant_from_absmax(_ptr(X), _ptr(absmax), M, K, _ptr(q), _ptr(scale), _ptr(rowsum), _stream()),
           "bl_quant_from_absmax")
    return q, scale, rowsum


def _wants(t, what, dtype, device, shape=None, rows=False):
    """The tensor as a call may take it: type, device, shape (None: any) and rows without gaps (all of it, unless `rows`)."""
    torch = _get_torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a tensor" % what)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, is %s" % (what, dtype, t.dtype))
    if t.device != device:
        raise ValueError("%s is on %s, not on %s" % (what, t.device, device))
    if shape is not None and (t.dim() != len(shape) or any(a is not None and a != b for a, b in zip(shape, t.shape))):
        raise ValueError("%s must have the shape %s, has %s" % (what, tuple(shape), tuple(t.shape)))
    if not (t.is_contiguous() or rows and t.dim() >= 2 and t[0].is_contiguous() and (t.shape[0] == 1 or t.stride(0) >= t[0].numel())):
        raise ValueError("%s has gaps or another order" % what)
    return t


def _wants_producer(p, M, K, device):
    """A producer whose tensors have M rows at least, each as wide as its kind has it (its values may be in several dimensions).  What the call itself
    refuses, and a descriptor that was filled in by hand, are left to it."""
    torch = _get_torch()
    width = _producer_width(p, K)
    if width is None or not hasattr(p, "tensors"):
        return
    in0, in1, aux_out, gain = p.tensors
    parts = [("in0", in0, width)] + ([("in1", in1, K), ("aux_out", aux_out, K)] if p.kind == BL_PROD_RESIDUAL else [])
    for name, t, wide in parts:
        if t is None:
            continue
        _wants(t, name, torch.bfloat16 if p.kind == BL_PROD_BF16 else torch.float32, device)
        if t.numel() < M * wide or (t.numel() % wide if t.dim() == 1 else wide not in (math.prod(t.shape[i:]) for i in range(t.dim()))):
            raise ValueError("%s must have %d rows of %d values, has the shape %s" % (name, M, wide, tuple(t.shape)))
    if p.norm and gain is not None:
        _wants(gain, "gain", torch.float32, device, (K,))


def _row_stride(t):
    """Elements from a row to the next (a single row may carry any stride, and there may be none)."""
    return t.stride(0) if t.shape[0] > 1 else math.prod(t.shape[1:])


class KVCache:
    """Key/value cache of 8-bit codes (bl_kv_cache): k [n_blocks][n_kv][block][head_dim], v [n_blocks][n_kv][head_dim][block], int8 or
    float8_e4m3fn; k_scale, v_scale fp32 [n_blocks][n_kv].  Blocks may lie apart (views into a pool of several layers)."""

    def __init__(self, k, v, k_scale, v_scale):
        torch = _get_torch()
        if k.dim() != 4 or k.dtype not in (torch.int8, torch.float8_e4m3fn):
            raise TypeError("k must be int8 or float8_e4m3fn [n_blocks][n_kv][block][head_dim]")
        n, h, block, dim = k.shape
        _wants(k, "k", k.dtype, k.device, rows=True)
        _wants(v, "v", k.dtype, k.device, (n, h, dim, block), rows=True)
        _wants(k_scale, "k_scale", torch.float32, k.device, (n, h), rows=True)
        _wants(v_scale, "v_scale", torch.float32, k.device, (n, h), rows=True)
        if _row_stride(k_scale) != _row_stride(v_scale):
            raise ValueError("k_scale and v_scale must have the same stride")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_blocks, self.n_kv, self.block, self.head_dim = n, h, block, dim
        self.desc = KVCacheDesc(BL_KV_INT8 if k.dtype == torch.int8 else BL_KV_E4M3, block, h, dim, n, _ptr(k), _ptr(v), _ptr(k_scale),
                                _ptr(v_scale), _row_stride(k), _row_stride(v), _row_stride(k_scale))

    @classmethod
    def empty(cls, n_blocks, n_kv, block, head_dim, device, kind=BL_KV_INT8):
        """A cache over memory of its own; nothing in it."""
        torch = _get_torch()
        dtype = torch.int8 if kind == BL_KV_INT8 else torch.float8_e4m3fn
        k = torch.empty((n_blocks, n_kv, block, head_dim), dtype=dtype, device=device)
        v = torch.empty((n_blocks, n_kv, head_dim, block), dtype=dtype, device=device)
        scales = [torch.empty((n_blocks, n_kv), dtype=torch.float32, device=device) for _ in range(2)]
        return cls(k, v, *scales)


class _KVCall:
    """A call whose descriptor stands over buffers that the caller keeps: filled once, run as often as wanted (their
    contents may change in between, HIP graphs may replay it)."""

    def run(self):
        out = (_native or _first_native()).kv(self._which, ctypes.addressof(self.desc))
        if out is not NotImplemented:
            return _result(out, self._where)
        _check(getattr(load(), self._where)(ctypes.byref(self.desc), _stream()), self._where)


class KVTables(_KVCall):
    """Block tables and slot maps of a step (bl_kv_tables).  seq_len, new_len int32 [B]; table int32 [B][max_blocks];
    free_list int32 [any]; free_count int32 [1]; rows: rows of the batch.  Outputs: start, q_start, positions, slots, bad, and
    seq_len_out, free_count_out (in_place: seq_len and free_count themselves, for a step that is run again and again).
    max_new: a request that brings more tokens is refused (bl_kv_tables_limited); None: no such limit.
    held: int32 [B], blocks in front of each row that an ended request does not give back (bl_kv_tables_held)."""
    _which, _where = 0, "bl_kv_tables"

    def __init__(self, seq_len, new_len, table, free_list, free_count, block, rows, in_place=False, max_new=None, held=None):
        torch = _get_torch()
        i32, dev, B = torch.int32, seq_len.device, seq_len.shape[0]
        _wants(seq_len, "seq_len", i32, dev, (B,))
        _wants(new_len, "new_len", i32, dev, (B,))
        _wants(table, "table", i32, dev, (B, None), rows=True)
        _wants(free_list, "free_list", i32, dev, (None,))
        _wants(free_count, "free_count", i32, dev, (1,))
        self.seq_len, self.new_len, self.table, self.free_list, self.free_count = seq_len, new_len, table, free_list, free_count

        def new(n):
            return torch.empty(n, dtype=i32, device=dev)
        self.seq_len_out, self.free_count_out = (seq_len, free_count) if in_place else (new(B), new(1))
        self.start, self.q_start, self.positions, self.slots, self.bad = new(B), new(B + 1), new(rows), new(rows), new(1)
        self.desc = KVBatchDesc(B, rows, _row_stride(table), free_list.shape[0], block, table.shape[1],
                                *(_ptr(t) for t in (seq_len, new_len, free_count, table, free_list, self.seq_len_out, self.free_count_out,
                                                    self.start, self.q_start, self.positions, self.slots, self.bad)))
        self.held = held
        if held is not None:
            _wants(held, "held", i32, dev, (B,))
            if max_new is not None and max_new < 1:
                raise ValueError("max_new must be at least 1, is %d" % max_new)
            self._which, self._where = 4, "bl_kv_tables_held"
            self.desc = KVHeldBatchDesc(self.desc, 0 if max_new is None else max_new, _ptr(held))
        elif max_new is not None:
            self._which, self._where = 3, "bl_kv_tables_limited"
            self.desc = KVLimitedBatchDesc(self.desc, max_new)


class KVAppend(_KVCall):
    """New tokens into the cache (bl_kv_append).  qkv fp32 or bf16 [T][(n_q + 2 n_kv) * head_dim]; slots, positions int32 [T];
    cos, sin fp32 [n_pos][head_dim / 2] or None (no rotation).  Output: q bf16 [T][n_q * head_dim].  bad: int32 [1] that counts, or None."""
    _which, _where = 1, "bl_kv_append"

    def __init__(self, cache, qkv, n_q, slots, positions=None, cos=None, sin=None, q=None, bad=None):
        torch = _get_torch()
        dev, dim = cache.k.device, cache.head_dim
        if qkv.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("qkv must be float32 or bfloat16")
        T = qkv.shape[0]
        _wants(qkv, "qkv", qkv.dtype, dev, (T, (n_q + 2 * cache.n_kv) * dim), rows=True)
        _wants(slots, "slots", torch.int32, dev, (T,))
        if cos is not None or sin is not None:
            _wants(cos, "cos", torch.float32, dev, (None, dim // 2))
            _wants(sin, "sin", torch.float32, dev, tuple(cos.shape))
            _wants(positions, "positions", torch.int32, dev, (T,))
        if q is None and n_q:
            q = torch.empty((T, n_q * dim), dtype=torch.bfloat16, device=dev)
        elif q is not None:
            _wants(q, "q", torch.bfloat16, dev, (T, n_q * dim), rows=True)
        if bad is not None:
            _wants(bad, "bad", torch.int32, dev, (1,))
        self.cache, self.qkv, self.slots, self.positions, self.cos, self.sin, self.q, self.bad = cache, qkv, slots, positions, cos, sin, q, bad
        self.desc = KVTokensDesc(cache.desc, _ptr(qkv), _row_stride(qkv), 0 if q is None else _row_stride(q), T,
                                 0 if cos is None else cos.shape[0], BL_KV_FROM_F32 if qkv.dtype == torch.float32 else BL_KV_FROM_BF16, n_q,
                                 *(_ptr(t) for t in (positions, slots, cos, sin, q, bad)))


class KVNormAppend(KVAppend):
    """KVAppend with an RMS norm of every Q and K head in front of the rotation (bl_kv_append_norm).  q_gain, k_gain: fp32 [head_dim] or None."""
    _which, _where = 5, "bl_kv_append_norm"

    def __init__(self, cache, qkv, n_q, slots, positions=None, cos=None, sin=None, q=None, bad=None, q_gain=None, k_gain=None, eps=1e-5):
        super().__init__(cache, qkv, n_q, slots, positions, cos, sin, q, bad)
        for t, name in ((q_gain, "q_gain"), (k_gain, "k_gain")):
            if t is not None:
                _wants(t, name, _get_torch().float32, cache.k.device, (cache.head_dim,))
        self.q_gain, self.k_gain = q_gain, k_gain
        self.desc = KVNormTokensDesc(self.desc, _ptr(q_gain), _ptr(k_gain), eps)


class KVAttention(_KVCall):
    """Causal attention over the cache (bl_attn_kv8).  q bf16 [T][n_q][head_dim] (or [T][n_q * head_dim] with n_q); q_start int32 [B + 1],
    seq_len int32 [B], table int32 [B][max_blocks].  max_q: no request has more queries (None: all T rows may be one request's; rows of
    one that has more may be NaN);
    max_len: about the longest length.  Output: out bf16 [T][n_q * head_dim].  The workspace may serve several handles whose runs
    follow each other on one stream."""
    _which, _where = 2, "bl_attn_kv8"

    def __init__(self, cache, q, q_start, seq_len, table, n_q=None, max_q=None, max_len=0, softmax_scale=None, window=0, out=None, workspace=None):
        torch = _get_torch()
        dev, dim, T, B = cache.k.device, cache.head_dim, q.shape[0], seq_len.shape[0]
        n_q = q.shape[1] if n_q is None else n_q
        _wants(q, "q", torch.bfloat16, dev, (T, n_q, dim) if q.dim() == 3 else (T, n_q * dim), rows=True)
        _wants(q_start, "q_start", torch.int32, dev, (B + 1,))
        _wants(seq_len, "seq_len", torch.int32, dev, (B,))
        _wants(table, "table", torch.int32, dev, (B, None), rows=True)
        if out is None:
            out = torch.empty((T, n_q * dim), dtype=torch.bfloat16, device=dev)
        else:
            _wants(out, "out", torch.bfloat16, dev, (T, n_q * dim), rows=True)
        self.cache, self.q, self.q_start, self.seq_len, self.table, self.out = cache, q, q_start, seq_len, table, out
        self.desc = AttnDesc(cache.desc, _ptr(q), _row_stride(q), _row_stride(out), _row_stride(table), B, T, _ptr(q_start), _ptr(seq_len),
                             _ptr(table), n_q, table.shape[1], T if max_q is None else max_q, max_len, window, dim ** -0.5 if softmax_scale is None else softmax_scale,
                             _ptr(out), None)
        self._space(workspace, dev)

    def _space(self, workspace, dev):
        self.workspace = _space_of(load().bl_attn_workspace_bytes(ctypes.byref(self.desc)), workspace, dev)
        self.desc.workspace = _ptr(self.workspace)


def _space_of(nbytes, workspace, dev):
    """A workspace of nbytes: the caller's, if it is large enough, or a new one."""
    if workspace is None:
        return _workspace(nbytes, dev)
    if _wants(workspace, "workspace", _get_torch().uint8, dev).numel() < nbytes:
        raise ValueError("workspace of %d bytes, %d are needed" % (workspace.numel(), nbytes))
    return workspace


class KVSharedAttention(KVAttention):
    """KVAttention where requests share prefixes, each read once for all of its requests (bl_attn_kv8_shared).  group: int32 [B], the group of
    each request (outside 0 .. n_groups - 1: none); shared_table int32 [n_groups][max_shared], shared_blocks int32 [n_groups]: the blocks of a
    group's prefix.  max_own: about the most tokens of a request behind its prefix.  max_q decides what shares a read, so it is worth giving (None: as if one request
    brought all rows; from 128 rows of n_q / n_kv heads on only requests of up to 16 rows share).  Everything else is KVAttention's."""
    _which, _where = 6, "bl_attn_kv8_shared"

    def __init__(self, cache, q, q_start, seq_len, table, group, shared_table, shared_blocks, n_q=None, max_q=None, max_len=0, max_own=0,
                 softmax_scale=None, window=0, out=None, workspace=None):
        i32, dev = _get_torch().int32, cache.k.device
        _wants(group, "group", i32, dev, (seq_len.shape[0],))
        _wants(shared_table, "shared_table", i32, dev, (None, None), rows=True)
        _wants(shared_blocks, "shared_blocks", i32, dev, (shared_table.shape[0],))
        self.group, self.shared_table, self.shared_blocks, self.max_own = group, shared_table, shared_blocks, max_own
        super().__init__(cache, q, q_start, seq_len, table, n_q, max_q, max_len, softmax_scale, window, out, workspace)

    def _space(self, workspace, dev):
        t = self.shared_table
        self.desc = AttnSharedDesc(self.desc, _ptr(self.group), _ptr(self.shared_blocks), _ptr(t), _row_stride(t), t.shape[0], t.shape[1], self.max_own)
        self.workspace = _space_of(load().bl_attn_shared_workspace_bytes(ctypes.byref(self.desc)), workspace, dev)
        self.desc.attn.workspace = _ptr(self.workspace)


class F8Matrix:
    """A matrix of 8-bit floating point codes (bl_f8_matrix): codes float8_e4m3fn [N][K] (rows may lie apart), scale fp32
    [ceil(N / 128)][ceil(K / 128)], one for each block of 128 x 128."""

    def __init__(self, codes, scale):
        torch = _get_torch()
        if codes.dim() != 2:
            raise ValueError("codes must be [N][K]")
        N, K = codes.shape
        _wants(codes, "codes", torch.float8_e4m3fn, codes.device, rows=True)
        _wants(scale, "scale", torch.float32, codes.device, (-(-N // 128), -(-K // 128)), rows=True)
        self.codes, self.scale, self.N, self.K = codes, scale, N, K
        self.desc = F8MatrixDesc(_ptr(codes), _ptr(scale), N, K, _row_stride(codes), _row_stride(scale))

    @classmethod
    def quantise(cls, W):
        """Codes and scales of a matrix of numbers, once when a model is loaded: a block's scale is its largest |value| / 448."""
        torch = _get_torch()
        N, K = W.shape
        high, wide = -(-N // 128), -(-K // 128)
        codes = torch.empty((N, K), dtype=torch.float8_e4m3fn, device=W.device)
        scale = torch.empty((high, wide), dtype=torch.float32, device=W.device)
        for i in range(0, high, 64):                             # (a vocabulary's matrix in 32 bits is not made whole)
            part = W[128 * i:128 * (i + 64)].float()
            rows = -(-part.shape[0] // 128)
            x = torch.zeros((rows * 128, wide * 128), dtype=torch.float32, device=W.device)
            x[:part.shape[0], :K] = part
            x = x.view(rows, 128, wide, 128)
            s = x.abs().amax((1, 3), keepdim=True).clamp(min=1e-12) / 448.0
            codes[128 * i:128 * i + part.shape[0]] = (x / s).clamp(-448.0, 448.0).view(rows * 128, wide * 128)[:part.shape[0], :K].to(codes.dtype)
            scale[i:i + rows] = s[:, 0, :, 0]
        return cls(codes, scale)


def _f8_kind(dtype):
    torch = _get_torch()
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("outputs are float32 or bfloat16, not %s" % dtype)
    return BL_F8_OUT_F32 if dtype == torch.float32 else BL_F8_OUT_BF16


class F8Linear(_KVCall):
    """y = rows times the matrix's transpose (bl_f8_linear).  x: bf16 or fp32 [M][K], with norm=True normalised on the way (gain fp32 [K] or
    None); or prod, a producer of make_producer whose tensors have M rows at least, and M.  Output: y [M][N] of `dtype` (or of y's).  The workspace
    may serve several handles whose runs follow each other on one stream."""
    _which, _where = 7, "bl_f8_linear"

    def __init__(self, matrix, x=None, y=None, dtype=None, norm=False, gain=None, eps=1e-5, workspace=None, prod=None, M=None):
        torch = _get_torch()
        dev = matrix.codes.device
        if (x is None) == (prod is None) or (prod is None) != (M is None):
            raise ValueError("x, or prod and M")
        if x is not None:
            if x.dtype not in (torch.float32, torch.bfloat16):
                raise TypeError("x must be float32 or bfloat16")
            _wants(x, "x", x.dtype, dev, (None, matrix.K))
            if gain is not None:
                _wants(gain, "gain", torch.float32, dev, (matrix.K,))
            M = x.shape[0]
            prod = make_producer(BL_PROD_F32 if x.dtype == torch.float32 else BL_PROD_BF16, x, norm=norm, gain=gain, eps=eps)
        else:
            _wants_producer(prod, M, matrix.K, dev)
        if y is None:
            y = torch.empty((M, matrix.N), dtype=torch.float32 if dtype is None else dtype, device=dev)
        else:
            _wants(y, "y", y.dtype if dtype is None else dtype, dev, (M, matrix.N), rows=True)
        self.matrix, self.prod, self.y = matrix, prod, y
        self.desc = F8ProductDesc(matrix.desc, prod, M, _row_stride(y), _ptr(y), _f8_kind(y.dtype), None)
        self.workspace = _space_of(load().bl_f8_workspace_bytes(ctypes.byref(self.desc)), workspace, dev)
        self.desc.workspace = _ptr(self.workspace)


class F8Embedding(_KVCall):
    """Rows of the matrix times a number (bl_f8_embed).  ids: int32 [T]; those outside the matrix give zeros, and but for -1 are counted in bad
    (int32 [1] or None).  Output: out [T][K] of `dtype` (or of out's)."""
    _which, _where = 8, "bl_f8_embed"

    def __init__(self, matrix, ids, out=None, dtype=None, multiplier=1.0, bad=None):
        torch = _get_torch()
        dev = matrix.codes.device
        _wants(ids, "ids", torch.int32, dev, (None,))
        if out is None:
            out = torch.empty((ids.shape[0], matrix.K), dtype=torch.float32 if dtype is None else dtype, device=dev)
        else:
            _wants(out, "out", out.dtype if dtype is None else dtype, dev, (ids.shape[0], matrix.K), rows=True)
        if bad is not None:
            _wants(bad, "bad", torch.int32, dev, (1,))
        self.matrix, self.ids, self.out, self.bad = matrix, ids, out, bad
        self.desc = F8LookupDesc(matrix.desc, _ptr(ids), ids.shape[0], _row_stride(out), _ptr(out), _f8_kind(out.dtype), multiplier, _ptr(bad))
