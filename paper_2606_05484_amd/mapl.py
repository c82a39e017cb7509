"""ctypes binding of libmapl (include/mapl.h): argument marshalling only.

Every entry point takes device pointers -- torch tensors (their data_ptr()),
plain integers, or None -- and the HIP stream to enqueue on (default: torch's
current stream on the current device).  All computation happens in the HIP
kernels of libmapl.so; this module never computes a result itself and raises
MaplError when the library is missing or a call fails.
"""
import ctypes
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmapl.so")

MAPL_OK = 0
STATUS = {0: "MAPL_OK", -1: "MAPL_E_NULL", -2: "MAPL_E_SHAPE", -3: "MAPL_E_DTYPE", -4: "MAPL_E_RANGE",
          -5: "MAPL_E_ALIGN", -6: "MAPL_E_ALIAS", -7: "MAPL_E_WORKSPACE", -8: "MAPL_E_UNSUPPORTED",
          -9: "MAPL_E_HIP"}
F32, BF16, U8, U16 = 0, 1, 2, 3
AMBIENT, COORD = 0, 1
CALL_ENCODE, CALL_DECODE, CALL_DECODE_BWD, CALL_ENCODE_BWD, CALL_STIEFEL = range(5)
SENDER, RECEIVER = 0, 1
XENT_FWD, XENT_BWD = 0, 1
NORM_PRE, NORM_BRANCH, NORM_POST = 1, 2, 4
STATES_F32, STATES_8BIT = 0, 1
_DT = {"f32": F32, "bf16": BF16, "u8": U8, "u16": U16}
_SPACE = {"ambient": AMBIENT, "coord": COORD}
_GATE = {"none": 0, "sigmoid": 1, "silu": 2}
_STATES = {"f32": STATES_F32, "8bit": STATES_8BIT}


class MaplError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("%s (%d): %s" % (STATUS.get(status, "?"), status, message))
        self.status = status


class CodecDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("d", ctypes.c_int64), ("r", ctypes.c_int64), ("V", ctypes.c_int64),
                ("k", ctypes.c_int64), ("anchor_space", ctypes.c_int32), ("L", ctypes.c_int32),
                ("K", ctypes.c_int32), ("x_dtype", ctypes.c_int32), ("ab_dtype", ctypes.c_int32),
                ("code_dtype", ctypes.c_int32), ("group_dim", ctypes.c_int32)]


class XentDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("d", ctypes.c_int64), ("V", ctypes.c_int64), ("x_dtype", ctypes.c_int32),
                ("dw_dtype", ctypes.c_int32)]


class NormDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("d", ctypes.c_int64), ("ld_h", ctypes.c_int64), ("ld_gate", ctypes.c_int64),
                ("x_dtype", ctypes.c_int32), ("h_dtype", ctypes.c_int32), ("parts", ctypes.c_int32),
                ("gate", ctypes.c_int32), ("alpha", ctypes.c_float), ("eps", ctypes.c_float)]


class Param(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("g", ctypes.c_void_p), ("p", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("e", ctypes.c_void_p), ("p16", ctypes.c_void_p),
                ("weight_decay", ctypes.c_float), ("lr_scale", ctypes.c_float)]


class AdamwDesc(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("eps", ctypes.c_float),
                ("g_dtype", ctypes.c_int32), ("states", ctypes.c_int32), ("step", ctypes.c_int32),
                ("seed", ctypes.c_uint32)]


_lib = None
_P = ctypes.c_void_p
_SIG = {
    "mapl_encode": [ctypes.POINTER(CodecDesc)] + [_P] * 7 + [_P, ctypes.c_size_t, _P],
    "mapl_encode_noalloc": [ctypes.POINTER(CodecDesc)] + [_P] * 7 + [_P],
    "mapl_codebook_pack": [ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, _P, _P, ctypes.c_int32, _P, _P],
    "mapl_codebook_unpack": [ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, _P, _P, ctypes.c_int32, _P, _P],
    "mapl_decode": [ctypes.POINTER(CodecDesc)] + [_P] * 7 + [_P, ctypes.c_size_t, _P],
    "mapl_decode_bwd": [ctypes.POINTER(CodecDesc)] + [_P] * 9 + [ctypes.c_int, _P, ctypes.c_size_t, _P],
    "mapl_encode_bwd": [ctypes.POINTER(CodecDesc)] + [_P] * 8 + [ctypes.c_int, _P, ctypes.c_size_t, _P],
    "mapl_decode_bwd_q": [ctypes.POINTER(CodecDesc)] + [_P] * 7 + [ctypes.c_int32] * 3 + [_P] * 3 +
                         [ctypes.c_int, _P, ctypes.c_size_t, _P],
    "mapl_decode_bwd_q_workspace_bytes": [ctypes.POINTER(CodecDesc), ctypes.c_int32, ctypes.c_int32],
    "mapl_anchor_bwd": [ctypes.POINTER(CodecDesc), ctypes.c_int] + [_P] * 5 + [ctypes.c_int, _P, ctypes.c_size_t,
                                                                              _P],
    "mapl_anchor_bwd_workspace_bytes": [ctypes.POINTER(CodecDesc), ctypes.c_int],
    "mapl_grad_dequantize": [ctypes.c_int64, ctypes.c_int64] + [ctypes.c_int32] * 3 + [_P, _P, ctypes.c_int32,
                                                                                        _P, _P],
    "mapl_ckpt_pack": [ctypes.c_int64, ctypes.c_int64, ctypes.c_int32] + [_P] * 4,
    "mapl_ckpt_unpack": [ctypes.c_int64, ctypes.c_int64, ctypes.c_int32] + [_P] * 4,
    "mapl_ckpt_encode_bwd": [ctypes.POINTER(CodecDesc)] + [_P] * 9 + [ctypes.c_int, _P, ctypes.c_size_t, _P],
    "mapl_ckpt_encode_bwd_workspace_bytes": [ctypes.POINTER(CodecDesc)],
    "mapl_xent_fwd": [ctypes.POINTER(XentDesc)] + [_P] * 5 + [_P, ctypes.c_size_t, _P],
    "mapl_xent_bwd": [ctypes.POINTER(XentDesc)] + [_P] * 5 + [ctypes.c_float] + [_P] * 2 + [ctypes.c_int, _P,
                                                                                          ctypes.c_size_t, _P],
    "mapl_xent_workspace_bytes": [ctypes.POINTER(XentDesc), ctypes.c_int],
    "mapl_norm_fwd": [ctypes.POINTER(NormDesc)] + [_P] * 9,
    "mapl_norm_bwd": [ctypes.POINTER(NormDesc)] + [_P] * 14 + [ctypes.c_int, _P, ctypes.c_size_t, _P],
    "mapl_norm_workspace_bytes": [ctypes.POINTER(NormDesc)],
    "mapl_grad_norm": [_P, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_float, _P, _P, _P, ctypes.c_size_t,
                       _P],
    "mapl_grad_norm_workspace_bytes": [_P, ctypes.c_int64, ctypes.c_int32],
    "mapl_adamw_step": [ctypes.POINTER(AdamwDesc), _P, ctypes.c_int64] + [_P] * 4,
    "mapl_adamw_unpack": [_P, _P, ctypes.c_int64, _P],
    "mapl_adamw_pack": [_P, _P, ctypes.c_int64, _P],
    "mapl_stiefel_step": [ctypes.c_int64] * 3 + [_P] * 3 + [ctypes.c_float, ctypes.c_float, ctypes.c_int,
                                                            ctypes.c_int, _P, ctypes.c_size_t, _P],
    "mapl_workspace_bytes": [ctypes.POINTER(CodecDesc), ctypes.c_int, ctypes.c_int64, ctypes.c_int64,
                             ctypes.c_int64],
    "mapl_last_error": [],
    "mapl_version": [],
    "mapl_profile": [ctypes.c_int],
    "mapl_profile_report": [ctypes.c_char_p, ctypes.c_size_t],
}
_RES = {"mapl_workspace_bytes": ctypes.c_size_t, "mapl_decode_bwd_q_workspace_bytes": ctypes.c_size_t,
        "mapl_anchor_bwd_workspace_bytes": ctypes.c_size_t, "mapl_ckpt_encode_bwd_workspace_bytes": ctypes.c_size_t,
        "mapl_xent_workspace_bytes": ctypes.c_size_t, "mapl_norm_workspace_bytes": ctypes.c_size_t,
        "mapl_grad_norm_workspace_bytes": ctypes.c_size_t,
        "mapl_last_error": ctypes.c_char_p}
EXPORTS = tuple(_SIG)


def lib():
    """Load libmapl.so (built in-tree by paper_2606_05484_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MaplError(-8, "libmapl.so not built at %s (run paper_2606_05484_amd.build)" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        for name, args in _SIG.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = _RES.get(name, ctypes.c_int)
        _lib = L
    return _lib


def last_error():
    return lib().mapl_last_error().decode()


def _check(status):
    if status != MAPL_OK:
        raise MaplError(status, last_error())


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _ptrs(*xs):
    """_ptr of several, without a Python call for each (0.04 to 0.15 us instead of 0.2 to 0.4)."""
    return [x if x is None or isinstance(x, int) else x.data_ptr() for x in xs]


_current = None  # torch's current raw stream, a function (torch is imported with the first use)


def _current_stream():
    global _current
    import torch
    raw = torch.cuda.current_stream().cuda_stream  # initialises the device
    C = torch._C
    if hasattr(C, "_cuda_getCurrentRawStream") and hasattr(C, "_cuda_getDevice"):
        # without a Stream object: 2 us less a call, a third of what a small call takes on the host
        _current = lambda: C._cuda_getCurrentRawStream(C._cuda_getDevice())
    else:
        _current = lambda: torch.cuda.current_stream().cuda_stream
    return raw


def _stream(stream):
    if stream is None:
        return _current() if _current is not None else _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def desc(T, d, r, V=0, k=0, L=0, K=0, x_dtype="bf16", anchor_space="ambient", code_dtype=None, group_dim=0):
    """Build a mapl_codec_desc; code_dtype defaults to u8 for K <= 256, else u16."""
    if code_dtype is None:
        code_dtype = "u8" if K <= 256 else "u16"
    dt = _DT[x_dtype] if isinstance(x_dtype, str) else x_dtype
    return CodecDesc(T, d, r, V, k, _SPACE[anchor_space] if isinstance(anchor_space, str) else anchor_space,
                     L, K, dt, dt, _DT[code_dtype] if isinstance(code_dtype, str) else code_dtype, group_dim)


def payload_bytes_per_token(D):
    """Bytes that cross the pipeline link per token (ids excluded)."""
    if D.L == 0:
        return D.r * (4 if D.x_dtype == F32 else 2)
    if D.group_dim == 2:
        return D.L * (D.r // 2)
    return D.L * (1 if D.code_dtype == U8 else 2)


def workspace_bytes(D, call, P=0, d=0, r=0):
    n = lib().mapl_workspace_bytes(ctypes.byref(D) if D is not None else None, call, P, d, r)
    if n == 0 and last_error():
        raise MaplError(-2, last_error())
    return n


def workspace(nbytes, device=None):
    """A device byte buffer for the workspace (torch's allocator aligns to 512 B)."""
    import torch
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device or "cuda")


def encode(D, X, ids, U, A_s, B_s, C, payload, ws, ws_bytes=None, stream=None):
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_encode(ctypes.byref(D), _ptr(X), _ptr(ids), _ptr(U), _ptr(A_s), _ptr(B_s), _ptr(C),
                             _ptr(payload), _ptr(ws), wb, _stream(stream)))


def encode_noalloc(D, X, ids, U, A_s, B_s, C, payload, stream=None):
    """mapl_encode on the library's static device scratch (no workspace)."""
    _check(lib().mapl_encode_noalloc(ctypes.byref(D), _ptr(X), _ptr(ids), _ptr(U), _ptr(A_s), _ptr(B_s), _ptr(C),
                                     _ptr(payload), _stream(stream)))


NOALLOC_SCRATCH_BYTES = 16 << 20


def decode(D, payload, ids, U, A_r, B_r, C, Xhat, ws, ws_bytes=None, stream=None):
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_decode(ctypes.byref(D), _ptr(payload), _ptr(ids), _ptr(U), _ptr(A_r), _ptr(B_r), _ptr(C),
                             _ptr(Xhat), _ptr(ws), wb, _stream(stream)))


def decode_bwd(D, dXhat, payload, ids, U, A_r, B_r, C, dZ, dU, accumulate_dU, ws, ws_bytes=None, stream=None):
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_decode_bwd(ctypes.byref(D), _ptr(dXhat), _ptr(payload), _ptr(ids), _ptr(U), _ptr(A_r),
                                 _ptr(B_r), _ptr(C), _ptr(dZ), _ptr(dU), int(accumulate_dU), _ptr(ws), wb,
                                 _stream(stream)))


def decode_bwd_q(D, dXhat, payload, ids, U, A_r, B_r, C, Lg, Kg, Cg, gcodes, dU, accumulate_dU, ws,
                 ws_bytes=None, stream=None, gcode_dtype=None):
    """decode_bwd with the returned gradient RVQ-encoded into gcodes [T,Lg]."""
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    gdt = (U8 if Kg <= 256 else U16) if gcode_dtype is None else _DT.get(gcode_dtype, gcode_dtype)
    _check(lib().mapl_decode_bwd_q(ctypes.byref(D), _ptr(dXhat), _ptr(payload), _ptr(ids), _ptr(U), _ptr(A_r),
                                   _ptr(B_r), _ptr(C), Lg, Kg, gdt, _ptr(Cg), _ptr(gcodes), _ptr(dU),
                                   int(accumulate_dU), _ptr(ws), wb, _stream(stream)))


def decode_bwd_q_workspace_bytes(D, Lg, Kg):
    n = lib().mapl_decode_bwd_q_workspace_bytes(ctypes.byref(D), Lg, Kg)
    if n == 0 and last_error():
        raise MaplError(-2, last_error())
    return n


def anchor_bwd(D, side, dY, ids, U, B, dA, accumulate, ws, ws_bytes=None, stream=None):
    """Gradient of the sender's (side 0) or receiver's (side 1) anchor table."""
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_anchor_bwd(ctypes.byref(D), int(side), _ptr(dY), _ptr(ids), _ptr(U), _ptr(B), _ptr(dA),
                                 int(accumulate), _ptr(ws), wb, _stream(stream)))


def anchor_bwd_workspace_bytes(D, side):
    n = lib().mapl_anchor_bwd_workspace_bytes(ctypes.byref(D), int(side))
    if n == 0 and last_error():
        raise MaplError(-2, last_error())
    return n


def grad_dequantize(T, r, Lg, Kg, gcodes, Cg, dZ, out_dtype="bf16", stream=None, gcode_dtype=None):
    """dZ[t] = sum_l Cg[l, gcodes[t, l]] as bf16 or fp32."""
    gdt = (U8 if Kg <= 256 else U16) if gcode_dtype is None else _DT.get(gcode_dtype, gcode_dtype)
    _check(lib().mapl_grad_dequantize(T, r, Lg, Kg, gdt, _ptr(gcodes), _ptr(Cg), _DT.get(out_dtype, out_dtype),
                                      _ptr(dZ), _stream(stream)))


def encode_bwd(D, dZ, X, ids, U, A_s, B_s, dX, dU, accumulate_dU, ws, ws_bytes=None, stream=None):
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_encode_bwd(ctypes.byref(D), _ptr(dZ), _ptr(X), _ptr(ids), _ptr(U), _ptr(A_s), _ptr(B_s),
                                 _ptr(dX), _ptr(dU), int(accumulate_dU), _ptr(ws), wb, _stream(stream)))


CKPT_BLOCK = 32  # tokens of one channel that share a scale


def ckpt_shapes(T, d):
    """Shapes of a checkpoint's int8 values and uint8 exponents."""
    nb = -(-T // CKPT_BLOCK)
    return (nb, d, CKPT_BLOCK), (nb, d)


def ckpt_pack(T, d, X, q, e, x_dtype="bf16", stream=None):
    """Keep X [T, d] in 8 bits: q int8 and e uint8 of ckpt_shapes(T, d)."""
    _check(lib().mapl_ckpt_pack(T, d, _DT.get(x_dtype, x_dtype), _ptr(X), _ptr(q), _ptr(e), _stream(stream)))


def ckpt_unpack(T, d, q, e, X, x_dtype="bf16", stream=None):
    """The values that a checkpoint stands for."""
    _check(lib().mapl_ckpt_unpack(T, d, _DT.get(x_dtype, x_dtype), _ptr(q), _ptr(e), _ptr(X), _stream(stream)))


def ckpt_encode_bwd(D, dZ, q, e, ids, U, A_s, B_s, dX, dU, accumulate_dU, ws, ws_bytes=None, stream=None):
    """encode_bwd with X read from its 8-bit checkpoint."""
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_ckpt_encode_bwd(ctypes.byref(D), _ptr(dZ), _ptr(q), _ptr(e), _ptr(ids), _ptr(U), _ptr(A_s),
                                      _ptr(B_s), _ptr(dX), _ptr(dU), int(accumulate_dU), _ptr(ws), wb,
                                      _stream(stream)))


def ckpt_encode_bwd_workspace_bytes(D):
    n = lib().mapl_ckpt_encode_bwd_workspace_bytes(ctypes.byref(D))
    if n == 0 and last_error():
        raise MaplError(-2, last_error())
    return n


def xent_desc(T, d, V, x_dtype="bf16", dw_dtype="f32"):
    """Build a mapl_xent_desc (dw_dtype: the type of dW)."""
    return XentDesc(T, d, V, _DT.get(x_dtype, x_dtype), _DT.get(dw_dtype, dw_dtype))


def xent_workspace_bytes(D, call):
    n = lib().mapl_xent_workspace_bytes(ctypes.byref(D), call)
    if n == 0 and last_error():
        raise MaplError(-2, last_error())
    return n


def xent_fwd(D, H, W, targets, loss, lse, ws, ws_bytes=None, stream=None):
    """Cross entropy of the logits H W^T: loss and log-sum-exp of every token."""
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_xent_fwd(ctypes.byref(D), _ptr(H), _ptr(W), _ptr(targets), _ptr(loss), _ptr(lse), _ptr(ws), wb,
                               _stream(stream)))


def xent_bwd(D, H, W, targets, lse, weight, scale, dH, dW, accumulate_dW, ws, ws_bytes=None, stream=None):
    """Its gradient: dH, and dW (added to with accumulate_dW); either may be None."""
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_xent_bwd(ctypes.byref(D), _ptr(H), _ptr(W), _ptr(targets), _ptr(lse), _ptr(weight), float(scale),
                               _ptr(dH), _ptr(dW), int(accumulate_dW), _ptr(ws), wb, _stream(stream)))


def norm_desc(T, d, x_dtype="bf16", h_dtype=None, branch=False, post=False, pre=True, gate="none", alpha=1.0, eps=1e-5,
              ld_h=0, ld_gate=0):
    """Build a mapl_norm_desc: pre (a norm in front of a block), branch (a block's output added to the
    residual stream, with post after a norm of its own), or both; h_dtype defaults to x_dtype."""
    parts = NORM_PRE * bool(pre) | NORM_BRANCH * bool(branch) | NORM_POST * bool(post)
    h_dtype = x_dtype if h_dtype is None else h_dtype
    return NormDesc(T, d, ld_h, ld_gate, _DT.get(x_dtype, x_dtype), _DT.get(h_dtype, h_dtype), parts,
                    _GATE.get(gate, gate), alpha, eps)


def norm_workspace_bytes(D):
    """Bytes that norm_bwd needs."""
    n = lib().mapl_norm_workspace_bytes(ctypes.byref(D))
    if n == 0 and last_error():
        raise MaplError(-2, last_error())
    return n


def norm_fwd(D, x, h, gate, w_post, scale, w_pre, xo, y, stream=None):
    """xo = x + alpha scale rms(h) w_post act(gate), y = rms(xo) w_pre; what D leaves out is None."""
    _check(lib().mapl_norm_fwd(ctypes.byref(D), *_ptrs(x, h, gate, w_post, scale, w_pre, xo, y), _stream(stream)))


def norm_bwd(D, dy, dxo, xo, h, gate, w_post, scale, w_pre, dx, dh, dgate, dw_post, dscale, dw_pre, accumulate_dw, ws,
             ws_bytes=None, stream=None):
    """Its gradient; the vectors' (any may be None) are added to with accumulate_dw."""
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_norm_bwd(ctypes.byref(D), *_ptrs(dy, dxo, xo, h, gate, w_post, scale, w_pre, dx, dh, dgate, dw_post,
                                                       dscale, dw_pre), int(accumulate_dw), _ptr(ws), wb, _stream(stream)))


def _type_name(t):
    """The name that _DT gives a tensor's type ("u8" for any of one byte), or torch's."""
    if t.element_size() == 1:
        return "u8"
    name = str(t.dtype)
    return {"torch.float32": "f32", "torch.bfloat16": "bf16"}.get(name, name)


class OptimParams:
    """A host array of mapl_param and the tensors that it points to (kept alive with it);
    types: the type of each kind that is given (_type_name), which the calls look at."""

    def __init__(self, array, count, tensors, types=None):
        self.array, self.count, self.tensors, self.types = array, count, tensors, types or {}
        self.seen = set()

    def need(self, *types):
        """Looks once whether the arrays have values of these types: (name, type) each."""
        if types in self.seen:
            return
        for name, want in types:
            if self.types.get(name, want) != want:
                raise ValueError("%s has values of type %s, this call takes %s" % (name, self.types[name], want))
        self.seen.add(types)


def optim_params(g, p=None, m=None, v=None, e=None, p16=None, weight_decay=0.0, lr_scale=1.0):
    """The tensors of an optimizer step: sequences of equal length (e, p16 and what a call does not
    use may be None); weight_decay and lr_scale are numbers or sequences of them."""
    count = len(g)
    lists = {name: None if x is None else tuple(x)  # (the caller's own lists may change)
             for name, x in (("g", g), ("p", p), ("m", m), ("v", v), ("e", e), ("p16", p16))}
    each = lambda x: list(x) if hasattr(x, "__len__") else [x] * count
    decay, lr = each(weight_decay), each(lr_scale)
    for name, x in list(lists.items()) + [("weight_decay", decay), ("lr_scale", lr)]:
        if x is not None and len(x) != count:
            raise ValueError("%s has %d entries, g %d" % (name, len(x), count))
    sizes = [t.numel() for t in lists["g"]]
    where, types = {}, {}
    for name, x in lists.items():
        if x is None:
            where[name] = [0] * count
            continue
        last = None
        for i, t in enumerate(x):
            if t is None:
                continue
            if t.dtype is not last:
                last, kind = t.dtype, _type_name(t)
                if types.setdefault(name, kind) != kind:
                    raise ValueError("%s has values of type %s and %s" % (name, types[name], kind))
            if not t.is_contiguous():
                raise ValueError("%s[%d] is not contiguous" % (name, i))
            if name == "e":
                if t.numel() < optim_exponents(sizes[i]):
                    raise ValueError("e[%d] has %d bytes, %d needed" % (i, t.numel(), optim_exponents(sizes[i])))
            elif t.numel() != sizes[i]:
                raise ValueError("%s[%d] has %d values, g[%d] %d" % (name, i, t.numel(), i, sizes[i]))
        where[name] = [0 if t is None else t.data_ptr() for t in x]
    a = (Param * count)()
    one = struct.Struct("=q6Q2f")  # Param's layout
    for i, row in enumerate(zip(sizes, *(where[name] for name, _ in Param._fields_[1:7]), decay, lr)):
        one.pack_into(a, i * one.size, *row)
    return OptimParams(a, count, lists, types)


def optim_exponents(n):
    """Exponent bytes of the 8-bit states of n values."""
    return -(-n // 128) * 2


def grad_norm_workspace_bytes(params, g_dtype="f32"):
    n = lib().mapl_grad_norm_workspace_bytes(params.array, params.count, _DT.get(g_dtype, g_dtype))
    if n == 0 and last_error():
        raise MaplError(-2, last_error())
    return n


def grad_norm(params, stats, ws, step=None, grad_scale=1.0, max_norm=float("inf"), g_dtype="f32", ws_bytes=None, stream=None):
    """stats[0]: the norm of all gradients, stats[1]: the factor that clips them; counts step up if it is finite."""
    params.need(("g", "bf16" if g_dtype in ("bf16", BF16) else "f32"))
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_grad_norm(params.array, params.count, _DT.get(g_dtype, g_dtype), grad_scale, max_norm, _ptr(stats),
                                _ptr(step), _ptr(ws), wb, _stream(stream)))


def adamw_desc(lr, beta1=0.9, beta2=0.95, eps=1e-8, g_dtype="f32", states="f32", step=0, seed=0):
    """Build a mapl_adamw_desc (step: the number of this step, from 1, where no device step is given)."""
    return AdamwDesc(lr, beta1, beta2, eps, _DT.get(g_dtype, g_dtype), _STATES.get(states, states), step, seed)


def adamw_step(A, params, stats=None, step=None, lr=None, stream=None):
    """One step over all of params; stats as grad_norm leaves it, step (int32) and lr (fp32) on the device."""
    state = "u8" if A.states == STATES_8BIT else "f32"
    params.need(("g", "bf16" if A.g_dtype == BF16 else "f32"), ("p", "f32"), ("m", state), ("v", state), ("e", "u8"), ("p16", "bf16"))
    _check(lib().mapl_adamw_step(ctypes.byref(A), params.array, params.count, _ptr(stats), _ptr(step), _ptr(lr),
                                 _stream(stream)))


def adamw_unpack(packed, values, stream=None):
    """The values of 8-bit states, as fp32 m and v."""
    if packed.count != values.count:
        raise ValueError("%d and %d tensors" % (packed.count, values.count))
    packed.need(("m", "u8"), ("v", "u8"), ("e", "u8"))
    values.need(("m", "f32"), ("v", "f32"))
    _check(lib().mapl_adamw_unpack(packed.array, values.array, packed.count, _stream(stream)))


def adamw_pack(values, packed, stream=None):
    """fp32 m and v in 8 bits, rounded to nearest."""
    if packed.count != values.count:
        raise ValueError("%d and %d tensors" % (packed.count, values.count))
    packed.need(("m", "u8"), ("v", "u8"), ("e", "u8"))
    values.need(("m", "f32"), ("v", "f32"))
    _check(lib().mapl_adamw_pack(values.array, packed.array, packed.count, _stream(stream)))


def stiefel_step(P, d, r, U, G, M, lr, beta, lmo_steps, retract_steps, ws, ws_bytes=None, stream=None):
    wb = ws_bytes if ws_bytes is not None else (ws.numel() if ws is not None else 0)
    _check(lib().mapl_stiefel_step(P, d, r, _ptr(U), _ptr(G), _ptr(M), lr, beta, lmo_steps, retract_steps,
                                   _ptr(ws), wb, _stream(stream)))


def codebook_pack(L, K, r, C, rows, n, buf, stream=None):
    """Sender side of the streaming codebook sync: buf[l, i] = C[l, rows[l, i]]."""
    _check(lib().mapl_codebook_pack(L, K, r, _ptr(C), _ptr(rows), n, _ptr(buf), _stream(stream)))


def codebook_unpack(L, K, r, buf, rows, n, C, stream=None):
    """Receiver side: C[l, rows[l, i]] = buf[l, i]."""
    _check(lib().mapl_codebook_unpack(L, K, r, _ptr(buf), _ptr(rows), n, _ptr(C), _stream(stream)))


def profile(enable):
    """Per-kernel event tracing: 0 off, 1 (True) on, 2 also RVQ decision
    counters (see mapl_profile_report)."""
    _check(lib().mapl_profile(int(enable)))


def profile_report():
    """{kernel name: (launches, total_ms)} for the launches since the last report."""
    buf = ctypes.create_string_buffer(1 << 16)
    _check(lib().mapl_profile_report(buf, len(buf)))
    out = {}
    for line in buf.value.decode().splitlines():
        name, n, ms = line.split()
        out[name] = (int(n), float(ms))
    return out
