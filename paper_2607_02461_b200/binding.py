"""Thin ctypes binding of liboq.so: same names as the C entry points, argument marshalling only.

Device buffers are torch CUDA tensors (torch owns memory and streams); every step of the path runs in
the library's kernels.  There is no fallback: if liboq.so is missing or a call fails, OqError is raised.
"""
import ctypes as C
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "liboq.so")
_lib = None

OQ_BF16, OQ_F32 = 0, 1
_INT_MAX = 2 ** 31 - 1
STATUS_NAMES = {0: "OQ_OK", 1: "OQ_ERR_INVALID_ARG", 2: "OQ_ERR_UNSUPPORTED", 3: "OQ_ERR_ALIGNMENT",
                4: "OQ_ERR_CUDA", 5: "OQ_ERR_DEVICE_TIMEOUT", 6: "OQ_ERR_NOMEM"}


class OqError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


def lib():
    """Loads liboq.so (built in-tree by paper_2607_02461_b200.build); fails loudly when absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise OqError(4, f"{_LIB_PATH} not found: run `python -m paper_2607_02461_b200.build`")
        L = C.CDLL(_LIB_PATH)
        vp, i, u64, sz = C.c_void_p, C.c_int, C.c_uint64, C.c_size_t
        pp = C.POINTER(C.c_void_p)
        sig = {
            "oq_build_codebook": (i, [i, i, pp]),
            "oq_codebook_get": (i, [vp, vp, vp, vp, vp]),
            "oq_codebook_dim": (i, [vp]), "oq_codebook_bits": (i, [vp]), "oq_codebook_destroy": (None, [vp]),
            "oq_make_rpbh": (i, [i, i, u64, pp]),
            "oq_rpbh_get": (i, [vp, vp, vp]),
            "oq_rpbh_dim": (i, [vp]), "oq_rpbh_block": (i, [vp]), "oq_rpbh_destroy": (None, [vp]),
            "oq_packed_bytes": (i, [i, i, i, C.POINTER(sz), C.POINTER(sz)]),
            "oq_rotate_quantize_act": (i, [vp, i, i, i, vp, vp, vp, vp, vp, vp]),
            "oq_quantize_weights": (i, [vp, i, i, i, vp, vp, vp, vp, vp, vp]),
            "oq_qlinear": (i, [vp, vp, i, vp, vp, vp, i, vp, i, vp, i, i, vp]),
            "oq_unpack_indices": (i, [vp, i, i, i, vp, vp]),
            "oq_linear_forward_noalloc": (i, [vp, i, i, i, vp, vp, vp, vp, i, vp, vp, i, i, vp]),
            "oq_forward_workspace_bytes": (i, [i, i, i, i, C.POINTER(sz)]),
            "oq_linear_forward_host": (i, [vp, i, i, vp, vp, vp, vp, i, vp, vp, vp, sz, vp]),
            "oq_device_status": (i, [C.POINTER(i)]),
            "oq_selftest_bounded_wait": (i, [vp]),
            "oq_debug_select_rq_kernel": (i, [i]),
            "oq_debug_select_gemm_kernel": (i, [i]),
            "oq_rq_plan": (i, [vp, vp, C.POINTER(i), C.POINTER(i), C.POINTER(i), C.POINTER(sz)]),
            "oq_rotate_quantize_act_levels": (i, [vp, i, i, i, vp, vp, vp, i, vp, vp, vp, vp]),
            "oq_decode_levels": (i, [vp, i, i, vp, vp, i, vp]),
            "oq_qlinear_levels": (i, [vp, i, vp, i, vp, vp, i, vp, i, vp, i, i, vp]),
            "oq_adaln_packed_bytes": (i, [i, i, C.POINTER(sz), C.POINTER(sz)]),
            "oq_adaln_quantize_weights": (i, [vp, i, i, i, vp, vp, vp]),
            "oq_adaln_linear": (i, [vp, i, i, vp, vp, i, i, vp, i, i, vp]),
            "oq_adaln_unpack": (i, [vp, vp, i, i, vp, vp, vp]),
            "oq_block_forward": (i, [i, vp, i, vp, i, vp]),
            "oq_make_rope": (i, [i, vp, vp, C.c_double, i, pp]),
            "oq_rope_dim": (i, [vp]), "oq_rope_destroy": (None, [vp]),
            "oq_qk_norm_rope": (i, [vp, vp, i, i, vp, vp, i, i, C.c_float, i, i, vp]),
            "oq_attention_workspace_bytes": (i, [vp, C.POINTER(sz)]),
            "oq_attention": (i, [vp, vp, sz, vp]),
            "oq_adapter_workspace_bytes": (i, [i, i, i, i, C.POINTER(sz)]),
            "oq_adapter_add": (i, [vp, i, i, i, vp, vp, i, i, vp, vp, vp, i, vp, i, vp, i, i, i, vp, sz, vp]),
            "oq_cache_block_bytes": (i, [i, i, i, C.POINTER(sz)]),
            "oq_cache_write": (i, [vp, vp, vp, i, vp, i, vp]),
            "oq_cache_read": (i, [vp, vp, vp, i, vp, i, vp]),
            "oq_cache_attention_workspace_bytes": (i, [vp, C.POINTER(sz)]),
            "oq_cache_attention": (i, [vp, vp, sz, vp]),
            "oq_last_error": (C.c_char_p, []), "oq_version": (C.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            if hasattr(L, name):
                f = getattr(L, name)
                f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def _check(code):
    if code != 0:
        raise OqError(code, lib().oq_last_error().decode())


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(0)


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


class Codebook:
    """Owns an oq_codebook handle."""

    def __init__(self, dim, bits):
        h = C.c_void_p()
        _check(lib().oq_build_codebook(dim, bits, C.byref(h)))
        self.handle, self.dim, self.bits = h, dim, bits
        L = 1 << bits
        self.centroids = np.zeros(L, np.float64)
        self.boundaries = np.zeros(L - 1, np.float64)
        self.boundaries_f32 = np.zeros(L - 1, np.float32)
        self.centroids_bf16_bits = np.zeros(L, np.uint16)
        _check(lib().oq_codebook_get(h, self.centroids.ctypes.data, self.boundaries.ctypes.data,
                                     self.boundaries_f32.ctypes.data, self.centroids_bf16_bits.ctypes.data))

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.oq_codebook_destroy(self.handle)
            self.handle = None


class Rpbh:
    """Owns an oq_rpbh handle."""

    def __init__(self, dim, block, seed):
        h = C.c_void_p()
        _check(lib().oq_make_rpbh(dim, block, seed, C.byref(h)))
        self.handle, self.dim, self.block, self.seed = h, dim, block, seed
        self.perm = np.zeros(dim, np.int32)
        self.signs = np.zeros(dim, np.int8)
        _check(lib().oq_rpbh_get(h, self.perm.ctypes.data, self.signs.ctypes.data))

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.oq_rpbh_destroy(self.handle)
            self.handle = None


class Rope:
    """Owns an oq_rope handle."""

    LAYOUTS = {"pairs": 0, "halves": 1}

    def __init__(self, axis_dims, max_pos, theta, layout):
        dims, top = np.asarray(axis_dims, np.int32), np.asarray(max_pos, np.int32)
        if dims.ndim != 1 or dims.shape != top.shape:
            raise OqError(1, "oq_make_rope: axis_dims and max_pos must be lists of one length")
        if layout not in self.LAYOUTS:
            raise OqError(1, f"oq_make_rope: layout must be one of {sorted(self.LAYOUTS)}")
        h = C.c_void_p()
        _check(lib().oq_make_rope(len(dims), dims.ctypes.data, top.ctypes.data, float(theta), self.LAYOUTS[layout], C.byref(h)))
        self.handle, self.axis_dims, self.max_pos = h, dims.tolist(), top.tolist()
        self.theta, self.layout, self.dim = theta, layout, int(dims.sum())

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.oq_rope_destroy(self.handle)
            self.handle = None


def oq_build_codebook(dim, bits):
    return Codebook(dim, bits)


def oq_make_rpbh(dim, block, seed):
    return Rpbh(dim, block, seed)


def oq_packed_bytes(rows, dim, bits):
    a, b = C.c_size_t(), C.c_size_t()
    _check(lib().oq_packed_bytes(rows, dim, bits, C.byref(a), C.byref(b)))
    return a.value, b.value


def _alloc_packed(rows, dim, bits, device):
    import torch
    total, pitch = oq_packed_bytes(rows, dim, bits)
    return torch.empty((rows, pitch), dtype=torch.uint8, device=device)


def oq_rotate_quantize_act(X, rot, cb_a, out_idx=None, out_norm=None, dbg_rotated=None):
    """X: CUDA bf16 [N, d] (row stride = ldx).  Returns (packed uint8 [N, pitch], norm fp32 [N])."""
    import torch
    n, d = X.shape
    if out_idx is None:
        out_idx = _alloc_packed(n, d, cb_a.bits, X.device)
    if out_norm is None:
        out_norm = torch.empty(n, dtype=torch.float32, device=X.device)
    _check(lib().oq_rotate_quantize_act(_ptr(X), n, d, X.stride(0) if n > 1 else d, rot.handle, cb_a.handle,
                                        _ptr(out_idx), _ptr(out_norm), _ptr(dbg_rotated), _stream()))
    return out_idx, out_norm


def oq_quantize_weights(W, rot, cb_w, out_idx=None, out_norm=None, dbg_rotated=None):
    """W: CUDA bf16 [m, d].  Returns (packed uint8 [m, pitch], row norms bf16 [m])."""
    import torch
    m, d = W.shape
    if out_idx is None:
        out_idx = _alloc_packed(m, d, cb_w.bits, W.device)
    if out_norm is None:
        out_norm = torch.empty(m, dtype=torch.bfloat16, device=W.device)
    _check(lib().oq_quantize_weights(_ptr(W), m, d, W.stride(0) if m > 1 else d, rot.handle, cb_w.handle,
                                     _ptr(out_idx), _ptr(out_norm), _ptr(dbg_rotated), _stream()))
    return out_idx, out_norm


def oq_qlinear(Xq_idx, Xq_norm, cb_a, Wq_idx, Wq_norm, cb_w, dim, out=None, out_dtype=None):
    """Returns Y [N, m] (bf16 by default, fp32 when out_dtype is torch.float32)."""
    import torch
    n, m = Xq_idx.shape[0], Wq_idx.shape[0]
    if out is None:
        out = torch.empty((n, m), dtype=out_dtype or torch.bfloat16, device=Xq_idx.device)
    ydt = OQ_F32 if out.dtype == torch.float32 else OQ_BF16
    _check(lib().oq_qlinear(_ptr(Xq_idx), _ptr(Xq_norm), n, cb_a.handle, _ptr(Wq_idx), _ptr(Wq_norm), m,
                            cb_w.handle, dim, _ptr(out), out.stride(0) if n > 1 else m, ydt, _stream()))
    return out


class _BlockInput(C.Structure):          # oq_block_input
    _fields_ = [("X_bf16", C.c_void_p), ("ldx", C.c_int), ("dim", C.c_int), ("rot", C.c_void_p), ("cb_a", C.c_void_p),
                ("Xq", C.c_void_p), ("Xq_norm", C.c_void_p)]


class _BlockLayer(C.Structure):          # oq_block_layer
    _fields_ = [("input", C.c_int), ("m", C.c_int), ("Wq_idx", C.c_void_p), ("Wq_norm_bf16", C.c_void_p),
                ("cb_w", C.c_void_p), ("Y", C.c_void_p), ("ldy", C.c_int), ("y_dtype", C.c_int)]


def oq_block_forward(inputs, layers):
    """The linear layers of one block on the current stream; every input is rotated and quantized once.
    inputs: list of dicts {X (CUDA bf16 [N, d]), rot, cb_a, xq (scratch: packed uint8 [N, pitch], or bf16 [N, d] at 6 bits),
    xs (fp32 [N])}; layers: list of dicts {input (index), wq, wr, cb_w, Y (CUDA [N, m] bf16 or fp32)}."""
    import torch
    n = inputs[0]["X"].shape[0] if inputs else 0
    ins = (_BlockInput * max(1, len(inputs)))()
    for k, a in enumerate(inputs):
        X = a["X"]
        d = X.shape[1]
        ins[k] = _BlockInput(X.data_ptr(), X.stride(0) if n > 1 else d, d, a["rot"].handle, a["cb_a"].handle,
                             a["xq"].data_ptr(), a["xs"].data_ptr())
    lys = (_BlockLayer * max(1, len(layers)))()
    for k, l in enumerate(layers):
        Y = l["Y"]
        m = Y.shape[1]
        lys[k] = _BlockLayer(l["input"], m, l["wq"].data_ptr(), l["wr"].data_ptr(), l["cb_w"].handle, Y.data_ptr(),
                             Y.stride(0) if n > 1 else m, OQ_F32 if Y.dtype == torch.float32 else OQ_BF16)
    _check(lib().oq_block_forward(n, C.cast(ins, C.c_void_p), len(inputs), C.cast(lys, C.c_void_p), len(layers), _stream()))


def oq_forward_workspace_bytes(n_tokens, dim, m, bits_a):
    b = C.c_size_t()
    _check(lib().oq_forward_workspace_bytes(n_tokens, dim, m, bits_a, C.byref(b)))
    return b.value


def oq_linear_forward_host(X_host, rot, cb_a, Wq_idx, Wq_norm, cb_w, Y_host, workspace):
    """X_host / Y_host: CPU bf16 tensors (pinned for asynchronous copies); workspace: CUDA uint8 tensor."""
    n, d = X_host.shape
    m = Wq_idx.shape[0]
    _check(lib().oq_linear_forward_host(_ptr(X_host), n, d, rot.handle, cb_a.handle, _ptr(Wq_idx), _ptr(Wq_norm), m,
                                        cb_w.handle, _ptr(Y_host), _ptr(workspace), workspace.numel(), _stream()))
    return Y_host


def oq_linear_forward_noalloc(X, rot, cb_a, Wq_idx, Wq_norm, cb_w, out):
    """Allocation-free layer call: X CUDA bf16 [N, d], `out` a preallocated CUDA [N, m] bf16 or fp32 tensor.
    Nothing is allocated here or in the library (the hand-over buffers are a static device array)."""
    import torch
    n, d = X.shape
    m = Wq_idx.shape[0]
    ydt = OQ_F32 if out.dtype == torch.float32 else OQ_BF16
    _check(lib().oq_linear_forward_noalloc(_ptr(X), n, d, X.stride(0) if n > 1 else d, rot.handle, cb_a.handle,
                                           _ptr(Wq_idx), _ptr(Wq_norm), m, cb_w.handle, _ptr(out),
                                           out.stride(0) if n > 1 else m, ydt, _stream()))
    return out


def oq_unpack_indices(idx, rows, dim, bits):
    import torch
    out = torch.empty((rows, dim), dtype=torch.uint8, device=idx.device)
    _check(lib().oq_unpack_indices(_ptr(idx), rows, dim, bits, _ptr(out), _stream()))
    return out


def oq_device_status():
    s = C.c_int(0)
    code = lib().oq_device_status(C.byref(s))
    if code not in (0, 5):
        _check(code)
    return s.value


def oq_selftest_bounded_wait():
    _check(lib().oq_selftest_bounded_wait(_stream()))


def oq_rq_plan(rot, cb):
    """(kernel, rows_per_group, tiles_per_group, smem_bytes) of the rotate+quantize launch for these handles."""
    k, r, t, m = C.c_int(0), C.c_int(0), C.c_int(0), C.c_size_t(0)
    _check(lib().oq_rq_plan(rot.handle, cb.handle, C.byref(k), C.byref(r), C.byref(t), C.byref(m)))
    return k.value, r.value, t.value, m.value


def oq_debug_select_rq_kernel(which):
    _check(lib().oq_debug_select_rq_kernel(int(which)))


def oq_debug_select_gemm_kernel(which):
    _check(lib().oq_debug_select_gemm_kernel(int(which)))


def oq_rotate_quantize_act_levels(X, rot, cb_a, out=None, out_norm=None, want_idx=False, dbg_rotated=None):
    """6-bit activations: X CUDA bf16 [N, d] -> (levels bf16 [N, d], norm fp32 [N], idx uint8 [N, d] or None)."""
    import torch
    n, d = X.shape
    if out is None:
        out = torch.empty((n, d), dtype=torch.bfloat16, device=X.device)
    if out_norm is None:
        out_norm = torch.empty(n, dtype=torch.float32, device=X.device)
    idx = torch.empty((n, d), dtype=torch.uint8, device=X.device) if want_idx else None
    _check(lib().oq_rotate_quantize_act_levels(_ptr(X), n, d, X.stride(0) if n > 1 else d, rot.handle, cb_a.handle,
                                               _ptr(out), out.stride(0) if n > 1 else d, _ptr(out_norm), _ptr(idx),
                                               _ptr(dbg_rotated), _stream()))
    return out, out_norm, idx


def oq_decode_levels(idx, rows, dim, cb, out=None):
    """Packed indices [rows, pitch] -> bf16 levels [rows, dim] (written once, read by oq_qlinear_levels)."""
    import torch
    if out is None:
        out = torch.empty((rows, dim), dtype=torch.bfloat16, device=idx.device)
    _check(lib().oq_decode_levels(_ptr(idx), rows, dim, cb.handle, _ptr(out), out.stride(0) if rows > 1 else dim, _stream()))
    return out


def oq_qlinear_levels(Xd, Xq_norm, Wq_idx, Wq_norm, cb_w, dim, out=None, out_dtype=None):
    """oq_qlinear with the activations given as bf16 levels [N, dim]."""
    import torch
    n, m = Xd.shape[0], Wq_idx.shape[0]
    if out is None:
        out = torch.empty((n, m), dtype=out_dtype or torch.bfloat16, device=Xd.device)
    ydt = OQ_F32 if out.dtype == torch.float32 else OQ_BF16
    _check(lib().oq_qlinear_levels(_ptr(Xd), Xd.stride(0) if n > 1 else dim, _ptr(Xq_norm), n, _ptr(Wq_idx),
                                   _ptr(Wq_norm), m, cb_w.handle, dim, _ptr(out), out.stride(0) if n > 1 else m, ydt,
                                   _stream()))
    return out


def oq_adaln_packed_bytes(m, dim):
    a, b = C.c_size_t(), C.c_size_t()
    _check(lib().oq_adaln_packed_bytes(m, dim, C.byref(a), C.byref(b)))
    return a.value, b.value


def oq_adaln_quantize_weights(W):
    """W: CUDA bf16 [m, d].  Returns (packed nibbles uint8 [m * d / 2], scales uint8 [2 * m * d / 64])."""
    import torch
    m, d = W.shape
    wq_bytes, sc_bytes = oq_adaln_packed_bytes(m, d)
    Wq = torch.empty(wq_bytes, dtype=torch.uint8, device=W.device)
    Sc = torch.empty(sc_bytes, dtype=torch.uint8, device=W.device)
    _check(lib().oq_adaln_quantize_weights(_ptr(W), m, d, W.stride(0) if m > 1 else d, _ptr(Wq), _ptr(Sc), _stream()))
    return Wq, Sc


def oq_adaln_linear(X, Wq, Sc, m, out=None, out_dtype=None):
    """X: CUDA bf16 [n, d].  Returns Y [n, m] (bf16 by default, fp32 when out_dtype is torch.float32)."""
    import torch
    n, d = X.shape
    if out is None:
        out = torch.empty((n, m), dtype=out_dtype or torch.bfloat16, device=X.device)
    ydt = OQ_F32 if out.dtype == torch.float32 else OQ_BF16
    _check(lib().oq_adaln_linear(_ptr(X), n, X.stride(0) if n > 1 else d, _ptr(Wq), _ptr(Sc), m, d, _ptr(out),
                                 out.stride(0) if n > 1 else m, ydt, _stream()))
    return out


def oq_adaln_unpack(Wq, Sc, m, dim):
    """Returns (q int8 [m, d], scale bf16 [m, d / 64]) on the device."""
    import torch
    q = torch.empty((m, dim), dtype=torch.int8, device=Wq.device)
    s = torch.empty((m, dim // 64), dtype=torch.bfloat16, device=Wq.device)
    _check(lib().oq_adaln_unpack(_ptr(Wq), _ptr(Sc), m, dim, _ptr(q), _ptr(s), _stream()))
    return q, s


def oq_make_rope(axis_dims, max_pos, theta=10000.0, layout="pairs"):
    """Rotation by position with len(axis_dims) axes; positions 0 .. max_pos[a] - 1 on axis a."""
    return Rope(axis_dims, max_pos, theta, layout)


def _dtype_code(dtype, what):
    import torch
    if dtype == torch.bfloat16:
        return OQ_BF16
    if dtype == torch.float32:
        return OQ_F32
    raise OqError(1, f"{what}: bf16 or fp32 expected, got {dtype}")


def _off_device(what):
    """Raised unless all tensors of a call are on one CUDA device (get_device() is -1 in host memory, whose pointers the kernels would
    follow).  The calls compare in place: a loop over their tensors takes half a microsecond more."""
    return OqError(1, f"{what}: all tensors must be on one CUDA device")


def _check_workspace(what, t, torch, device):
    if t.dtype != torch.uint8 or not t.is_contiguous() or t.get_device() != device:
        raise OqError(1, f"{what}: the workspace must be a contiguous uint8 tensor on the inputs' device")


# The calls below are short on the GPU at small sizes (3 to 7 us), so their marshalling looks at every property of a tensor
# once, and outputs that are allocated here are not looked at again.
_QK_SIDE = struct.Struct("@PqqiPPqq")               # oq_qk_side
NORMS = {"none": 0, "head": 1, "row": 2}


def _qk_side(torch, X, w, Y, norm, n, head_dim, dtype, out_dtype):
    """Checks one side of oq_qk_norm_rope, allocates its output if there is none, and packs its oq_qk_side."""
    shape = X.shape
    if len(shape) != 3 or shape[0] != n or shape[2] != head_dim or X.dtype != dtype:
        raise OqError(1, "oq_qk_norm_rope: queries and keys must be [T, heads, head_dim] of one T, head_dim and type")
    heads = shape[1]
    lt, lh, lc = X.stride()
    if Y is None:
        Y = X.new_empty(shape) if out_dtype is None else X.new_empty(shape, dtype=out_dtype)
        yt, yh = heads * head_dim, head_dim
    else:
        if Y.shape != shape:
            raise OqError(1, "oq_qk_norm_rope: outputs must have the inputs' shape")
        yt, yh, yc = Y.stride()
        if yc != 1 and n:
            lc = yc
        if n == 1:                                   # torch leaves the stride of a single row or head free
            yt = 0
        if heads == 1:
            yh = 0
    if lc != 1 and n:
        raise OqError(3, "oq_qk_norm_rope: the coordinates of a head must be adjacent")
    if n == 1:
        lt = 0
    if heads == 1:
        lh = 0
    at = 0
    if w is not None:
        if w.dtype != torch.bfloat16 or w.numel() != (head_dim if norm == "head" else heads * head_dim) or not w.is_contiguous():
            raise OqError(1, "oq_qk_norm_rope: weights must be contiguous bf16, one for each normed coordinate")
        at = w.data_ptr()
    return Y, _QK_SIDE.pack(X.data_ptr(), lt, lh, heads, at, Y.data_ptr(), yt, yh)


def oq_qk_norm_rope(Q, K, rope=None, pos=None, wq=None, wk=None, norm="head", eps=1e-6, out_q=None, out_k=None, out_dtype=None):
    """Q, K: CUDA [T, heads, head_dim] (bf16 or fp32, any token and head strides, unit stride inside a head); K may be
    None.  pos: CUDA int32 [T, axes].  wq, wk: CUDA bf16, head_dim values (norm="head") or heads * head_dim (norm="row").
    Returns (Q', K'), of out_dtype (the inputs' by default); out_q, out_k may be Q and K themselves."""
    import torch
    shape, dtype = Q.shape, Q.dtype
    if len(shape) != 3:
        raise OqError(1, "oq_qk_norm_rope: queries and keys must be [T, heads, head_dim]")
    n, _, head_dim = shape
    device = Q.get_device()
    if device < 0 or (wq is not None and wq.get_device() != device) or (out_q is not None and out_q.get_device() != device):
        raise _off_device("oq_qk_norm_rope")
    if K is not None and (K.get_device() != device or (wk is not None and wk.get_device() != device) or
                          (out_k is not None and out_k.get_device() != device)):
        raise _off_device("oq_qk_norm_rope")
    norm_code = NORMS.get(norm)
    if norm_code is None:
        raise OqError(1, f"oq_qk_norm_rope: norm must be one of {sorted(NORMS)}")
    x_code = y_code = _dtype_code(dtype, "oq_qk_norm_rope")
    out_q, q_side = _qk_side(torch, Q, wq, out_q, norm, n, head_dim, dtype, out_dtype)
    if out_q.dtype != dtype:
        y_code = _dtype_code(out_q.dtype, "oq_qk_norm_rope")
    k_side = None
    if K is not None:
        out_k, k_side = _qk_side(torch, K, wk, out_k, norm, n, head_dim, dtype, out_dtype)
        if out_k.dtype != out_q.dtype:
            raise OqError(1, "oq_qk_norm_rope: outputs must have one type")
    else:
        out_k = None
    ldpos, table, at = 0, None, None
    if rope is not None:
        axes = len(rope.axis_dims)
        if pos is None or pos.dtype != torch.int32 or pos.shape != (n, axes):
            raise OqError(1, "oq_qk_norm_rope: pos must be int32 [T, axes]")
        if pos.get_device() != device:
            raise _off_device("oq_qk_norm_rope")
        ldpos, step = pos.stride()
        if step != 1 and axes > 1 and n:
            raise OqError(3, "oq_qk_norm_rope: the positions of a token must be adjacent")
        if n <= 1:
            ldpos = axes
        if ldpos > _INT_MAX:                         # (ctypes would cut it to 32 bits)
            raise OqError(2, "oq_qk_norm_rope: a stride of positions above 2^31 - 1")
        table, at = rope.handle, pos.data_ptr()
    code = (_lib or lib()).oq_qk_norm_rope(q_side, k_side, n, head_dim, table, at, ldpos, norm_code, eps, x_code, y_code,
                                           torch._C._cuda_getCurrentRawStream(device))
    if code:
        _check(code)
    return out_q, out_k


_ATTENTION_ARGS = struct.Struct("@PPPqqqqqqPqqPPPiiiiiiiiif")      # oq_attention_args


def oq_attention(Q, K, V, q_start=None, k_start=None, left=-1, right=-1, sinks=0, scale=0.0, out=None, want_lse=False,
                 workspace=None):
    """Q: CUDA bf16 [Tq, heads, head_dim], K, V: [Tk, kv_heads, head_dim] (token and head strides of at least head_dim, or a
    head stride of 0: a head expanded over all; unit stride inside a head); q_start, k_start: CUDA int32 [sequences + 1], or None for one sequence.  left, right, sinks: see oq.h.
    Returns out [Tq, heads, head_dim], or (out, lse fp32 [heads, Tq]) with want_lse.  workspace: CUDA uint8 tensor, by
    default one is taken from torch's allocator when the call needs it."""
    import torch
    bf16 = torch.bfloat16
    qs, ks = Q.shape, K.shape
    if len(qs) != 3 or len(ks) != 3 or ks != V.shape or qs[2] != ks[2]:
        raise OqError(1, "oq_attention: Q must be [Tq, heads, head_dim], K and V [Tk, kv_heads, head_dim]")
    if Q.dtype != bf16 or K.dtype != bf16 or V.dtype != bf16:
        raise OqError(1, "oq_attention: bf16 expected")
    device = Q.get_device()
    if device < 0 or not device == K.get_device() == V.get_device():
        raise _off_device("oq_attention")
    tq, heads, head_dim = qs
    tk, kv_heads, _ = ks
    n_seqs, q_at, k_at = 1, 0, 0
    if q_start is not None or k_start is not None:
        for t in (q_start, k_start):
            if t is None or t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous() or t.get_device() != device:
                raise OqError(1, "oq_attention: q_start and k_start must both be contiguous int32 [sequences + 1] on Q's device")
        n_seqs = len(q_start) - 1
        if len(k_start) != n_seqs + 1:
            raise OqError(1, "oq_attention: q_start and k_start must have one length")
        q_at, k_at = q_start.data_ptr(), k_start.data_ptr()
    (qt, qh, qc), (kt, kh, kc), (vt, vh, vc) = Q.stride(), K.stride(), V.stride()
    if out is None:
        out = Q.new_empty(qs)
        ot, oh = heads * head_dim, head_dim
    else:
        if out.shape != qs or out.dtype != bf16 or out.get_device() != device:
            raise OqError(1, "oq_attention: out must be bf16, shaped like Q and on its device")
        ot, oh, oc = out.stride()
        if oc != 1 and tq:
            qc = oc
    if qc != 1 and tq or (kc != 1 or vc != 1) and tk:
        raise OqError(3, "oq_attention: the coordinates of a head must be adjacent")
    if tq <= 1:                                      # torch leaves the stride of a single row or head free
        qt = ot = 0
    if heads == 1:
        qh = oh = 0
    if tk <= 1:
        kt = vt = 0
    if kv_heads == 1:
        kh = vh = 0
    lse, lse_at = None, 0
    if want_lse:
        lse = Q.new_empty((heads, tq), dtype=torch.float32)
        lse_at = lse.data_ptr()
    try:
        args = _ATTENTION_ARGS.pack(Q.data_ptr(), K.data_ptr(), V.data_ptr(), qt, qh, kt, kh, vt, vh, out.data_ptr(), ot, oh, lse_at,
                                    q_at, k_at, n_seqs, tq, tk, heads, kv_heads, head_dim, left, right, sinks, scale)
    except (struct.error, OverflowError):
        raise OqError(1, "oq_attention: sizes and the window must be whole numbers of 32 bits, scale a number in fp32") from None
    L = _lib or lib()
    space = size = 0
    if workspace is not None:
        _check_workspace("oq_attention", workspace, torch, device)
        space, size = workspace.data_ptr(), workspace.numel()
    else:
        need = C.c_size_t()
        code = L.oq_attention_workspace_bytes(args, C.byref(need))
        if code:
            _check(code)
        size = need.value
        if size:
            workspace = Q.new_empty(size, dtype=torch.uint8)
            space = workspace.data_ptr()
    code = L.oq_attention(args, space, size, torch._C._cuda_getCurrentRawStream(device))
    if code:
        _check(code)
    return (out, lse) if want_lse else out


def oq_adapter_add(X, A, Bm, scale, seg_start, seg_adapter, base, out=None, workspace=None):
    """base + scale_a B_a (A_a x) for the tokens of each segment.  X: CUDA bf16 [T, d]; A: bf16 [adapters, rank, d]; Bm: bf16
    [adapters, m, rank]; scale: fp32 [adapters]; seg_start: int32 [segments + 1]; seg_adapter: int32 [segments] (-1: none);
    base: bf16 or fp32 [T, m].  Returns out (new by default; out=base adds in place).  workspace: CUDA uint8 tensor, by default
    one is taken from torch's allocator when the call needs it."""
    import torch
    bf16, i32 = torch.bfloat16, torch.int32
    xs, sa, sb, shape = X.shape, A.shape, Bm.shape, base.shape
    if len(xs) != 2 or len(sa) != 3 or len(sb) != 3 or len(shape) != 2:
        raise OqError(1, "oq_adapter_add: X [T, d], A [adapters, rank, d], B [adapters, m, rank], base [T, m] expected")
    device = X.get_device()
    if device < 0 or not (device == A.get_device() == Bm.get_device() == scale.get_device() == seg_start.get_device() ==
                          seg_adapter.get_device() == base.get_device()):
        raise _off_device("oq_adapter_add")
    n, d = xs
    na, rank, m = sa[0], sa[1], sb[1]
    segs = seg_adapter.numel()
    if sa[2] != d or sb[0] != na or sb[2] != rank or shape[0] != n or shape[1] != m or scale.shape != (na,):
        raise OqError(1, "oq_adapter_add: sizes do not match")
    if X.dtype != bf16 or A.dtype != bf16 or Bm.dtype != bf16 or scale.dtype != torch.float32:
        raise OqError(1, "oq_adapter_add: X, A, B must be bf16 and scale fp32")
    if seg_start.dtype != i32 or seg_adapter.dtype != i32 or seg_adapter.dim() != 1 or seg_start.shape != (segs + 1,):
        raise OqError(1, "oq_adapter_add: seg_start int32 [segments + 1], seg_adapter int32 [segments] expected")
    if not (A.is_contiguous() and Bm.is_contiguous() and scale.is_contiguous() and seg_start.is_contiguous() and seg_adapter.is_contiguous()):
        raise OqError(1, "oq_adapter_add: adapters, scales and segment tables must be contiguous")
    if out is None:
        out = base.new_empty(shape)
    elif out.shape != shape or out.dtype != base.dtype or out.get_device() != device:
        raise OqError(1, "oq_adapter_add: out must have base's shape, type and device")
    (ldx, xc), (ldb, bc), (ldy, yc) = X.stride(), base.stride(), out.stride()
    if n and (xc != 1 or bc != 1 or yc != 1):
        raise OqError(3, "oq_adapter_add: the elements of a row must be adjacent")
    if n <= 1:
        ldx, ldb, ldy = d, m, m
    if max(ldx, ldb, ldy) > _INT_MAX:                # (ctypes would cut it to 32 bits)
        raise OqError(2, "oq_adapter_add: a leading dimension above 2^31 - 1")
    space = size = 0
    if workspace is not None:
        _check_workspace("oq_adapter_add", workspace, torch, device)
    else:
        need = C.c_size_t()
        _check(lib().oq_adapter_workspace_bytes(n, segs, d, rank, C.byref(need)))
        if need.value:
            workspace = torch.empty(need.value, dtype=torch.uint8, device=X.device)
    if workspace is not None:
        space, size = workspace.data_ptr(), workspace.numel()
    _check(lib().oq_adapter_add(X.data_ptr(), n, ldx, d, A.data_ptr(), Bm.data_ptr(), na, rank, scale.data_ptr(), seg_start.data_ptr(),
                                seg_adapter.data_ptr(), segs, base.data_ptr(), ldb, out.data_ptr(), ldy, m,
                                _dtype_code(base.dtype, "oq_adapter_add"), space, size, torch._C._cuda_getCurrentRawStream(device)))
    return out


_CACHE = struct.Struct("@PPPqiiiiiii4x")             # oq_cache
_CACHE_ROWS = struct.Struct("@Pqq")                  # oq_cache_rows
_CACHE_ATTENTION = struct.Struct("@PPPqiiiiiii4xPqqPqqPPiiiiiif")      # oq_cache_attention_args
CACHE_KINDS = {"fp8": 8, "fp4": 4}


def oq_cache_block_bytes(page_size, head_dim, kind="fp8"):
    """Bytes of one head's block in a page of page_size tokens."""
    n = C.c_size_t()
    _check(lib().oq_cache_block_bytes(CACHE_KINDS.get(kind, 0), page_size, head_dim, C.byref(n)))
    return n.value


def oq_cache_alloc(n_pages, page_size, kv_heads, head_dim, kind="fp8", device="cuda"):
    """A pool of pages: uint8 [n_pages, kv_heads, bytes of a block], cleared."""
    import torch
    return torch.zeros((n_pages, kv_heads, oq_cache_block_bytes(page_size, head_dim, kind)), dtype=torch.uint8, device=device)


def _cache_fields(what, torch, pages, head_dim, kind, table, lens, start, device, page_size):
    """Checks what the calls on a cache have in common.  Returns the fields of oq_cache and the address of start."""
    bits = CACHE_KINDS.get(kind)
    if bits is None:
        raise OqError(1, f"{what}: kind must be one of {sorted(CACHE_KINDS)}")
    if device < 0 or not device == pages.get_device() == table.get_device() == lens.get_device():
        raise _off_device(what)
    if device != torch._C._cuda_getDevice():
        raise OqError(1, f"{what}: the tensors' device must be the current one")
    shape, tshape, lshape, i32 = pages.shape, table.shape, lens.shape, torch.int32
    if len(shape) != 3 or pages.dtype != torch.uint8 or not pages.is_contiguous():
        raise OqError(1, f"{what}: pages must be contiguous uint8 [pages, kv_heads, bytes of a block]")
    if head_dim != 64 and head_dim != 128:
        raise OqError(2, f"{what}: head_dim must be 64 or 128")
    n_pages, heads, block = shape
    size, odd = divmod(block, head_dim * (4 * bits + 1) // 16)        # bytes of a token's keys, values and scales: 2 (d * bits / 8 + d / 32)
    if odd:
        raise OqError(1, f"{what}: no number of tokens of this kind and head_dim fills a block of these pages")
    if page_size is not None and page_size != size:
        raise OqError(1, f"{what}: with this kind and head_dim, blocks of these pages hold {size} tokens, not {page_size}")
    if len(lshape) != 1 or len(tshape) != 2 or tshape[0] != lshape[0] or table.dtype != i32 or lens.dtype != i32 or not lens.is_contiguous():
        raise OqError(1, f"{what}: table must be int32 [sequences, pages], lens contiguous int32 [sequences]")
    seqs, most = tshape
    ld, step = table.stride()
    if step != 1 and most > 1:
        raise OqError(3, f"{what}: the entries of a row of the table must be adjacent")
    at = 0
    if start is not None:
        if start.get_device() != device:
            raise _off_device(what)
        if start.dtype != i32 or start.shape != (seqs + 1,) or not start.is_contiguous():
            raise OqError(1, f"{what}: start must be contiguous int32 [sequences + 1]")
        at = start.data_ptr()
    elif seqs != 1:
        raise OqError(1, f"{what}: several sequences need start")
    if n_pages > _INT_MAX or heads > _INT_MAX or most > _INT_MAX:
        raise OqError(2, f"{what}: sizes above 2^31 - 1")
    return (pages.data_ptr(), table.data_ptr(), lens.data_ptr(), ld, n_pages, size, heads, head_dim, bits, seqs, most), at


def _cache_rows(what, X, heads, head_dim):
    """oq_cache_rows of keys or values [T, kv_heads, head_dim]."""
    n, h, d = X.shape
    lt, lh, lc = X.stride()
    if h != heads or d != head_dim:
        raise OqError(1, f"{what}: keys and values must be [T, {heads}, {head_dim}]")
    if lc != 1 and n:
        raise OqError(3, f"{what}: the coordinates of a head must be adjacent")
    return _CACHE_ROWS.pack(X.data_ptr(), lt if n > 1 else head_dim * heads, lh if h > 1 else head_dim)


def oq_cache_write(pages, K, V, table, lens, start=None, kind="fp8", page_size=None):
    """Quantizes keys and values of new tokens into the pages of their sequences.  pages: CUDA uint8 [pages, kv_heads, bytes of a
    block] (oq_cache_alloc); K, V: CUDA bf16 or fp32 [T, kv_heads, head_dim], any strides of multiples of 16 bytes, unit stride
    inside a head; table: int32 [sequences, pages]; lens: int32 [sequences], the new tokens included; start: int32 [sequences + 1]
    or None for one sequence.  The tokens of a page follow from its bytes, kind and head_dim; page_size, where it is given, has to agree
    (pages of head_dim 128 pass for pages of twice as many tokens of 64 without it)."""
    import torch
    if K.dim() != 3 or K.shape != V.shape or K.dtype != V.dtype:
        raise OqError(1, "oq_cache_write: K and V must be [T, kv_heads, head_dim] of one type")
    device = K.get_device()
    if V.get_device() != device:
        raise _off_device("oq_cache_write")
    code = _dtype_code(K.dtype, "oq_cache_write")
    n, heads, head_dim = K.shape
    fields, at = _cache_fields("oq_cache_write", torch, pages, head_dim, kind, table, lens, start, device, page_size)
    if heads != fields[6]:
        raise OqError(1, "oq_cache_write: the pages are of another number of heads")
    if n > _INT_MAX:
        raise OqError(2, "oq_cache_write: too many tokens")
    rc = (_lib or lib()).oq_cache_write(_CACHE.pack(*fields), _cache_rows("oq_cache_write", K, heads, head_dim),
                                        _cache_rows("oq_cache_write", V, heads, head_dim), code, at, n,
                                        torch._C._cuda_getCurrentRawStream(device))
    if rc:
        _check(rc)


def oq_cache_read(pages, head_dim, table, lens, start=None, total=None, kind="fp8", out_k=None, out_v=None, out_dtype=None, page_size=None):
    """Reads the last start[s + 1] - start[s] tokens of each sequence back.  total: tokens of all sequences together (the tensors'
    first size where out_k or out_v is given).  Returns (K, V) [total, kv_heads, head_dim] of out_dtype (bf16 or fp32, bf16 by default).
    With out_k or out_v given, only what is given is read.  page_size: see oq_cache_write."""
    import torch
    device = pages.get_device()
    fields, at = _cache_fields("oq_cache_read", torch, pages, head_dim, kind, table, lens, start, device, page_size)
    heads = fields[6]
    if out_k is None and out_v is None:
        if total is None or not 0 <= total <= _INT_MAX:
            raise OqError(1, "oq_cache_read: total, or out_k or out_v, is needed")
        shape, dtype = (total, heads, head_dim), out_dtype or torch.bfloat16
        code = _dtype_code(dtype, "oq_cache_read")
        out_k, out_v = pages.new_empty(shape, dtype=dtype), pages.new_empty(shape, dtype=dtype)
        k = _CACHE_ROWS.pack(out_k.data_ptr(), heads * head_dim, head_dim)
        v = _CACHE_ROWS.pack(out_v.data_ptr(), heads * head_dim, head_dim)
    else:
        given = [x for x in (out_k, out_v) if x is not None]
        total = given[0].shape[0] if total is None and given[0].dim() else total
        for x in given:
            if x.dim() != 3 or x.shape[0] != total or x.dtype != given[0].dtype or (out_dtype is not None and x.dtype != out_dtype):
                raise OqError(1, "oq_cache_read: out_k and out_v must be [total, kv_heads, head_dim] of one type")
            if x.get_device() != device:
                raise _off_device("oq_cache_read")
        code = _dtype_code(given[0].dtype, "oq_cache_read")
        k, v = (None if x is None else _cache_rows("oq_cache_read", x, heads, head_dim) for x in (out_k, out_v))
    rc = (_lib or lib()).oq_cache_read(_CACHE.pack(*fields), k, v, code, at, total, torch._C._cuda_getCurrentRawStream(device))
    if rc:
        _check(rc)
    return out_k, out_v


def oq_cache_attention(Q, pages, table, lens, q_start=None, kind="fp8", left=-1, right=0, sinks=0, scale=0.0, max_q=0, out=None,
                       want_lse=False, workspace=None, page_size=None):
    """Attention of new tokens over the pages of their sequences, which hold the new tokens' keys and values already.  Q: CUDA bf16
    [T, heads, head_dim] (any strides of multiples of 8, unit stride inside a head); pages, table, lens, q_start, page_size: see oq_cache_write.  left, right,
    sinks, max_q: see oq.h.  Returns out [T, heads, head_dim], or (out, lse fp32 [heads, T]) with want_lse.  workspace: CUDA uint8
    tensor, by default one is taken from torch's allocator when the call needs it."""
    import torch
    qs, bf16 = Q.shape, torch.bfloat16
    if len(qs) != 3 or Q.dtype != bf16:
        raise OqError(1, "oq_cache_attention: Q must be bf16 [T, heads, head_dim]")
    device = Q.get_device()
    n, heads, head_dim = qs
    fields, at = _cache_fields("oq_cache_attention", torch, pages, head_dim, kind, table, lens, q_start, device, page_size)
    qt, qh, qc = Q.stride()
    if out is None:
        out = Q.new_empty(qs)
        ot, oh = heads * head_dim, head_dim
    else:
        if out.shape != qs or out.dtype != bf16 or out.get_device() != device:
            raise OqError(1, "oq_cache_attention: out must be bf16, shaped like Q and on its device")
        ot, oh, oc = out.stride()
        if oc != 1 and n:
            qc = oc
    if qc != 1 and n:
        raise OqError(3, "oq_cache_attention: the coordinates of a head must be adjacent")
    if n <= 1:                                       # torch leaves the stride of a single row or head free
        qt = ot = 0
    if heads == 1:
        qh = oh = 0
    lse, lse_at = None, 0
    if want_lse:
        lse = Q.new_empty((heads, n), dtype=torch.float32)
        lse_at = lse.data_ptr()
    try:
        args = _CACHE_ATTENTION.pack(*fields, Q.data_ptr(), qt, qh, out.data_ptr(), ot, oh, lse_at, at, n, heads, max_q, left, right, sinks,
                                     scale)
    except (struct.error, OverflowError):
        raise OqError(1, "oq_cache_attention: sizes and the window must be whole numbers of 32 bits, scale a number in fp32") from None
    L = _lib or lib()
    space = size = 0
    if workspace is not None:
        _check_workspace("oq_cache_attention", workspace, torch, device)
        space, size = workspace.data_ptr(), workspace.numel()
    else:
        need = C.c_size_t()
        code = L.oq_cache_attention_workspace_bytes(args, C.byref(need))
        if code:
            _check(code)
        size = need.value
        if size:
            workspace = Q.new_empty(size, dtype=torch.uint8)
            space = workspace.data_ptr()
    code = L.oq_cache_attention(args, space, size, torch._C._cuda_getCurrentRawStream(device))
    if code:
        _check(code)
    return (out, lse) if want_lse else out


def oq_version():
    return lib().oq_version().decode()
