"""ctypes binding over libfgattn.so: same names as the C ABI in include/fgattn.h.

Argument marshalling only -- every step of the path runs in the library's HIP kernels.
torch is used for device memory and streams.  There is no fallback: if the library has
not been built, importing a symbol from it raises.
"""
import ctypes
import os
import struct

from . import build as _build


class FgattnParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32), ("d", ctypes.c_int32),
                ("M", ctypes.c_int32), ("N", ctypes.c_int32),
                ("q_stride_b", ctypes.c_int64), ("q_stride_h", ctypes.c_int64), ("q_stride_l", ctypes.c_int64),
                ("k_stride_b", ctypes.c_int64), ("k_stride_h", ctypes.c_int64), ("k_stride_l", ctypes.c_int64),
                ("v_stride_b", ctypes.c_int64), ("v_stride_h", ctypes.c_int64), ("v_stride_l", ctypes.c_int64),
                ("o_stride_b", ctypes.c_int64), ("o_stride_h", ctypes.c_int64), ("o_stride_l", ctypes.c_int64),
                ("scale", ctypes.c_float), ("flags", ctypes.c_int32)]


class FgattnRopeAxis(ctypes.Structure):
    _fields_ = [("size", ctypes.c_int32), ("pairs", ctypes.c_int32), ("theta", ctypes.c_double), ("offset", ctypes.c_double),
                ("step", ctypes.c_double), ("factor", ctypes.c_double), ("original", ctypes.c_double),
                ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double)]


class FgattnRopeParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hk", ctypes.c_int32), ("L", ctypes.c_int32), ("d", ctypes.c_int32),
                ("rot_dims", ctypes.c_int32), ("layout", ctypes.c_int32), ("dtype", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("eps", ctypes.c_float)] + [("%s_stride_%s" % (t, x), ctypes.c_int64) for t in ("q", "k", "qo", "ko") for x in "bhl"]


class FgattnCrossParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("Lq", ctypes.c_int32), ("Lk", ctypes.c_int32),
                ("d", ctypes.c_int32)] + \
        [("%s_stride_%s" % (t, x), ctypes.c_int64) for t in ("q", "k", "v", "o", "do", "dq", "dk", "dv") for x in "bhl"] + \
        [("scale", ctypes.c_float), ("flags", ctypes.c_int32)]


FLAG_STATIC_ASSIGN, FLAG_FIFO_QUEUE, FLAG_REUSE_PLAN, FLAG_MASK_ROWS_IN_HBM, FLAG_MASK_ONE_TILE_CHUNKS = 1, 2, 4, 8, 16
E_NULL, E_SHAPE, E_STRIDE, E_ALIGN, E_WORKSPACE, E_SCALE, E_DEVICE, E_MASK, E_FLAGS, E_STATIC_LIMIT, E_DTYPE = range(-1, -12, -1)
STATIC_MAX_ITEMS = 65536
BF16, FP16, FP32 = 0, 1, 2
ROPE_INTERLEAVED, ROPE_HALF = 0, 1
FLAG_ROPE_NORM, FLAG_ROPE_WEIGHT_FP32 = 1, 2

_lib = None


class FgattnError(RuntimeError):
    def __init__(self, code):
        self.code = code
        super().__init__("fgattn error %d: %s" % (code, fgattn_strerror(code)))


def lib():
    """The loaded C-ABI library; raises if it has not been built (there is no CPU fallback)."""
    global _lib
    if _lib is None:
        path = _build.LIBFGATTN
        if not os.path.exists(path):
            raise RuntimeError("libfgattn.so is missing: run __graft_entry__.build() (hipcc, gfx950) first")
        L = ctypes.CDLL(path)
        vp, i64p, pp = ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(FgattnParams)
        L.fgattn_workspace_bytes.argtypes = [pp]
        L.fgattn_workspace_bytes.restype = ctypes.c_size_t
        L.fgattn_forward.argtypes = [vp, vp, vp, i64p, vp, pp, vp, vp, vp, ctypes.c_size_t, vp]
        L.fgattn_forward.restype = ctypes.c_int
        L.fgattn_forward_static.argtypes = [vp, vp, vp, i64p, vp, pp, vp, vp, vp]
        L.fgattn_forward_static.restype = ctypes.c_int
        L.fgattn_forward_part.argtypes = [vp, vp, vp, i64p, vp, pp, vp, vp, vp, ctypes.c_size_t, ctypes.c_int, vp]
        L.fgattn_forward_part.restype = ctypes.c_int
        L.fgattn_issue_probe.argtypes = [ctypes.c_int, ctypes.c_int, vp, ctypes.c_size_t, ctypes.POINTER(ctypes.c_double), vp]
        L.fgattn_issue_probe.restype = ctypes.c_int
        L.fgattn_forward_grouped.argtypes = [vp, vp, vp, vp, i64p, vp, vp, pp, vp, vp, vp, ctypes.c_size_t, vp]
        L.fgattn_forward_grouped.restype = ctypes.c_int
        L.fgattn_dense_forward.argtypes = [vp, vp, vp, pp, vp, vp, vp, ctypes.c_size_t, vp]
        L.fgattn_dense_forward.restype = ctypes.c_int
        L.fgattn_plan.argtypes = [i64p, pp, vp, ctypes.c_size_t, vp]
        L.fgattn_plan.restype = ctypes.c_int
        L.fgattn_validate_mask.argtypes = [i64p, vp, pp, vp, ctypes.c_size_t, vp]
        L.fgattn_validate_mask.restype = ctypes.c_int
        L.fgattn_mask_workspace_bytes.argtypes = [pp]
        L.fgattn_mask_workspace_bytes.restype = ctypes.c_size_t
        L.fgattn_mask_select.argtypes = [vp, vp, pp, ctypes.c_float, vp, vp, ctypes.c_size_t, vp]
        L.fgattn_mask_select.restype = ctypes.c_int
        L.fgattn_mask_emit.argtypes = [pp, vp, vp, ctypes.c_int64, vp, ctypes.c_size_t, vp]
        L.fgattn_mask_emit.restype = ctypes.c_int
        L.fgattn_group_workspace_bytes.argtypes = [pp, ctypes.c_int]
        L.fgattn_group_workspace_bytes.restype = ctypes.c_size_t
        L.fgattn_group_select.argtypes = [i64p, vp, pp, ctypes.c_int, vp, vp, vp, ctypes.c_size_t, vp]
        L.fgattn_group_select.restype = ctypes.c_int
        L.fgattn_group_emit.argtypes = [pp, ctypes.c_int, vp, vp, vp, vp, ctypes.c_int64, vp, ctypes.c_size_t, vp]
        L.fgattn_group_emit.restype = ctypes.c_int
        rp, xp, sz = ctypes.POINTER(FgattnRopeParams), ctypes.POINTER(FgattnCrossParams), ctypes.c_size_t
        L.fgattn_rope_table.argtypes = [ctypes.POINTER(FgattnRopeAxis), ctypes.c_int, ctypes.c_double, vp, vp, vp]
        L.fgattn_rope_table.restype = ctypes.c_int
        L.fgattn_rope_forward.argtypes = [vp] * 6 + [ctypes.c_int32, vp, rp, vp, vp, vp]
        L.fgattn_rope_forward.restype = ctypes.c_int
        L.fgattn_rope_workspace_bytes.argtypes = [rp]
        L.fgattn_rope_workspace_bytes.restype = sz
        L.fgattn_rope_backward.argtypes = [vp] * 6 + [ctypes.c_int32, vp, rp] + [vp] * 7 + [sz, vp]
        L.fgattn_rope_backward.restype = ctypes.c_int
        L.fgattn_cross_workspace_bytes.argtypes = [xp]
        L.fgattn_cross_workspace_bytes.restype = sz
        L.fgattn_cross_forward.argtypes = [vp] * 5 + [xp, vp, vp, vp, sz, vp]
        L.fgattn_cross_forward.restype = ctypes.c_int
        L.fgattn_cross_backward_workspace_bytes.argtypes = [xp]
        L.fgattn_cross_backward_workspace_bytes.restype = sz
        L.fgattn_cross_backward.argtypes = [vp] * 8 + [xp] + [vp] * 4 + [sz, vp]
        L.fgattn_cross_backward.restype = ctypes.c_int
        L.fgattn_grid_size.argtypes = [pp]
        L.fgattn_grid_size.restype = ctypes.c_int
        L.fgattn_strerror.argtypes = [ctypes.c_int]
        L.fgattn_strerror.restype = ctypes.c_char_p
        _lib = L
    return _lib


def fgattn_strerror(code):
    return lib().fgattn_strerror(int(code)).decode()


def make_params(q, k, v, out, M, N, scale, flags=0):
    """fgattn_params for [B, H, L, d] tensors (any strides with a contiguous last dim)."""
    B, H, L, d = q.shape
    for t in (q, k, v, out):
        assert t.dim() == 4 and t.stride(3) == 1
    p = FgattnParams(B, H, L, d, M, N,
                     q.stride(0), q.stride(1), q.stride(2), k.stride(0), k.stride(1), k.stride(2),
                     v.stride(0), v.stride(1), v.stride(2), out.stride(0), out.stride(1), out.stride(2),
                     float(scale), int(flags))
    return p


def fgattn_workspace_bytes(params):
    return int(lib().fgattn_workspace_bytes(ctypes.byref(params)))


def _stream_ptr(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _check(rc):
    if rc != 0:
        raise FgattnError(rc)


def fgattn_forward(q, k, v, mask_indptr, mask_indices, params, out, lse, workspace, stream=None):
    """Enqueue the sparse forward pass on `stream` (default: torch's current stream)."""
    _check(lib().fgattn_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), mask_indptr.data_ptr(),
                                mask_indices.data_ptr(), ctypes.byref(params), out.data_ptr(), lse.data_ptr(),
                                workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                _stream_ptr(stream)))


def fgattn_forward_static(q, k, v, mask_indptr, mask_indices, params, out, lse, stream=None):
    """The sparse forward pass without a workspace argument (scratch inside the library's device image)."""
    _check(lib().fgattn_forward_static(q.data_ptr(), k.data_ptr(), v.data_ptr(), mask_indptr.data_ptr(),
                                       mask_indices.data_ptr(), ctypes.byref(params), out.data_ptr(), lse.data_ptr(),
                                       _stream_ptr(stream)))


PART_GATHER, PART_COMPUTE, PART_GATHER_RING3, PART_GATHER_ONE_WG = 1, 2, 3, 4


def fgattn_forward_grouped(q, k, v, group_tiles, union_indptr, union_indices, union_members, params, out, lse, workspace,
                           stream=None):
    """Sparse forward pass over grouped query tiles (union key lists with per-member masks)."""
    _check(lib().fgattn_forward_grouped(q.data_ptr(), k.data_ptr(), v.data_ptr(), group_tiles.data_ptr(),
                                        union_indptr.data_ptr(), union_indices.data_ptr(), union_members.data_ptr(),
                                        ctypes.byref(params), out.data_ptr(), lse.data_ptr(), workspace.data_ptr(),
                                        workspace.numel() * workspace.element_size(), _stream_ptr(stream)))


def fgattn_forward_part(q, k, v, mask_indptr, mask_indices, params, out, lse, workspace, part, stream=None):
    """Measurement aid: one half of the forward kernel (results in out / lse are meaningless)."""
    _check(lib().fgattn_forward_part(q.data_ptr(), k.data_ptr(), v.data_ptr(), mask_indptr.data_ptr(),
                                     mask_indices.data_ptr(), ctypes.byref(params), out.data_ptr(), lse.data_ptr(),
                                     workspace.data_ptr(), workspace.numel() * workspace.element_size(), int(part),
                                     _stream_ptr(stream)))


def fgattn_issue_probe(other_valu_per_16_mfma, iters, scratch, stream=None):
    """Measurement aid: enqueues the instruction-issue probe; returns the MFMA FLOP count of the launch."""
    flop = ctypes.c_double(0.0)
    _check(lib().fgattn_issue_probe(int(other_valu_per_16_mfma), int(iters), scratch.data_ptr(),
                                    scratch.numel() * scratch.element_size(), ctypes.byref(flop), _stream_ptr(stream)))
    return flop.value


def fgattn_dense_forward(q, k, v, params, out, lse, workspace, stream=None):
    _check(lib().fgattn_dense_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), ctypes.byref(params),
                                      out.data_ptr(), lse.data_ptr(), workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(), _stream_ptr(stream)))


def fgattn_mask_workspace_bytes(params):
    return int(lib().fgattn_mask_workspace_bytes(ctypes.byref(params)))


def fgattn_mask_select(q, k, params, top_p, mask_indptr, workspace, stream=None):
    """Top-p mask, first half: fills mask_indptr (device int64) and the per-block cuts in `workspace`."""
    _check(lib().fgattn_mask_select(q.data_ptr(), k.data_ptr(), ctypes.byref(params), float(top_p), mask_indptr.data_ptr(),
                                    workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(stream)))


def fgattn_mask_emit(params, mask_indptr, mask_indices, workspace, stream=None):
    """Top-p mask, second half: writes the kept key-block ids (ascending per query block) into mask_indices."""
    _check(lib().fgattn_mask_emit(ctypes.byref(params), mask_indptr.data_ptr(), mask_indices.data_ptr(),
                                  int(mask_indices.numel()), workspace.data_ptr(),
                                  workspace.numel() * workspace.element_size(), _stream_ptr(stream)))


GROUP_CONSECUTIVE, GROUP_XOR = 0, 1


def fgattn_group_workspace_bytes(params, mode):
    return int(lib().fgattn_group_workspace_bytes(ctypes.byref(params), int(mode)))


def fgattn_group_select(mask_indptr, mask_indices, params, mode, group_tiles, union_indptr, workspace, stream=None):
    """Query-tile grouping, first half: fills group_tiles and union_indptr (device tensors)."""
    _check(lib().fgattn_group_select(mask_indptr.data_ptr(), mask_indices.data_ptr(), ctypes.byref(params), int(mode),
                                     group_tiles.data_ptr(), union_indptr.data_ptr(), workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(), _stream_ptr(stream)))


def fgattn_group_emit(params, mode, group_tiles, union_indptr, union_indices, union_members, workspace, stream=None):
    """Query-tile grouping, second half: fills union_indices / union_members."""
    _check(lib().fgattn_group_emit(ctypes.byref(params), int(mode), group_tiles.data_ptr(), union_indptr.data_ptr(),
                                   union_indices.data_ptr(), union_members.data_ptr(), int(union_indices.numel()),
                                   workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                   _stream_ptr(stream)))


def fgattn_plan(mask_indptr, params, workspace, stream=None):
    _check(lib().fgattn_plan(mask_indptr.data_ptr(), ctypes.byref(params), workspace.data_ptr(),
                             workspace.numel() * workspace.element_size(), _stream_ptr(stream)))


def fgattn_validate_mask(mask_indptr, mask_indices, params, workspace, stream=None):
    """Returns 0 or E_MASK (synchronous)."""
    rc = lib().fgattn_validate_mask(mask_indptr.data_ptr(), mask_indices.data_ptr(), ctypes.byref(params),
                                    workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                    _stream_ptr(stream))
    if rc not in (0, E_MASK):
        raise FgattnError(rc)
    return rc


def fgattn_grid_size(params):
    return int(lib().fgattn_grid_size(ctypes.byref(params)))


# ---- rotary positions, norms of queries and keys, cross attention ----
# These bindings also compare every tensor with the params (the C ABI sees pointers only) and run on the tensors' own device,
# whichever is current.  Small calls take as long as this file does, so the comparisons are made in one loop and the
# params are packed as bytes.

_ROPE_FIELDS, _CROSS_FIELDS = struct.Struct("9if12q"), struct.Struct("6i24qfi")


def _refuse(code):
    raise FgattnError(code)


def _addresses(device, tensors):
    """Addresses of tensors (None: NULL) given as (tensor, dtype, shape, strides or None where it has to be contiguous), all on device
    number `device`."""
    found = []
    for t, dtype, shape, strides in tensors:
        if t is None:
            found.append(None)
            continue
        if t.dtype is not dtype or t.get_device() != device or t.shape != shape or \
                (not t.is_contiguous() if strides is None else t.stride() != strides):
            _compare(t, device, dtype, shape, strides)
        found.append(t.data_ptr())
    return found


def _compare(t, device, dtype, shape, strides):
    """Refuses a tensor that differs from what the params say (the stride of a dimension of one does not matter)."""
    if t.get_device() != device:
        _refuse(E_DEVICE)
    if t.dtype is not dtype:
        _refuse(E_DTYPE)
    if t.shape != shape or (strides is None and not t.is_contiguous()):
        _refuse(E_SHAPE)
    if strides is not None and any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), strides)):
        _refuse(E_STRIDE)


def _launch(call, args, device, stream, tensors):
    """call(*args, stream) with device number `device` current; a stream of another device is refused, and the allocator learns
    of tensors that are used on a stream other than the current one."""
    import torch
    if device < 0:
        _refuse(E_DEVICE)
    if device != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _launch(call, args, device, stream, tensors)
    if stream is None:
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # (a pointer at a tenth of a Stream object's cost)
        at = torch.cuda.current_stream().cuda_stream if raw is None else raw(device)
    else:
        at = stream.cuda_stream
        if stream.device.index != device:
            _refuse(E_DEVICE)
        if stream != torch.cuda.current_stream():
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)
    rc = call(*args, at)
    if rc != 0:
        raise FgattnError(rc)


def fgattn_rope_table(axes, cos, sin, mscale=1.0, stream=None):
    """Fills cos and sin (fp32 [rows, pairs]) with the angles of a token grid.  axes: one to three tuples (size, pairs, theta,
    offset, step, factor, original, beta_fast, beta_slow), later ones optional from `offset` on (0, 1, 1, 0, 32, 1)."""
    import torch
    n = len(axes)
    if not 1 <= n <= 3:
        _refuse(E_SHAPE)
    rows, pairs, table = 1, 0, []
    for x in axes:
        if not 3 <= len(x) <= 9:
            _refuse(E_SHAPE)
        rows, pairs = rows * x[0], pairs + x[1]
        table.append(FgattnRopeAxis(*x, *(0.0, 1.0, 1.0, 0.0, 32.0, 1.0)[len(x) - 3:]))
    device, f32, shape = cos.get_device(), torch.float32, (rows, pairs)
    c, s = _addresses(device, ((cos, f32, shape, None), (sin, f32, shape, None)))
    _launch(lib().fgattn_rope_table, ((FgattnRopeAxis * n)(*table), n, mscale, c, s), device, stream, (cos, sin))


_DTYPES = {}


def _dtype_code(dtype):
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32})
    code = _DTYPES.get(dtype)
    return _refuse(E_DTYPE) if code is None else code


def make_rope_params(q, k, q_out, k_out, rot_dims, layout=ROPE_INTERLEAVED, eps=1e-6, flags=FLAG_ROPE_NORM):
    """fgattn_rope_params for [B, H, L, d] tensors (any strides with a contiguous last dim); k and k_out may be None.  For the
    backward call q_out and k_out are the gradients that come in, and dq and dk have the strides of q and k."""
    shape, Hk = q.shape, 0
    if len(shape) != 4 or q_out.shape != shape or (k is None) != (k_out is None):
        _refuse(E_SHAPE)
    B, Hq, L, d = shape
    a, c = q.stride(), q_out.stride()
    b = e = (0, 0, 0, 1)
    if k is not None:
        shape = k.shape
        if len(shape) != 4 or shape[0] != B or shape[2] != L or shape[3] != d or k_out.shape != shape:
            _refuse(E_SHAPE)
        Hk, b, e = shape[1], k.stride(), k_out.stride()
    if a[3] != 1 or b[3] != 1 or c[3] != 1 or e[3] != 1:
        _refuse(E_STRIDE)
    return FgattnRopeParams.from_buffer_copy(_ROPE_FIELDS.pack(
        B, Hq, Hk, L, d, rot_dims, layout, _dtype_code(q.dtype), flags, eps, *a[:3], *b[:3], *c[:3], *e[:3]))


def fgattn_rope_workspace_bytes(params):
    return int(lib().fgattn_rope_workspace_bytes(ctypes.byref(params)))


def _rope_operands(params, q, k, cos, sin, positions, q_weight, k_weight, results, backward, dtype, device):
    """Addresses of q, k, weights, cos, sin, positions and `results` (forward: q_out, k_out; backward: dq_out, dk_out, dq, dk), and the
    table's rows."""
    import torch
    B, Hq, Hk, L, d, rot, _, code, flags, _, *s = _ROPE_FIELDS.unpack_from(params)
    if _dtype_code(dtype) != code:
        _refuse(E_DTYPE)
    if (cos is None) != (sin is None):
        _refuse(E_NULL)
    f32 = torch.float32
    w_type = f32 if flags & FLAG_ROPE_WEIGHT_FP32 else dtype
    rows = 0 if cos is None else cos.shape[0]
    if rows > 0x7FFFFFFF:   # (the call takes the count in 32 bits)
        _refuse(E_SHAPE)
    of_q, of_k, weight, table = (B, Hq, L, d), (B, Hk, L, d), (d,), (rows, rot // 2)
    sq, sk = (s[0], s[1], s[2], 1), (s[3], s[4], s[5], 1)
    given = [(q, dtype, of_q, sq), (k, dtype, of_k, sk), (q_weight, w_type, weight, None), (k_weight, w_type, weight, None),
             (cos, f32, table, None), (sin, f32, table, None), (positions, torch.int32, (B, L), None),
             (results[0], dtype, of_q, (s[6], s[7], s[8], 1)), (results[1], dtype, of_k, (s[9], s[10], s[11], 1))]
    if backward:
        given += [(results[2], dtype, of_q, sq), (results[3], dtype, of_k, sk)]
    return _addresses(device, given), rows


def fgattn_rope_forward(q, k, params, q_out, k_out, cos=None, sin=None, positions=None, q_weight=None, k_weight=None, stream=None):
    """Queries and keys normed per head and turned by their positions (see include/fgattn.h)."""
    device = q.get_device()
    a, rows = _rope_operands(params, q, k, cos, sin, positions, q_weight, k_weight, (q_out, k_out), False, q.dtype, device)
    _launch(lib().fgattn_rope_forward, (*a[:6], rows, a[6], ctypes.byref(params), a[7], a[8]), device, stream,
            (q, k, q_out, k_out, cos, sin, positions, q_weight, k_weight))


def fgattn_rope_backward(q, k, params, dq_out, dk_out, dq, dk, cos=None, sin=None, positions=None, q_weight=None, k_weight=None,
                         dq_weight=None, dk_weight=None, workspace=None, stream=None):
    """Gradients of fgattn_rope_forward: dq, dk and, where given, dq_weight and dk_weight (fp32).  q and k may be None without
    FLAG_ROPE_NORM."""
    import torch
    device, f32, weight = dq_out.get_device(), torch.float32, (params.d,)
    a, rows = _rope_operands(params, q, k, cos, sin, positions, q_weight, k_weight, (dq_out, dk_out, dq, dk), True, dq_out.dtype,
                             device)
    dw = _addresses(device, ((dq_weight, f32, weight, None), (dk_weight, f32, weight, None)))
    _launch(lib().fgattn_rope_backward, (*a[:6], rows, a[6], ctypes.byref(params), *a[7:], *dw, *_scratch(workspace, device)), device, stream,
            (q, k, dq_out, dk_out, dq, dk, cos, sin, positions, q_weight, k_weight, dq_weight, dk_weight, workspace))


def _scratch(workspace, device):
    if workspace is None:
        return None, 0
    if workspace.get_device() != device:
        _refuse(E_DEVICE)
    if not workspace.is_contiguous():   # (elements that share memory do not count as bytes)
        _refuse(E_SHAPE)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def make_cross_params(q, k, v, out, scale, dout=None, dq=None, dk=None, dv=None):
    """fgattn_cross_params for q, out [B, H, Lq, d] and k, v [B, Hkv, Lk, d] (any strides with a contiguous last dim); for the
    backward call also the incoming gradient and the three gradients."""
    of_q, of_k = q.shape, k.shape
    if len(of_q) != 4 or len(of_k) != 4 or of_k[0] != of_q[0] or of_k[3] != of_q[3]:
        _refuse(E_SHAPE)
    strides = []
    for t, shape in ((q, of_q), (k, of_k), (v, of_k), (out, of_q), (dout, of_q), (dq, of_q), (dk, of_k), (dv, of_k)):
        if t is None:
            strides += (0, 0, 0)
            continue
        if t.shape != shape:
            _refuse(E_SHAPE)
        s = t.stride()
        if s[3] != 1:
            _refuse(E_STRIDE)
        strides += s[:3]
    return FgattnCrossParams.from_buffer_copy(_CROSS_FIELDS.pack(of_q[0], of_q[1], of_k[1], of_q[2], of_k[2], of_q[3], *strides, scale, 0))


def fgattn_cross_workspace_bytes(params):
    return int(lib().fgattn_cross_workspace_bytes(ctypes.byref(params)))


def fgattn_cross_backward_workspace_bytes(params):
    return int(lib().fgattn_cross_backward_workspace_bytes(ctypes.byref(params)))


def fgattn_cross_forward(q, k, v, params, out, lse, workspace=None, q_lens=None, k_lens=None, stream=None):
    """Attention of q's tokens to k and v, another sequence with its own lengths (see include/fgattn.h)."""
    import torch
    device, bf16, i32 = q.get_device(), torch.bfloat16, torch.int32
    B, H, Hkv, Lq, Lk, d, *s = _CROSS_FIELDS.unpack_from(params)
    of_q, of_k, lens = (B, H, Lq, d), (B, Hkv, Lk, d), (B,)
    a = _addresses(device, ((q, bf16, of_q, (s[0], s[1], s[2], 1)),
                            (k, bf16, of_k, (s[3], s[4], s[5], 1)),
                            (v, bf16, of_k, (s[6], s[7], s[8], 1)),
                            (q_lens, i32, lens, None), (k_lens, i32, lens, None),
                            (out, bf16, of_q, (s[9], s[10], s[11], 1)),
                            (lse, torch.float32, of_q[:3], None)))
    _launch(lib().fgattn_cross_forward, (*a[:5], ctypes.byref(params), a[5], a[6], *_scratch(workspace, device)), device, stream,
            (q, k, v, out, lse, workspace, q_lens, k_lens))


def fgattn_cross_backward(q, k, v, out, lse, dout, params, dq, dk, dv, workspace, q_lens=None, k_lens=None, stream=None):
    """Gradients of fgattn_cross_forward with respect to q, k and v, from its inputs and results and the gradient of out."""
    import torch
    device, bf16, i32 = q.get_device(), torch.bfloat16, torch.int32
    B, H, Hkv, Lq, Lk, d, *s = _CROSS_FIELDS.unpack_from(params)
    of_q, of_k, lens = (B, H, Lq, d), (B, Hkv, Lk, d), (B,)
    a = _addresses(device, ((q, bf16, of_q, (s[0], s[1], s[2], 1)),
                            (k, bf16, of_k, (s[3], s[4], s[5], 1)),
                            (v, bf16, of_k, (s[6], s[7], s[8], 1)),
                            (out, bf16, of_q, (s[9], s[10], s[11], 1)),
                            (lse, torch.float32, of_q[:3], None),
                            (dout, bf16, of_q, (s[12], s[13], s[14], 1)),
                            (q_lens, i32, lens, None), (k_lens, i32, lens, None),
                            (dq, bf16, of_q, (s[15], s[16], s[17], 1)),
                            (dk, bf16, of_k, (s[18], s[19], s[20], 1)),
                            (dv, bf16, of_k, (s[21], s[22], s[23], 1))))
    _launch(lib().fgattn_cross_backward, (*a[:8], ctypes.byref(params), *a[8:], *_scratch(workspace, device)), device, stream,
            (q, k, v, out, lse, dout, dq, dk, dv, workspace, q_lens, k_lens))
