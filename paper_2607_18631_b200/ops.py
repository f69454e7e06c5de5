"""The operators of one decode layer (include/planfront_ops.h): argument marshalling only.

What the serving model prices per layer and step -- attention over the cached keys and values, the experts of a few
tokens -- and the norm and the cache append that go with it, as hand-written CUDA on the current device.  Function names
mirror the C ABI.
Tensors stay with the caller; outputs and workspaces that are not passed in come from PyTorch's allocator, on the
stream the call runs on (`stream`, or the current one).  There is no CPU path.

`stream`: the call is enqueued there, and the tensors given to it are marked as used there (they may be dropped at once).
That they are ready on that stream, and that its results are not used elsewhere before they are, is up to the caller.

8-bit tensors are torch.float8_e4m3fn.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import math

from .binding import PF_EINVAL, PF_ERANGE, PF_OK, PlanfrontError, _check, _torch, i32, i64, load_library

EXPORTS = ("pf_add_rms_norm", "pf_kv_append", "pf_decode_attention_workspace", "pf_decode_attention",
           "pf_moe_packed_bytes", "pf_moe_pack", "pf_moe_workspace", "pf_moe_forward")
DT_BF16, DT_F16, DT_F32, DT_E4M3 = 0, 1, 2, 3
SCALE_GROUP = 128
MOE_MAX_TOKENS = 512

_vp, _sz = C.c_void_p, C.c_size_t


class PfKvCache(C.Structure):
    _fields_ = [(n, i32) for n in ("n_pages", "n_kv", "page", "hd")] + [(n, _vp) for n in ("d_k", "d_v", "d_k_scale", "d_v_scale")]


class PfMoe(C.Structure):
    _fields_ = [(n, i32) for n in ("H", "F", "n_experts", "first", "n_local", "n_shared", "top_k", "wtype")]


_ready = None
_dtypes = None
_attention_workspace = {}


def _lib():
    """The library with this header's signatures declared, and torch; raises without a CUDA device."""
    global _ready, _dtypes
    if _ready is not None:
        return _ready
    torch = _torch()
    L = declare(load_library())
    _dtypes = {torch.bfloat16: DT_BF16, torch.float16: DT_F16, torch.float32: DT_F32}
    _ready = L, torch
    return _ready


def declare(L):
    """Declare the argument types of planfront_ops.h on a loaded library."""
    cache, moe = C.POINTER(PfKvCache), C.POINTER(PfMoe)
    f32 = C.c_float
    for name, args in (("pf_add_rms_norm", [i32, i64, i32, _vp, i64, _vp, i64, _vp, f32, i32, _vp, i64, _vp, i64, _vp, _vp, _vp]),
                       ("pf_kv_append", [cache, i32, i32, i64, i32, _vp, i64, _vp, i64, _vp, _vp, _vp, i32, _vp]),
                       ("pf_decode_attention", [cache, i32, i32, i32, _vp, i64, _vp, _vp, i32, f32, _vp, i64, _vp, _vp, _sz, _vp]),
                       ("pf_moe_pack", [moe] + [_vp] * 8),
                       ("pf_moe_forward", [moe, i32, _vp, i64] + [_vp] * 8 + [_vp, _sz, _vp])):
        fn = getattr(L, name)
        fn.restype, fn.argtypes = C.c_int, args
    for name, args in (("pf_decode_attention_workspace", [cache, i32, i32]), ("pf_moe_packed_bytes", [moe]), ("pf_moe_workspace", [moe, i32])):
        fn = getattr(L, name)
        fn.restype, fn.argtypes = _sz, args
    return L


def _refuse(what: str):
    raise PlanfrontError(PF_EINVAL, what)


def _cut_off(what):
    """For counts that do not fit the C call's 32-bit arguments: ctypes would cut them off without a word."""
    raise PlanfrontError(PF_ERANGE, f"{what}: a count does not fit 32 bits")


def _on_device(torch, what, *tensors):
    """Every tensor on the current CUDA device; returns its index."""
    dev = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            _refuse(f"{what}: a tensor is not on the current CUDA device (cuda:{dev})")
    return dev


def _stream(torch, dev, stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        _refuse(f"the stream belongs to cuda:{stream.device_index}, the current device is cuda:{dev}")
    return stream.cuda_stream


def _used_on(torch, stream, *tensors):
    """A stream of the current device; the allocator is not to hand these tensors' memory out again before the work now enqueued there is done."""
    _stream(torch, torch._C._cuda_getDevice(), stream)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


def _like(torch, t, dtype=None):
    """A new contiguous tensor of t's shape."""
    if t.is_contiguous():
        return torch.empty_like(t) if dtype is None else torch.empty_like(t, dtype=dtype)
    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


def _matrix(torch, rows, cols, dtype, device):
    return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)      # the quickest way to a new tensor


def _rows(t, what, width):
    """A 2-D tensor with contiguous rows of `width`; returns its row stride in elements."""
    if t.dim() != 2 or t.shape[1] != width or (t.stride(1) != 1 and width > 1):
        _refuse(f"{what}: expected rows of {width} contiguous elements, got shape {tuple(t.shape)}, strides {t.stride()}")
    return t.stride(0) if t.shape[0] > 1 else width      # below the width (an expanded row): the library refuses it


def _work_bytes(t, what):
    """Size of a caller's workspace: what lies behind data_ptr() (an expanded tensor has fewer bytes than elements)."""
    if not t.is_contiguous():
        _refuse(f"{what}: the workspace has to be contiguous")
    return t.numel() * t.element_size()


def _ptr(t):
    return None if t is None else t.data_ptr()


def pf_add_rms_norm(x, residual=None, weight=None, *, eps: float = 1e-6, group: int = SCALE_GROUP, y: bool = False, q: bool = True,
                    sum_out=None, stream=None) -> dict:
    """a = x + residual; y = a / sqrt(mean a^2 + eps) * weight; 8-bit form of y with a scale per `group` elements (128, or 0: per row).

    x, residual: [rows, H] bf16, fp16 or fp32, rows contiguous.  Returns a dict: "sum" (a rounded to x's type; where a
    residual is given; `sum_out` to write it in place, x and residual themselves allowed), "y" if asked for, and "q" (e4m3) with "scale" (fp32)
    unless q=False."""
    L, torch = _ready or _lib()
    if stream is not None:      # the caching allocator hands memory out per stream
        _used_on(torch, stream, x, residual, weight, sum_out)
        with torch.cuda.stream(stream):
            return pf_add_rms_norm(x, residual, weight, eps=eps, group=group, y=y, q=q, sum_out=sum_out)
    what = "pf_add_rms_norm"
    dev = _on_device(torch, what, x, residual, weight, sum_out)
    dt = _dtypes.get(x.dtype)
    if dt is None:
        _refuse(f"{what}: {x.dtype} is not supported")
    if x.dim() != 2:
        _refuse(f"{what}: x has to be [rows, H]")
    rows, H = shape = x.shape
    if group >> 31 or H >> 31:
        _cut_off(what)
    if H < 1:
        raise PlanfrontError(PF_ERANGE, f"{what}: rows without elements")
    if weight is not None and (weight.dtype != x.dtype or weight.shape != (H,) or not weight.is_contiguous()):
        _refuse(f"{what}: weight has to be a contiguous [{H}] of x's type")
    out = {}
    s_ptr = r_ptr = y_ptr = q_ptr = scale_ptr = None
    s_stride = r_stride = 0
    if residual is not None:
        if residual.dtype != x.dtype or residual.shape != shape:
            _refuse(f"{what}: residual has x's shape and type")
        r_ptr, r_stride = residual.data_ptr(), _rows(residual, what, H)
    if residual is not None or sum_out is not None:
        if sum_out is not None and (sum_out.dtype != x.dtype or sum_out.shape != shape):
            _refuse(f"{what}: sum_out has x's shape and type")
        out["sum"] = s = _like(torch, x) if sum_out is None else sum_out
        s_ptr, s_stride = s.data_ptr(), H if sum_out is None else _rows(s, what, H)
    if y:
        out["y"] = t = _like(torch, x)
        y_ptr = t.data_ptr()
    if q:
        out["q"] = t = _like(torch, x, torch.float8_e4m3fn)
        q_ptr = t.data_ptr()
        out["scale"] = t = _matrix(torch, rows, -(-H // group) if group else 1, torch.float32, x.device)
        scale_ptr = t.data_ptr()
    status = L.pf_add_rms_norm(dt, rows, H, x.data_ptr(), _rows(x, what, H), r_ptr, r_stride, None if weight is None else weight.data_ptr(), eps, group,
                               s_ptr, s_stride, y_ptr, H, q_ptr, scale_ptr, _stream(torch, dev, None))
    if status != PF_OK:
        _check(status, what)
    return out


def _cache(torch, what, k_cache, v_cache, k_scale, v_scale):
    shape = k_cache.shape
    if len(shape) != 4 or shape != v_cache.shape or k_scale.shape != shape[:2] or v_scale.shape != shape[:2]:
        _refuse(f"{what}: caches are [pages, kv heads, page, head_dim], scales [pages, kv heads]")
    f8, f32 = torch.float8_e4m3fn, torch.float32
    if k_cache.dtype != f8 or v_cache.dtype != f8 or k_scale.dtype != f32 or v_scale.dtype != f32:
        _refuse(f"{what}: caches are float8_e4m3fn, scales float32")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()):
        _refuse(f"{what}: the cache has to be contiguous")
    return PfKvCache(*shape, k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())


def _heads(t, what, heads, hd):
    """[rows, heads, hd], contiguous within a row; returns the row stride in elements."""
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != hd or t.stride(2) != 1 or (heads > 1 and t.stride(1) != hd):
        _refuse(f"{what}: expected [rows, {heads}, {hd}] with contiguous rows, got shape {tuple(t.shape)}, strides {t.stride()}")
    return t.stride(0) if t.shape[0] > 1 else heads * hd


def _int32(torch, what, t, dims):
    if t.dtype != torch.int32 or t.dim() != dims or not t.is_contiguous():
        _refuse(f"{what}: lengths, offsets and tables are contiguous int32")
    return t.data_ptr()


def pf_kv_append(k_cache, v_cache, k_scale, v_scale, k, v, cu_new, lengths, table, *, max_new: int, stream=None) -> None:
    """Write new tokens into the paged 8-bit cache, in place.

    k_cache, v_cache: [pages, kv_heads, page, head_dim] float8_e4m3fn; k_scale, v_scale: [pages, kv_heads] fp32.
    k, v: [new tokens, kv_heads, head_dim] bf16 or fp16; tokens cu_new[b] .. cu_new[b + 1] - 1 go behind the lengths[b] cached
    ones of sequence b, whose pages are table[b].  max_new: the most tokens a sequence gets.  `lengths` is not advanced."""
    L, torch = _ready or _lib()
    what = "pf_kv_append"
    dev = _on_device(torch, what, k_cache, v_cache, k_scale, v_scale, k, v, cu_new, lengths, table)
    c = _cache(torch, what, k_cache, v_cache, k_scale, v_scale)
    dt = _dtypes.get(k.dtype)
    if dt is None or v.dtype != k.dtype or v.shape != k.shape:
        _refuse(f"{what}: k and v have the same shape and type (bf16 or fp16)")
    n_seq = lengths.shape[0]
    if cu_new.shape != (n_seq + 1,) or table.dim() != 2 or table.shape[0] != n_seq:
        _refuse(f"{what}: cu_new is [sequences + 1], table [sequences, columns]")
    if (n_seq | max_new | table.shape[1]) >> 31:
        _cut_off(what)
    if stream is not None:
        _used_on(torch, stream, k_cache, v_cache, k_scale, v_scale, k, v, cu_new, lengths, table)
    status = L.pf_kv_append(c, dt, n_seq, k.shape[0], max_new, k.data_ptr(), _heads(k, what, c.n_kv, c.hd), v.data_ptr(), _heads(v, what, c.n_kv, c.hd),
                            _int32(torch, what, cu_new, 1), _int32(torch, what, lengths, 1), _int32(torch, what, table, 2), table.shape[1],
                            _stream(torch, dev, stream))
    if status != PF_OK:
        _check(status, what)


def pf_decode_attention(q, k_cache, v_cache, k_scale, v_scale, lengths, table, *, sm_scale: float | None = None, lse: bool = False, out=None,
                        workspace=None, stream=None) -> dict:
    """Attention of one query token per sequence over its cached tokens.

    q: [sequences, heads, head_dim] bf16 or fp16; head h reads key / value head h // (heads // kv_heads).  sm_scale: 1 / sqrt(head_dim)
    if None.  Returns {"out": like q} and, if asked for, {"lse": [sequences, heads] fp32}.  A sequence without tokens gives
    zeros and -inf."""
    L, torch = _ready or _lib()
    if stream is not None:
        _used_on(torch, stream, q, k_cache, v_cache, k_scale, v_scale, lengths, table, out, workspace)
        with torch.cuda.stream(stream):
            return pf_decode_attention(q, k_cache, v_cache, k_scale, v_scale, lengths, table, sm_scale=sm_scale, lse=lse, out=out, workspace=workspace)
    what = "pf_decode_attention"
    dev = _on_device(torch, what, q, k_cache, v_cache, k_scale, v_scale, lengths, table, out, workspace)
    c = _cache(torch, what, k_cache, v_cache, k_scale, v_scale)
    dt = _dtypes.get(q.dtype)
    shape = q.shape
    if dt is None or len(shape) != 3:
        _refuse(f"{what}: q has to be [sequences, heads, head_dim] of bf16 or fp16")
    n_seq, heads, _ = shape
    hd = c.hd
    if lengths.shape != (n_seq,) or table.dim() != 2 or table.shape[0] != n_seq:
        _refuse(f"{what}: lengths is [sequences], table [sequences, columns]")
    if (n_seq | heads | table.shape[1]) >> 31:
        _cut_off(what)
    res = {}
    if out is None:
        out = _like(torch, q)
    elif out.dtype != q.dtype or out.shape != shape:
        _refuse(f"{what}: out has q's shape and type")
    res["out"] = out
    lse_ptr = None
    if lse:
        res["lse"] = t = _matrix(torch, n_seq, heads, torch.float32, q.device)
        lse_ptr = t.data_ptr()
    if workspace is None:
        size = _attention_workspace.get((dev, hd))
        if size is None:        # depends on the device and the head size only
            size = _attention_workspace[dev, hd] = L.pf_decode_attention_workspace(c, max(n_seq, 1), max(heads, 1))
        workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
        size_ws = size
    else:
        size_ws = _work_bytes(workspace, what)
    status = L.pf_decode_attention(c, dt, n_seq, heads, q.data_ptr(), _heads(q, what, heads, hd), _int32(torch, what, lengths, 1),
                                   _int32(torch, what, table, 2), table.shape[1], 1.0 / math.sqrt(hd) if sm_scale is None else sm_scale,
                                   out.data_ptr(), _heads(out, what, heads, hd), lse_ptr, workspace.data_ptr(), size_ws, _stream(torch, dev, None))
    if status != PF_OK:
        _check(status, what)
    return res


class MoeLayer:
    """A mixture-of-experts layer's weights, laid out for few-token calls (pf_moe_pack), and its forward (pf_moe_forward).

    router: [experts, H] bf16.  gate, up: [local + shared, F, H], down: [local + shared, H, F], bf16, or float8_e4m3fn with
    fp32 scales per 128 x 128 block ([local + shared, ceil(rows / 128), ceil(columns / 128)]).  Experts
    first_expert .. first_expert + local - 1 live here; the last n_shared of the weight tensors are taken by every token.
    The layer keeps a packed copy; gate, up, down and their scales may be dropped afterwards.  With `stream` the packing runs there, behind what
    the current stream holds already.  A forward on another stream than the packing's waits for the packing; one that is
    captured there cannot, so the packing has to be done by then (torch.cuda.graph synchronizes before it captures)."""

    def __init__(self, router, gate, up, down, *, top_k: int, first_expert: int = 0, n_shared: int = 0, gate_scale=None, up_scale=None,
                 down_scale=None, stream=None):
        L, torch = _lib()
        what = "MoeLayer"
        dev = _on_device(torch, what, router, gate, up, down, gate_scale, up_scale, down_scale)
        if router.dim() != 2 or router.dtype != torch.bfloat16 or not router.is_contiguous():
            _refuse(f"{what}: router has to be a contiguous [experts, H] of bf16")
        if gate.dim() != 3:
            _refuse(f"{what}: gate has to be [local + shared, F, H]")
        (E, H), (n, F) = router.shape, gate.shape[:2]
        if gate.shape != (n, F, H) or up.shape != gate.shape or down.shape != (n, H, F):
            _refuse(f"{what}: gate and up are [n, F, H], down [n, H, F]")
        wtype = {torch.bfloat16: DT_BF16, torch.float8_e4m3fn: DT_E4M3}.get(gate.dtype)
        if wtype is None or up.dtype != gate.dtype or down.dtype != gate.dtype:
            _refuse(f"{what}: weights are bf16 or float8_e4m3fn")
        if not (gate.is_contiguous() and up.is_contiguous() and down.is_contiguous()):
            _refuse(f"{what}: weights have to be contiguous")
        blocks = lambda r, c: (n, -(-r // SCALE_GROUP), -(-c // SCALE_GROUP))  # noqa: E731
        for t, shape in ((gate_scale, blocks(F, H)), (up_scale, blocks(F, H)), (down_scale, blocks(H, F))):
            if (t is None) != (wtype == DT_BF16):
                _refuse(f"{what}: block scales come with float8 weights, and only with them")
            if t is not None and (t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous()):
                _refuse(f"{what}: expected contiguous fp32 block scales of shape {shape}")
        if any(v >> 31 for v in (H, F, E, n, first_expert, n_shared, top_k)):
            _cut_off(what)
        self.m = PfMoe(H, F, E, first_expert, n - n_shared, n_shared, top_k, wtype)
        size = L.pf_moe_packed_bytes(self.m)
        if size == 0:
            _refuse(f"{what}: inconsistent sizes")
        self._L, self._torch, self._dev = L, torch, dev
        self.router = router
        if stream is not None:
            _used_on(torch, stream, gate, up, down, gate_scale, up_scale, down_scale)
            stream.wait_stream(torch.cuda.current_stream())
        with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
            self.packed = torch.empty(size, dtype=torch.uint8, device=router.device)
            self._home = _stream(torch, dev, None)         # the packing's stream
            _check(L.pf_moe_pack(self.m, gate.data_ptr(), up.data_ptr(), down.data_ptr(), _ptr(gate_scale), _ptr(up_scale), _ptr(down_scale),
                                 self.packed.data_ptr(), self._home), "pf_moe_pack")
            self._pack_done = torch.cuda.current_stream().record_event()
        self._router_ptr, self._packed_ptr, self._workspace, self._visited = router.data_ptr(), self.packed.data_ptr(), {}, set()

    def _visit(self, raw):
        """The first forward on a stream that is not the packing's: it comes after the packing, and the layer's memory is marked as
        used there."""
        torch = self._torch
        stream = torch.cuda.current_stream()
        _used_on(torch, stream, self.packed, self.router)
        if not torch.cuda.is_current_stream_capturing():
            stream.wait_event(self._pack_done)
            self._visited.add(raw)

    def forward(self, x, xq=None, xq_scale=None, *, out=None, status=None, workspace=None, stream=None) -> dict:
        """x: [tokens, H] bf16, 1 .. 512 tokens; xq, xq_scale: the same tokens in 8 bits from pf_add_rms_norm (group 128), which
        e4m3 weights then multiply (the router reads x).  Returns {"out": [tokens, H] bf16, "ids": [tokens, top_k] int32, "weights": [tokens, top_k]
        fp32}.  status: int32 tensor of one element, 0 after a complete call, 1 if a wait inside the kernel ran out; "out" is then NaN, with or
        without it."""
        L, torch, m = self._L, self._torch, self.m
        if stream is not None:
            _used_on(torch, stream, x, xq, xq_scale, out, status, workspace)
            with torch.cuda.stream(stream):
                return self.forward(x, xq, xq_scale, out=out, status=status, workspace=workspace)
        what = "pf_moe_forward"
        dev = _on_device(torch, what, x, xq, xq_scale, out, status, workspace, self.packed)
        if x.dtype != torch.bfloat16:
            _refuse(f"{what}: x has to be bf16")
        xs = _rows(x, what, m.H)
        T = x.shape[0]
        if T > MOE_MAX_TOKENS:
            raise PlanfrontError(PF_ERANGE, f"{what}: at most {MOE_MAX_TOKENS} tokens a call")
        if xq is not None and (xq_scale is None or xq.dtype != torch.float8_e4m3fn or xq.shape != x.shape or not xq.is_contiguous() or
                               xq_scale.dtype != torch.float32 or xq_scale.shape != (T, -(-m.H // SCALE_GROUP)) or not xq_scale.is_contiguous()):
            _refuse(f"{what}: xq is a contiguous float8_e4m3fn of x's shape, xq_scale [tokens, ceil(H / 128)] fp32")
        if out is not None and (out.dtype != x.dtype or out.shape != x.shape or not out.is_contiguous()):
            _refuse(f"{what}: out is a contiguous bf16 of x's shape")
        if status is not None and (status.dtype != torch.int32 or status.numel() != 1):
            _refuse(f"{what}: status is one int32")
        if out is None:
            out = _like(torch, x)
        ids, weights = (_matrix(torch, T, m.top_k, t, x.device) for t in (torch.int32, torch.float32))
        raw = _stream(torch, dev, None)
        if raw != self._home and raw not in self._visited:
            self._visit(raw)
        if workspace is None:
            size = self._workspace.get(T)
            if size is None:
                size = self._workspace[T] = L.pf_moe_workspace(m, T)
            workspace = torch.empty(size, dtype=torch.uint8, device=x.device)
        else:
            size = _work_bytes(workspace, what)
        status_of = L.pf_moe_forward(m, T, x.data_ptr(), xs, _ptr(xq), _ptr(xq_scale), self._router_ptr, self._packed_ptr, out.data_ptr(), ids.data_ptr(),
                                     weights.data_ptr(), _ptr(status), workspace.data_ptr(), size, raw)
        if status_of != PF_OK:
            _check(status_of, what)
        return {"out": out, "ids": ids, "weights": weights}
