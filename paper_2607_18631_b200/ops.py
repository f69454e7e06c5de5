"""The operators of one decode layer (include/planfront_ops.h): argument marshalling only.

What the serving model prices per layer and step -- the norm in front of it, attention over the cached keys and
values, the experts of a few tokens -- as hand-written CUDA on the current device.  Function names mirror the C ABI.
Tensors stay with the caller; outputs and workspaces that are not passed in come from PyTorch's allocator, on the
stream the call runs on (`stream`, or the current one).  There is no CPU path.

8-bit tensors are torch.float8_e4m3fn.
"""
from __future__ import annotations

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


def _on_device(torch, what, *tensors):
    """Every tensor on the current CUDA device; returns its index."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and (not t.is_cuda or t.device.index != dev):
            _refuse(f"{what}: a tensor is not on the current CUDA device (cuda:{dev})")
    return dev


def _stream(torch, dev, stream):
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(dev)


class _On:
    """Allocate on the given stream (the caching allocator hands memory out per stream); no-op for the current one."""

    def __new__(cls, torch, stream):
        import contextlib
        return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _rows(t, what, width):
    """A 2-D tensor with contiguous rows of `width`; returns its row stride in elements."""
    if t.dim() != 2 or t.shape[1] != width or (t.stride(1) != 1 and width > 1):
        _refuse(f"{what}: expected rows of {width} contiguous elements, got shape {tuple(t.shape)}, strides {t.stride()}")
    return max(t.stride(0), width) if t.shape[0] > 1 else width


def _ptr(t):
    return None if t is None else t.data_ptr()


def pf_add_rms_norm(x, residual=None, weight=None, *, eps: float = 1e-6, group: int = SCALE_GROUP, y: bool = False, q: bool = True,
                    sum_out=None, stream=None) -> dict:
    """a = x + residual; y = a / sqrt(mean a^2 + eps) * weight; 8-bit form of y with a scale per `group` elements (128, or 0: per row).

    x, residual: [rows, H] bf16, fp16 or fp32, rows contiguous.  Returns a dict: "sum" (a rounded to x's type; where a
    residual is given; `sum_out` to write it in place, x and residual themselves allowed), "y" if asked for, and "q" (e4m3) with "scale" (fp32)
    unless q=False."""
    L, torch = _lib()
    what = "pf_add_rms_norm"
    dev = _on_device(torch, what, x, residual, weight, sum_out)
    dt = _dtypes.get(x.dtype)
    if dt is None:
        _refuse(f"{what}: {x.dtype} is not supported")
    if x.dim() != 2:
        _refuse(f"{what}: x has to be [rows, H]")
    rows, H = x.shape
    if H < 1:
        raise PlanfrontError(PF_ERANGE, f"{what}: rows without elements")
    xs = _rows(x, what, H)
    for t in (residual, sum_out):
        if t is not None and (t.dtype != x.dtype or t.shape != x.shape):
            _refuse(f"{what}: residual and sum_out have x's shape and type")
    if weight is not None and (weight.dtype != x.dtype or weight.shape != (H,) or not weight.is_contiguous()):
        _refuse(f"{what}: weight has to be a contiguous [{H}] of x's type")
    out = {}
    with _On(torch, stream):
        if residual is not None or sum_out is not None:
            out["sum"] = torch.empty((rows, H), dtype=x.dtype, device=x.device) if sum_out is None else sum_out
        if y:
            out["y"] = torch.empty((rows, H), dtype=x.dtype, device=x.device)
        if q:
            out["q"] = torch.empty((rows, H), dtype=torch.float8_e4m3fn, device=x.device)
            out["scale"] = torch.empty((rows, -(-H // group) if group else 1), dtype=torch.float32, device=x.device)
    s = out.get("sum")
    _check(L.pf_add_rms_norm(dt, rows, H, x.data_ptr(), xs, _ptr(residual), 0 if residual is None else _rows(residual, what, H), _ptr(weight),
                             eps, group, _ptr(s), 0 if s is None else _rows(s, what, H), _ptr(out.get("y")), H, _ptr(out.get("q")),
                             _ptr(out.get("scale")), _stream(torch, dev, stream)), what)
    return out


def _cache(torch, what, k_cache, v_cache, k_scale, v_scale):
    if k_cache.dim() != 4 or k_cache.shape != v_cache.shape or k_scale.shape != k_cache.shape[:2] or v_scale.shape != k_cache.shape[:2]:
        _refuse(f"{what}: caches are [pages, kv heads, page, head_dim], scales [pages, kv heads]")
    if k_cache.dtype != torch.float8_e4m3fn or v_cache.dtype != torch.float8_e4m3fn or k_scale.dtype != torch.float32 or v_scale.dtype != torch.float32:
        _refuse(f"{what}: caches are float8_e4m3fn, scales float32")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()):
        _refuse(f"{what}: the cache has to be contiguous")
    n_pages, n_kv, page, hd = k_cache.shape
    return PfKvCache(n_pages, n_kv, page, hd, k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())


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
    L, torch = _lib()
    what = "pf_kv_append"
    dev = _on_device(torch, what, k_cache, v_cache, k_scale, v_scale, k, v, cu_new, lengths, table)
    c = _cache(torch, what, k_cache, v_cache, k_scale, v_scale)
    dt = _dtypes.get(k.dtype)
    if dt is None or v.dtype != k.dtype or v.shape != k.shape:
        _refuse(f"{what}: k and v have the same shape and type (bf16 or fp16)")
    n_seq = lengths.shape[0]
    if cu_new.shape != (n_seq + 1,) or table.dim() != 2 or table.shape[0] != n_seq:
        _refuse(f"{what}: cu_new is [sequences + 1], table [sequences, columns]")
    _check(L.pf_kv_append(c, dt, n_seq, k.shape[0], max_new, k.data_ptr(), _heads(k, what, c.n_kv, c.hd), v.data_ptr(), _heads(v, what, c.n_kv, c.hd),
                          _int32(torch, what, cu_new, 1), _int32(torch, what, lengths, 1), _int32(torch, what, table, 2), table.shape[1],
                          _stream(torch, dev, stream)), what)


def pf_decode_attention(q, k_cache, v_cache, k_scale, v_scale, lengths, table, *, sm_scale: float | None = None, lse: bool = False, out=None,
                        workspace=None, stream=None) -> dict:
    """Attention of one query token per sequence over its cached tokens.

    q: [sequences, heads, head_dim] bf16 or fp16; head h reads key / value head h // (heads // kv_heads).  sm_scale: 1 / sqrt(head_dim)
    if None.  Returns {"out": like q} and, if asked for, {"lse": [sequences, heads] fp32}.  A sequence without tokens gives
    zeros and -inf."""
    L, torch = _lib()
    what = "pf_decode_attention"
    dev = _on_device(torch, what, q, k_cache, v_cache, k_scale, v_scale, lengths, table, out, workspace)
    c = _cache(torch, what, k_cache, v_cache, k_scale, v_scale)
    dt = _dtypes.get(q.dtype)
    if dt is None or q.dim() != 3:
        _refuse(f"{what}: q has to be [sequences, heads, head_dim] of bf16 or fp16")
    n_seq, heads, hd = q.shape
    if lengths.shape != (n_seq,) or table.dim() != 2 or table.shape[0] != n_seq:
        _refuse(f"{what}: lengths is [sequences], table [sequences, columns]")
    if out is not None and (out.dtype != q.dtype or out.shape != q.shape):
        _refuse(f"{what}: out has q's shape and type")
    res = {}
    with _On(torch, stream):
        res["out"] = torch.empty((n_seq, heads, hd), dtype=q.dtype, device=q.device) if out is None else out
        if lse:
            res["lse"] = torch.empty((n_seq, heads), dtype=torch.float32, device=q.device)
        if workspace is None:
            workspace = torch.empty(L.pf_decode_attention_workspace(c, n_seq, heads), dtype=torch.uint8, device=q.device)
    _check(L.pf_decode_attention(c, dt, n_seq, heads, q.data_ptr(), _heads(q, what, heads, c.hd), _int32(torch, what, lengths, 1),
                                 _int32(torch, what, table, 2), table.shape[1], 1.0 / math.sqrt(c.hd) if sm_scale is None else sm_scale,
                                 res["out"].data_ptr(), _heads(res["out"], what, heads, c.hd), _ptr(res.get("lse")), workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream(torch, dev, stream)), what)
    return res


class MoeLayer:
    """A mixture-of-experts layer's weights, laid out for few-token calls (pf_moe_pack), and its forward (pf_moe_forward).

    router: [experts, H] bf16.  gate, up: [local + shared, F, H], down: [local + shared, H, F], bf16, or float8_e4m3fn with
    fp32 scales per 128 x 128 block ([local + shared, ceil(rows / 128), ceil(columns / 128)]).  Experts
    first_expert .. first_expert + local - 1 live here; the last n_shared of the weight tensors are taken by every token.
    The layer keeps a packed copy; gate, up, down and their scales may be dropped afterwards."""

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
        self.m = PfMoe(H, F, E, first_expert, n - n_shared, n_shared, top_k, wtype)
        size = L.pf_moe_packed_bytes(self.m)
        if size == 0:
            _refuse(f"{what}: inconsistent sizes")
        self._L, self._torch, self._dev = L, torch, dev
        self.router = router
        with _On(torch, stream):
            self.packed = torch.empty(size, dtype=torch.uint8, device=router.device)
        _check(L.pf_moe_pack(self.m, gate.data_ptr(), up.data_ptr(), down.data_ptr(), _ptr(gate_scale), _ptr(up_scale), _ptr(down_scale),
                             self.packed.data_ptr(), _stream(torch, dev, stream)), "pf_moe_pack")

    def forward(self, x, xq=None, xq_scale=None, *, out=None, status=None, workspace=None, stream=None) -> dict:
        """x: [tokens, H] bf16, 1 .. 512 tokens; xq, xq_scale: the same tokens in 8 bits from pf_add_rms_norm (group 128), which
        e4m3 weights then multiply (the router reads x).  Returns {"out": [tokens, H] bf16, "ids": [tokens, top_k] int32, "weights": [tokens, top_k]
        fp32}.  status: int32 tensor of one element, see pf_moe_forward."""
        L, torch, m = self._L, self._torch, self.m
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
        with _On(torch, stream):
            if out is None:
                out = torch.empty((T, m.H), dtype=x.dtype, device=x.device)
            ids = torch.empty((T, m.top_k), dtype=torch.int32, device=x.device)
            weights = torch.empty((T, m.top_k), dtype=torch.float32, device=x.device)
            if workspace is None:
                workspace = torch.empty(L.pf_moe_workspace(m, T), dtype=torch.uint8, device=x.device)
        status_of = L.pf_moe_forward(m, T, x.data_ptr(), xs, _ptr(xq), _ptr(xq_scale), self.router.data_ptr(), self.packed.data_ptr(), out.data_ptr(), ids.data_ptr(), weights.data_ptr(), _ptr(status), workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(), _stream(torch, dev, stream))
        if status_of != PF_OK:
            _check(status_of, what)
        return {"out": out, "ids": ids, "weights": weights}
