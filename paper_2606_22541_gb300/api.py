"""Python binding of the C ABI, one function per entry point with the same name.

Tensors are torch CUDA tensors (the binding passes their device pointers);
``stream`` is a torch.cuda.Stream or None for the current stream.  Every step
of the layer runs in libasap_moe's kernels; nothing here computes.
"""
import ctypes
import threading

import torch

from . import _native
from ._native import AsapMoeConfig, AsapMoeWeights, check, fast, lib
from .configs import GATING, DTYPE


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


# this thread's pending asap_moe_time_layer events (kept alive for the C side)
_timing = threading.local()


def _stream(stream):
    if stream is None:  # (the current stream's handle without its Python object, which takes 3 us to make)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def make_config(cfg, max_tokens):
    """C config from a configs.LayerConfig."""
    return AsapMoeConfig(hidden=cfg.hidden, n_experts=cfg.n_experts, top_k=cfg.top_k, inter=cfg.inter,
                         n_shared=cfg.n_shared, shared_inter=cfg.shared_inter, gating=GATING[cfg.gating],
                         n_groups=cfg.n_groups, topk_groups=cfg.topk_groups,
                         route_scale=float(cfg.route_scale), dtype=DTYPE[cfg.dtype],
                         max_tokens=int(max_tokens))


class Handle:
    """Owns an asap_moe_t; destroyed on close() or garbage collection."""

    def __init__(self, ptr, cfg, ccfg):
        self.ptr = ptr
        self.cfg = cfg
        self.ccfg = ccfg

    @property
    def max_tokens(self):
        return self.ccfg.max_tokens

    def close(self):
        """Frees the handle; raises AsapError (and keeps it) while a mailbox
        created on it is open."""
        if self.ptr:
            check("asap_moe_destroy", lib().asap_moe_destroy(self.ptr))
            self.ptr = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def asap_moe_check_config(cfg, max_tokens=1):
    c = make_config(cfg, max_tokens)
    return lib().asap_moe_check_config(ctypes.byref(c))


def _weights_struct(weights, w):
    for name, _ in AsapMoeWeights._fields_:
        t = weights.get(name)
        setattr(w, name, None if t is None else t.data_ptr())


def asap_moe_create(cfg, weights, max_tokens):
    """weights: dict of CUDA tensors named like asap_moe_weights' fields."""
    c = make_config(cfg, max_tokens)
    w = AsapMoeWeights()
    _weights_struct(weights, w)
    out = ctypes.c_void_p()
    check("asap_moe_create", lib().asap_moe_create(ctypes.byref(c), ctypes.byref(w), ctypes.byref(out)))
    return Handle(out, cfg, c)


def asap_moe_create_layers(cfg, layers, max_tokens):
    """One handle over several layers of the same shape; layers: a list of
    weight dicts, one per layer (layer l = layers[l])."""
    c = make_config(cfg, max_tokens)
    ws = (AsapMoeWeights * len(layers))()
    for i, weights in enumerate(layers):
        _weights_struct(weights, ws[i])
    out = ctypes.c_void_p()
    check("asap_moe_create_layers", lib().asap_moe_create_layers(ctypes.byref(c), ws, len(layers), ctypes.byref(out)))
    return Handle(out, cfg, c)


def asap_moe_n_layers(h):
    out = ctypes.c_int32()
    check("asap_moe_n_layers", lib().asap_moe_n_layers(h.ptr, ctypes.byref(out)))
    return out.value


def asap_moe_destroy(h):
    h.close()


def asap_moe_workspace_size(cfg, n_tokens, max_tokens=None):
    c = make_config(cfg, max_tokens if max_tokens is not None else max(n_tokens, 1))
    out = ctypes.c_size_t()
    check("asap_moe_workspace_size", lib().asap_moe_workspace_size(ctypes.byref(c), int(n_tokens), ctypes.byref(out)))
    return out.value


def workspace(h, n_tokens, device="cuda"):
    """A workspace tensor large enough for one call with n_tokens tokens."""
    nbytes = asap_moe_workspace_size(h.cfg, n_tokens, h.max_tokens)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def _ws(ws):
    return (_ptr(ws), ctypes.c_size_t(0 if ws is None else ws.numel() * ws.element_size()))


def asap_moe_router_logits(h, x, logits, ws, stream=None):
    p, n = _ws(ws)
    check("asap_moe_router_logits",
          lib().asap_moe_router_logits(h.ptr, _ptr(x), x.shape[0], _ptr(logits), p, n, _stream(stream)))


def asap_moe_route(h, x, idx, w, counts, offsets, ws, stream=None):
    p, n = _ws(ws)
    check("asap_moe_route", lib().asap_moe_route(h.ptr, _ptr(x), x.shape[0], _ptr(idx), _ptr(w), _ptr(counts),
                                                 _ptr(offsets), p, n, _stream(stream)))


def asap_moe_route_logits(h, logits, idx, w, counts, offsets, ws, stream=None):
    p, n = _ws(ws)
    check("asap_moe_route_logits",
          lib().asap_moe_route_logits(h.ptr, _ptr(logits), logits.shape[0], _ptr(idx), _ptr(w), _ptr(counts),
                                      _ptr(offsets), p, n, _stream(stream)))


def asap_moe_dispatch(h, x, idx, x_perm, perm_src, perm_dst, ws, stream=None, x_perm_scales=None):
    p, n = _ws(ws)
    check("asap_moe_dispatch",
          lib().asap_moe_dispatch(h.ptr, _ptr(x), x.shape[0], _ptr(idx), _ptr(x_perm), _ptr(x_perm_scales),
                                  _ptr(perm_src), _ptr(perm_dst), p, n, _stream(stream)))


def asap_moe_expert_ffn(h, x_perm, offsets, x, y_perm, y_shared, ws, stream=None, x_perm_scales=None):
    p, n = _ws(ws)
    check("asap_moe_expert_ffn",
          lib().asap_moe_expert_ffn(h.ptr, _ptr(x_perm), _ptr(x_perm_scales), _ptr(offsets), _ptr(x),
                                    x.shape[0], _ptr(y_perm), _ptr(y_shared), p, n, _stream(stream)))


def asap_moe_expert_gate_up(h, x_perm, offsets, x, h_perm, h_shared, stream=None, x_perm_scales=None, ws=None):
    """ws (optional): a workspace for x.shape[0] tokens; with it the GEMM claims
    its tiles dynamically."""
    p, nb = _ws(ws)
    check("asap_moe_expert_gate_up",
          lib().asap_moe_expert_gate_up(h.ptr, _ptr(x_perm), _ptr(x_perm_scales), _ptr(offsets), _ptr(x),
                                        x.shape[0], _ptr(h_perm), _ptr(h_shared), p, nb, _stream(stream)))


def asap_moe_expert_down(h, h_perm, offsets, h_shared, n, y_perm, y_shared, stream=None, h_perm_scales=None,
                         ws=None):
    p, nb = _ws(ws)
    check("asap_moe_expert_down",
          lib().asap_moe_expert_down(h.ptr, _ptr(h_perm), _ptr(h_perm_scales), _ptr(offsets), _ptr(h_shared),
                                     int(n), _ptr(y_perm), _ptr(y_shared), p, nb, _stream(stream)))


def asap_moe_combine(h, y_perm, y_shared, w, perm_dst, out, stream=None):
    check("asap_moe_combine", lib().asap_moe_combine(h.ptr, _ptr(y_perm), _ptr(y_shared), _ptr(w), _ptr(perm_dst),
                                                     out.shape[0], _ptr(out), _stream(stream)))


def asap_moe_layer(h, x, out, ws, stream=None):
    p, n = _ws(ws)
    try:
        check("asap_moe_layer", lib().asap_moe_layer(h.ptr, _ptr(x), x.shape[0], _ptr(out), p, n, _stream(stream)))
    finally:
        _timing.events = None   # the call has taken this thread's timing request


FEW_MAX_TOKENS = 64


def asap_moe_layer_few(h, x, out, ws, stream=None, layer_id=None):
    """The whole layer for 1 to FEW_MAX_TOKENS tokens in two kernels (the
    decode steps of a handle whose prompt batches go through asap_moe_layer).
    x [n, hidden] and out (n rows or more) are bf16 and contiguous.
    layer_id: None (layer 0) or a one-element int32 CUDA tensor."""
    rows = x.shape[0]
    size = rows * h.cfg.hidden
    if x.dtype is not _BF16 or out.dtype is not _BF16 or x.numel() != size or out.numel() < size or \
            not (x.is_cuda and out.is_cuda and x.is_contiguous() and out.is_contiguous()):
        _refuse(f"x [n, {h.cfg.hidden}] and out of as many rows or more, bf16 contiguous CUDA tensors", x=x, out=out)
    if ws is not None and not (ws.is_cuda and ws.is_contiguous()):
        _refuse("a contiguous CUDA tensor for the workspace", ws=ws)
    if layer_id is not None and (not layer_id.is_cuda or layer_id.is_floating_point() or
                                 layer_id.numel() * layer_id.element_size() < 4):
        _refuse("layer_id: an int32 on the GPU", layer_id=layer_id)
    p, n = _ws(ws)
    check("asap_moe_layer_few", lib().asap_moe_layer_few(h.ptr, _ptr(layer_id), _ptr(x), rows, _ptr(out), p, n,
                                                         _stream(stream)))


def asap_moe_layer_batched(h, xs, outs, ws, stream=None):
    """Serve several ready micro-batches in one pass (one grouped GEMM per
    weight matrix); outs[i] equals asap_moe_layer on xs[i] bit for bit."""
    cnt = len(xs)
    xa = (ctypes.c_void_p * cnt)(*[x.data_ptr() for x in xs])
    na = (ctypes.c_int32 * cnt)(*[x.shape[0] for x in xs])
    oa = (ctypes.c_void_p * cnt)(*[o.data_ptr() for o in outs])
    p, n = _ws(ws)
    check("asap_moe_layer_batched",
          lib().asap_moe_layer_batched(h.ptr, cnt, xa, na, oa, p, n, _stream(stream)))


def asap_moe_layer_dyn(h, layer_id, x, out, ws, stream=None):
    """asap_moe_layer for the layer whose id the kernels read from layer_id
    (a one-element int32 CUDA tensor) when they run."""
    p, n = _ws(ws)
    try:
        check("asap_moe_layer_dyn", lib().asap_moe_layer_dyn(h.ptr, _ptr(layer_id), _ptr(x), x.shape[0], _ptr(out), p,
                                                             n, _stream(stream)))
    finally:
        _timing.events = None   # the call has taken this thread's timing request


def asap_moe_layer_batched_dyn(h, layer_id, xs, outs, ws, stream=None):
    """asap_moe_layer_batched for micro-batches of the layer at layer_id."""
    cnt = len(xs)
    xa = (ctypes.c_void_p * cnt)(*[x.data_ptr() for x in xs])
    na = (ctypes.c_int32 * cnt)(*[x.shape[0] for x in xs])
    oa = (ctypes.c_void_p * cnt)(*[o.data_ptr() for o in outs])
    p, n = _ws(ws)
    check("asap_moe_layer_batched_dyn",
          lib().asap_moe_layer_batched_dyn(h.ptr, _ptr(layer_id), cnt, xa, na, oa, p, n, _stream(stream)))


def asap_moe_time_layer(events):
    """Events (torch.cuda.Event, enable_timing=True; up to 6) for this
    thread's next asap_moe_layer / _dyn call to record: before its first
    kernel and after route, dispatch, gate/up, down and combine."""
    events = list(events)
    for ev in events:
        if ev.cuda_event == 0:   # torch creates the CUDA event at its first record
            ev.record()
    arr = (ctypes.c_void_p * max(1, len(events)))(*[ev.cuda_event for ev in events])
    check("asap_moe_time_layer", lib().asap_moe_time_layer(len(events), arr))
    _timing.events = events     # alive until the layer call that records them returns


def asap_moe_route_noalloc(h, x, idx, w, counts, offsets, stream=None):
    """asap_moe_route with its scratch in the library's static device array
    (at most 4096 tokens; calls overlapping on the GPU race)."""
    check("asap_moe_route_noalloc",
          lib().asap_moe_route_noalloc(h.ptr, _ptr(x), x.shape[0], _ptr(idx), _ptr(w), _ptr(counts),
                                       _ptr(offsets), _stream(stream)))


_BF16, _F32, _F8, _U8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.uint8
_WORD = (torch.int32, torch.uint32)


def _ld(t):
    """Row stride of a 2-D CUDA tensor whose columns are contiguous, else 0.  (A
    single row's stride says nothing: one that any row may have.)"""
    if not t.is_cuda:
        return 0
    s0, s1 = t.stride()
    rows, cols = t.shape
    if s1 != 1 and cols > 1:
        return 0
    return s0 if rows > 1 else (cols + 15) // 16 * 16


def _refuse(what, **tensors):
    raise ValueError(what + "; got " + ", ".join(
        f"{k} {tuple(t.shape)} {t.dtype} strides {tuple(t.stride())} on {t.device}" for k, t in tensors.items()))


def asap_moe_fp8_quantize(x, q, scales, stream=None):
    """bf16 rows x [n, c] to e4m3 q [n, c] with scales [n, ceil(c / 128)]
    (fp32); any row strides."""
    f = fast()
    code = f.quantize(x, q, scales, stream) if f else None
    if code is None:
        code = _quantize(x, q, scales, stream)
    if code:
        check("asap_moe_fp8_quantize", code)


def _quantize(x, q, scales, stream):
    shape = x.shape
    if len(shape) != 2 or x.dtype is not _BF16 or q.shape != shape or (q.dtype is not _F8 and q.dtype is not _U8) or \
            scales.dtype is not _F32 or scales.shape != (shape[0], (shape[1] + 127) // 128):
        _refuse("x [n, c] bf16, q [n, c] e4m3, scales [n, ceil(c / 128)] fp32", x=x, q=q, scales=scales)
    n, c = shape
    ld, ldq, lds = _ld(x), _ld(q), _ld(scales)
    if not (ld and ldq and lds) and n and c:
        _refuse("CUDA tensors with contiguous columns", x=x, q=q, scales=scales)
    code = lib().asap_moe_fp8_quantize(x.data_ptr(), ld, n, c, q.data_ptr(), ldq, scales.data_ptr(), lds,
                                       _stream(stream))
    return code


def asap_moe_fp8_swiglu_quantize(gate, up, q, scales, stream=None):
    """silu(gate) * up of bf16 [n, c] tensors with one row stride (the halves of
    a product's rows) to e4m3 q [n, c] with scales [n, ceil(c / 128)]."""
    f = fast()
    code = f.swiglu_quantize(gate, up, q, scales, stream) if f else None
    if code is None:
        code = _swiglu_quantize(gate, up, q, scales, stream)
    if code:
        check("asap_moe_fp8_swiglu_quantize", code)


def _swiglu_quantize(gate, up, q, scales, stream):
    shape = gate.shape
    if len(shape) != 2 or gate.dtype is not _BF16 or up.shape != shape or up.dtype is not _BF16 or \
            q.shape != shape or (q.dtype is not _F8 and q.dtype is not _U8) or \
            scales.dtype is not _F32 or scales.shape != (shape[0], (shape[1] + 127) // 128):
        _refuse("gate, up [n, c] bf16, q [n, c] e4m3, scales [n, ceil(c / 128)] fp32", gate=gate, up=up, q=q,
                scales=scales)
    n, c = shape
    ld, ldq, lds = _ld(gate), _ld(q), _ld(scales)
    if not (ld and ldq and lds and _ld(up) == ld) and n and c:
        _refuse("CUDA tensors with contiguous columns, gate and up with one row stride", gate=gate, up=up, q=q,
                scales=scales)
    code = lib().asap_moe_fp8_swiglu_quantize(gate.data_ptr(), up.data_ptr(), ld, n, c, q.data_ptr(), ldq,
                                              scales.data_ptr(), lds, _stream(stream))
    return code


def asap_moe_fp8_matmul(a, a_scales, b, b_scales, out, stream=None, status=None):
    """out [m, n] (bf16) = a b^T of e4m3 a [m, k], b [n, k] (rows on 16-byte
    boundaries) with fp32 scales [m, ceil(k / 128)] and [ceil(n / 128),
    ceil(k / 128)].  status: None or a one-element int32 CUDA tensor that gets
    error bits."""
    if status is not None and not (status.is_cuda and status.dtype in _WORD and status.numel()):
        _refuse("status: an int32 on the GPU", status=status)
    f = fast()
    code = f.matmul(a, a_scales, b, b_scales, out, stream, status) if f else None
    if code is None:
        code = _matmul(a, a_scales, b, b_scales, out, stream, status)
    if code:
        check("asap_moe_fp8_matmul", code)


def _matmul(a, a_scales, b, b_scales, out, stream, status):
    sa, sb = a.shape, b.shape
    if len(sa) != 2 or len(sb) != 2:
        _refuse("a [m, k], b [n, k]", a=a, b=b)
    m, k = sa
    n = sb[0]
    blocks = (k + 127) // 128
    if (a.dtype is not _F8 and a.dtype is not _U8) or (b.dtype is not _F8 and b.dtype is not _U8) or sb[1] != k or \
            out.dtype is not _BF16 or out.shape != (m, n) or \
            a_scales.dtype is not _F32 or a_scales.shape != (m, blocks) or \
            b_scales.dtype is not _F32 or b_scales.shape != ((n + 127) // 128, blocks):
        _refuse("a [m, k], b [n, k] e4m3, a_scales [m, ceil(k / 128)], b_scales [ceil(n / 128), ceil(k / 128)] fp32, "
                "out [m, n] bf16", a=a, a_scales=a_scales, b=b, b_scales=b_scales, out=out)
    lda, lsa, ldb, lsb, ldc = _ld(a), _ld(a_scales), _ld(b), _ld(b_scales), _ld(out)
    if not (lda and lsa and ldb and lsb and ldc) and m and n and k:
        _refuse("CUDA tensors with contiguous columns", a=a, a_scales=a_scales, b=b, b_scales=b_scales, out=out)
    code = lib().asap_moe_fp8_matmul(a.data_ptr(), lda, a_scales.data_ptr(), lsa, b.data_ptr(), ldb,
                                     b_scales.data_ptr(), lsb, out.data_ptr(), ldc, m, n, k,
                                     None if status is None else status.data_ptr(), _stream(stream))
    return code


# ------------------------------------------------------------ around the expert products of a training step
# The compiled marshalling takes the calls without a status, and asap_moe_unpermute_backward with both gradients (3 to 4 us
# on the host); those with a status, or without one of the gradients, go through the checks here (7 to 11).

SORT_MAX_EXPERTS = 1024
_ELEM = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_BYTES = {torch.float8_e4m3fn: 3, torch.uint8: 3, **_ELEM}   # what asap_moe_permute copies


def asap_moe_sort_workspace_size(n, k, n_experts):
    out = ctypes.c_size_t()
    check("asap_moe_sort_workspace_size",
          lib().asap_moe_sort_workspace_size(int(n), int(k), int(n_experts), ctypes.byref(out)))
    return out.value


def sort_workspace(n, k, n_experts, device="cuda"):
    """A workspace tensor large enough for asap_moe_sort of n tokens or fewer."""
    return torch.empty(max(asap_moe_sort_workspace_size(n, k, n_experts), 256), dtype=torch.uint8, device=device)


def _data(t):
    return None if t is None else t.data_ptr()


def _here(*tensors):
    """All on the current device, where the calls without a handle launch."""
    index = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            return False
        if index is None:
            index = torch.cuda.current_device()
        if t.get_device() != index:
            return False
    return True


def _dense(t, dtype, shape):
    return t.dtype is dtype and t.shape == shape and t.is_contiguous()


def asap_moe_sort(idx, n_experts, offsets, perm_dst, ws=None, perm_src=None, stream=None):
    """Entries sorted by expert: idx [n, k] int32 (outside [0, n_experts): no
    expert takes it) to offsets [n_experts + 1], perm_dst [n, k] (the entry's
    row, -1: none) and, if given, perm_src [n * k] (row -> token), all int32 and
    contiguous.  ws: sort_workspace(n, k, n_experts), None where its size is 0."""
    f = fast()
    code = f.sort(idx, n_experts, offsets, perm_dst, ws, perm_src, stream) if f else None
    if code is None:
        code = _sort(idx, n_experts, offsets, perm_dst, ws, perm_src, stream)
    if code:
        check("asap_moe_sort", code)


def _sort(idx, n_experts, offsets, perm_dst, ws, perm_src, stream):
    shape = idx.shape
    if len(shape) != 2 or not _dense(idx, torch.int32, shape) or not _dense(perm_dst, torch.int32, shape) or \
            not _dense(offsets, torch.int32, (n_experts + 1,)) or \
            (perm_src is not None and not _dense(perm_src, torch.int32, (shape[0] * shape[1],))) or \
            (ws is not None and not ws.is_contiguous()) or not _here(idx, offsets, perm_dst, perm_src, ws):
        _refuse("contiguous int32 tensors on the current CUDA device, idx, perm_dst [n, k], offsets [n_experts + 1], "
                "perm_src [n * k] or None, and a workspace", idx=idx, offsets=offsets, perm_dst=perm_dst,
                **{k: t for k, t in (("perm_src", perm_src), ("ws", ws)) if t is not None})
    p, nb = (None, 0) if ws is None else (ws.data_ptr(), ws.numel() * ws.element_size())
    return lib().asap_moe_sort(idx.data_ptr(), shape[0], shape[1], n_experts, offsets.data_ptr(), perm_dst.data_ptr(),
                               _data(perm_src), p, nb, _stream(stream))


def _check_status(status):
    if status is not None and not (status.is_cuda and status.dtype in _WORD and status.numel()):
        _refuse("status: an int32 on the GPU", status=status)


def asap_moe_permute(x, perm_dst, x_perm, stream=None, status=None):
    """x_perm[perm_dst[t, j]] = x[t]: x [n, c] and x_perm [rows, c] of one type
    (bf16, fp16, fp32, e4m3 or uint8), perm_dst [n, k] int32 contiguous; any row
    strides.  Rows of x_perm that nothing names stay as they were.  status: None
    or a one-element int32 CUDA tensor that gets bit 2 for a row that does not
    exist (other than -1)."""
    f = fast()
    code = f.permute(x, perm_dst, x_perm, stream, status) if f else None
    if code is None:
        code = _permute(x, perm_dst, x_perm, stream, status)
    if code:
        check("asap_moe_permute", code)


def _permute(x, perm_dst, x_perm, stream, status):
    _check_status(status)
    if x.dim() != 2 or x_perm.dim() != 2 or perm_dst.dim() != 2 or x.dtype not in _BYTES or x_perm.dtype is not x.dtype or \
            x_perm.shape[1] != x.shape[1] or not _dense(perm_dst, torch.int32, (x.shape[0], perm_dst.shape[1])) or \
            not _here(x, x_perm, perm_dst, status):
        _refuse("tensors on the current CUDA device, x [n, c], x_perm [rows, c] of one type, perm_dst [n, k] int32", x=x,
                perm_dst=perm_dst, x_perm=x_perm)
    n, c = x.shape
    rows, ld, ldp = x_perm.shape[0], _ld(x), _ld(x_perm)
    if not (ld and ldp) and n and c and rows:
        _refuse("CUDA tensors with contiguous columns", x=x, x_perm=x_perm)
    return lib().asap_moe_permute(_BYTES[x.dtype], x.data_ptr(), ld, n, c, perm_dst.data_ptr(), perm_dst.shape[1],
                                  x_perm.data_ptr(), ldp, rows, _data(status), _stream(stream))


def asap_moe_unpermute(y_perm, w, perm_dst, out, stream=None, status=None):
    """out[t] = sum_j w[t, j] y_perm[perm_dst[t, j]] over the entries that have a
    row: y_perm [rows, c], out [n, c] of one type (bf16, fp16 or fp32), w [n, k]
    fp32 or None (ones: the gradient of asap_moe_permute), perm_dst [n, k] int32,
    both contiguous.  status as for asap_moe_permute."""
    f = fast()
    code = f.unpermute(y_perm, w, perm_dst, out, stream, status) if f else None
    if code is None:
        code = _unpermute(y_perm, w, perm_dst, out, stream, status)
    if code:
        check("asap_moe_unpermute", code)


def _unpermute(y_perm, w, perm_dst, out, stream, status):
    _check_status(status)
    if y_perm.dim() != 2 or out.dim() != 2 or perm_dst.dim() != 2 or y_perm.dtype not in _ELEM or \
            out.dtype is not y_perm.dtype or y_perm.shape[1] != out.shape[1] or \
            not _dense(perm_dst, torch.int32, (out.shape[0], perm_dst.shape[1])) or \
            (w is not None and not _dense(w, _F32, perm_dst.shape)) or not _here(y_perm, w, perm_dst, out, status):
        _refuse("tensors on the current CUDA device, y_perm [rows, c], out [n, c] of one type, perm_dst [n, k] int32, w "
                "[n, k] fp32 or None", y_perm=y_perm, perm_dst=perm_dst, out=out, **({} if w is None else {"w": w}))
    n, c = out.shape
    rows, ldy, ldo = y_perm.shape[0], _ld(y_perm), _ld(out)
    if not (ldy and ldo) and n and c and rows:
        _refuse("CUDA tensors with contiguous columns", y_perm=y_perm, out=out)
    return lib().asap_moe_unpermute(_ELEM[out.dtype], y_perm.data_ptr(), ldy, rows, c, _data(w), perm_dst.data_ptr(), n,
                                    perm_dst.shape[1], out.data_ptr(), ldo, _data(status), _stream(stream))


def asap_moe_unpermute_backward(d_out, y_perm, w, perm_dst, d_y_perm, d_w, stream=None, status=None):
    """The gradients of asap_moe_unpermute: d_y_perm[perm_dst[t, j]] = w[t, j]
    d_out[t] and d_w[t, j] = <d_out[t], y_perm[perm_dst[t, j]]> (0 where the entry
    has no row).  d_out [n, c], y_perm and d_y_perm [rows, c] of one type, w and
    d_w [n, k] fp32.  w None: ones; d_y_perm or d_w None: not wanted; y_perm may be
    None where d_w is."""
    f = fast()
    code = f.unpermute_backward(d_out, y_perm, w, perm_dst, d_y_perm, d_w, stream, status) if f else None
    if code is None:
        code = _unpermute_backward(d_out, y_perm, w, perm_dst, d_y_perm, d_w, stream, status)
    if code:
        check("asap_moe_unpermute_backward", code)


def _unpermute_backward(d_out, y_perm, w, perm_dst, d_y_perm, d_w, stream, status):
    _check_status(status)
    y = {k: t for k, t in (("y_perm", y_perm), ("d_y_perm", d_y_perm)) if t is not None}
    rows = next(iter(y.values())).shape[0] if y else 0
    if d_out.dim() != 2 or perm_dst.dim() != 2 or d_out.dtype not in _ELEM or \
            any(t.dtype is not d_out.dtype or t.shape != (rows, d_out.shape[1]) for t in y.values()) or \
            not _dense(perm_dst, torch.int32, (d_out.shape[0], perm_dst.shape[1])) or \
            any(t is not None and not _dense(t, _F32, perm_dst.shape) for t in (w, d_w)) or \
            (d_w is not None and y_perm is None) or \
            not _here(d_out, y_perm, w, perm_dst, d_y_perm, d_w, status):
        _refuse("tensors on the current CUDA device, d_out [n, c], y_perm and d_y_perm [rows, c] of one type, perm_dst "
                "[n, k] int32, w and d_w [n, k] fp32", d_out=d_out, perm_dst=perm_dst, **y,
                **{k: t for k, t in (("w", w), ("d_w", d_w)) if t is not None})
    n, c = d_out.shape
    ldo, lds = _ld(d_out), {k: _ld(t) for k, t in y.items()}
    if not (ldo and all(lds.values())) and n and c and rows:
        _refuse("CUDA tensors with contiguous columns", d_out=d_out, **y)
    return lib().asap_moe_unpermute_backward(_ELEM[d_out.dtype], d_out.data_ptr(), ldo, _data(y_perm), lds.get("y_perm", 0),
                                             _data(w), perm_dst.data_ptr(), n, perm_dst.shape[1], c, _data(d_y_perm),
                                             lds.get("d_y_perm", 0), rows, _data(d_w), _data(status), _stream(stream))


def _swiglu_kept(rows, cols, gate_q, gate_s, up_q, up_s, n_rows, **others):
    """Row strides of the kept tensors' values and scales; refuses what does not fit (others: [rows, cols] of one type)."""
    shape, blocks = (rows, cols), (rows, (cols + 127) // 128)
    first = next(iter(others.values()))
    tensors = dict(others, gate_q=gate_q, gate_s=gate_s, up_q=up_q, up_s=up_s)
    if first.dtype not in _ELEM or any(t.dtype is not first.dtype or t.shape != shape for t in others.values()) or \
            any(t.dtype not in (_F8, _U8) or t.shape != shape for t in (gate_q, up_q)) or \
            any(t.dtype is not _F32 or t.shape != blocks for t in (gate_s, up_s)) or \
            (n_rows is not None and (n_rows.dtype is not torch.int32 or n_rows.numel() != 1)) or \
            not _here(*tensors.values(), n_rows):
        _refuse(f"tensors on the current CUDA device, {', '.join(others)} [n, c] of one type (bf16, fp16, fp32), gate_q, "
                "up_q [n, c] e4m3, gate_s, up_s [n, ceil(c / 128)] fp32, n_rows None or one int32", **tensors,
                **({} if n_rows is None else {"n_rows": n_rows}))
    lds = {k: _ld(t) for k, t in tensors.items()}
    pairs = [("gate_q", "up_q"), ("gate_s", "up_s"), ("gate", "up"), ("d_gate", "d_up")]
    if rows and cols and (not all(lds.values()) or any(lds[a] != lds[b] for a, b in pairs if a in lds)):
        _refuse("CUDA tensors with contiguous columns, gate and up (values, scales, gradients) with one row stride", **tensors)
    return lds


def asap_moe_swiglu_save(gate, up, h, gate_q, gate_s, up_q, up_s, stream=None, n_rows=None):
    """h = silu(gate) * up, with gate and up kept for asap_moe_swiglu_backward as
    asap_moe_fp8_quantize would quantise them.  gate, up, h [n, c] of one type
    (bf16, fp16 or fp32), gate_q, up_q [n, c] e4m3, gate_s, up_s [n, ceil(c /
    128)] fp32; gate and up have one row stride each time (the halves of a
    product's rows).  n_rows: None or a one-element int32 CUDA tensor, the rows
    that are read and written (offsets[-1:] of asap_moe_sort)."""
    f = fast()
    code = f.swiglu_save(gate, up, h, gate_q, gate_s, up_q, up_s, stream, n_rows) if f else None
    if code is None:
        code = _swiglu_save(gate, up, h, gate_q, gate_s, up_q, up_s, stream, n_rows)
    if code:
        check("asap_moe_swiglu_save", code)


def _swiglu_save(gate, up, h, gate_q, gate_s, up_q, up_s, stream, n_rows):
    if gate.dim() != 2:
        _refuse("gate [n, c]", gate=gate)
    n, c = gate.shape
    ld = _swiglu_kept(n, c, gate_q, gate_s, up_q, up_s, n_rows, gate=gate, up=up, h=h)
    return lib().asap_moe_swiglu_save(_ELEM[gate.dtype], gate.data_ptr(), up.data_ptr(), ld["gate"], n, c, _data(n_rows),
                                      h.data_ptr(), ld["h"], gate_q.data_ptr(), up_q.data_ptr(), ld["gate_q"],
                                      gate_s.data_ptr(), up_s.data_ptr(), ld["gate_s"], _stream(stream))


def asap_moe_swiglu_backward(d_h, gate_q, gate_s, up_q, up_s, d_gate, d_up, h=None, stream=None, n_rows=None):
    """The gradients of silu(gate) * up at the values kept by asap_moe_swiglu_save,
    and (h not None) silu(gate) * up at them.  d_h, d_gate, d_up, h [n, c] of one
    type, d_gate and d_up with one row stride; n_rows as there."""
    f = fast()
    code = f.swiglu_backward(d_h, gate_q, gate_s, up_q, up_s, d_gate, d_up, h, stream, n_rows) if f else None
    if code is None:
        code = _swiglu_backward(d_h, gate_q, gate_s, up_q, up_s, d_gate, d_up, h, stream, n_rows)
    if code:
        check("asap_moe_swiglu_backward", code)


def _swiglu_backward(d_h, gate_q, gate_s, up_q, up_s, d_gate, d_up, h, stream, n_rows):
    if d_h.dim() != 2:
        _refuse("d_h [n, c]", d_h=d_h)
    n, c = d_h.shape
    more = {} if h is None else {"h": h}
    ld = _swiglu_kept(n, c, gate_q, gate_s, up_q, up_s, n_rows, d_h=d_h, d_gate=d_gate, d_up=d_up, **more)
    return lib().asap_moe_swiglu_backward(_ELEM[d_h.dtype], d_h.data_ptr(), ld["d_h"], gate_q.data_ptr(), up_q.data_ptr(),
                                          ld["gate_q"], gate_s.data_ptr(), up_s.data_ptr(), ld["gate_s"], n, c,
                                          _data(n_rows), d_gate.data_ptr(), d_up.data_ptr(), ld["d_gate"], _data(h),
                                          ld.get("h", 0), _stream(stream))


def asap_moe_fp8_dequantize(q, scales, x, perm_dst=None, stream=None, status=None):
    """e4m3 rows q [n, c] with scales [n, ceil(c / 128)] (asap_moe_fp8_quantize's)
    back to x of bf16, fp16 or fp32: row t to every row perm_dst[t, j] of x [rows,
    c], or, without perm_dst, to row t of x [n, c].  status as for
    asap_moe_permute."""
    f = fast()
    code = f.dequantize(q, scales, x, perm_dst, stream, status) if f else None
    if code is None:
        code = _dequantize(q, scales, x, perm_dst, stream, status)
    if code:
        check("asap_moe_fp8_dequantize", code)


def _dequantize(q, scales, x, perm_dst, stream, status):
    _check_status(status)
    if q.dim() != 2 or x.dim() != 2 or q.dtype not in (_F8, _U8) or x.dtype not in _ELEM or x.shape[1] != q.shape[1] or \
            scales.dtype is not _F32 or scales.shape != (q.shape[0], (q.shape[1] + 127) // 128) or \
            (x.shape[0] != q.shape[0] if perm_dst is None else
             perm_dst.dim() != 2 or not _dense(perm_dst, torch.int32, (q.shape[0], perm_dst.shape[1]))) or \
            not _here(q, scales, x, perm_dst, status):
        _refuse("tensors on the current CUDA device, q [n, c] e4m3, scales [n, ceil(c / 128)] fp32, x [rows, c], perm_dst "
                "[n, k] int32 or None", q=q, scales=scales, x=x, **({} if perm_dst is None else {"perm_dst": perm_dst}))
    n, c = q.shape
    ldq, lds, ldx = _ld(q), _ld(scales), _ld(x)
    if not (ldq and lds and ldx) and n and c and x.shape[0]:
        _refuse("CUDA tensors with contiguous columns", q=q, scales=scales, x=x)
    k = 1 if perm_dst is None else perm_dst.shape[1]
    return lib().asap_moe_fp8_dequantize(_ELEM[x.dtype], q.data_ptr(), ldq, scales.data_ptr(), lds, n, c, _data(perm_dst), k,
                                         x.data_ptr(), ldx, x.shape[0], _data(status), _stream(stream))


class Mailbox:
    """Owns an asap_moe_mailbox_t (slots that DP-group streams post routed
    micro-batches into and that service rounds on the MoE stream claim on the
    device); destroyed on close() or garbage collection.  Keeps the tensors
    of every post alive until the mailbox is closed or the slot is reposted."""

    def __init__(self, ptr, handle, n_slots, slot_tokens):
        self.ptr = ptr
        self.handle = handle          # the weights must outlive the mailbox
        self.n_slots = n_slots
        self.slot_tokens = slot_tokens
        self._keep = {}

    def close(self):
        if self.ptr:
            lib().asap_moe_mailbox_destroy(self.ptr)
            self.ptr = None
            self._keep.clear()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def asap_moe_mailbox_create(h, n_slots, slot_tokens, layer_id=None, wait_ns=2_000_000_000):
    """A mailbox of n_slots slots of up to slot_tokens tokens on h (layer_id:
    None for layer 0, or a one-element int32 CUDA tensor)."""
    out = ctypes.c_void_p()
    check("asap_moe_mailbox_create",
          lib().asap_moe_mailbox_create(h.ptr, int(n_slots), int(slot_tokens), _ptr(layer_id), int(wait_ns),
                                        ctypes.byref(out)))
    m = Mailbox(out, h, n_slots, slot_tokens)
    m._layer = layer_id
    return m


def asap_moe_mailbox_post(m, slot, x, out, stream=None, layer_id=None):
    """Post x (n tokens) into slot; returns the post's epoch.  layer_id: None
    (the mailbox's default layer) or a one-element int32 CUDA tensor.  The
    mailbox keeps x, out and layer_id alive until the slot is posted again or
    the mailbox is closed."""
    s = torch.cuda.current_stream() if stream is None else stream
    ep = ctypes.c_uint64()
    check("asap_moe_mailbox_post",
          lib().asap_moe_mailbox_post(m.ptr, int(slot), _ptr(x), x.shape[0], _ptr(out), _ptr(layer_id),
                                      _stream(s), ctypes.byref(ep)))
    old = m._keep.get(int(slot))
    if old is not None:
        # The post just enqueued on s waits for the round that served the
        # slot's previous post, so once s reaches this point that round is
        # done with the previous tensors.  Recording s on them keeps the
        # caching allocator from handing their memory to another stream
        # before then, even when this reference was the last one.
        for t in old:
            if t is not None:
                t.record_stream(s)
    m._keep[int(slot)] = (x, out, layer_id)
    return ep.value


def asap_moe_mailbox_serve(m, slot, epoch, stream=None):
    try:
        check("asap_moe_mailbox_serve", lib().asap_moe_mailbox_serve(m.ptr, int(slot), int(epoch), _stream(stream)))
    finally:
        m._timing = None


def asap_moe_mailbox_serve_many(m, slots, epochs, stream=None):
    """One service round for the posts (slots[i], epochs[i]) already made."""
    n = len(slots)
    cs = (ctypes.c_int32 * n)(*[int(v) for v in slots])
    ce = (ctypes.c_uint64 * n)(*[int(v) for v in epochs])
    try:
        check("asap_moe_mailbox_serve_many", lib().asap_moe_mailbox_serve_many(m.ptr, n, cs, ce, _stream(stream)))
    finally:
        m._timing = None


def asap_moe_mailbox_wait(m, slot, stream=None):
    check("asap_moe_mailbox_wait", lib().asap_moe_mailbox_wait(m.ptr, int(slot), _stream(stream)))


def asap_moe_mailbox_served(m, slot):
    ep = ctypes.c_uint64()
    check("asap_moe_mailbox_served", lib().asap_moe_mailbox_served(m.ptr, int(slot), ctypes.byref(ep)))
    return ep.value


def asap_moe_mailbox_time_gemms(m, ev_before, ev_after):
    """torch.cuda.Event pair (enable_timing=True) recorded around the next
    serve call's GEMMs."""
    for ev in (ev_before, ev_after):
        if ev.cuda_event == 0:   # torch creates the CUDA event at its first record
            ev.record()
    check("asap_moe_mailbox_time_gemms",
          lib().asap_moe_mailbox_time_gemms(m.ptr, ctypes.c_void_p(ev_before.cuda_event),
                                            ctypes.c_void_p(ev_after.cuda_event)))
    m._timing = (ev_before, ev_after)   # alive until the serve call that records them returns


def asap_moe_mailbox_rounds(m, cap=4096):
    """(rounds run so far, list of the posts each round claimed); synchronises."""
    n = ctypes.c_int32()
    buf = (ctypes.c_int32 * cap)()
    check("asap_moe_mailbox_rounds", lib().asap_moe_mailbox_rounds(m.ptr, ctypes.byref(n), buf, cap))
    return n.value, list(buf[:min(cap, n.value)])


COMBINE_SEPARATE, COMBINE_FUSED = 0, 1


def asap_moe_set_combine(h, mode):
    """Where asap_moe_layer combines on a bf16 handle: COMBINE_SEPARATE (a
    kernel after the down GEMM, the default) or COMBINE_FUSED (inside the down
    GEMM); bit-identical outputs."""
    check("asap_moe_set_combine", lib().asap_moe_set_combine(h.ptr, int(mode)))


TILING_AUTO, TILING_SINGLE, TILING_PAIRED = 0, 1, 2


def asap_moe_set_tiling(h, mode):
    """Tile shape of the BF16 grouped expert GEMMs: TILING_AUTO, _SINGLE or
    _PAIRED (bit-identical results; only the speed differs)."""
    check("asap_moe_set_tiling", lib().asap_moe_set_tiling(h.ptr, int(mode)))


def asap_moe_status(h):
    """(code, raw status word); code is ASAP_OK or ASAP_ERR_DEVICE_STATUS."""
    word = ctypes.c_uint32()
    code = lib().asap_moe_status(h.ptr, ctypes.byref(word))
    return code, word.value


def asap_moe_last_error():
    return lib().asap_moe_last_error().decode(errors="replace")
