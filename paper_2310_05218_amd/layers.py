"""Thin binding of the layer norm and linear attention entry points: argument marshalling, scratch memory, no arithmetic.

Tensors may have any strides as long as the innermost dimension is contiguous (a slice of a fused projection, heads before
tokens).  Outputs that are not given, and the scratch memory of a call, are allocated on the stream that the call runs on, so
that the caching allocator hands them to nothing else before the call's kernels are done with them.

Calls on the current stream without `out` go the native short way of `binding`, which takes them or leaves them to the checks here.
"""
from __future__ import annotations

import contextlib

from . import binding
from .binding import SW_BF16, SW_ERR_SHAPE, SW_F16, SW_F32, SwError, SwLinearAttentionDims, SwStrides, _check, _done, _stream, lib

_types = None


def _type(t, what):
    """The sw_type of a tensor's elements."""
    global _types
    if _types is None:
        import torch

        _types = {torch.float32: SW_F32, torch.bfloat16: SW_BF16, torch.float16: SW_F16}
    try:
        return _types[t.dtype]
    except KeyError:
        raise ValueError(f"{what}: expected float32, bfloat16 or float16, got {t.dtype}") from None


def _on(stream):
    """Allocations within belong to the stream that the call runs on."""
    if stream is None:
        return contextlib.nullcontext()
    import torch

    return torch.cuda.stream(stream)


def _plain(t, dtype, shape, name):
    """The address of a contiguous tensor of that type and shape; None for None."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _rows(t, like, name):
    """(address, rows, channels, stride) of a tensor as rows of its last dimension, evenly apart."""
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if like is not None and (t.dtype != like.dtype or t.shape != like.shape):
        raise ValueError(f"{name}: expected {like.dtype} {tuple(like.shape)}, got {t.dtype} {tuple(t.shape)}")
    if t.dim() < 1:
        raise ValueError(f"{name}: expected rows of channels, got a single value")
    c = t.shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), t.numel() // c if c else 0, c, c
    rows, stride = 1, None
    if t.stride(-1) != 1 and c > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous, got strides {t.stride()}")
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1:
            continue
        if stride is None:
            stride = s
        elif s != rows * stride:
            raise ValueError(f"{name}: rows must be evenly apart, got strides {t.stride()}")
        rows *= n
    return t.data_ptr(), rows, c, c if stride is None else stride


def sw_layer_norm(x, weight=None, bias=None, eps: float = 1e-5, stats: bool = False, out=None, stream=None):
    """Layer norm over the last dimension: x [..., C] fp32, bf16 or half, weight and bias [C] fp32 or None -> y as x;
    with `stats` (y, mean, rstd), the statistics [...] fp32 that sw_layer_norm_backward takes."""
    if out is None and stream is None:
        y = binding._native(binding._LAYER_NORM, x, weight, bias, eps, stats)
        if y is not None:
            return _done(y, "sw_layer_norm")
    import torch

    code = _type(x, "x")
    px, rows, c, x_stride = _rows(x, None, "x")
    w, b = _plain(weight, torch.float32, (c,), "weight"), _plain(bias, torch.float32, (c,), "bias")
    mean = rstd = None
    with _on(stream):
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        if stats:
            mean, rstd = (torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) for _ in range(2))
    py, _, _, y_stride = _rows(out, x, "out")
    rc = lib().sw_layer_norm(px, w, b, py, mean.data_ptr() if stats else None, rstd.data_ptr() if stats else None, rows, c, x_stride, y_stride,
                             eps, code, _stream(stream))
    _check(rc, "sw_layer_norm")
    return (out, mean, rstd) if stats else out


def sw_layer_norm_backward(dy, x, weight, mean, rstd, params: bool = True, out=None, stream=None):
    """Gradients of sw_layer_norm: dy and x [..., C], weight [C] fp32 or None, mean and rstd [...] as the forward call returned
    them -> (dx, dweight, dbias), dx as x (`out` where given), dweight and dbias [C] fp32, or None with `params` False."""
    if out is None and stream is None:
        y = binding._native(binding._LAYER_NORM_BACKWARD, dy, x, weight, mean, rstd, params)
        if y is not None:
            return _done(y, "sw_layer_norm_backward")
    import torch

    code = _type(x, "x")
    px, rows, c, x_stride = _rows(x, None, "x")
    pdy, _, _, dy_stride = _rows(dy, x, "dy")
    w = _plain(weight, torch.float32, (c,), "weight")
    m, r = _plain(mean, torch.float32, x.shape[:-1], "mean"), _plain(rstd, torch.float32, x.shape[:-1], "rstd")
    if m is None or r is None:
        raise ValueError("mean and rstd are those that sw_layer_norm returned")
    L = lib()
    dweight = dbias = work = None
    need = 0
    with _on(stream):
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        if params:
            dweight, dbias = (torch.empty(c, dtype=torch.float32, device=x.device) for _ in range(2))
            need = L.sw_layer_norm_backward_workspace_bytes(rows, c)
            work = torch.empty(need, dtype=torch.uint8, device=x.device)
    pdx, _, _, dx_stride = _rows(out, x, "out")
    rc = L.sw_layer_norm_backward(pdy, px, w, m, r, pdx, dweight.data_ptr() if params else None, dbias.data_ptr() if params else None, rows, c,
                                  dy_stride, x_stride, dx_stride, code, work.data_ptr() if params else None, need, _stream(stream))
    _check(rc, "sw_layer_norm_backward")
    return out, dweight, dbias


def _heads(t, shape, dtype, name):
    """(address, strides) of a tensor of that shape, [..., heads, width] with two, one or no dimensions in front."""
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dtype != dtype or tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected {dtype} {shape}, got {t.dtype} {tuple(t.shape)}")
    s = t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous, got strides {s}")
    return t.data_ptr(), SwStrides(s[0] if len(s) == 4 else 0, s[-3], s[-2])


def _states(t, dims, count, name):
    """The address of contiguous fp32 states [count, heads, dk, dv] (count None: any number); None for None."""
    if t is None:
        return None
    import torch

    want = (t.shape[0] if count is None and t.dim() else count, dims.heads, dims.dk, dims.dv)
    return _plain(t, torch.float32, want, name)


def _attention(q, k, v, log_decay, scale, starts, slots, what):
    """Shapes of an attention call: its dims, the shape of q without its width, and the plain tensors' addresses."""
    import torch

    lead = 1 if starts is not None else 2
    if q.dim() != lead + 2 or k.dim() != lead + 2 or v.dim() != lead + 2:
        raise ValueError(f"{what}: q, k and v have {lead + 2} dimensions, got {tuple(q.shape)}, {tuple(k.shape)}, {tuple(v.shape)}")
    front, (heads, dk), (kv_heads, dv) = tuple(q.shape[:lead]), q.shape[-2:], v.shape[-2:]
    B = front[0] if lead == 2 else starts.shape[0] - 1 if starts.dim() == 1 else 0
    if B <= 0 or 0 in front or 0 in (heads, kv_heads, dk, dv) or heads % kv_heads:
        raise SwError(SW_ERR_SHAPE, what)
    dims = SwLinearAttentionDims(front[-1], B, heads, kv_heads, dk, dv, 0, _type(q, "q"), dk ** -0.5 if scale is None else scale)
    return (dims, front, _plain(log_decay, torch.float32, (heads,), "log_decay"), _plain(starts, torch.int32, (B + 1,), "starts"),
            _plain(slots, torch.int32, (B,), "slots"))


def _workspace(need, q):
    import torch

    return torch.empty(need, dtype=torch.uint8, device=q.device) if need else None


def sw_linear_attention(q, k, v, log_decay, scale=None, starts=None, state=None, slots=None, final_state=None, out=None, stream=None):
    """Linear attention with a decay for each head: q [B,T,heads,dk], k [B,T,kv_heads,dk], v [B,T,kv_heads,dv], log_decay [heads] fp32
    -> o [B,T,heads,dv];  S_t = exp(log_decay) * S_{t-1} + k_t v_t^T,  o_t = scale * S_t^T q_t  (scale: dk ** -0.5 unless given).

    Packed sequences of different lengths: starts [B+1] int32, and q, k, v, o without the first dimension.
    state [n,heads,dk,dv] fp32: what the sequences start from (None: zeros); final_state, as state: where their last states are
    written (may be `state`; None: not kept); slots [B] int32: the sequences' entries of both (None: in order)."""
    if out is None and stream is None:
        y = binding._native(binding._ATTENTION, q, k, v, log_decay, scale, starts, state, slots, final_state)
        if y is not None:
            return _done(y, "sw_linear_attention")
    import torch

    dims, front, g, s, at = _attention(q, k, v, log_decay, scale, starts, slots, "sw_linear_attention")
    held = state if state is not None else final_state
    if held is not None:
        dims.n_states = held.shape[0] if held.dim() else 0
    ps, pf = _states(state, dims, dims.n_states, "state"), _states(final_state, dims, dims.n_states, "final_state")
    pq, sq = _heads(q, (*front, dims.heads, dims.dk), q.dtype, "q")
    pk, sk = _heads(k, (*front, dims.kv_heads, dims.dk), q.dtype, "k")
    pv, sv = _heads(v, (*front, dims.kv_heads, dims.dv), q.dtype, "v")
    L = lib()
    need = L.sw_linear_attention_workspace_bytes(dims, starts is not None)
    with _on(stream):
        if out is None:
            out = torch.empty((*front, dims.heads, dims.dv), dtype=q.dtype, device=q.device)
        work = _workspace(need, q)
    po, so = _heads(out, (*front, dims.heads, dims.dv), q.dtype, "out")
    rc = L.sw_linear_attention(pq, pk, pv, po, g, ps, pf, at, s, dims, sq, sk, sv, so, work.data_ptr() if need else None, need, _stream(stream))
    _check(rc, "sw_linear_attention")
    return out


def sw_linear_attention_backward(do, q, k, v, log_decay, scale=None, starts=None, state=None, slots=None, d_final_state=None, d_state=None,
                                 out=None, stream=None):
    """Gradients of sw_linear_attention, from do (as o) and, where the final states went on, d_final_state [B,heads,dk,dv] fp32
    -> (dq, dk, dv) as q, k, v (`out`: the three to write into); d_state [B,heads,dk,dv] fp32 is filled where given (it may be
    d_final_state).  The other arguments are the forward call's."""
    if out is None and stream is None:
        y = binding._native(binding._ATTENTION_BACKWARD, do, q, k, v, log_decay, scale, starts, state, slots, d_final_state, d_state)
        if y is not None:
            return _done(y, "sw_linear_attention_backward")
    import torch

    dims, front, g, s, at = _attention(q, k, v, log_decay, scale, starts, slots, "sw_linear_attention_backward")
    if state is not None:
        dims.n_states = state.shape[0] if state.dim() else 0
    ps = _states(state, dims, dims.n_states, "state")
    pdf, pds = _states(d_final_state, dims, dims.B, "d_final_state"), _states(d_state, dims, dims.B, "d_state")
    pdo, sdo = _heads(do, (*front, dims.heads, dims.dv), q.dtype, "do")
    shapes = (*front, dims.heads, dims.dk), (*front, dims.kv_heads, dims.dk), (*front, dims.kv_heads, dims.dv)
    (pq, sq), (pk, sk), (pv, sv) = (_heads(t, shape, q.dtype, n) for t, shape, n in zip((q, k, v), shapes, "qkv"))
    L = lib()
    need = L.sw_linear_attention_backward_workspace_bytes(dims, starts is not None)
    with _on(stream):
        if out is None:
            out = tuple(torch.empty(shape, dtype=q.dtype, device=q.device) for shape in shapes)
        work = _workspace(need, q)
    (pdq, sdq), (pdk, sdk), (pdv, sdv) = (_heads(t, shape, q.dtype, n) for t, shape, n in zip(out, shapes, ("dq", "dk", "dv")))
    rc = L.sw_linear_attention_backward(pdo, pq, pk, pv, g, ps, pdf, pdq, pdk, pdv, pds, at, s, dims, sdo, sq, sk, sv, sdq, sdk, sdv,
                                        work.data_ptr() if need else None, need, _stream(stream))
    _check(rc, "sw_linear_attention_backward")
    return tuple(out)


def sw_linear_attention_step(q, k, v, log_decay, state, slots=None, scale=None, out=None, stream=None):
    """One token of each of B requests on a cache of states, brought up to date in place: q [B,heads,dk], k [B,kv_heads,dk],
    v [B,kv_heads,dv], state [n,heads,dk,dv] fp32, slots [B] int32 (None: in order) -> o [B,heads,dv].  A row whose slot is
    out of range (-1: unused) gets zeros and touches no state."""
    if out is None and stream is None:
        y = binding._native(binding._ATTENTION_STEP, q, k, v, log_decay, scale, state, slots)
        if y is not None:
            return _done(y, "sw_linear_attention_step")
    import torch

    if q.dim() != 3 or k.dim() != 3 or v.dim() != 3:
        raise ValueError(f"sw_linear_attention_step: q, k and v have 3 dimensions, got {tuple(q.shape)}, {tuple(k.shape)}, {tuple(v.shape)}")
    (B, heads, dk), (kv_heads, dv) = q.shape, v.shape[1:]
    if 0 in (B, heads, kv_heads, dk, dv) or heads % kv_heads:
        raise SwError(SW_ERR_SHAPE, "sw_linear_attention_step")
    dims = SwLinearAttentionDims(1, B, heads, kv_heads, dk, dv, state.shape[0] if state.dim() else 0, _type(q, "q"), dk ** -0.5 if scale is None else scale)
    g, ps, at = _plain(log_decay, torch.float32, (heads,), "log_decay"), _states(state, dims, None, "state"), _plain(slots, torch.int32, (B,), "slots")
    tensors = (q, (B, heads, dk)), (k, (B, kv_heads, dk)), (v, (B, kv_heads, dv))
    (pq, sq), (pk, sk), (pv, sv) = (_step_rows(t, shape, q.dtype, n) for (t, shape), n in zip(tensors, "qkv"))
    if out is None:
        with _on(stream):
            out = torch.empty((B, heads, dv), dtype=q.dtype, device=q.device)
    po, so = _step_rows(out, (B, heads, dv), q.dtype, "out")
    _check(lib().sw_linear_attention_step(pq, pk, pv, po, g, ps, at, dims, sq, sk, sv, so, _stream(stream)), "sw_linear_attention_step")
    return out


def _step_rows(t, shape, dtype, name):
    p, s = _heads(t, shape, dtype, name)
    return p, SwStrides(s.token, 0, s.head)
