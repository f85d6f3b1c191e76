"""Thin binding of the gated recurrence, the norms of heads with their rotation and the adapters: argument marshalling, scratch memory,
no arithmetic.  Strides, outputs and streams as in `layers`.
"""
from __future__ import annotations

from . import binding
from .binding import SW_ERR_SHAPE, SwAdaptersDims, SwError, SwGatedRecurrenceDims, SwHeadNormDims, SwStrides, _check, _done, _stream, lib
from .layers import _heads, _on, _plain, _rows, _type, _workspace


def _elsewhere(*tensors):
    """The GPU of a call's tensors where it is not the current one (None: it is, or there is none: tensors off the GPU are refused by name)."""
    import torch

    there = [t.device for t in tensors if t is not None and t.is_cuda]
    for device in there:
        if device != there[0]:
            raise ValueError(f"tensors on {there[0]} and {device} in one call")
    return there[0] if there and there[0].index != torch.cuda.current_device() else None


def _channels(t, shape, dtype, name):
    """(address, strides) of a tensor of that shape, [..., C] with one or two dimensions in front, channels contiguous."""
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dtype != dtype or tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected {dtype} {shape}, got {t.dtype} {tuple(t.shape)}")
    s = t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous, got strides {s}")
    return t.data_ptr(), SwStrides(s[0] if len(s) == 3 else 0, s[-2], 0)


def _recurrence(x, log_decay, starts, slots, what):
    """Shapes of a recurrence call: its dims, and the plain tensors' addresses."""
    import torch

    lead = 1 if starts is not None else 2
    if x.dim() != lead + 1:
        raise ValueError(f"{what}: x has {lead + 1} dimensions, got {tuple(x.shape)}")
    B = x.shape[0] if lead == 2 else starts.shape[0] - 1 if starts.dim() == 1 else 0
    if B <= 0 or 0 in x.shape:
        raise SwError(SW_ERR_SHAPE, what)
    dims = SwGatedRecurrenceDims(x.shape[-2], x.shape[-1], B, 0, _type(x, "x"))
    return (dims, _plain(log_decay, torch.float32, (x.shape[-1],), "log_decay"), _plain(starts, torch.int32, (B + 1,), "starts"),
            _plain(slots, torch.int32, (B,), "slots"))


def _vectors(t, dims, count, name):
    """The address of contiguous fp32 states [count, C]; None for None."""
    if t is None:
        return None
    import torch

    return _plain(t, torch.float32, (count, dims.C), name)


def _tensors(tensors, shape, dtype):
    """Addresses and an array of strides of (tensor, name) pairs."""
    both = [_channels(t, shape, dtype, name) for t, name in tensors]
    return [p for p, _ in both], (SwStrides * len(both))(*(s for _, s in both))


def sw_gated_recurrence(x, decay_gate, input_gate, log_decay, starts=None, state=None, slots=None, final_state=None, out=None, stream=None):
    """Gated linear recurrence: x, decay_gate, input_gate [B,T,C], log_decay [C] fp32 -> h [B,T,C];  a_t = exp(log_decay * sigmoid(decay_gate_t)),
    h_t = a_t * h_{t-1} + sqrt(1 - a_t^2) * sigmoid(input_gate_t) * x_t.

    Packed sequences of different lengths: starts [B+1] int32, and the tensors without the first dimension.  state [n,C] fp32: what the
    sequences start from (None: zeros); final_state, as state: where their last states are written (may be `state`; None: not kept);
    slots [B] int32: the sequences' entries of both (None: in order)."""
    if out is None and stream is None:
        y = binding._native(binding._RECURRENCE, x, decay_gate, input_gate, log_decay, starts, state, slots, final_state)
        if y is not None:
            return _done(y, "sw_gated_recurrence")
    import torch

    other = _elsewhere(x, decay_gate, input_gate, log_decay, starts, state, slots, final_state, out)
    if other is not None:
        with torch.cuda.device(other):
            return sw_gated_recurrence(x, decay_gate, input_gate, log_decay, starts, state, slots, final_state, out, stream)
    dims, g, s, at = _recurrence(x, log_decay, starts, slots, "sw_gated_recurrence")
    held = state if state is not None else final_state
    if held is not None:
        dims.n_states = held.shape[0] if held.dim() else 0
    ps, pf = _vectors(state, dims, dims.n_states, "state"), _vectors(final_state, dims, dims.n_states, "final_state")
    L = lib()
    need = L.sw_gated_recurrence_workspace_bytes(dims, starts is not None)
    with _on(stream):
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        work = _workspace(need, x)
    (px, pr, pi, ph), strides = _tensors(((x, "x"), (decay_gate, "decay_gate"), (input_gate, "input_gate"), (out, "out")), tuple(x.shape), x.dtype)
    rc = L.sw_gated_recurrence(px, pr, pi, g, ph, ps, pf, at, s, dims, strides, work.data_ptr() if need else None, need, _stream(stream))
    _check(rc, "sw_gated_recurrence")
    return out


def sw_gated_recurrence_backward(dh, x, decay_gate, input_gate, log_decay, h, starts=None, state=None, slots=None, d_final_state=None,
                                 d_state=None, params: bool = True, out=None, stream=None):
    """Gradients of sw_gated_recurrence, from dh (as h), its result h and, where the final states went on, d_final_state [B,C] fp32
    -> (dx, d_decay_gate, d_input_gate, d_log_decay), the first three as x (`out`: the three to write into), d_log_decay [C] fp32 or
    None with `params` False; d_state [B,C] fp32 is filled where given (it may be d_final_state).  The other arguments are the forward call's."""
    if out is None and stream is None:
        y = binding._native(binding._RECURRENCE_BACKWARD, dh, x, decay_gate, input_gate, log_decay, h, starts, state, slots, d_final_state, d_state, params)
        if y is not None:
            return _done(y, "sw_gated_recurrence_backward")
    import torch

    other = _elsewhere(dh, x, decay_gate, input_gate, log_decay, h, starts, state, slots, d_final_state, d_state, *(out or ()))
    if other is not None:
        with torch.cuda.device(other):
            return sw_gated_recurrence_backward(dh, x, decay_gate, input_gate, log_decay, h, starts, state, slots, d_final_state, d_state, params, out, stream)
    dims, g, s, at = _recurrence(x, log_decay, starts, slots, "sw_gated_recurrence_backward")
    if state is not None:
        dims.n_states = state.shape[0] if state.dim() else 0
    ps = _vectors(state, dims, dims.n_states, "state")
    pdf, pds = _vectors(d_final_state, dims, dims.B, "d_final_state"), _vectors(d_state, dims, dims.B, "d_state")
    L = lib()
    need = L.sw_gated_recurrence_backward_workspace_bytes(dims, starts is not None)
    with _on(stream):
        if out is None:
            out = tuple(torch.empty(x.shape, dtype=x.dtype, device=x.device) for _ in range(3))
        sums = torch.empty(dims.C, dtype=torch.float32, device=x.device) if params else None
        work = _workspace(need, x)
    names = "dh", "x", "decay_gate", "input_gate", "h", "dx", "d_decay_gate", "d_input_gate"
    (pdh, px, pr, pi, ph, pdx, pdr, pdi), strides = _tensors(tuple(zip((dh, x, decay_gate, input_gate, h, *out), names)), tuple(x.shape), x.dtype)
    rc = L.sw_gated_recurrence_backward(pdh, px, pr, pi, g, ph, ps, pdf, pdx, pdr, pdi, sums.data_ptr() if params else None, pds, at, s, dims, strides,
                                        work.data_ptr() if need else None, need, _stream(stream))
    _check(rc, "sw_gated_recurrence_backward")
    return (*out, sums)


def sw_gated_recurrence_step(x, decay_gate, input_gate, log_decay, state, slots=None, out=None, stream=None):
    """One token of each of B requests on a cache of states, brought up to date in place: x, decay_gate, input_gate [B,C], log_decay [C] fp32,
    state [n,C] fp32, slots [B] int32 (None: in order) -> h [B,C].  A row whose slot is out of range (-1: unused) gets zeros and touches no state."""
    if out is None and stream is None:
        y = binding._native(binding._RECURRENCE_STEP, x, decay_gate, input_gate, log_decay, state, slots)
        if y is not None:
            return _done(y, "sw_gated_recurrence_step")
    import torch

    other = _elsewhere(x, decay_gate, input_gate, log_decay, state, slots, out)
    if other is not None:
        with torch.cuda.device(other):
            return sw_gated_recurrence_step(x, decay_gate, input_gate, log_decay, state, slots, out, stream)
    if x.dim() != 2:
        raise ValueError(f"sw_gated_recurrence_step: x has 2 dimensions, got {tuple(x.shape)}")
    if 0 in x.shape:
        raise SwError(SW_ERR_SHAPE, "sw_gated_recurrence_step")
    B, C = x.shape
    dims = SwGatedRecurrenceDims(1, C, B, state.shape[0] if state.dim() else 0, _type(x, "x"))
    g, ps, at = _plain(log_decay, torch.float32, (C,), "log_decay"), _vectors(state, dims, dims.n_states, "state"), _plain(slots, torch.int32, (B,), "slots")
    if out is None:
        with _on(stream):
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    (px, pr, pi, ph), rows = _tensors(((x, "x"), (decay_gate, "decay_gate"), (input_gate, "input_gate"), (out, "out")), (B, C), x.dtype)
    strides = (SwStrides * 4)(*(SwStrides(s.token, 0, 0) for s in rows))
    _check(lib().sw_gated_recurrence_step(px, pr, pi, g, ph, ps, at, dims, strides, _stream(stream)), "sw_gated_recurrence_step")
    return out


def _head_norm(q, k, q_weight, k_weight, frequencies, positions, eps, interleaved, what):
    """Shapes of a head norm: its dims, the shapes of queries and keys, and the plain tensors' addresses."""
    import torch

    if q.dim() not in (3, 4) or k.dim() != q.dim():
        raise ValueError(f"{what}: q and k have 3 or 4 dimensions, got {tuple(q.shape)}, {tuple(k.shape)}")
    front, (heads, d), kv_heads = tuple(q.shape[:-2]), q.shape[-2:], k.shape[-2]
    if 0 in (*front, heads, kv_heads, d):
        raise SwError(SW_ERR_SHAPE, what)
    if frequencies is not None and frequencies.dim() != 1:
        raise ValueError(f"frequencies: expected one dimension, got {tuple(frequencies.shape)}")
    pairs = 0 if frequencies is None else frequencies.shape[0]
    dims = SwHeadNormDims(front[0] if len(front) == 2 else 1, front[-1], heads, kv_heads, d, pairs, bool(interleaved), _type(q, "q"), eps)
    return (dims, (*front, heads, d), (*front, kv_heads, d), _plain(q_weight, torch.float32, (d,), "q_weight"),
            _plain(k_weight, torch.float32, (d,), "k_weight"), _plain(frequencies, torch.float32, (pairs,), "frequencies"),
            _plain(positions, torch.int32, front, "positions"))


def sw_head_norm(q, k, q_weight=None, k_weight=None, frequencies=None, positions=None, eps: float = 1e-6, interleaved: bool = False, out=None,
                 stream=None):
    """Norms of the heads of queries and keys and their rotation by position, in one pass: q [B,T,heads,d] or [T,heads,d], k the same with
    kv_heads -> (q, k);  n = x / sqrt(mean(x^2) + eps) * weight, then the pairs (k, k + pairs), or (2k, 2k+1) with `interleaved`, turned by
    position * frequencies[k].  Weights [d] fp32 or None (ones); frequencies [pairs] fp32 or None (no rotation), 2 * pairs <= d;
    positions [B,T] or [T] int32 or None (places in the sequence); out: the two to write into (they may be q and k)."""
    if out is None and stream is None:
        y = binding._native(binding._HEAD_NORM, q, k, q_weight, k_weight, frequencies, positions, eps, interleaved)
        if y is not None:
            return _done(y, "sw_head_norm")
    import torch

    other = _elsewhere(q, k, q_weight, k_weight, frequencies, positions, *(out or ()))
    if other is not None:
        with torch.cuda.device(other):
            return sw_head_norm(q, k, q_weight, k_weight, frequencies, positions, eps, interleaved, out, stream)
    dims, shape, kv_shape, wq, wk, f, at = _head_norm(q, k, q_weight, k_weight, frequencies, positions, eps, interleaved, "sw_head_norm")
    with _on(stream):
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device), torch.empty(kv_shape, dtype=q.dtype, device=q.device)
    both = [_heads(t, s, q.dtype, n) for t, s, n in ((q, shape, "q"), (k, kv_shape, "k"), (out[0], shape, "out"), (out[1], kv_shape, "out"))]
    pq, pk, oq, ok = (p for p, _ in both)
    _check(lib().sw_head_norm(pq, pk, wq, wk, f, at, oq, ok, dims, (SwStrides * 4)(*(s for _, s in both)), _stream(stream)), "sw_head_norm")
    return tuple(out)


def sw_head_norm_backward(dq, dk, q, k, q_weight=None, k_weight=None, frequencies=None, positions=None, eps: float = 1e-6,
                          interleaved: bool = False, params: bool = True, out=None, stream=None):
    """Gradients of sw_head_norm, from those of its results and its inputs -> (q_grad, k_grad, q_weight_grad, k_weight_grad), the first two
    as q and k (`out`: the two to write into; they may be dq and dk or q and k), the others [d] fp32, or None with `params` False."""
    if out is None and stream is None:
        y = binding._native(binding._HEAD_NORM_BACKWARD, dq, dk, q, k, q_weight, k_weight, frequencies, positions, eps, interleaved, params)
        if y is not None:
            return _done(y, "sw_head_norm_backward")
    import torch

    other = _elsewhere(dq, dk, q, k, q_weight, k_weight, frequencies, positions, *(out or ()))
    if other is not None:
        with torch.cuda.device(other):
            return sw_head_norm_backward(dq, dk, q, k, q_weight, k_weight, frequencies, positions, eps, interleaved, params, out, stream)
    dims, shape, kv_shape, wq, wk, f, at = _head_norm(q, k, q_weight, k_weight, frequencies, positions, eps, interleaved, "sw_head_norm_backward")
    L = lib()
    sums, work, need = (None, None), None, 0
    with _on(stream):
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device), torch.empty(kv_shape, dtype=q.dtype, device=q.device)
        if params:
            sums = tuple(torch.empty(dims.d, dtype=torch.float32, device=q.device) for _ in range(2))
            need = L.sw_head_norm_backward_workspace_bytes(dims)
            work = _workspace(need, q)
    tensors = (dq, shape, "dq"), (dk, kv_shape, "dk"), (q, shape, "q"), (k, kv_shape, "k"), (out[0], shape, "out"), (out[1], kv_shape, "out")
    both = [_heads(t, s, q.dtype, n) for t, s, n in tensors]
    pdq, pdk, pq, pk, oq, ok = (p for p, _ in both)
    sq, sk = (t.data_ptr() if params else None for t in sums)
    rc = L.sw_head_norm_backward(pdq, pdk, pq, pk, wq, wk, f, at, oq, ok, sq, sk, dims, (SwStrides * 6)(*(s for _, s in both)),
                                 work.data_ptr() if need else None, need, _stream(stream))
    _check(rc, "sw_head_norm_backward")
    return (*out, *sums)


def sw_adapters(x, a, b, y, scales=None, slots=None, starts=None, out=None, stream=None):
    """Low-rank adapters of many requests beside a projection that they share: y + scales[s] * b[s] (a[s] x) for every row, s = slots[sequence].

    x [B,T,C_in] or, a row for each of B sequences, [B,C_in]; y the same with C_out; a [n,rank,C_in], b [n,C_out,rank], scales [n] fp32 or None
    (ones), slots [B] int32 or None (in order).  Packed sequences: starts [B+1] int32, x [T,C_in].  Rows of a sequence whose slot is out
    of range (-1: no adapter), and rows in no sequence, are y's.  -> a new tensor, or `out` (it may be y)."""
    if out is None and stream is None:
        z = binding._native(binding._ADAPTERS, x, a, b, y, scales, slots, starts)
        if z is not None:
            return _done(z, "sw_adapters")
    import torch

    other = _elsewhere(x, a, b, y, scales, slots, starts, out)
    if other is not None:
        with torch.cuda.device(other):
            return sw_adapters(x, a, b, y, scales, slots, starts, out, stream)
    what = "sw_adapters"
    if x.dim() not in ((2,) if starts is not None else (2, 3)) or y.dim() != x.dim() or a.dim() != 3:
        raise ValueError(f"{what}: x and y have 2 or 3 dimensions (2 with starts), a 3, got {tuple(x.shape)}, {tuple(y.shape)}, {tuple(a.shape)}")
    B = x.shape[0] if starts is None else starts.shape[0] - 1 if starts.dim() == 1 else 0
    n, rank, c_in = a.shape
    c_out = y.shape[-1]
    if B <= 0 or 0 in (*x.shape, *a.shape, c_out):
        raise SwError(SW_ERR_SHAPE, what)
    dims = SwAdaptersDims(x.shape[0] if starts is not None else x.shape[1] if x.dim() == 3 else 1, B, c_in, c_out, rank, n, _type(x, "x"))
    pa, pb = _plain(a, x.dtype, (n, rank, c_in), "a"), _plain(b, x.dtype, (n, c_out, rank), "b")
    if pa is None or pb is None:
        raise ValueError("a and b are the adapters' factors")
    if x.shape[-1] != c_in:
        raise ValueError(f"x: expected rows of {c_in}, got {tuple(x.shape)}")
    if y.dtype != x.dtype or y.shape[:-1] != x.shape[:-1]:
        raise ValueError(f"y: expected {x.dtype} rows {tuple(x.shape[:-1])}, got {y.dtype} {tuple(y.shape)}")
    ps = _plain(scales, torch.float32, (n,), "scales")
    at, ends = _plain(slots, torch.int32, (B,), "slots"), _plain(starts, torch.int32, (B + 1,), "starts")
    px, _, _, x_stride = _rows(x, None, "x")
    py, _, _, y_stride = _rows(y, None, "y")
    L = lib()
    need = L.sw_adapters_workspace_bytes(dims, starts is not None)
    with _on(stream):
        if out is None:
            out = torch.empty(y.shape, dtype=y.dtype, device=y.device)
        work = _workspace(need, x)
    po, _, _, out_stride = _rows(out, y, "out")
    rc = L.sw_adapters(px, pa, pb, py, ps, at, ends, po, dims, x_stride, y_stride, out_stride, work.data_ptr() if need else None, need, _stream(stream))
    _check(rc, what)
    return out
