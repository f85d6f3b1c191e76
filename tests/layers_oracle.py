"""Layer norm and linear attention in 64 bits, token by token, on the CPU: the definitions, sharing no code with the library."""
import torch


def layer_norm(x, weight, bias, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    rstd = (((x - mean) ** 2).mean(-1, keepdim=True) + eps) ** -0.5
    hat = (x - mean) * rstd
    y = hat if weight is None else hat * weight.double()
    return (y if bias is None else y + bias.double()), mean.squeeze(-1), rstd.squeeze(-1)


def layer_norm_backward(dy, x, weight, eps):
    """By autograd of the definition."""
    x = x.double().detach().requires_grad_(True)
    w = (torch.ones(x.shape[-1]) if weight is None else weight).double().detach().requires_grad_(True)
    b = torch.zeros(x.shape[-1], dtype=torch.float64, requires_grad=True)
    hat = (x - x.mean(-1, keepdim=True)) * ((x - x.mean(-1, keepdim=True)) ** 2).mean(-1, keepdim=True).add(eps) ** -0.5
    return torch.autograd.grad(hat * w + b, (x, w, b), dy.double())


def attention(q, k, v, log_decay, scale, state=None):
    """One sequence: q [T,H,dk], k [T,Hk,dk], v [T,Hk,dv], state [H,dk,dv] -> o [T,H,dv], the last state."""
    share = q.shape[1] // k.shape[1]
    q, k, v = q.double(), k.double().repeat_interleave(share, 1), v.double().repeat_interleave(share, 1)
    decay = torch.exp(log_decay.double())[:, None, None]
    s = torch.zeros(q.shape[1], q.shape[2], v.shape[2], dtype=torch.float64) if state is None else state.double().clone()
    o = torch.zeros(*q.shape[:2], v.shape[2], dtype=torch.float64)
    for t in range(q.shape[0]):
        s = decay * s + k[t][:, :, None] * v[t][:, None, :]
        o[t] = scale * (q[t][:, :, None] * s).sum(1)
    return o, s


def attention_backward(do, q, k, v, log_decay, scale, state=None, d_final=None):
    """One sequence -> dq, dk, dv, d_state: the recurrence backwards, from the states of the forward one."""
    h, share = q.shape[1], q.shape[1] // k.shape[1]
    do, q, ks, vs = do.double(), q.double(), k.double().repeat_interleave(share, 1), v.double().repeat_interleave(share, 1)
    decay = torch.exp(log_decay.double())[:, None, None]
    s = torch.zeros(h, q.shape[2], vs.shape[2], dtype=torch.float64) if state is None else state.double().clone()
    g = torch.zeros_like(s) if d_final is None else d_final.double().clone()
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(ks), torch.zeros_like(vs)
    for t in range(q.shape[0]):
        s = decay * s + ks[t][:, :, None] * vs[t][:, None, :]
        dq[t] = scale * (s * do[t][:, None, :]).sum(2)
    for t in reversed(range(q.shape[0])):
        g = g + scale * q[t][:, :, None] * do[t][:, None, :]
        dk[t], dv[t] = (g * vs[t][:, None, :]).sum(2), (g * ks[t][:, :, None]).sum(1)
        g = decay * g
    fold = lambda x, like: x.reshape(x.shape[0], like.shape[1], share, like.shape[2]).sum(2)
    return dq, fold(dk, k), fold(dv, v), g


def sequences(starts, T, B):
    """Rows of each packed sequence; starts None: of one batch entry each."""
    if starts is None:
        return [(b, slice(0, T)) for b in range(B)]
    clip = lambda x, lo: max(lo, min(int(x), T))
    rows = []
    for b in range(B):
        lo = clip(starts[b], 0)
        rows.append((None, slice(lo, clip(starts[b + 1], lo))))
    return rows
