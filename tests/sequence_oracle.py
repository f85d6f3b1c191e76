"""The gated recurrence, the norms of heads with their rotation and the adapters in 64 bits, token by token, on the CPU: the definitions,
sharing no code with the library.  Beside a value that is a sum, the sum of its terms' magnitudes, for tolerances."""
import torch


def gates(x, r, i, log_decay):
    """s, p, log of the decay, decay, weight sqrt(1 - decay^2), all in 64 bits.  A gate below fp32's normal numbers is shut: -infinity
    times it is 0."""
    s, p = torch.sigmoid(r.double()), torch.sigmoid(i.double())
    s, log_decay = torch.where(s < 2.0 ** -126, 0.0, s), log_decay.double().clamp(min=-3e38)
    la = log_decay * s
    return s, p, la, torch.exp(la), torch.sqrt(-torch.expm1(2 * la))


def recurrence(x, r, i, log_decay, state=None):
    """One sequence [T,C] -> h [T,C], the last state [C], the same of the terms' magnitudes."""
    s, p, la, a, w = gates(x, r, i, log_decay)
    now = torch.zeros(x.shape[1], dtype=torch.float64) if state is None else state.double()
    mag = now.abs()
    h, m = torch.zeros(x.shape, dtype=torch.float64), torch.zeros(x.shape, dtype=torch.float64)
    for t in range(x.shape[0]):
        new = w[t] * p[t] * x[t].double()
        now, mag = a[t] * now + new, a[t] * mag + new.abs()
        h[t], m[t] = now, mag
    return h, now, m, mag


def recurrence_backward(dh, x, r, i, log_decay, h, state=None, d_final=None):
    """One sequence -> the gradients and their magnitudes, from the forward pass's result as it was rounded."""
    T, C = x.shape
    s, p, la, a, w = gates(x, r, i, log_decay)
    x, h, dh = x.double(), h.double(), dh.double()
    first = torch.zeros(C, dtype=torch.float64) if state is None else state.double()
    later = torch.zeros(C, dtype=torch.float64) if d_final is None else d_final.double()
    mag = later.abs()
    names = ("dx", "dr", "di")
    g, m = {n: torch.zeros(T, C, dtype=torch.float64) for n in names}, {n: torch.zeros(T, C, dtype=torch.float64) for n in names}
    g["dl"], m["dl"] = torch.zeros(C, dtype=torch.float64), torch.zeros(C, dtype=torch.float64)
    for t in range(T - 1, -1, -1):
        u, um = dh[t] + later, dh[t].abs() + mag
        before = h[t - 1] if t else first
        dw = torch.where(w[t] > 0, a[t] * a[t] / w[t], 0.0)
        l, lm = u * (a[t] * before - p[t] * x[t] * dw), um * (a[t] * before.abs() + p[t] * x[t].abs() * dw)
        g["dx"][t], m["dx"][t] = u * w[t] * p[t], um * w[t] * p[t]
        g["di"][t], m["di"][t] = u * w[t] * x[t] * p[t] * (1 - p[t]), um * w[t] * x[t].abs() * p[t] * (1 - p[t])
        g["dr"][t], m["dr"][t] = l * la[t] * (1 - s[t]), lm * la[t].abs() * (1 - s[t])
        g["dl"], m["dl"] = g["dl"] + l * s[t], m["dl"] + lm * s[t]
        later, mag = a[t] * u, a[t] * um
    g["state"], m["state"] = later, mag
    return g, m


def head_norm(x, w, frequencies, positions, eps, interleaved):
    """x [rows, heads, d], positions [rows] -> the result, the magnitudes of its terms."""
    x = x.double()
    n = x * (x.square().mean(-1, keepdim=True) + eps) ** -0.5
    if w is not None:
        n = n * w.double()
    y, m = n.clone(), n.abs()
    for k in range(0 if frequencies is None else frequencies.shape[0]):
        i, j = (2 * k, 2 * k + 1) if interleaved else (k, k + frequencies.shape[0])
        f = (positions.double() * frequencies[k].double())[:, None]
        y[..., i], y[..., j] = n[..., i] * f.cos() - n[..., j] * f.sin(), n[..., i] * f.sin() + n[..., j] * f.cos()
        m[..., i], m[..., j] = ((n[..., i] * f.cos()).abs() + (n[..., j] * f.sin()).abs(), (n[..., i] * f.sin()).abs() + (n[..., j] * f.cos()).abs())
    return y, m


def head_norm_backward(dy, x, w, frequencies, positions, eps, interleaved):
    """By autograd of the definition, written once more with matrices of rotation: dx, dw; the magnitudes of dw's terms."""
    x = x.double().detach().requires_grad_(True)
    d = x.shape[-1]
    weight = (torch.ones(d) if w is None else w).double().detach().requires_grad_(True)
    turn = torch.eye(d, dtype=torch.float64).repeat(x.shape[0], 1, 1)
    for k in range(0 if frequencies is None else frequencies.shape[0]):
        i, j = (2 * k, 2 * k + 1) if interleaved else (k, k + frequencies.shape[0])
        f = positions.double() * frequencies[k].double()
        turn[:, i, i], turn[:, i, j], turn[:, j, i], turn[:, j, j] = f.cos(), -f.sin(), f.sin(), f.cos()
    hat = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + eps)
    y = torch.matmul(turn[:, None], (hat * weight)[..., None])[..., 0]
    dx, dw = torch.autograd.grad(y, (x, weight), dy.double())
    back = torch.matmul(turn.abs().transpose(1, 2)[:, None], dy.double().abs()[..., None])[..., 0]
    return dx, dw, (back * hat.detach().abs()).sum((0, 1)), back


def adapters(x, a, b, y, scales, of):
    """x [rows, C_in], `of`: the adapter of each row, -1 none -> the result and the magnitudes of its terms."""
    out, m = y.double().clone(), y.double().abs()
    for row, s in enumerate(of):
        if s >= 0:
            scale = 1.0 if scales is None else float(scales[s].double())
            out[row] += scale * (b[s].double() @ (a[s].double() @ x[row].double()))
            m[row] += abs(scale) * (b[s].double().abs() @ (a[s].double().abs() @ x[row].double().abs()))
    return out, m
