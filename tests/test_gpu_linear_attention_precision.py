"""Linear attention on the GPU: how far its results are from the definition in 64 bits, rounded once.

Inputs' products and states are summed in 32 bits (u = 2^-24).  With sums of up to T terms in runs of a chunk each, whose roundings are independent,
a result before its last rounding is held to 8 u of it in the 2-norm, and a state, each value, to 16 u of the sum of its terms' magnitudes.
The last rounding then gives another value than that of the exact result where a boundary lies between the two: with a probability of
|error| / step, one step off (at most eps of the value), so that the squared 2-norm of what is off is at most eps * |error| * |value|
summed, and its 2-norm sqrt(8 u eps) of the result's: 2^-14 in bf16, 2^-15.5 in half.  (Operands of 16 or 17 bits: 2^-13.3 and 2^-14.9.)  fp32
results are off by their last rounding besides: 9 u."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def sw():
    import paper_2310_05218_amd as _sw
    from paper_2310_05218_amd import binding

    assert torch.cuda.is_available(), "these tests need the GPU"
    binding.lib()            # fails loudly if the library is not built
    return _sw


def definition(q, k, v, do, g, scale, s0, df, mag):
    """Every pair of tokens of every head, in 64 bits, on magnitudes where `mag` -> o, the last state, dq, dk, dv, the first state's gradient."""
    f = (lambda x: x.double().abs()) if mag else (lambda x: x.double())
    (B, T, H, dk), (Hk, dv) = q.shape, v.shape[2:]
    share = H // Hk
    q, k, v, do, s0, df = (f(x) for x in (q, k, v, do, s0, df))
    o, gq, gk, gv = do.new_zeros(B, T, H, dv), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    last, first = torch.zeros_like(s0), torch.zeros_like(s0)
    t = torch.arange(T, dtype=torch.float64)
    gap = t[:, None] - t[None, :]
    for b in range(B):
        for h in range(H):
            u, l = h // share, g[h].double()
            fade = torch.exp(l * gap.clamp(min=0)) * (gap >= 0)
            up, after, whole = torch.exp(l * (t + 1))[:, None], torch.exp(l * (T - 1 - t))[:, None], torch.exp(l * T)
            Q, K, V, D = q[b, :, h], k[b, :, u], v[b, :, u], scale * do[b, :, h]
            pair, back = (Q @ K.T) * fade, (D @ V.T) * fade
            o[b, :, h] = scale * (pair @ V + up * (Q @ s0[b, h]))
            last[b, h] = K.T @ (after * V) + whole * s0[b, h]
            gq[b, :, h] = back @ K + up * (D @ s0[b, h].T)
            gk[b, :, u] += back.T @ Q + after * (V @ df[b, h].T)
            gv[b, :, u] += pair.T @ D + after * (K @ df[b, h])
            first[b, h] = Q.T @ (up * D) + whole * df[b, h]
    return o, last, gq, gk, gv, first


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,T,H,Hk,dk,dv", [(1, 1000, 4, 4, 128, 128), (2, 200, 16, 16, 64, 64), (3, 600, 8, 2, 64, 96), (1, 900, 4, 4, 136, 200)])
def test_one_rounding(sw, B, T, H, Hk, dk, dv, t):
    r = torch.Generator().manual_seed(T + dk)
    n = lambda *s: torch.randn(s, generator=r)
    q, k, v, do = (n(B, T, h, d).to(TYPES[t]) for h, d in ((H, dk), (Hk, dk), (Hk, dv), (H, dv)))
    s0, df = n(B, H, dk, dv), n(B, H, dk, dv)
    g = torch.log1p(-torch.exp2(-torch.linspace(2, 8, H)))
    scale = dk ** -0.5
    Q, K, V, D, G, S, F = (x.cuda() for x in (q, k, v, do, g, s0, df))
    last, first = torch.empty_like(S), torch.empty_like(S)
    o = sw.sw_linear_attention(Q, K, V, G, scale, state=S, final_state=last)
    grads = sw.sw_linear_attention_backward(D, Q, K, V, G, scale, state=S, d_final_state=F, d_state=first)
    want, mag = (definition(q, k, v, do, g, scale, s0, df, m) for m in (False, True))
    bound = 9 * U if t == "f32" else (8 * U * torch.finfo(TYPES[t]).eps) ** 0.5
    for name, x, w in zip(("o", "dq", "dk", "dv"), (o, *grads), (want[0], *want[2:5])):
        w = w if t == "f32" else w.to(TYPES[t]).double()
        off = float((x.cpu().double() - w).norm() / w.norm())
        assert off <= bound, f"{name}: {off:.3g} off the rounded result, {bound:.3g} allowed"
    for name, x, w, a in (("final_state", last, want[1], mag[1]), ("d_state", first, want[5], mag[5])):
        off = float(((x.cpu().double() - w).abs() / a).max())
        assert off <= 16 * U, f"{name}: {off:.3g} of the terms' magnitudes"


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,T,H,dk,dv", [(1, 1000, 4, 128, 128), (2, 200, 16, 64, 96)])
def test_columns_of_different_magnitudes(sw, B, T, H, dk, dv, t):
    """Neighbouring columns of values, and of what comes of them, 2^20 apart: each keeps its own bits."""
    r = torch.Generator().manual_seed(T)
    n = lambda *s: torch.randn(s, generator=r)
    apart = lambda d: torch.where(torch.arange(d) % 2 == 0, 2.0 ** 8, 2.0 ** -12)
    q, k, v, do = n(B, T, H, dk).to(TYPES[t]), n(B, T, H, dk), (n(B, T, H, dv) * apart(dv)).to(TYPES[t]), n(B, T, H, dv).to(TYPES[t])
    s0 = n(B, H, dk, dv) * apart(dv)
    k = k.to(TYPES[t])
    g = torch.log1p(-torch.exp2(-torch.linspace(2, 8, H)))
    o = sw.sw_linear_attention(*(x.cuda() for x in (q, k, v, g)), state=s0.cuda()).cpu().double()
    w = definition(q, k, v, do, g, dk ** -0.5, s0, torch.zeros_like(s0), False)[0]
    w = w if t == "f32" else w.to(TYPES[t]).double()
    bound = 9 * U if t == "f32" else (8 * U * torch.finfo(TYPES[t]).eps) ** 0.5
    for first in (0, 1):
        off = float((o - w)[..., first::2].norm() / w[..., first::2].norm())
        assert off <= bound, f"columns {first}, {first + 2} ...: {off:.3g} off the rounded result, {bound:.3g} allowed"
