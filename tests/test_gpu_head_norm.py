"""Norms of queries' and keys' heads with their rotation, and the backward pass, on the GPU against the definition in 64 bits.

Tolerances.  A result is rounded once to its format (half a step, e = eps / 2 of it).  With u = 2^-24: a sum of d <= 256 squares is off by at most 16 u (trees and
runs of 16), 1 / sqrt of it by half of that and 3 u, the norm by 4 u more for its products: 16 u.  Sine and cosine are off by 4 u at any angle (taken in 64
bits), so that a turned pair is off by 24 u of its two terms' magnitudes.  The gradient has the rotation (8 u), its product with the weight, a sum over d (16 u of
the magnitudes) and the norm twice: 64 u of its terms' magnitudes.  The weights' gradients are sums over rows and heads in runs and
trees no deeper than 512: 512 u of the magnitudes, beside the 40 u of a term."""
import pytest

import sequence_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}


@pytest.fixture(scope="module")
def sw():
    import paper_2310_05218_amd as _sw
    from paper_2310_05218_amd import binding

    assert torch.cuda.is_available(), "these tests need the GPU"
    binding.lib()            # fails loudly if the library is not built
    return _sw


def make(rows, heads, kv, d, pairs, t, seed, far=100000):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=g)
    q, k, dq, dk = ((f(rows, h, d) * 1.5).to(TYPES[t]) for h in (heads, kv, heads, kv))
    wq, wk = 1 + 0.2 * f(d), 1 + 0.2 * f(d)
    frequencies = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))).float() if pairs else None
    positions = torch.randint(-far, far, (rows,), generator=g).int()
    return q, k, dq, dk, wq, wk, frequencies, positions


def check(got, want, mag, t, k):
    e = torch.finfo(TYPES[t]).eps / 2 if t else 0.0
    tol = e * want.abs() + k * U * mag * (1 + e) + (TINY[t] if t else 1e-37)
    off = (got.cpu().double() - want).abs()
    assert torch.all(off <= tol), f"{float((off / tol).max()):.2f} of the tolerance"


def check_both(t, made, eps, interleaved, out, grads):
    q, k, dq, dk, wq, wk, f, at = made
    for x, dy, w, y, gx, gw in ((q, dq, wq, out[0], grads[0], grads[2]), (k, dk, wk, out[1], grads[1], grads[3])):
        want, m = O.head_norm(x, w, f, at, eps, interleaved)
        check(y, want, m, t, 40)
        dx, dw, dwm, back = O.head_norm_backward(dy, x, w, f, at, eps, interleaved)
        r = (x.double().square().mean(-1, keepdim=True) + eps) ** -0.5
        g = back * (1.0 if w is None else w.double().abs())
        hat = x.double().abs() * r
        check(gx, dx, r * (g + hat * (g * hat).mean(-1, keepdim=True)), t, 64)
        if gw is not None:
            check(gw, dw, dwm, None, 552)


def run(sw, made, eps=1e-6, interleaved=False):
    q, k, dq, dk, wq, wk, f, at = (None if v is None else v.cuda() for v in made)
    out = sw.sw_head_norm(q, k, wq, wk, f, at, eps, interleaved)
    grads = sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f, at, eps, interleaved)
    again = sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f, at, eps, interleaved)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    only = sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f, at, eps, interleaved, params=False)
    assert only[2] is None and only[3] is None and torch.equal(only[0], grads[0]) and torch.equal(only[1], grads[1])
    return out, grads


# d, pairs
WIDTHS = [(1, 0), (2, 1), (3, 1), (4, 2), (6, 3), (8, 4), (8, 2), (10, 5), (16, 8), (20, 10), (24, 12), (31, 15), (32, 16), (32, 8), (34, 17), (48, 24), (64, 32),
          (64, 16), (64, 0), (66, 33), (72, 36), (80, 20), (80, 40), (96, 48), (96, 24), (100, 50), (112, 56), (126, 63), (127, 63), (128, 64), (128, 32),
          (128, 1), (130, 65), (144, 72), (160, 80), (192, 96), (200, 50), (222, 111), (240, 120), (250, 62), (255, 127), (256, 128), (256, 64), (256, 7), (256, 12), (254, 11)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,pairs", WIDTHS)
def test_widths(sw, d, pairs, interleaved, t):
    made = make(9, 3, 2, d, pairs, t, d + pairs)
    check_both(t, made, 1e-6, interleaved, *run(sw, made, 1e-6, interleaved))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,heads,kv,d", [(1, 1, 1, 64), (1, 16, 4, 128), (4, 1, 7, 96), (2, 40, 1, 128), (33, 5, 5, 64), (1000, 6, 3, 80), (257, 32, 8, 128),
                                             (3001, 2, 1, 32), (7, 130, 3, 256), (70, 9, 4, 100)])
def test_rows_and_heads(sw, rows, heads, kv, d, t):
    made = make(rows, heads, kv, d, d // 2, t, rows)
    check_both(t, made, 1e-5, False, *run(sw, made, 1e-5))


@pytest.mark.parametrize("t", TYPES)
def test_no_weights_no_rotation_no_epsilon(sw, t):
    q, k, dq, dk, wq, wk, f, at = make(20, 3, 2, 64, 32, t, 1)
    for made, eps in (((q, k, dq, dk, None, None, f, at), 1e-6), ((q, k, dq, dk, wq, None, None, None), 0.0), ((q, k, dq, dk, None, wk, f, at), 0.5)):
        check_both(t, made, eps, False, *run(sw, made, eps))


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(sw, interleaved):
    """The angle is taken in 64 bits, at any 32-bit position and with frequencies above 1."""
    q, k, dq, dk, wq, wk, f, at = make(64, 2, 1, 64, 32, "f32", 2)
    at[:8] = torch.tensor([2 ** 31 - 1, -2 ** 31, 0, 1, -1, 2 ** 30 + 7, 2 ** 24 + 1, -(2 ** 24) - 1]).int()
    f = torch.cat([f[:28], torch.tensor([3.14159274, 100.3, 0.0, -0.7])])
    made = q, k, dq, dk, wq, wk, f, at
    check_both("f32", made, 1e-6, interleaved, *run(sw, made, 1e-6, interleaved))


@pytest.mark.parametrize("t", TYPES)
def test_positions_are_places_unless_given(sw, t):
    B, T = 3, 50
    q, k, dq, dk, wq, wk, f, _ = make(B * T, 4, 2, 64, 32, t, 3)
    shape = lambda v: v.unflatten(0, (B, T)).cuda()
    at = torch.arange(T).int().repeat(B, 1).cuda()
    q, k, dq, dk, wq, wk, f = shape(q), shape(k), shape(dq), shape(dk), wq.cuda(), wk.cuda(), f.cuda()
    for a, b in zip(sw.sw_head_norm(q, k, wq, wk, f), sw.sw_head_norm(q, k, wq, wk, f, at)):
        assert torch.equal(a, b)
    for a, b in zip(sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f), sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f, at)):
        assert torch.equal(a, b)
    assert torch.equal(sw.sw_head_norm(q[0], k[0], wq, wk, f)[0], sw.sw_head_norm(q, k, wq, wk, f)[0][0])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("d,first", [(64, 0), (64, 1), (128, 8), (80, 4), (48, 3), (100, 2), (33, 5)])
def test_slices_of_a_projection(sw, d, first, t):
    """Queries and keys as slices of a fused projection's rows, results into slices, in place as well; what lies beside them is not touched."""
    rows, heads, kv = 30, 5, 2
    made = make(rows, heads, kv, d, d // 2, t, d)
    q, k, dq, dk, wq, wk, f, at = (v.cuda() for v in made)
    want, grads = sw.sw_head_norm(q, k, wq, wk, f, at), sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f, at)

    def fused(a=None, b=None):
        big = torch.full((rows, first + (heads + 2 * kv) * d + 3), 7.0, dtype=TYPES[t], device="cuda")
        parts = big[:, first:first + heads * d].unflatten(1, (heads, d)), big[:, first + heads * d:first + (heads + kv) * d].unflatten(1, (kv, d))
        if a is not None:
            parts[0].copy_(a), parts[1].copy_(b)
        return big, *parts

    def untouched(big):
        return torch.all(big[:, :first] == 7.0) and torch.all(big[:, first + (heads + kv) * d:] == 7.0)

    src, Q, K = fused(q, k)
    into, A, B = fused()
    sw.sw_head_norm(Q, K, wq, wk, f, at, out=(A, B))
    assert torch.equal(A, want[0]) and torch.equal(B, want[1]) and untouched(into)
    gsrc, DQ, DK = fused(dq, dk)
    into, A, B = fused()
    sums = sw.sw_head_norm_backward(DQ, DK, Q, K, wq, wk, f, at, out=(A, B))[2:]
    assert torch.equal(A, grads[0]) and torch.equal(B, grads[1]) and untouched(into) and all(torch.equal(x, y) for x, y in zip(sums, grads[2:]))
    sw.sw_head_norm_backward(DQ, DK, Q, K, wq, wk, f, at, out=(DQ, DK))
    assert torch.equal(DQ, grads[0]) and torch.equal(DK, grads[1]) and untouched(gsrc)
    src2, Q2, K2 = fused(q, k)
    sw.sw_head_norm_backward(dq, dk, Q2, K2, wq, wk, f, at, out=(Q2, K2))
    assert torch.equal(Q2, grads[0]) and torch.equal(K2, grads[1]) and untouched(src2)
    sw.sw_head_norm(Q, K, wq, wk, f, at, out=(Q, K))
    assert torch.equal(Q, want[0]) and torch.equal(K, want[1]) and untouched(src)


def test_heads_before_tokens(sw):
    q, k, dq, dk, wq, wk, f, at = (v.cuda() for v in make(24, 3, 2, 64, 32, "bf16", 4))
    turned = lambda v: v.unflatten(0, (2, 12)).transpose(1, 2).contiguous().transpose(1, 2)
    at = at.reshape(2, 12)
    four = lambda v: v.unflatten(0, (2, 12))
    for a, b in zip(sw.sw_head_norm(turned(q), turned(k), wq, wk, f, at), sw.sw_head_norm(four(q), four(k), wq, wk, f, at)):
        assert torch.equal(a, b)
    wide = q[:1].expand(24, 3, 64)
    assert torch.equal(sw.sw_head_norm(wide, k, wq, wk, f)[0], sw.sw_head_norm(wide.contiguous(), k, wq, wk, f)[0])


@pytest.mark.parametrize("t", TYPES)
def test_zeros_infinities_and_nans(sw, t):
    """A head of zeros gives zeros (eps > 0) and a gradient scaled by 1 / sqrt(eps); a value that is not finite spoils its own head alone."""
    q, k, dq, dk, wq, wk, f, at = (v.cuda() for v in make(6, 4, 2, 64, 16, t, 5))
    clean, gclean = sw.sw_head_norm(q, k, wq, wk, f, at), sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f, at)
    q[1, 2] = 0
    q[3, 0, 5] = float("nan")
    q[4, 1, 63] = float("inf")
    out, grads = sw.sw_head_norm(q, k, wq, wk, f, at), sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f, at)
    assert torch.all(out[0][1, 2] == 0) and torch.isfinite(grads[0][1, 2]).all()
    assert torch.isnan(out[0][3, 0]).all() and torch.isnan(grads[0][3, 0]).all()
    assert not torch.isfinite(out[0][4, 1]).all()
    left = torch.ones(6, 4, dtype=torch.bool, device="cuda")
    left[1, 2] = left[3, 0] = left[4, 1] = False
    assert torch.equal(out[0][left], clean[0][left]) and torch.equal(grads[0][left], gclean[0][left])
    assert torch.equal(out[1], clean[1]) and torch.equal(grads[1], gclean[1])


def test_gradients_against_differences(sw):
    q, k, dq, dk, wq, wk, f, at = made = make(3, 2, 1, 20, 7, "f32", 6, far=50)
    Q, K, DQ, DK, *rest = (v.cuda() for v in made)
    grads = sw.sw_head_norm_backward(DQ, DK, Q, K, *rest, 1e-3, True)

    def loss(q, k, wq, wk):
        return float((O.head_norm(q, wq, f, at, 1e-3, True)[0] * dq.double()).sum() + (O.head_norm(k, wk, f, at, 1e-3, True)[0] * dk.double()).sum())

    given, step = [v.double() for v in (q, k, wq, wk)], 1e-5
    for n, g in enumerate(grads):
        for i in range(0, g.numel(), 3):
            plus, minus = ([v.clone() for v in given] for _ in range(2))
            plus[n].view(-1)[i] += step
            minus[n].view(-1)[i] -= step
            want = (loss(*plus) - loss(*minus)) / (2 * step)
            assert abs(float(g.reshape(-1)[i]) - want) <= 2e-5 * (1 + abs(want)), (n, i)


def test_another_stream_and_graphs(sw):
    made = [[v.cuda() for v in make(700, 8, 2, 128, 64, "bf16", s)] for s in range(3)]
    held = [v.clone() for v in made[0]]
    q, k, dq, dk, wq, wk, f, at = held
    both = lambda: (*sw.sw_head_norm(q, k, wq, wk, f, at), *sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f, at))
    want = [v.clone() for v in both()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = sw.sw_head_norm(q, k, wq, wk, f, at, stream=side)
    b = sw.sw_head_norm_backward(dq, dk, q, k, wq, wk, f, at, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((*a, *b), want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = both()
    for turn in range(4):
        for v, new in zip(held, made[turn % 3]):
            v.copy_(new)
        want = [v.clone() for v in both()]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_offsets_beyond_32_bits(sw):
    """Rows that lie so far apart that their places take more than 31 bits of elements."""
    rows, d, far = 3, 64, (1 << 30) + 64
    big = torch.zeros(2 * far + d + 64, dtype=torch.bfloat16, device="cuda")
    q = big.as_strided((rows, 1, d), (far, d, 1))
    src = torch.randn(rows, 1, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    q.copy_(src)
    f, at = torch.rand(32).cuda(), torch.arange(rows).int().cuda()
    want = sw.sw_head_norm(src, src, None, None, f, at)
    got = sw.sw_head_norm(q, src, None, None, f, at, out=(q, torch.empty_like(src)))
    assert torch.equal(got[0], want[0])
