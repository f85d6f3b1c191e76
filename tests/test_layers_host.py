"""Layer norm and linear attention without a GPU: the refusals of the C entry points on addresses that are never used, those of the
Python ones, and the 64-bit definitions against each other and against differences."""
import ctypes

import pytest

from paper_2310_05218_amd import binding as B

torch = pytest.importorskip("torch")

import layers_oracle as O  # noqa: E402  (tests/ is on the path)

X, W, Y, M, R, Z = (0x10000000 * i for i in range(1, 7))


@pytest.fixture(scope="module")
def L():
    import os

    if not os.path.exists(B.LIB_PATH):
        from paper_2310_05218_amd import build
        build.build()
    return B.lib()


def test_layer_norm_refusals(L):
    f = lambda x=X, w=W, b=W + 0x1000, y=Y, m=M, r=R, rows=4, C=64, xs=64, ys=64, eps=1e-5, t=B.SW_F32: \
        L.sw_layer_norm(x, w, b, y, m, r, rows, C, xs, ys, eps, t, None)
    assert f(x=None) == f(y=None) == B.SW_ERR_NULL
    for bad in (dict(rows=0), dict(rows=-1), dict(C=0), dict(xs=63), dict(ys=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(rows=1 << 62), dict(xs=1 << 60)):
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    assert f(C=(1 << 20) + 1, xs=1 << 21, ys=1 << 21) == B.SW_ERR_UNSUPPORTED
    assert f(t=3) == f(t=-1) == B.SW_ERR_UNSUPPORTED
    for bad in (dict(x=X + 2), dict(y=Y + 1), dict(w=W + 1), dict(b=W + 0x1002), dict(m=M + 2), dict(r=R + 3), dict(x=X + 1, t=B.SW_BF16)):
        assert f(**bad) == B.SW_ERR_ALIGN, bad
    for bad in (dict(y=X + 64), dict(y=X, ys=128), dict(m=X), dict(r=M + 4), dict(y=W - 64), dict(m=Y + 4 * 255)):
        assert f(**bad) == B.SW_ERR_ALIAS, bad


def test_layer_norm_backward_refusals(L):
    need = L.sw_layer_norm_backward_workspace_bytes(4, 64)
    assert need > 0 and L.sw_layer_norm_backward_workspace_bytes(0, 64) == L.sw_layer_norm_backward_workspace_bytes(4, 0) == 0
    f = lambda dy=X, x=Y, w=W, m=M, r=R, dx=Z, dw=Z + 0x100000, db=Z + 0x200000, rows=4, C=64, s=(64, 64, 64), t=B.SW_F32, ws=Z + 0x300000, \
        n=need: L.sw_layer_norm_backward(dy, x, w, m, r, dx, dw, db, rows, C, *s, t, ws, n, None)
    for bad in (dict(dy=None), dict(x=None), dict(m=None), dict(r=None), dict(dx=None, dw=None, db=None)):
        assert f(**bad) == B.SW_ERR_NULL, bad
    for bad in (dict(rows=0), dict(C=0), dict(s=(63, 64, 64)), dict(s=(64, 1, 64)), dict(s=(64, 64, 63))):
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    assert f(t=7) == B.SW_ERR_UNSUPPORTED
    for bad in (dict(dy=X + 1), dict(dx=Z + 2), dict(dw=Z + 0x100001), dict(m=M + 1)):
        assert f(**bad) == B.SW_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(n=need - 1), dict(ws=Z + 0x300004)):
        assert f(**bad) == B.SW_ERR_WORKSPACE, bad
    for bad in (dict(dx=X, s=(64, 64, 65)), dict(dx=Y + 4), dict(dw=X), dict(db=Z + 0x100000), dict(ws=Y), dict(ws=Z + 0x100000)):
        assert f(**bad) == B.SW_ERR_ALIAS, bad


def dims(**k):
    d = dict(T=10, B=2, heads=4, kv_heads=2, dk=16, dv=32, n_states=2, type=B.SW_F32, scale=0.25)
    d.update(k)
    return B.SwLinearAttentionDims(**d)


def strides(tokens, heads, width):
    return B.SwStrides(tokens * heads * width, heads * width, width)


BAD_DIMS = [dict(T=0), dict(T=-3), dict(B=0), dict(heads=0), dict(kv_heads=3), dict(kv_heads=0), dict(dk=0), dict(dv=-1), dict(n_states=-1),
            dict(n_states=1), dict(scale=float("nan")), dict(scale=float("inf")), dict(T=1 << 60)]


def test_attention_refusals(L):
    sq, sk, sv, so = strides(10, 4, 16), strides(10, 2, 16), strides(10, 2, 32), strides(10, 4, 32)
    ws = Z + 0x8000000

    def f(q=X, k=Y, v=W, o=M, g=R, s=R + 0x1000, fs=Z, slots=None, starts=None, d=None, a=sq, b=sk, c=sv, e=so, w=ws, n=1 << 26, **k2):
        return L.sw_linear_attention(q, k, v, o, g, s, fs, slots, starts, dims(**k2) if d is None else d, a, b, c, e, w, n, None)

    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(g=None), dict(a=None), dict(e=None)):
        assert f(**bad) == B.SW_ERR_NULL, bad
    assert L.sw_linear_attention(X, Y, W, M, R, None, None, None, None, None, sq, sk, sv, so, ws, 1 << 26, None) == B.SW_ERR_NULL
    for bad in BAD_DIMS:
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    for bad in (dict(a=B.SwStrides(640, -1, 16)), dict(e=B.SwStrides(1280, 128, 31)), dict(e=B.SwStrides(0, 128, 32)), dict(e=B.SwStrides(1280, 32, 32)),
                dict(c=B.SwStrides(1 << 60, 64, 32))):
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    assert f(starts=R + 0x20000, T=1 << 31, o=1 << 46) == B.SW_ERR_SHAPE
    for bad in (dict(dk=257, a=strides(10, 4, 257), b=strides(10, 2, 257)), dict(dv=300, c=strides(10, 2, 300), e=strides(10, 4, 300)), dict(type=5)):
        assert f(**bad) == B.SW_ERR_UNSUPPORTED, bad
    for bad in (dict(q=X + 2), dict(v=W + 1), dict(g=R + 2), dict(s=R + 0x1002), dict(fs=Z + 1), dict(slots=R + 0x20001), dict(starts=R + 0x20002)):
        assert f(**bad) == B.SW_ERR_ALIGN, bad
    for bad in (dict(o=X), dict(fs=Y), dict(fs=R + 0x1004), dict(o=R + 0x1000), dict(fs=M)):
        assert f(**bad) == B.SW_ERR_ALIAS, bad
    need = L.sw_linear_attention_workspace_bytes(dims(T=5000), 0)
    if need:
        big = [strides(5000, h, w) for h, w in ((4, 16), (2, 16), (2, 32), (4, 32))]
        far = dict(zip("abce", big), T=5000)
        assert f(**far, w=None) == f(**far, n=need - 1) == f(**far, w=ws + 8) == B.SW_ERR_WORKSPACE
    assert L.sw_linear_attention_workspace_bytes(dims(T=0), 0) == 0


def test_attention_sizes_of_a_launch(L):
    """Packed rows count once, not once a sequence; what no launch has threads for is refused, workspace and call alike."""
    many = dims(T=1 << 23, B=1000, heads=16, kv_heads=16, dk=64, dv=64, n_states=0)
    state = 16 * 64 * 64 * 4
    assert 1000 * state <= L.sw_linear_attention_workspace_bytes(many, 1) <= 2000 * state
    assert L.sw_linear_attention_backward_workspace_bytes(many, 1) == 2 * L.sw_linear_attention_workspace_bytes(many, 1)
    most = dims(T=64, B=(1 << 24) // 96, heads=32, kv_heads=16, n_states=0)         # 2^24 / 3 heads of sequences
    assert L.sw_linear_attention_backward_workspace_bytes(most, 0) > 0
    more = dims(T=64, B=(1 << 24) // 96 + 1, heads=32, kv_heads=16, n_states=0)
    assert L.sw_linear_attention_backward_workspace_bytes(more, 0) == 0
    s = B.SwStrides(64 * 32 * 16, 32 * 16, 16), B.SwStrides(64 * 16 * 16, 16 * 16, 16), B.SwStrides(64 * 16 * 32, 16 * 32, 32), B.SwStrides(64 * 32 * 32, 32 * 32, 32)
    T = 1 << 44
    call = lambda d: L.sw_linear_attention_backward(T, 2 * T, 3 * T, 4 * T, X, None, None, 5 * T, 6 * T, 7 * T, None, None, None, d, s[3], *s[:3], *s[:3], None, 0, None)
    assert call(more) == B.SW_ERR_SHAPE and call(most) == B.SW_ERR_WORKSPACE


def test_attention_backward_refusals(L):
    sq, sk, sv, so = strides(10, 4, 16), strides(10, 2, 16), strides(10, 2, 32), strides(10, 4, 32)
    need = L.sw_linear_attention_backward_workspace_bytes(dims(), 0)
    assert need > 0 and L.sw_linear_attention_backward_workspace_bytes(dims(kv_heads=3), 0) == 0
    at = 0x1000000

    def f(do=X, q=X + at, k=X + 2 * at, v=X + 3 * at, g=X + 4 * at, s=Y, df=Y + at, gq=W, gk=W + at, gv=W + 2 * at, gs=W + 3 * at, slots=None,
          starts=None, st=None, w=Z, n=need, **k2):
        st = st or (so, sq, sk, sv, sq, sk, sv)
        return L.sw_linear_attention_backward(do, q, k, v, g, s, df, gq, gk, gv, gs, slots, starts, dims(**k2), *st, w, n, None)

    for bad in (dict(do=None), dict(q=None), dict(gq=None), dict(gk=None), dict(gv=None), dict(g=None)):
        assert f(**bad) == B.SW_ERR_NULL, bad
    for bad in BAD_DIMS:
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    assert f(st=(so, sq, sk, sv, sq, B.SwStrides(0, 32, 16), sv)) == B.SW_ERR_SHAPE
    assert f(gq=W + 2) == f(gs=W + 3 * at + 1) == B.SW_ERR_ALIGN
    for bad in (dict(w=None), dict(n=need - 1), dict(w=Z + 4)):
        assert f(**bad) == B.SW_ERR_WORKSPACE, bad
    for bad in (dict(gq=X), dict(gk=X + 2 * at), dict(gs=Y), dict(gs=W), dict(w=W + at), dict(gv=Y + at)):
        assert f(**bad) == B.SW_ERR_ALIAS, bad


def test_attention_step_refusals(L):
    s4, s2 = B.SwStrides(4 * 16, 0, 16), B.SwStrides(2 * 16, 0, 16)

    def f(q=X, k=Y, v=W, o=M, g=R, s=Z, slots=None, a=s4, b=s2, c=s2, e=s4, **k2):
        return L.sw_linear_attention_step(q, k, v, o, g, s, slots, dims(**{**dict(T=1, dv=16), **k2}), a, b, c, e, None)

    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(g=None), dict(s=None), dict(a=None)):
        assert f(**bad) == B.SW_ERR_NULL, bad
    for bad in BAD_DIMS + [dict(T=2), dict(n_states=0), dict(e=B.SwStrides(15, 0, 16))]:
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    assert f(dk=300, a=B.SwStrides(1200, 0, 300), b=B.SwStrides(600, 0, 300)) == B.SW_ERR_UNSUPPORTED
    for bad in (dict(q=X + 1), dict(s=Z + 4), dict(slots=R + 0x1001)):
        assert f(**bad) == B.SW_ERR_ALIGN, bad
    for bad in (dict(o=X), dict(s=Y), dict(o=Z), dict(g=Z)):
        assert f(**bad) == B.SW_ERR_ALIAS, bad


def test_python_refusals():
    import paper_2310_05218_amd as sw

    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="x must live on the GPU"):
        sw.sw_layer_norm(x)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        sw.sw_layer_norm(x.double())
    with pytest.raises(ValueError, match="3 dimensions"):
        sw.sw_linear_attention_step(x, x, x, x, x)
    with pytest.raises(ValueError, match="4 dimensions"):
        sw.sw_linear_attention(x, x, x, x)
    q = torch.zeros(2, 3, 4, 8)
    with pytest.raises(ValueError, match="log_decay must live on the GPU"):
        sw.sw_linear_attention(q, q, q, torch.zeros(4))
    with pytest.raises(sw.SwError):                                   # 4 heads on 3 rows of keys and values
        sw.sw_linear_attention(q, q[:, :, :3], q[:, :, :3], torch.zeros(4))
    with pytest.raises(sw.SwError):
        sw.sw_linear_attention(q[:, :0], q[:, :0], q[:, :0], torch.zeros(4))


@pytest.mark.parametrize("T", [1, 2, 7])
def test_gradients_of_the_definition_by_differences(T):
    """The backward recurrence against central differences of the forward one in 64 bits (both linear in each operand, so the
    differences are exact up to rounding)."""
    g = torch.Generator().manual_seed(T)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    q, k, v, s0, do, df = r(T, 4, 3), r(T, 2, 3), r(T, 2, 5), r(4, 3, 5), r(T, 4, 5), r(4, 3, 5)
    decay = -torch.rand(4, generator=g, dtype=torch.float64)

    def loss(q, k, v, s0):
        o, s = O.attention(q, k, v, decay, 0.7, s0)
        return float((o * do).sum() + (s * df).sum())

    grads = O.attention_backward(do, q, k, v, decay, 0.7, s0, df)
    base = [q, k, v, s0]
    for i, grad in enumerate(grads):
        step = r(*base[i].shape)
        ends = [loss(*(b + e * step if j == i else b for j, b in enumerate(base))) for e in (0.5, -0.5)]
        assert abs(ends[0] - ends[1] - float((grad * step).sum())) < 1e-9


def test_layer_norm_gradient_by_differences():
    g = torch.Generator().manual_seed(3)
    x, w, dy, dirx = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 11), (11,), (3, 11), (3, 11)))
    dx, dw, db = O.layer_norm_backward(dy, x, w, 1e-5)
    e = 1e-5
    f = lambda x, w: float((O.layer_norm(x, w, None, 1e-5)[0] * dy).sum())
    assert abs((f(x + e * dirx, w) - f(x - e * dirx, w)) / (2 * e) - float((dx * dirx).sum())) < 1e-7
    assert abs(f(x, w + dirx[0]) - f(x, w) - float((dw * dirx[0]).sum())) < 1e-9
    assert torch.allclose(db, dy.sum(0))
