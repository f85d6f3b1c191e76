"""The gated recurrence, the norms of heads and the adapters without a GPU: the refusals of the C entry points on addresses that are never used,
those of the Python ones, and the 64-bit definitions against each other and against differences."""
import pytest

from paper_2310_05218_amd import binding as B

torch = pytest.importorskip("torch")

import paper_2310_05218_amd as sw  # noqa: E402
import sequence_oracle as O  # noqa: E402  (tests/ is on the path)

AT = [0x10000000 * i for i in range(1, 20)]


@pytest.fixture(scope="module")
def L():
    import os

    if not os.path.exists(B.LIB_PATH):
        from paper_2310_05218_amd import build
        build.build()
    return B.lib()


def strides(*of):
    return (B.SwStrides * len(of))(*(B.SwStrides(*s) for s in of))


def recurrence(L, t=None, state=AT[5], final=AT[6], slots=None, starts=None, s=None, work=AT[9], bytes_=1 << 27, g=AT[4], **k):
    d = B.SwGatedRecurrenceDims(**{**dict(T=10, C=16, B=2, n_states=2, type=B.SW_F32), **k})
    t, s = t or AT[:4], s or [(160, 16, 0)] * 4
    return L.sw_gated_recurrence(t[0], t[1], t[2], g, t[3], state, final, slots, starts, d, strides(*s), work, bytes_, None)


def replaced(v, k, new):
    return [new if i == k else x for i, x in enumerate(v)]


BAD_EXTENTS = [dict(T=0), dict(T=-1), dict(B=0), dict(C=0), dict(n_states=-1), dict(n_states=1), dict(T=1 << 60), dict(C=1 << 20, T=1 << 40)]


def test_recurrence_refusals(L):
    f = lambda **k: recurrence(L, **k)
    for i in range(4):
        assert f(t=replaced(AT[:4], i, None)) == B.SW_ERR_NULL
    assert f(g=None) == B.SW_ERR_NULL
    for bad in BAD_EXTENTS + [dict(s=[(160, 16, 0)] * 3 + [(160, 15, 0)]), dict(s=[(160, 16, 0)] * 3 + [(150, 16, 0)]), dict(s=[(-1, 16, 0)] + [(160, 16, 0)] * 3),
                              dict(starts=AT[8], T=1 << 31, t=[1 << 46, 1 << 47, 3 << 46, 5 << 46])]:
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    assert f(C=(1 << 20) + 1, s=[(1 << 26, 1 << 21, 0)] * 4) == f(type=3) == B.SW_ERR_UNSUPPORTED
    for bad in (dict(t=replaced(AT[:4], 1, AT[1] + 2)), dict(g=AT[4] + 1), dict(state=AT[5] + 2), dict(final=AT[6] + 1), dict(slots=AT[7] + 2), dict(starts=AT[8] + 1)):
        assert f(**bad) == B.SW_ERR_ALIGN, bad
    for bad in (dict(t=replaced(AT[:4], 3, AT[0])), dict(t=replaced(AT[:4], 3, AT[1] + 64)), dict(final=AT[3]), dict(final=AT[5] + 64), dict(final=AT[4]),
                dict(t=replaced(AT[:4], 3, AT[5]))):
        assert f(**bad) == B.SW_ERR_ALIAS, bad
    # slices of one tensor's rows: apart, and not apart
    wide = [(480, 48, 0)] * 4
    assert f(t=[AT[0], AT[1], AT[2], AT[0] + 60], s=wide) == B.SW_ERR_ALIAS
    assert f(t=[AT[0], AT[1], AT[2], AT[0] + 64], s=[(480, 48, 0)] * 3 + [(480, 40, 0)]) == B.SW_ERR_ALIAS
    d = B.SwGatedRecurrenceDims(20000, 512, 1, 0, B.SW_BF16)
    need = L.sw_gated_recurrence_workspace_bytes(d, 0)
    if need:
        far = dict(T=20000, C=512, B=1, type=B.SW_BF16, s=[(0, 512, 0)] * 4)
        assert f(**far, work=None) == f(**far, bytes_=need - 1) == f(**far, work=AT[9] + 8) == B.SW_ERR_WORKSPACE
        assert f(**far, work=AT[0]) == B.SW_ERR_ALIAS
    assert L.sw_gated_recurrence_workspace_bytes(B.SwGatedRecurrenceDims(0, 512, 1, 0, 0), 0) == 0


def test_recurrence_backward_refusals(L):
    d0 = dict(T=1000, C=16, B=2, n_states=2, type=B.SW_F32)
    need = L.sw_gated_recurrence_backward_workspace_bytes(B.SwGatedRecurrenceDims(**d0), 0)
    assert need > 0

    def f(t=None, g=AT[8], state=AT[9], df=AT[10], dl=AT[11], ds=AT[12], s=None, work=AT[13], bytes_=need, slots=None, starts=None, **k):
        t, s = t or AT[:8], s or [(16000, 16, 0)] * 8
        dims = B.SwGatedRecurrenceDims(**{**d0, **k})
        return L.sw_gated_recurrence_backward(t[0], t[1], t[2], t[3], g, t[4], state, df, t[5], t[6], t[7], dl, ds, slots, starts, dims, strides(*s), work, bytes_, None)

    for i in range(8):
        assert f(t=replaced(AT[:8], i, None)) == B.SW_ERR_NULL
        assert f(t=replaced(AT[:8], i, AT[i] + 2)) == B.SW_ERR_ALIGN
    for bad in BAD_EXTENTS + [dict(s=[(16000, 16, 0)] * 7 + [(16000, 8, 0)])]:
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    for bad in (dict(work=None), dict(bytes_=need - 1), dict(work=AT[13] + 4)):
        assert f(**bad) == B.SW_ERR_WORKSPACE, bad
    for bad in (dict(t=replaced(AT[:8], 5, AT[0])), dict(t=replaced(AT[:8], 6, AT[5])), dict(t=replaced(AT[:8], 7, AT[5] + 64)), dict(ds=AT[9]), dict(dl=AT[8]),
                dict(ds=AT[10] + 64), dict(work=AT[7]), dict(dl=AT[12])):
        assert f(**bad) == B.SW_ERR_ALIAS, bad
    assert f(t=[*AT[:5], AT[5], AT[5] + 60, AT[5] + 128], s=[(16000, 16, 0)] * 5 + [(48000, 48, 0)] * 3) == B.SW_ERR_ALIAS


def test_recurrence_step_refusals(L):
    def f(t=None, g=AT[4], state=AT[5], slots=None, s=None, **k):
        t, s = t or AT[:4], s or [(16, 0, 0)] * 4
        dims = B.SwGatedRecurrenceDims(**{**dict(T=1, C=16, B=2, n_states=2, type=B.SW_F32), **k})
        return L.sw_gated_recurrence_step(t[0], t[1], t[2], g, t[3], state, slots, dims, strides(*s), None)

    for i in range(4):
        assert f(t=replaced(AT[:4], i, None)) == B.SW_ERR_NULL and f(t=replaced(AT[:4], i, AT[i] + 1)) == B.SW_ERR_ALIGN
    assert f(state=None) == f(g=None) == B.SW_ERR_NULL
    for bad in BAD_EXTENTS[:7] + [dict(T=2), dict(n_states=0), dict(s=[(16, 0, 0)] * 3 + [(15, 0, 0)]),
                                  dict(B=1 << 24, n_states=1 << 24, t=[1 << 45, 2 << 45, 3 << 45, 4 << 45], g=5 << 45, state=6 << 45)]:
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    for bad in (dict(t=replaced(AT[:4], 3, AT[0])), dict(state=AT[0]), dict(state=AT[3] + 64), dict(state=AT[4])):
        assert f(**bad) == B.SW_ERR_ALIAS, bad


HEADS = dict(B=2, T=10, heads=4, kv_heads=2, d=16, pairs=8, interleaved=0, type=B.SW_F32, eps=1e-6)
BAD_HEADS = [dict(B=0), dict(T=0), dict(heads=0), dict(kv_heads=-1), dict(d=0), dict(pairs=-1), dict(pairs=9), dict(eps=-1.0), dict(eps=float("nan")),
             dict(eps=float("inf")), dict(T=1 << 60)]
SQ, SK = (640, 64, 16), (320, 32, 16)


def test_head_norm_refusals(L):
    def f(t=None, w=(AT[4], AT[5]), fr=AT[6], at=AT[7], s=None, **k):
        t, s = t or AT[:4], s or [SQ, SK, SQ, SK]
        return L.sw_head_norm(t[0], t[1], *w, fr, at, t[2], t[3], B.SwHeadNormDims(**{**HEADS, **k}), strides(*s), None)

    for i in range(4):
        assert f(t=replaced(AT[:4], i, None)) == B.SW_ERR_NULL and f(t=replaced(AT[:4], i, AT[i] + 2)) == B.SW_ERR_ALIGN
    assert f(fr=None) == B.SW_ERR_NULL
    for bad in BAD_HEADS + [dict(s=[SQ, SK, (640, 60, 16), SK]), dict(s=[SQ, SK, SQ, (320, 32, 8)]), dict(s=[(640, -64, 16), SK, SQ, SK]),
                            dict(at=None, B=1, T=1 << 31, t=[1 << 45, 2 << 45, 3 << 45, 4 << 45])]:
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    assert f(d=257, s=[(1 << 20, 1 << 16, 300)] * 4) == f(type=4) == f(heads=65536, s=[(1 << 30, 1 << 24, 16)] * 4) == B.SW_ERR_UNSUPPORTED
    for bad in (dict(w=(AT[4] + 1, AT[5])), dict(fr=AT[6] + 2), dict(at=AT[7] + 1)):
        assert f(**bad) == B.SW_ERR_ALIGN, bad
    for bad in (dict(t=[AT[0], AT[1], AT[0] + 64, AT[3]]), dict(t=[AT[0], AT[1], AT[1], AT[3]]), dict(t=[AT[0], AT[1], AT[2], AT[2]]),
                dict(t=[AT[0], AT[1], AT[0], AT[3]], s=[SQ, SK, (1280, 128, 16), SK]), dict(t=[AT[0], AT[1], AT[4], AT[3]]), dict(t=[AT[0], AT[1], AT[2], AT[7]])):
        assert f(**bad) == B.SW_ERR_ALIAS, bad


def test_head_norm_backward_refusals(L):
    need = L.sw_head_norm_backward_workspace_bytes(B.SwHeadNormDims(**HEADS))
    assert need > 0 and L.sw_head_norm_backward_workspace_bytes(B.SwHeadNormDims(**{**HEADS, "d": 0})) == 0

    def f(t=None, w=(AT[6], AT[7]), fr=AT[8], at=AT[9], g=(AT[10], AT[11]), s=None, work=AT[12], bytes_=need, **k):
        t, s = t or AT[:6], s or [SQ, SK] * 3
        return L.sw_head_norm_backward(t[0], t[1], t[2], t[3], *w, fr, at, t[4], t[5], *g, B.SwHeadNormDims(**{**HEADS, **k}), strides(*s), work, bytes_, None)

    for i in range(6):
        assert f(t=replaced(AT[:6], i, None)) == B.SW_ERR_NULL and f(t=replaced(AT[:6], i, AT[i] + 1)) == B.SW_ERR_ALIGN
    for bad in BAD_HEADS + [dict(s=[SQ, SK, SQ, SK, SQ, (320, 16, 16)])]:
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    for bad in (dict(work=None), dict(bytes_=need - 1), dict(work=AT[12] + 4), dict(g=(None, AT[11]), work=None)):
        assert f(**bad) == B.SW_ERR_WORKSPACE, bad
    for bad in (dict(t=replaced(AT[:6], 4, AT[1])), dict(t=replaced(AT[:6], 4, AT[2] + 64)), dict(t=replaced(AT[:6], 5, AT[2])), dict(g=(AT[10], AT[10])),
                dict(g=(AT[4], AT[11])), dict(work=AT[0])):
        assert f(**bad) == B.SW_ERR_ALIAS, bad


def test_adapters_refusals(L):
    d0 = dict(T=10, B=2, C_in=16, C_out=24, rank=4, n=2, type=B.SW_F32)
    need = L.sw_adapters_workspace_bytes(B.SwAdaptersDims(**d0), 0)
    assert L.sw_adapters_workspace_bytes(B.SwAdaptersDims(**{**d0, "rank": 0}), 0) == 0

    def f(t=None, scales=AT[5], slots=None, starts=None, s=(16, 24, 24), work=AT[8], bytes_=1 << 27, **k):
        t = t or AT[:5]
        return L.sw_adapters(t[0], t[1], t[2], t[3], scales, slots, starts, t[4], B.SwAdaptersDims(**{**d0, **k}), *s, work, bytes_, None)

    for i in range(5):
        assert f(t=replaced(AT[:5], i, None)) == B.SW_ERR_NULL and f(t=replaced(AT[:5], i, AT[i] + 2)) == B.SW_ERR_ALIGN
    for bad in (dict(T=0), dict(B=0), dict(C_in=0), dict(C_out=-1), dict(rank=0), dict(n=0), dict(n=1), dict(s=(15, 24, 24)), dict(s=(16, 23, 24)),
                dict(s=(16, 24, 20)), dict(T=1 << 31), dict(T=1 << 30, B=4, n=4), dict(s=(1 << 60, 24, 24))):
        assert f(**bad) == B.SW_ERR_SHAPE, bad
    assert f(rank=257) == f(C_in=(1 << 20) + 1, s=(1 << 21, 24, 24)) == f(type=9) == B.SW_ERR_UNSUPPORTED
    for bad in (dict(scales=AT[5] + 1), dict(slots=AT[6] + 2), dict(starts=AT[7] + 1)):
        assert f(**bad) == B.SW_ERR_ALIGN, bad
    for bad in (dict(t=replaced(AT[:5], 4, AT[0])), dict(t=replaced(AT[:5], 4, AT[3] + 96)), dict(t=replaced(AT[:5], 4, AT[3]), s=(16, 24, 48)),
                dict(t=replaced(AT[:5], 4, AT[1])), dict(t=replaced(AT[:5], 4, AT[5]))):
        assert f(**bad) == B.SW_ERR_ALIAS, bad
    if need:
        assert f(work=None) == f(bytes_=need - 1) == f(work=AT[8] + 8) == B.SW_ERR_WORKSPACE
        assert f(work=AT[4]) == B.SW_ERR_ALIAS


def test_python_refusals():
    """Tensors off the GPU, of other types and shapes: an exception that says so, before anything is touched."""
    f = lambda *s, t=torch.float32: torch.zeros(s, dtype=t)
    x, g, s = f(2, 5, 8), f(8), f(2, 8)
    with pytest.raises(ValueError, match="GPU"):
        sw.sw_gated_recurrence(x, x, x, g)
    with pytest.raises(ValueError, match="dimensions"):
        sw.sw_gated_recurrence(x[0], x[0], x[0], g)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        sw.sw_gated_recurrence(x.double(), x.double(), x.double(), g)
    with pytest.raises(sw.SwError):
        sw.sw_gated_recurrence(x[:, :0], x[:, :0], x[:, :0], g)
    with pytest.raises(ValueError, match="GPU"):
        sw.sw_gated_recurrence_backward(x, x, x, x, g, x)
    with pytest.raises(ValueError, match="2 dimensions"):
        sw.sw_gated_recurrence_step(x, x, x, g, s)
    with pytest.raises(ValueError, match="GPU"):
        sw.sw_gated_recurrence_step(s, s, s, g, s)
    q, k = f(5, 4, 16), f(5, 2, 16)
    with pytest.raises(ValueError, match="GPU"):
        sw.sw_head_norm(q, k)
    with pytest.raises(ValueError, match="3 or 4 dimensions"):
        sw.sw_head_norm(q[0], k)
    with pytest.raises(ValueError, match="one dimension"):
        sw.sw_head_norm(q, k, frequencies=f(2, 2))
    with pytest.raises(sw.SwError):
        sw.sw_head_norm(q[:0], k[:0])
    with pytest.raises(ValueError, match="GPU"):
        sw.sw_head_norm_backward(q, k, q, k)
    a, b = f(3, 4, 16), f(3, 24, 4)
    with pytest.raises(ValueError, match="GPU"):
        sw.sw_adapters(f(3, 16), a, b, f(3, 24))
    with pytest.raises(ValueError, match="dimensions"):
        sw.sw_adapters(f(1, 3, 16), a, b, f(1, 3, 24), starts=torch.tensor([0, 3]))
    with pytest.raises(sw.SwError):
        sw.sw_adapters(f(0, 16), a, b, f(0, 24))


def test_definitions_against_each_other():
    """The oracle's recurrences against autograd of one that is written out, its norms against matrices, its adapters against one product."""
    g = torch.Generator().manual_seed(1)
    f = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    T, C = 9, 5
    x, r, i, dh, s0, df, ld = f(T, C), f(T, C), f(T, C), f(T, C), f(C), f(C), -torch.rand(C, generator=g, dtype=torch.float64) - 0.01
    leaves = [v.clone().requires_grad_(True) for v in (x, r, i, ld, s0)]
    a = torch.exp(leaves[3] / (1 + torch.exp(-leaves[1])))
    now, hs = leaves[4], []
    for t in range(T):
        now = a[t] * now + torch.sqrt(1 - a[t] ** 2) / (1 + torch.exp(-leaves[2][t])) * leaves[0][t]
        hs.append(now)
    h = torch.stack(hs)
    want = torch.autograd.grad((h * dh).sum() + (now * df).sum(), leaves)
    got, last, _, _ = O.recurrence(x, r, i, ld, s0)
    assert torch.allclose(got, h.detach(), rtol=1e-12) and torch.allclose(last, now.detach(), rtol=1e-12)
    grads, _ = O.recurrence_backward(dh, x, r, i, ld, got, s0, df)
    for n, w in zip(("dx", "dr", "di", "dl", "state"), want):
        assert torch.allclose(grads[n], w, rtol=1e-9, atol=1e-12), n
    for interleaved in (False, True):
        q, w, fr, at = f(4, 2, 10), f(10), torch.rand(3, generator=g), torch.tensor([0, 5, -7, 100000])
        y, _ = O.head_norm(q, w, fr, at, 1e-3, interleaved)
        dy = f(4, 2, 10)
        dx, dw, _, _ = O.head_norm_backward(dy, q, w, fr, at, 1e-3, interleaved)
        step = f(4, 2, 10)
        d = 1e-6
        moved = (O.head_norm(q + d * step, w, fr, at, 1e-3, interleaved)[0] - O.head_norm(q - d * step, w, fr, at, 1e-3, interleaved)[0]) / (2 * d)
        assert abs(float((moved * dy).sum() - (dx * step).sum())) < 1e-6
        assert torch.allclose((y * dy).sum(), (dw * w).sum())                       # y is linear in w
    xs, A, Bf, ys = f(3, 6), f(2, 4, 6), f(2, 5, 4), f(3, 5)
    out, _ = O.adapters(xs, A, Bf, ys, torch.tensor([2.0, 0.5]), [1, -1, 0])
    assert torch.allclose(out[0], ys[0] + 0.5 * xs[0] @ (Bf[1] @ A[1]).T) and torch.equal(out[1], ys[1]) and torch.allclose(out[2], ys[2] + 2 * xs[2] @ (Bf[0] @ A[0]).T)
