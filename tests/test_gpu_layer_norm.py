"""Layer norm and its backward pass on the GPU against the definition in 64 bits.

Tolerances: a result is rounded once to its format (half a step, e = eps / 2 of it) from a value computed in fp32 (u = 2^-24).  Sums of C
or of all rows are added in runs and trees no deeper than 64 additions a run in the norms and 512 in the sums over rows, so a sum
is off by at most that many u of the sum of its magnitudes; a mean that is off moves every x - mean by as much."""
import pytest

import layers_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = {"f32": 1e-38, "bf16": 1e-38, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def sw():
    import paper_2310_05218_amd as _sw
    from paper_2310_05218_amd import binding

    assert torch.cuda.is_available(), "these tests need the GPU"
    binding.lib()            # fails loudly if the library is not built
    return _sw


def make(rows, C, t, seed, offset=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, C, generator=g) * 1.5 + offset * torch.randn(rows, 1, generator=g)).to(TYPES[t])
    return x, 1 + 0.2 * torch.randn(C, generator=g), 0.3 * torch.randn(C, generator=g), torch.randn(rows, C, generator=g).to(TYPES[t])


def check_forward(x, w, b, eps, t, y, mean=None, rstd=None):
    ry, rm, rr = O.layer_norm(x, w, b, eps)
    e = torch.finfo(TYPES[t]).eps / 2
    a = x.double().abs()
    wa = torch.ones(x.shape[-1]) if w is None else w.double().abs()
    off = 64 * U * a.mean(-1)
    tol = e * ry.abs() + 64 * U * (x.double() - rm[..., None]).abs() * rr[..., None] * wa + off[..., None] * rr[..., None] * wa
    tol = tol + 4 * U * (ry.abs() + (0 if b is None else b.double().abs())) + TINY[t]
    assert torch.all((y.cpu().double() - ry).abs() <= tol)
    if mean is not None:
        assert torch.all((mean.cpu().double() - rm).abs() <= off + 1e-38)
        var = ((x.double() - rm[..., None]) ** 2).mean(-1)
        assert torch.all((rstd.cpu().double() - rr).abs() <= (64 * U + off ** 2 / (var + eps)) * rr)


def check_backward(dy, x, w, eps, t, dx, dw, db):
    rdx, rdw, rdb = O.layer_norm_backward(dy, x, w, eps)
    _, m, r = O.layer_norm(x, None, None, eps)
    e = torch.finfo(TYPES[t]).eps / 2
    r = r[:, None]
    h = (x.double() - m[:, None]) * r
    g = dy.double() * (1 if w is None else w.double())
    dh = 64 * U * (x.double().abs().mean(-1, keepdim=True) * r + h.abs())          # how far h may be off
    mean = lambda v: v.mean(-1, keepdim=True)
    tol = e * rdx.abs() + 64 * U * (rdx.abs() + r * (g.abs() + mean(g.abs()) + h.abs() * mean((g * h).abs())))
    tol = tol + r * (dh * mean(g * h).abs() + h.abs() * mean(g.abs() * dh)) + TINY[t]
    assert torch.all((dx.cpu().double() - rdx).abs() <= tol)
    if dw is not None:
        assert torch.all((dw.cpu().double() - rdw).abs() <= (512 * U * (dy.double() * h).abs() + dy.double().abs() * dh).sum(0) + 1e-38)
        assert torch.all((db.cpu().double() - rdb).abs() <= 512 * U * dy.double().abs().sum(0) + 1e-38)


SHAPES = [(1, 1), (3, 1), (1, 2), (2, 3), (5, 7), (4, 8), (67, 8), (3, 16), (9, 31), (130, 32), (33, 33), (1000, 40), (17, 63), (300, 64), (5, 65),
          (9, 100), (64, 127), (65, 128), (7, 129), (12, 192), (257, 200), (3, 255), (40, 256), (5, 257), (21, 384), (2, 511), (9, 512), (3, 513),
          (1, 777), (300, 999), (5, 1000), (4, 1024), (3, 1025), (2, 1536), (600, 2048), (3, 2050), (2, 4095), (70, 4096), (3, 4097), (1, 5000),
          (2, 8192), (3, 8193), (1, 10240), (2, 12345), (2, 16384), (1, 20001), (2, 32768), (1, 40000), (1, 65536), (1, 65537), (1, 100003)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,C", SHAPES)
def test_forward_and_backward(sw, rows, C, t):
    x, w, b, dy = make(rows, C, t, rows * 7 + C)
    y, mean, rstd = sw.sw_layer_norm(x.cuda(), w.cuda(), b.cuda(), 1e-5, stats=True)
    check_forward(x, w, b, 1e-5, t, y, mean, rstd)
    assert torch.equal(y, sw.sw_layer_norm(x.cuda(), w.cuda(), b.cuda(), 1e-5))
    dx, dw, db = sw.sw_layer_norm_backward(dy.cuda(), x.cuda(), w.cuda(), mean, rstd)
    check_backward(dy, x, w, 1e-5, t, dx, dw, db)
    again = sw.sw_layer_norm_backward(dy.cuda(), x.cuda(), w.cuda(), mean, rstd)
    assert all(torch.equal(a, c) for a, c in zip((dx, dw, db), again))               # a fixed order of additions


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,C", [(6, 24), (5, 301), (3, 1024), (2, 9001)])
def test_optional_operands(sw, rows, C, t):
    x, w, b, dy = make(rows, C, t, 5)
    X = x.cuda()
    check_forward(x, None, None, 1e-3, t, sw.sw_layer_norm(X, None, None, 1e-3))
    check_forward(x, w, None, 0.0, t, sw.sw_layer_norm(X, w.cuda(), None, 0.0))
    check_forward(x, None, b, 1e-5, t, *sw.sw_layer_norm(X, None, b.cuda(), 1e-5, stats=True))
    _, mean, rstd = sw.sw_layer_norm(X, None, None, 1e-5, stats=True)
    dx, dw, db = sw.sw_layer_norm_backward(dy.cuda(), X, None, mean, rstd)
    check_backward(dy, x, None, 1e-5, t, dx, dw, db)
    only, none1, none2 = sw.sw_layer_norm_backward(dy.cuda(), X, None, mean, rstd, params=False)
    assert none1 is None and none2 is None and torch.equal(only, dx)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C,first,stride", [(24, 3, 40), (64, 8, 96), (100, 1, 101), (512, 0, 1024), (1000, 5, 1011), (4096, 8, 4112)])
def test_strides_and_alignment(sw, C, first, stride, t):
    """Slices of wider rows, at addresses off 16 bytes; what lies between the rows is not touched."""
    rows = 7
    x, w, b, dy = make(rows, C, t, C)
    hold = lambda v: (lambda big: (big, big[:, first:first + C]))(torch.full((rows, stride), 7.0, dtype=TYPES[t], device="cuda"))
    (_, X), (_, DY), (bigy, Y), (bigd, DX) = (hold(v) for v in range(4))
    X.copy_(x), DY.copy_(dy)
    y, mean, rstd = sw.sw_layer_norm(X, w.cuda(), b.cuda(), 1e-5, stats=True, out=Y)
    check_forward(x, w, b, 1e-5, t, y, mean, rstd)
    dx, dw, db = sw.sw_layer_norm_backward(DY, X, w.cuda(), mean, rstd, out=DX)
    check_backward(dy, x, w, 1e-5, t, dx, dw, db)
    for big, part in ((bigy, Y), (bigd, DX)):
        part.fill_(7.0)
        assert torch.all(big == 7.0)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,C", [(50, 64), (9, 1000), (3, 9000), (2, 70000)])
def test_in_place(sw, rows, C, t):
    x, w, b, dy = make(rows, C, t, 9)
    X = x.cuda()
    want, mean, rstd = sw.sw_layer_norm(X, w.cuda(), b.cuda(), stats=True)
    dwant = sw.sw_layer_norm_backward(dy.cuda(), X, w.cuda(), mean, rstd)
    for target in ("dy", "x"):
        a, c = dy.cuda(), x.cuda()
        got = sw.sw_layer_norm_backward(a, c, w.cuda(), mean, rstd, out=a if target == "dy" else c)
        assert all(torch.equal(p, q) for p, q in zip(got, dwant))
    assert sw.sw_layer_norm(X, w.cuda(), b.cuda(), out=X) is X and torch.equal(X, want)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [5, 64, 1000, 4096, 9000, 70000])
def test_rows_of_one_value_and_far_off_centre(sw, C, t):
    """Rows without variance give the bias (a mean that is off by its rounding is magnified by 1 / sqrt(eps), no further), rows far
    from zero keep their spread."""
    x = torch.full((4, C), 3.0)
    x[1] = -0.0
    x[2] = 1000.0 + torch.randn(C, generator=torch.Generator().manual_seed(1))
    x[3, 0] = 4.0
    x = x.to(TYPES[t])
    b = torch.randn(C, generator=torch.Generator().manual_seed(2))
    check_forward(x, None, b, 1e-5, t, *sw.sw_layer_norm(x.cuda(), None, b.cuda(), 1e-5, stats=True))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [8, 100, 1024, 9000])
def test_nonfinite_rows_stay_to_themselves(sw, C, t):
    x, w, b, dy = make(9, C, t, 11)
    want, mean, rstd = sw.sw_layer_norm(x.cuda(), w.cuda(), b.cuda(), stats=True)
    dwant = sw.sw_layer_norm_backward(dy.cuda(), x.cuda(), w.cuda(), mean, rstd)[0]
    bad = x.clone()
    bad[2, C // 2], bad[5, C - 1], bad[7, 0] = float("nan"), float("inf"), -float("inf")
    y, m, r = sw.sw_layer_norm(bad.cuda(), w.cuda(), b.cuda(), stats=True)
    rows = torch.tensor([0, 1, 3, 4, 6, 8]).cuda()
    assert torch.equal(y[rows], want[rows]) and torch.equal(m[rows], mean[rows]) and torch.equal(r[rows], rstd[rows])
    assert all(torch.isnan(y[i]).all() for i in (2, 5, 7))
    dx, dw, db = sw.sw_layer_norm_backward(dy.cuda(), bad.cuda(), w.cuda(), m, r)
    assert torch.equal(dx[rows], dwant[rows]) and all(torch.isnan(dx[i]).all() for i in (2, 5, 7))
    assert torch.isnan(dw).all() and torch.isfinite(db).all()


def test_many_rows_and_leading_dimensions(sw):
    x, w, b, dy = make(70001, 12, "f32", 4)
    y, mean, rstd = sw.sw_layer_norm(x.cuda(), w.cuda(), b.cuda(), stats=True)
    check_forward(x, w, b, 1e-5, "f32", y, mean, rstd)
    four = x[:60].reshape(3, 4, 5, 12).cuda()
    y4, m4, _ = sw.sw_layer_norm(four, w.cuda(), b.cuda(), stats=True)
    assert y4.shape == four.shape and m4.shape == (3, 4, 5) and torch.equal(y4.reshape(60, 12), y[:60])
    one = sw.sw_layer_norm(x[0].cuda(), w.cuda(), b.cuda())
    assert one.shape == (12,) and torch.equal(one, y[0])
    turned = four.permute(2, 1, 0, 3)
    with pytest.raises(ValueError, match="evenly apart"):
        sw.sw_layer_norm(turned)


def test_offsets_beyond_32_bits(sw):
    """Two rows 3 GiB apart."""
    C, stride = 300, 3 << 29
    big = torch.empty(stride + C, dtype=torch.bfloat16, device="cuda")
    x, w, b, dy = make(2, C, "bf16", 6)
    X = big.as_strided((2, C), (stride, 1))
    X.copy_(x)
    y, mean, rstd = sw.sw_layer_norm(X, w.cuda(), b.cuda(), stats=True)
    check_forward(x, w, b, 1e-5, "bf16", y, mean, rstd)
    check_backward(dy, x, w, 1e-5, "bf16", *sw.sw_layer_norm_backward(dy.cuda(), X, w.cuda(), mean, rstd))
    assert sw.sw_layer_norm(X, w.cuda(), b.cuda(), out=X) is X and torch.equal(X, y)


def test_refusals(sw):
    x = torch.randn(4, 8, device="cuda")
    for call in (lambda: sw.sw_layer_norm(x, x[0].bfloat16()), lambda: sw.sw_layer_norm(x, x[0, :7]), lambda: sw.sw_layer_norm(x, out=x[:3]),
                 lambda: sw.sw_layer_norm(x, x[0].cpu()), lambda: sw.sw_layer_norm(x.t()[:, ::2]), lambda: sw.sw_layer_norm_backward(x, x, None, None, None),
                 lambda: sw.sw_layer_norm_backward(x[:, :4], x, None, x[:, 0].contiguous(), x[:, 0].contiguous())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: sw.sw_layer_norm(x[:0]), lambda: sw.sw_layer_norm(x, eps=-1.0), lambda: sw.sw_layer_norm(x[:2], out=x[1:3]),
                 lambda: sw.sw_layer_norm(x[:1].expand(4, 8))):
        with pytest.raises(sw.SwError):
            call()


def test_another_stream_and_graph_replays(sw):
    x, w, b, dy = make(500, 768, "bf16", 8)
    X, W, Bi, DY = x.cuda(), w.cuda(), b.cuda(), dy.cuda()

    def step(stream=None):
        y, m, r = sw.sw_layer_norm(X, W, Bi, stats=True, stream=stream)
        return (y, m, r, *sw.sw_layer_norm_backward(DY, X, W, m, r, stream=stream))

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    gen = torch.Generator(device="cuda").manual_seed(3)
    for _ in range(4):
        X.copy_(torch.randn(X.shape, generator=gen, device="cuda"))
        DY.copy_(torch.randn(X.shape, generator=gen, device="cuda"))
        assert (X.float() * 2).sum().isfinite().item()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert all(torch.equal(p, q) for p, q in zip(got, step()))
