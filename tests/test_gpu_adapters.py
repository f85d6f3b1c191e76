"""Low-rank adapters of many requests beside a shared projection on the GPU against the definition in 64 bits.

Tolerances.  The result is rounded once to its format (half a step, e = eps / 2 of it).  With u = 2^-24: products of 16-bit values are exact in fp32, those of
fp32 ones off by u; a sum of C_in of them, in any order of runs and trees, by at most C_in u of the magnitudes (runs are shorter: 64 to 512 of
them one after another, a few tens of partial sums: 512 u); the sum over the rank by rank u <= 256 u more, its products by 2 u, and scale and y by 3 u."""
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


def make(rows, n, c_in, c_out, rank, t, seed):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=g)
    x, y = f(rows, c_in).to(TYPES[t]), f(rows, c_out).to(TYPES[t])
    a, b = (f(n, rank, c_in) * c_in ** -0.5).to(TYPES[t]), (f(n, c_out, rank) * rank ** -0.5).to(TYPES[t])
    return x, a, b, y, 0.5 + f(n).abs()


def check(got, x, a, b, y, scales, of, t):
    want, m = O.adapters(x, a, b, y, scales, of)
    e = torch.finfo(TYPES[t]).eps / 2
    tol = e * want.abs() + (520 + a.shape[1]) * U * m * (1 + e) + TINY[t]
    off = (got.cpu().double() - want).abs()
    assert torch.all(off <= tol), f"{float((off / tol).max()):.2f} of the tolerance"
    none = torch.tensor([s < 0 for s in of])
    assert torch.equal(got.cpu()[none], y[none])


def i32(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


SIZES = [(1, 1, 1), (8, 8, 1), (16, 24, 2), (33, 17, 3), (64, 64, 4), (63, 130, 5), (128, 96, 8), (200, 264, 12), (256, 512, 16), (255, 1000, 17), (1024, 72, 24),
         (520, 520, 32), (2048, 256, 33), (1000, 999, 48), (384, 2048, 64), (300, 300, 65), (512, 128, 100), (136, 136, 128), (96, 264, 200), (264, 96, 256)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("c_in,c_out,rank", SIZES)
def test_tokens(sw, c_in, c_out, rank, t):
    """A row for each request; several with one adapter, some with none."""
    rows, n = 13, 5
    x, a, b, y, scales = make(rows, n, c_in, c_out, rank, t, c_in + rank)
    of = torch.randint(0, n, (rows,), generator=torch.Generator().manual_seed(rank)).tolist()
    of[3], of[7] = -1, -1
    slots = list(of)
    slots[7] = n
    dev = [v.cuda() for v in (x, a, b, y)]
    got = sw.sw_adapters(*dev, scales.cuda(), i32(slots))
    check(got, x, a, b, y, scales, of, t)
    assert torch.equal(dev[3].cpu(), y) and torch.equal(got, sw.sw_adapters(*dev, scales.cuda(), i32(slots)))
    assert sw.sw_adapters(*dev, scales.cuda(), i32(slots), out=dev[3]) is dev[3] and torch.equal(dev[3], got)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("c_in,c_out,rank", SIZES)
def test_packed(sw, c_in, c_out, rank, t):
    lengths, before, after, n = [40, 0, 1, 70, 3, 0, 17, 16, 33], 2, 5, 4
    rows = before + sum(lengths) + after
    x, a, b, y, scales = make(rows, n, c_in, c_out, rank, t, c_in * 3 + rank)
    slots = [0, 1, 2, 3, -1, 2, 0, 9, 1]
    of, starts = [-1] * before, [before]
    for length, s in zip(lengths, slots):
        of += [s if 0 <= s < n else -1] * length
        starts.append(starts[-1] + length)
    of += [-1] * after
    got = sw.sw_adapters(x.cuda(), a.cuda(), b.cuda(), y.cuda(), scales.cuda(), i32(slots), i32(starts))
    check(got, x, a, b, y, scales, of, t)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,T", [(1, 1), (1, 300), (3, 65), (5, 16), (70, 2), (2, 1000)])
def test_sequences(sw, B, T, t):
    n = 70
    x, a, b, y, scales = make(B * T, n, 96, 160, 16, t, B + T)
    of = torch.arange(B).repeat_interleave(T).tolist()
    shape = lambda v: v.unflatten(0, (B, T)).cuda()
    got = sw.sw_adapters(shape(x), a.cuda(), b.cuda(), shape(y))
    check(got.flatten(0, 1), x, a, b, y, None, of, t)
    same = sw.sw_adapters(x.cuda(), a.cuda(), b.cuda(), y.cuda(), None, i32(list(range(B))), i32([k * T for k in range(B + 1)]))
    assert torch.allclose(same.float(), got.flatten(0, 1).float(), rtol=2 * torch.finfo(TYPES[t]).eps, atol=1e-5)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_many_rows_and_adapters(sw, t):
    """Hundreds of sequences, most of them short; more rows than a launch has at a time."""
    g = torch.Generator().manual_seed(4)
    lengths = torch.cat([torch.randint(0, 5, (500,), generator=g), torch.tensor([3000, 1, 700])]).tolist()
    rows, n = sum(lengths), 40
    x, a, b, y, scales = make(rows, n, 64, 80, 8, t, 9)
    slots = torch.randint(-1, n, (len(lengths),), generator=g).tolist()
    of = [s for length, s in zip(lengths, slots) for _ in range(length)]
    starts = [0]
    for length in lengths:
        starts.append(starts[-1] + length)
    check(sw.sw_adapters(x.cuda(), a.cuda(), b.cuda(), y.cuda(), scales.cuda(), i32(slots), i32(starts)), x, a, b, y, scales, of, t)
    tokens = torch.randint(-1, n, (rows,), generator=g).tolist()
    check(sw.sw_adapters(x.cuda(), a.cuda(), b.cuda(), y.cuda(), scales.cuda(), i32(tokens)), x, a, b, y, scales, tokens, t)


@pytest.mark.parametrize("starts", [(-5, 3, 90), (0, 50, 20), (60, 10, 70), (0, 200, 300), (2000000000, -2000000000, 5)])
def test_starts_out_of_range_stay_within(sw, starts):
    rows, c_out = 70, 40
    x, a, b, y, scales = make(rows, 2, 48, c_out, 4, "bf16", 3)
    big = torch.full((3 * rows, c_out), 7.0, dtype=torch.bfloat16, device="cuda")
    sw.sw_adapters(x.cuda(), a.cuda(), b.cuda(), y.cuda(), scales.cuda(), None, i32(starts), out=big[rows:2 * rows])
    assert torch.all(big[:rows] == 7.0) and torch.all(big[2 * rows:] == 7.0)
    if starts == (-5, 3, 90):
        check(big[rows:2 * rows], x, a, b, y, scales, [0] * 3 + [1] * 67, "bf16")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("c_in,c_out,rank,first", [(64, 64, 16, 3), (72, 100, 7, 1), (256, 128, 16, 8), (256, 128, 64, 1)])
def test_slices(sw, c_in, c_out, rank, first, t):
    """Rows of wider tensors, results into slices of others; what lies beside them is not touched."""
    rows, n = 50, 3
    x, a, b, y, scales = make(rows, n, c_in, c_out, rank, t, first)
    slots, starts = i32([2, 0, 1]), i32([0, 20, 21, 50])
    rest = a.cuda(), b.cuda()
    want = sw.sw_adapters(x.cuda(), *rest, y.cuda(), scales.cuda(), slots, starts)
    hold = lambda v: (lambda big: (big, big[:, first:first + v.shape[1]]))(torch.full((rows, v.shape[1] + first + 6), 7.0, dtype=TYPES[t], device="cuda"))
    (_, X), (ybig, Y), (big, O_) = hold(x), hold(y), hold(y)
    X.copy_(x), Y.copy_(y)
    sw.sw_adapters(X, *rest, Y, scales.cuda(), slots, starts, out=O_)
    e = 2 * torch.finfo(TYPES[t]).eps
    assert torch.allclose(O_.float(), want.float(), rtol=e, atol=1e-5)
    check(O_, x, a, b, y, scales, [2] * 20 + [0] + [1] * 29, t)
    sw.sw_adapters(X, *rest, Y, scales.cuda(), slots, starts, out=Y)
    assert torch.equal(Y, O_)
    for held, part in ((big, O_), (ybig, Y)):
        part.fill_(7.0)
        assert torch.all(held == 7.0)
    odd = torch.zeros(a.numel() + 1, dtype=TYPES[t], device="cuda")[1:].view(a.shape)        # factors off 16 bytes
    odd.copy_(rest[0])
    check(sw.sw_adapters(x.cuda(), odd, rest[1], y.cuda(), scales.cuda(), slots, starts), x, a, b, y, scales, [2] * 20 + [0] + [1] * 29, t)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rank,c_in", [(16, 256), (5, 70)])
def test_values_that_are_not_finite(sw, rank, c_in, t):
    """They stay in their row; what a row has no adapter for is never looked at; large values of half tensors' products do not overflow on the way."""
    rows, n = 40, 3
    x, a, b, y, scales = make(rows, n, c_in, 96, rank, t, 2)
    slots, starts = i32([0, -1, 1]), i32([0, 10, 20, 40])
    run = lambda: sw.sw_adapters(x.cuda(), a.cuda(), b.cuda(), y.cuda(), scales.cuda(), slots, starts)
    clean = run()
    x[5, 3], x[12, 0], x[30, 7] = float("nan"), float("nan"), float("inf")
    a[2], b[2] = float("nan"), float("inf")
    got = run()
    left = torch.ones(rows, dtype=torch.bool)
    left[5] = left[30] = False
    assert torch.equal(got.cpu()[left], clean.cpu()[left])
    assert torch.isnan(got[5]).all() and not torch.isfinite(got[30]).any()
    if t == "f16":
        x[:], a[:], b[:] = 100.0, 100.0, 2.0 ** -20
        want = float(y[0, 0]) + 100.0 * 100.0 * c_in * rank * 2.0 ** -20 * float(scales[0])        # a x is beyond half's largest value for c_in 70 and up
        assert abs(float(run()[0, 0]) - want) <= 2e-3 * abs(want) + 1e-3


def test_another_stream_and_graphs(sw):
    rows, n = 600, 6
    made = [[v.cuda() for v in make(rows, n, 256, 320, 32, "bf16", s)] for s in range(3)]
    held = [v.clone() for v in made[0]]
    x, a, b, y, scales = held
    slots, starts = i32([3, 0, 5]), i32([0, 100, 101, 600])
    tokens = i32([k % (n + 1) - 1 for k in range(rows)])
    both = lambda: (sw.sw_adapters(x, a, b, y, scales, slots, starts), sw.sw_adapters(x, a, b, y, scales, tokens))
    want = [v.clone() for v in both()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = sw.sw_adapters(x, a, b, y, scales, slots, starts, stream=side), sw.sw_adapters(x, a, b, y, scales, tokens, stream=side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = both()
    for turn in range(4):
        for v, new in zip(held, made[turn % 3]):
            v.copy_(new)
        want = [v.clone() for v in both()]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


@pytest.mark.parametrize("packed", [False, True])
def test_offsets_beyond_32_bits(sw, packed):
    """Rows so far apart that their places take more than 32 bits of bytes."""
    rows, far = 16, (1 << 28) + 16
    x, a, b, y, scales = make(rows, 2, 64, 72, 8, "bf16", 6)
    big = torch.zeros(rows * far, dtype=torch.bfloat16, device="cuda")
    X, Y = big.as_strided((rows, 64), (far, 1)), big[64:].as_strided((rows, 72), (far, 1))
    X.copy_(x), Y.copy_(y)
    slots = i32([1, 0]) if packed else i32([k % 2 for k in range(rows)])
    args = scales.cuda(), slots, i32([0, 5, rows]) if packed else None
    of = [1] * 5 + [0] * 11 if packed else [k % 2 for k in range(rows)]
    check(sw.sw_adapters(X, a.cuda(), b.cuda(), y.cuda(), *args), x, a, b, y, scales, of, "bf16")
    check(sw.sw_adapters(X, a.cuda(), b.cuda(), Y, *args, out=Y), x, a, b, y, scales, of, "bf16")
    assert torch.equal(X.cpu(), x)
