"""The gated recurrence, its backward pass and its form for single tokens on the GPU against the definition in 64 bits.

Tolerances.  A result is rounded once to its format (half a step, e = eps / 2 of it).  Before that it is a sum of terms, each a product of
decays a and of a weight and gates.  With u = 2^-24: an exponential of fp32 tensors is off by 2 u, of 16-bit ones by |x| u + u more where the gates are
|x| <= 8 (10 u), a reciprocal by 2 u, so sigmoids are off by at most 14 u of themselves; a decay's exponent L = log_decay s, |L| <= |log_decay| <= 2,
by 16 u |L| <= 32 u; a by 32 u + 4 u.  sqrt(1 - a^2) has half the relative error of 1 - a^2, which is that of 16 u (L) and of the
series or the subtraction: 2^-22 = 4 u, in 16-bit formats 2^-18 = 64 u.  A term that has gone through n decays is off by n (36 u + u) of itself,
but has itself shrunk by a^n = e^(n L): n 37 u e^(n L) with the error of a relative to |L|, 16 u n |L| e^(-n |L|) <= 6 u where the error of L counts, and
n 5 u e^(-n |L|) <= 5 u / |L| where that of the exponential and the products does.  Tests' decays have |L| >= 2^-12 where gates are open, so of the
sum of magnitudes in a sequence of T tokens at most min(T, 2^12) 5 u + 64 u + 40 u are lost."""
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


def lost(T):
    return (5 * min(T, 4096) + 104) * U


def make(rows, C, t, seed, count=1):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=g)
    x, r, i, dh = (f(rows, C).to(TYPES[t]) for _ in range(4))
    log_decay = torch.log1p(-torch.exp2(-0.5 - 9 * torch.rand(C, generator=g)))
    return x, r, i, dh, log_decay, f(count, C), f(count, C)


def close(got, want, mag, t, T, extra=0.0):
    e = torch.finfo(TYPES[t]).eps / 2 if t else 0.0
    tol = e * want.abs() + (lost(T) * (1 + e) + extra) * mag + (TINY[t] if t else 1e-37)
    bad = (got.cpu().double() - want).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} off, worst {float(((got.cpu().double() - want).abs() / tol).max()):.2f} of the tolerance"


# a gradient with respect to a gate has the derivative of a sigmoid (2 x 14 u) and that of the weight, whose 1 / w doubles w's error, beside the sum's terms
GRADIENT = 200 * U

LENGTHS = [1, 2, 3, 7, 15, 16, 17, 31, 32, 33, 37, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 300, 513, 777, 1025, 2100]
WIDTHS = [1, 2, 3, 63, 64, 65, 127, 128, 129, 130, 200, 257]


def check_sequences(sw, t, C, T, B, initial, seed):
    x, r, i, dh, ld, s0, df = make(B * T, C, t, seed, B)
    shape = lambda v: v.reshape(B, T, C).cuda()
    state = s0.cuda() if initial else None
    final = torch.full((B, C), 7.0, device="cuda")
    h = sw.sw_gated_recurrence(shape(x), shape(r), shape(i), ld.cuda(), state=state, final_state=final)
    assert torch.equal(h, sw.sw_gated_recurrence(shape(x), shape(r), shape(i), ld.cuda(), state=state))
    d_state = torch.full((B, C), 7.0, device="cuda") if initial else None
    args = shape(dh), shape(x), shape(r), shape(i), ld.cuda(), h
    more = dict(state=state, d_final_state=df.cuda() if initial else None)
    grads = sw.sw_gated_recurrence_backward(*args, d_state=d_state, **more)
    again = sw.sw_gated_recurrence_backward(*args, **more)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))                     # a fixed order of additions
    dl, dlm = 0, 0
    for b in range(B):
        cut = slice(b * T, (b + 1) * T)
        want, last, m, lm = O.recurrence(x[cut], r[cut], i[cut], ld, s0[b] if initial else None)
        close(h[b], want, m, t, T)
        close(final[b], last, lm, None, T)
        g, gm = O.recurrence_backward(dh[cut], x[cut], r[cut], i[cut], ld, h[b].cpu(), s0[b] if initial else None, df[b] if initial else None)
        for n, got in zip(("dx", "dr", "di"), grads):
            close(got[b], g[n], gm[n], t, T, GRADIENT)
        if initial:
            close(d_state[b], g["state"], gm["state"], None, T)
        dl, dlm = dl + g["dl"], dlm + gm["dl"]
    close(grads[3], dl, dlm, None, T, GRADIENT + 512 * U)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", LENGTHS)
def test_lengths(sw, T, t):
    check_sequences(sw, t, 130 if T % 2 else 67, T, 1 + T % 3, T % 4 != 0, T)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", WIDTHS)
def test_widths(sw, C, t):
    check_sequences(sw, t, C, 70, 2, C % 2 == 0, C)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,C", [(1, 5000, 64), (2, 4100, 192), (40, 3, 512), (300, 1, 96), (5, 600, 1030), (48, 300, 130), (48, 70, 131), (24, 200, 1030), (60, 200, 1030),
                                   (700, 3, 130), (1201, 9, 64)])
def test_larger(sw, B, T, C, t):
    check_sequences(sw, t, C, T, B, True, B + T)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("lengths,before,after", [((5,), 0, 0), ((3, 0, 1, 60, 0), 0, 0), ((17, 0, 0, 33, 1, 1, 100), 3, 5), ((0, 0), 4, 4), ((1,) * 50, 1, 0),
                                                  ((700, 2, 333), 0, 40), ((0,) * 70 + (9, 0, 300) + (0,) * 70, 0, 1), ((256, 256, 16, 16), 0, 0)])
@pytest.mark.parametrize("slots", [False, True])
@pytest.mark.parametrize("C", [131])
def test_packed(sw, lengths, before, after, slots, t, C):
    """Sequences one after the other, empty ones among them, rows of none around them; entries of a cache, some of them none."""
    B, n = len(lengths), sum(lengths)
    T = before + n + after
    x, r, i, dh, ld, s0, df = make(T, C, t, n + B, B + 3)
    starts = torch.tensor([before + sum(lengths[:k]) for k in range(B + 1)])
    at = (torch.randperm(B + 3, generator=torch.Generator().manual_seed(B))[:B] if slots else torch.arange(B)).tolist()
    if slots:
        at[B // 2] = (-1, B + 3)[n % 2]
    dev = lambda v: v.cuda()
    cache, final, d_state = s0.cuda(), torch.full((B + 3, C), 7.0, device="cuda"), df[:B].cuda()
    kw = dict(starts=starts.int().cuda(), slots=torch.tensor(at, dtype=torch.int32).cuda() if slots else None, state=cache)
    h = sw.sw_gated_recurrence(dev(x), dev(r), dev(i), dev(ld), final_state=final, **kw)
    grads = sw.sw_gated_recurrence_backward(dev(dh), dev(x), dev(r), dev(i), dev(ld), h, d_final_state=d_state, d_state=d_state, **kw)
    assert torch.equal(cache.cpu(), s0)
    in_place = s0.cuda()
    assert torch.equal(h, sw.sw_gated_recurrence(dev(x), dev(r), dev(i), dev(ld), **{**kw, "state": in_place}, final_state=in_place))
    outside = torch.ones(T, dtype=torch.bool)
    untouched = torch.ones(B + 3, dtype=torch.bool)
    dl, dlm = 0, 0
    for b, length in enumerate(lengths):
        cut = slice(int(starts[b]), int(starts[b + 1]))
        outside[cut] = False
        first = s0[at[b]] if 0 <= at[b] < B + 3 else None
        want, last, m, lm = O.recurrence(x[cut], r[cut], i[cut], ld, first)
        close(h[cut], want, m, t, length)
        if first is not None:
            untouched[at[b]] = False
            close(final[at[b]], last, lm, None, length)
        g, gm = O.recurrence_backward(dh[cut], x[cut], r[cut], i[cut], ld, h[cut].cpu(), first, df[b])
        for k, got in zip(("dx", "dr", "di"), grads):
            close(got[cut], g[k], gm[k], t, length, GRADIENT)
        close(d_state[b], g["state"], gm["state"], None, length)
        dl, dlm = dl + g["dl"], dlm + gm["dl"]
    for v in (h, *grads[:3]):
        assert torch.all(v.cpu()[outside] == 0)
    assert torch.all(final.cpu()[untouched] == 7.0) and torch.equal(in_place.cpu()[untouched], s0[untouched])
    assert torch.equal(in_place.cpu()[~untouched], final.cpu()[~untouched])
    close(grads[3], dl + torch.zeros(C), dlm + torch.zeros(C), None, n, GRADIENT + 512 * U)


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("lengths,before,after", [((700, 2, 333), 0, 40), ((0, 129, 1, 0, 1000, 15), 3, 0)])
@pytest.mark.parametrize("C", [2101, 4101])
def test_packed_on_many_workgroups(sw, C, lengths, before, after, t):
    test_packed(sw, lengths, before, after, True, t, C)


def test_packed_without_states(sw):
    lengths, C = (40, 0, 300), 70
    x, r, i, dh, ld, _, _ = make(340, C, "bf16", 5)
    starts = torch.tensor([0, 40, 40, 340], dtype=torch.int32).cuda()
    final = torch.full((3, C), 7.0, device="cuda")
    h = sw.sw_gated_recurrence(x.cuda(), r.cuda(), i.cuda(), ld.cuda(), starts=starts, final_state=final)
    d_state = torch.full((3, C), 7.0, device="cuda")
    sw.sw_gated_recurrence_backward(dh.cuda(), x.cuda(), r.cuda(), i.cuda(), ld.cuda(), h, starts=starts, d_state=d_state)
    assert torch.all(final[1] == 0) and torch.all(d_state[1] == 0)
    for b, cut in ((0, slice(0, 40)), (2, slice(40, 340))):
        want, last, m, lm = O.recurrence(x[cut], r[cut], i[cut], ld)
        close(h[cut], want, m, "bf16", 300)
        close(final[b], last, lm, None, 300)


@pytest.mark.parametrize("before", [3, 300])
def test_rows_in_no_sequence_are_not_looked_at(sw, before):
    """Whatever they hold: padding around sequences, and between them and the next."""
    n, C = 200, 70
    T = before + n + 5
    x, r, i, dh, ld, _, df = make(T, C, "bf16", 5)
    starts = torch.tensor([before, before + n], dtype=torch.int32).cuda()
    got = []
    for fill in (0.0, float("nan")):
        tensors = [v.clone() for v in (x, r, i, dh)]
        for v in tensors:
            v[:before] = v[before + n:] = fill
        xs, rs, gs, dhs = (v.cuda() for v in tensors)
        final = torch.empty(1, C, device="cuda")
        h = sw.sw_gated_recurrence(xs, rs, gs, ld.cuda(), starts=starts, final_state=final)
        grads = sw.sw_gated_recurrence_backward(dhs, xs, rs, gs, ld.cuda(), h, starts=starts, d_final_state=df[:1].cuda())
        got.append((h, final, *grads))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.all(got[1][0][:before] == 0) and torch.all(got[1][0][before + n:] == 0)


@pytest.mark.parametrize("starts", [(-5, 3, 90), (0, 50, 20), (60, 10, 70), (0, 200, 300), (2000000000, -2000000000, 5)])
def test_starts_out_of_range_stay_within(sw, starts):
    """Whatever starts holds, nothing outside of the tensors is written; in range and in order, every row has its sequence."""
    T, C = 70, 66
    x, r, i, dh, ld, s0, df = make(T, C, "bf16", 8, 2)
    hold = lambda: torch.full((3 * T, C), 7.0, dtype=torch.bfloat16, device="cuda")
    big = [hold() for _ in range(4)]
    out = [v[T:2 * T] for v in big]
    at = torch.tensor(starts, dtype=torch.int32).cuda()
    final = torch.full((4, C), 7.0, device="cuda")
    sw.sw_gated_recurrence(x.cuda(), r.cuda(), i.cuda(), ld.cuda(), starts=at, final_state=final[1:3], out=out[0])
    sw.sw_gated_recurrence_backward(dh.cuda(), x.cuda(), r.cuda(), i.cuda(), ld.cuda(), out[0], starts=at, d_state=final[1:3], out=out[1:])
    for v in big:
        assert torch.all(v[:T] == 7.0) and torch.all(v[2 * T:] == 7.0)
    assert torch.all(final[0] == 7.0) and torch.all(final[3] == 7.0)
    if starts == (-5, 3, 90):
        for cut in (slice(0, 3), slice(3, 70)):
            want, _, m, _ = O.recurrence(x[cut], r[cut], i[cut], ld)
            close(out[0][cut], want, m, "bf16", 70)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("B", [2, 140])
def test_slices_of_a_projection(sw, t, packed, B):
    """x and the gates as slices of one tensor's rows, the gradients into slices of another's; what lies beside them is not touched."""
    T, C = 150, 75
    g = torch.Generator().manual_seed(1)
    fused = torch.randn(B, T, 3 * C + 5, generator=g).to(TYPES[t])
    dh, ld = torch.randn(B, T, C, generator=g).to(TYPES[t]), -torch.rand(C, generator=g) - 1e-3
    starts = torch.tensor([0, 90, B * T], dtype=torch.int32).cuda() if packed else None
    lead = (lambda v: v.flatten(0, 1)) if packed else (lambda v: v)
    cut = lambda v: [v[..., k * C + 1:(k + 1) * C + 1] for k in range(3)]
    F = lead(fused.cuda())
    dense = [v.contiguous() for v in cut(F)]
    h = sw.sw_gated_recurrence(*cut(F), ld.cuda(), starts=starts)
    assert torch.equal(h, sw.sw_gated_recurrence(*dense, ld.cuda(), starts=starts))
    into = torch.full_like(F, 7.0)
    got = sw.sw_gated_recurrence_backward(lead(dh.cuda()), *cut(F), ld.cuda(), h, starts=starts, out=cut(into))
    want = sw.sw_gated_recurrence_backward(lead(dh.cuda()), *dense, ld.cuda(), h, starts=starts)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.all(into[..., 0] == 7.0) and torch.all(into[..., 3 * C + 1:] == 7.0)
    wide = torch.full((*F.shape[:-1], C + 3), 7.0, dtype=TYPES[t], device="cuda")
    assert torch.equal(sw.sw_gated_recurrence(*cut(F), ld.cuda(), starts=starts, out=wide[..., 2:C + 2]), h)
    assert torch.all(wide[..., :2] == 7.0) and torch.all(wide[..., -1] == 7.0)
    if not packed:      # tokens before sequences
        turned = [v.transpose(0, 1).contiguous().transpose(0, 1) for v in dense]
        assert torch.equal(h, sw.sw_gated_recurrence(*turned, ld.cuda()))
        zero = torch.zeros_like(dense[0][:1]).expand(B, T, C)
        assert torch.equal(sw.sw_gated_recurrence(dense[0], zero, dense[2], ld.cuda()), sw.sw_gated_recurrence(dense[0], zero.contiguous(), dense[2], ld.cuda()))


@pytest.mark.parametrize("t", TYPES)
def test_gates_at_their_ends(sw, t):
    """Gates far open and far shut, decays of -infinity, 0 and beyond fp32's exponents: finite, and the definition's."""
    ends = [0.0, 1.0, -1.0, 8.0, -8.0, 20.0, -20.0, 60.0, -60.0, 100.0, -100.0, 200.0, -200.0, float("inf"), float("-inf"), 1e4, -1e4]
    decays = [0.0, -1e-12, -1e-6, -1e-3, -0.1, -1.0, -20.0, -100.0, -1e10, -3e38, float("-inf")]
    n = len(ends)
    r, i = torch.tensor(ends).repeat_interleave(n), torch.tensor(ends).repeat(n)
    ld = torch.tensor(decays)
    C, T = len(decays), n * n
    x, _, _, dh, _, s0, df = make(T, C, t, 4)
    gr, gi = (v[:, None].expand(T, C).to(TYPES[t]).contiguous() for v in (r, i))
    B = lambda v: v[None].cuda()
    final = torch.empty(1, C, device="cuda")
    h = sw.sw_gated_recurrence(B(x), B(gr), B(gi), ld.cuda(), state=s0.cuda(), final_state=final)
    want, last, m, lm = O.recurrence(x, gr.float(), gi.float(), ld, s0[0])
    assert torch.isfinite(h).all()
    # (gates of up to 20 in 16-bit formats: 20 u more in each exponential; beyond, sigmoids are 0 or 1 to fp32's bits or shut to 1e-9)
    close(h[0], want, m + 1e-6, t, T, 60 * U)
    grads = sw.sw_gated_recurrence_backward(B(dh), B(x), B(gr), B(gi), ld.cuda(), h, state=s0.cuda(), d_final_state=df.cuda())
    g, gm = O.recurrence_backward(dh, x, gr.float(), gi.float(), ld, h[0].cpu(), s0[0], df[0])
    for k, got in zip(("dx", "dr", "di"), grads):
        assert torch.isfinite(got).all()
        close(got[0], g[k], gm[k] + 1e-6, t, T, GRADIENT + 60 * U)
    assert torch.isfinite(grads[3]).all()


@pytest.mark.parametrize("T", [40, 700])
@pytest.mark.parametrize("value,where", [(float(v), w) for v in ("nan", "inf", "-inf") for w in ("x", "state")] + [(float("nan"), "r")])
def test_non_finite_values_stay_in_their_sequence_and_channel(sw, T, value, where):
    """Of packed sequences only the one that holds the value has it, from its token on, in its channel; backwards, from its token to its beginning."""
    C, at, ch = 70, T // 2, 33
    x, r, i, dh, ld, s0, _ = make(3 * T, C, "f32", 3, 3)
    starts = torch.tensor([0, T, 2 * T, 3 * T], dtype=torch.int32).cuda()
    run = lambda: sw.sw_gated_recurrence(x.cuda(), r.cuda(), i.cuda(), ld.cuda(), starts=starts, state=s0.cuda())
    clean = run()
    if where == "state":
        s0[1, ch], at = value, 0
    elif where == "x":
        x[T + at, ch] = value
    else:
        r[T + at, ch] = value
    h = run().cpu()
    touched = torch.zeros(3 * T, C, dtype=torch.bool)
    touched[T + at:2 * T, ch] = True
    assert torch.equal(h[~touched], clean.cpu()[~touched])
    assert not torch.isfinite(h[touched]).any()
    # backwards: the same value in dh
    args = x.clone().nan_to_num(0, 0, 0), r.nan_to_num(0), i, ld
    back = lambda d: sw.sw_gated_recurrence_backward(d.cuda(), *(v.cuda() for v in args), clean, starts=starts, params=False)
    plain = back(dh)
    dh[T + at, ch] = value
    for a, b in zip(back(dh)[:3], plain[:3]):
        reached = torch.zeros(3 * T, C, dtype=torch.bool)
        reached[T:T + at + 1, ch] = True
        assert torch.equal(a.cpu()[~reached], b.cpu()[~reached])
        assert not torch.isfinite(a.cpu()[reached]).any()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,C,n", [(1, 1, 1), (1, 4096, 1), (5, 63, 9), (128, 520, 160), (3, 1001, 3), (70, 8, 70)])
def test_step(sw, B, C, n, t):
    x, r, i, _, ld, s0, _ = make(B, C, t, B + C, n)
    at = torch.randperm(n, generator=torch.Generator().manual_seed(n))[:B].tolist()
    if B > 2:
        at[1], at[2] = -1, n
    state = s0.cuda()
    h = sw.sw_gated_recurrence_step(x.cuda(), r.cuda(), i.cuda(), ld.cuda(), state, torch.tensor(at, dtype=torch.int32).cuda())
    left = torch.ones(n, dtype=torch.bool)
    for b, slot in enumerate(at):
        if not 0 <= slot < n:
            assert torch.all(h[b] == 0)
            continue
        left[slot] = False
        want, last, m, lm = O.recurrence(x[b:b + 1], r[b:b + 1], i[b:b + 1], ld, s0[slot])
        close(h[b:b + 1], want, m, t, 1)
        close(state[slot], last, lm, None, 1)
    assert torch.equal(state.cpu()[left], s0[left])
    if B == n:
        other = s0.cuda()
        assert torch.equal(sw.sw_gated_recurrence_step(x.cuda(), r.cuda(), i.cuda(), ld.cuda(), other)[:1], sw.sw_gated_recurrence_step(
            x.cuda(), r.cuda(), i.cuda(), ld.cuda(), s0.cuda(), torch.arange(B, dtype=torch.int32).cuda())[:1])


def test_step_slices(sw):
    B, C = 6, 45
    fused = torch.randn(B, 3 * C + 2, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    cut = [fused[:, k * C + 1:(k + 1) * C + 1] for k in range(3)]
    ld, s = torch.full((C,), -0.2, device="cuda"), torch.ones(B, C, device="cuda")
    wide = torch.full((B, C + 2), 7.0, dtype=torch.bfloat16, device="cuda")
    a, b = s.clone(), s.clone()
    want = sw.sw_gated_recurrence_step(*(v.contiguous() for v in cut), ld, a)
    assert torch.equal(sw.sw_gated_recurrence_step(*cut, ld, b, out=wide[:, 1:C + 1]), want) and torch.equal(a, b)
    assert torch.all(wide[:, 0] == 7.0) and torch.all(wide[:, -1] == 7.0)


def test_tokens_one_by_one_are_the_prompt(sw):
    B, T, C = 3, 40, 200
    x, r, i, _, ld, s0, _ = make(B * T, C, "f32", 6, B)
    shape = lambda v: v.reshape(B, T, C).cuda()
    final, state = torch.empty(B, C, device="cuda"), s0.cuda()
    h = sw.sw_gated_recurrence(shape(x), shape(r), shape(i), ld.cuda(), state=s0.cuda(), final_state=final)
    steps = torch.stack([sw.sw_gated_recurrence_step(shape(x)[:, k], shape(r)[:, k], shape(i)[:, k], ld.cuda(), state) for k in range(T)], 1)
    # (terms are |N(0, 1)| times weights below 1, |h| stays below the magnitudes' sum: four times the largest value covers it here)
    scale = max(float(h.abs().max()), 1.0)
    assert float((steps - h).abs().max()) <= 2 * lost(T) * scale * 4 and float((state - final).abs().max()) <= 2 * lost(T) * scale * 4


def test_gradients_against_differences(sw):
    """fp32, central differences of the definition's loss in 64 bits."""
    T, C = 20, 6
    x, r, i, dh, ld, s0, df = make(T, C, "f32", 12)
    loss = lambda x, r, i, ld, s: (lambda h, last: float((h * dh.double()).sum() + (last * df[0].double()).sum()))(*O.recurrence(x, r, i, ld, s)[:2])
    h = sw.sw_gated_recurrence(x[None].cuda(), r[None].cuda(), i[None].cuda(), ld.cuda(), state=s0.cuda())
    d_state = df.cuda()
    grads = sw.sw_gated_recurrence_backward(dh[None].cuda(), x[None].cuda(), r[None].cuda(), i[None].cuda(), ld.cuda(), h, state=s0.cuda(),
                                            d_final_state=d_state, d_state=d_state)
    given, step = [v.double() for v in (x, r, i, ld, s0[0])], 1e-5
    got = [*(v[0].cpu() for v in grads[:3]), grads[3].cpu(), d_state[0].cpu()]
    for k, g in enumerate(got):
        for at in range(0, g.numel(), 7):
            plus, minus = ([v.clone() for v in given] for _ in range(2))
            plus[k].view(-1)[at] += step
            minus[k].view(-1)[at] -= step
            want = (loss(*plus) - loss(*minus)) / (2 * step)
            assert abs(float(g.reshape(-1)[at]) - want) <= 2e-4 * (1 + abs(want)), (k, at)


def test_another_stream_and_graphs(sw):
    """On a stream of its own; captured, replayed on new inputs with eager calls between; two graphs that share their workspace's memory."""
    B, T, C = 2, 1500, 260
    made = [make(B * T, C, "bf16", seed, B) for seed in range(3)]
    dev = lambda m: [v.reshape(B, T, C).cuda() for v in m[:4]] + [m[4].cuda(), m[5].cuda()]
    x, r, i, dh, ld, s = dev(made[0])

    def both():
        f = torch.empty_like(s)
        h = sw.sw_gated_recurrence(x, r, i, ld, state=s, final_state=f)
        return (h, f, *sw.sw_gated_recurrence_backward(dh, x, r, i, ld, h, state=s))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = [v.clone() for v in both()]
    out = torch.empty_like(x)
    sw.sw_gated_recurrence(x, r, i, ld, state=s, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want[0])
    graphs = []
    pool = None
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            held = both()
        pool = g.pool()
        graphs.append((g, held))
    for turn in range(4):
        for v, new in zip((x, r, i, dh, ld, s), dev(made[turn % 3])):
            v.copy_(new)
        want = [v.clone() for v in both()]
        for g, held in graphs:
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_calls_side_by_side(sw):
    """Two streams at once, each with its own workspace."""
    B, T, C = 1, 4000, 512
    x, r, i, dh, ld, s0, _ = make(B * T, C, "f16", 9, B)
    args = [v.reshape(B, T, C).cuda() for v in (x, r, i)] + [ld.cuda()]
    want = sw.sw_gated_recurrence(*args)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    outs = [[torch.empty_like(want) for _ in range(5)] for _ in streams]
    for k in range(5):
        for st, o in zip(streams, outs):
            sw.sw_gated_recurrence(*args, out=o[k], stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(v, want) for o in outs for v in o)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_offsets_beyond_32_bits(sw, t):
    """Tokens and sequences so far apart that their places take more than 32 bits of bytes."""
    T, C = 5, 40
    far = (1 << 30) // (2 if t == "f32" else 1) + 8
    x, r, i, dh, ld, _, _ = make(T, C, t, 2)
    big = torch.zeros(T * far, dtype=TYPES[t], device="cuda")
    X = big.as_strided((T, C), (far, 1))
    X.copy_(x)
    args = r[None].cuda(), i[None].cuda(), ld.cuda()
    want = sw.sw_gated_recurrence(x[None].cuda(), *args)
    assert torch.equal(sw.sw_gated_recurrence(X[None], *args), want)
    grads = sw.sw_gated_recurrence_backward(dh[None].cuda(), x[None].cuda(), *args, want)
    assert all(torch.equal(a, b) for a, b in zip(sw.sw_gated_recurrence_backward(dh[None].cuda(), X[None], *args, want), grads))
    sw.sw_gated_recurrence(x[None].cuda(), *args, out=X[None])
    assert torch.equal(X, want[0])
    rows = sw.sw_gated_recurrence(x[:, None].cuda(), r[:, None].cuda(), i[:, None].cuda(), ld.cuda())
    X.copy_(x)
    assert torch.equal(sw.sw_gated_recurrence(X[:, None], r[:, None].cuda(), i[:, None].cuda(), ld.cuda()), rows)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [1, 2, 3, 65, 127, 128, 129, 131, 255, 257, 385])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("B", [6, 48])
def test_states_in_place(sw, C, packed, t, B):
    """States and gradients of states that replace what they come from, at widths whose last channels are a lane's or a workgroup's of their own: several times over,
    the same bits as into tensors of their own."""
    T = 300
    x, r, i, dh, ld, s0, df = make(B * T, C, t, C, B)
    shape = (lambda v: v.cuda()) if packed else (lambda v: v.reshape(B, T, C).cuda())
    args = shape(x), shape(r), shape(i), ld.cuda()
    starts = torch.arange(0, (B + 1) * T, T).int().cuda() if packed else None
    final, d_state = torch.empty(B, C, device="cuda"), torch.empty(B, C, device="cuda")
    h = sw.sw_gated_recurrence(*args, starts=starts, state=s0.cuda(), final_state=final)
    grads = sw.sw_gated_recurrence_backward(shape(dh), *args, h, starts=starts, state=s0.cuda(), d_final_state=df.cuda(), d_state=d_state)
    for _ in range(5):
        s, d = s0.cuda(), df.cuda()
        assert torch.equal(sw.sw_gated_recurrence(*args, starts=starts, state=s, final_state=s), h) and torch.equal(s, final)
        again = sw.sw_gated_recurrence_backward(shape(dh), *args, h, starts=starts, state=s0.cuda(), d_final_state=d, d_state=d)
        assert all(torch.equal(a, b) for a, b in zip(again, grads)) and torch.equal(d, d_state)
