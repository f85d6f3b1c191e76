"""Linear attention with a decay for each head on the GPU (prompts, gradients, single tokens) against the recurrence in 64 bits.

Tolerances.  A sum is compared with the same sum of its terms' magnitudes, A (the definition on absolute values).  A result is rounded
once to its format, at most e = eps / 2 of itself.  Within, a product may meet two factors rounded to the format (pair products and
states as operands of matrix instructions): 2 e of A for 16-bit formats; in fp32 additions count, u = 2^-24 each, 256 deep.  States
stay in fp32 and their terms keep at least 16 bits: 2^-16 of A, in fp32 256 u.  Over a whole head the roundings are independent:
the 2-norm of its error is held to 2 e of the head's 2-norm (fp32: 64 u), plus 8 u of A's for what cancels in the pair products."""
import math

import pytest

import layers_oracle as O

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


def decays(H):
    """From 1/4 a token to 1 - 2^-8."""
    return torch.tensor([math.log1p(-2.0 ** -(0.42 + 7.58 * i / max(1, H - 1))) for i in range(H)])


class Case:
    """Inputs, and what the definition makes of them, sequence by sequence."""

    def __init__(self, t, B, T, H, Hk, dk, dv, starts=None, states=True, seed=0, log_decay=None, scale=None):
        g = torch.Generator().manual_seed(seed)
        lead = (T,) if starts is not None else (B, T)
        r = lambda *s: torch.randn(*s, generator=g)
        self.t, self.B, self.T, self.starts = t, B, T, starts
        self.q, self.k, self.v, self.do = (r(*lead, h, d).to(TYPES[t]) for h, d in ((H, dk), (Hk, dk), (Hk, dv), (H, dv)))
        self.g = decays(H) if log_decay is None else log_decay
        self.scale = dk ** -0.5 if scale is None else scale
        self.state, self.d_final = (r(B, H, dk, dv), r(B, H, dk, dv)) if states else (None, None)

    def rows(self, x, b, r):
        return x[r] if b is None else x[b, r]

    def forward(self, mag=False):
        f = (lambda x: x.double().abs()) if mag else (lambda x: x)
        o = torch.zeros(*self.q.shape[:-1], self.v.shape[-1], dtype=torch.float64)
        last = []
        for i, (b, r) in enumerate(O.sequences(self.starts, self.T, self.B)):
            s0 = None if self.state is None else f(self.state[i])
            y, s = O.attention(*(f(self.rows(x, b, r)) for x in (self.q, self.k, self.v)), self.g, abs(self.scale) if mag else self.scale, s0)
            self.rows(o, b, r).copy_(y)
            last.append(s)
        return o, torch.stack(last)

    def backward(self, mag=False):
        f = (lambda x: x.double().abs()) if mag else (lambda x: x)
        grads = [torch.zeros(x.shape, dtype=torch.float64) for x in (self.q, self.k, self.v)]
        first = []
        for i, (b, r) in enumerate(O.sequences(self.starts, self.T, self.B)):
            s0, df = (None, None) if self.state is None else (f(self.state[i]), f(self.d_final[i]))
            *out, ds = O.attention_backward(*(f(self.rows(x, b, r)) for x in (self.do, self.q, self.k, self.v)), self.g,
                                              abs(self.scale) if mag else self.scale, s0, df)
            for x, y in zip(grads, out):
                self.rows(x, b, r).copy_(y)
            first.append(ds)
        return *grads, torch.stack(first)

    def on_gpu(self, *names):
        return [None if getattr(self, n) is None else getattr(self, n).cuda() for n in names]

    def cu(self):
        return None if self.starts is None else torch.tensor(self.starts, dtype=torch.int32).cuda()


def near(got, want, mag, t, what):
    got, e = got.cpu().double(), torch.finfo(TYPES[t]).eps / 2
    c = 256 * U if t == "f32" else 2 * e
    off = (got - want).abs()
    tol = e * want.abs() + c * mag + TINY[t]
    assert torch.all(off <= tol), f"{what}: {float((off / tol).max())} of the tolerance"
    norm = lambda x: x.reshape(-1, *x.shape[-2:]).pow(2).sum((0, 2)).sqrt()         # of each head
    assert torch.all(norm(got - want) <= (64 * U if t == "f32" else 2 * e) * norm(want) + 8 * U * norm(mag) + 16 * TINY[t]), what


def near_state(got, want, mag, t, what):
    got = got.cpu().double()
    assert torch.all((got - want).abs() <= (256 * U if t == "f32" else 2.0 ** -16) * mag + 1e-37), what


def check(sw, c):
    q, k, v, do, g, s0, df = c.on_gpu("q", "k", "v", "do", "g", "state", "d_final")
    final = torch.full((c.B, c.q.shape[-2], c.q.shape[-1], c.v.shape[-1]), float("nan"), device="cuda")
    o = sw.sw_linear_attention(q, k, v, g, c.scale, starts=c.cu(), state=s0, final_state=final)
    (ro, rf), (ao, af) = c.forward(), c.forward(True)
    near(o, ro, ao, c.t, "o")
    near_state(final, rf, af, c.t, "final_state")
    ds = torch.full_like(final, float("nan"))
    grads = sw.sw_linear_attention_backward(do, q, k, v, g, c.scale, starts=c.cu(), state=s0, d_final_state=df, d_state=ds)
    want, mag = c.backward(), c.backward(True)
    for x, y, a, n in zip(grads, want, mag, ("dq", "dk", "dv")):
        near(x, y, a, c.t, n)
    near_state(ds, want[3], mag[3], c.t, "d_state")


LENGTHS = [1, 2, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 127, 128, 129, 191, 200, 255, 256, 257, 300, 511, 513, 640, 1000]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", LENGTHS)
def test_lengths(sw, T, t):
    check(sw, Case(t, 2, T, 2, 2, 32, 32, states=T % 2 == 1, seed=T))


WIDTHS = [(1, 1), (1, 64), (64, 1), (3, 5), (8, 16), (16, 8), (17, 31), (33, 32), (32, 65), (48, 80), (64, 64), (64, 128), (72, 40), (80, 48), (96, 64),
          (100, 100), (128, 64), (128, 128), (129, 127), (136, 200), (192, 96), (200, 33), (256, 64), (64, 256), (256, 256)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("dk,dv", WIDTHS)
def test_widths(sw, dk, dv, t):
    check(sw, Case(t, 1, 150, 2, 1, dk, dv, seed=dk * 3 + dv))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,T,H,Hk", [(1, 70, 1, 1), (3, 70, 4, 2), (2, 130, 6, 1), (5, 40, 12, 4), (1, 2100, 4, 2), (2, 1100, 3, 3)])
def test_batches_and_shared_heads(sw, B, T, H, Hk, t):
    check(sw, Case(t, B, T, H, Hk, 64, 64, seed=T))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("starts,T", [
    ([0, 1], 1), ([0, 0], 1), ([0, 0, 0, 3], 3), ([0, 1, 2, 3, 4], 4), ([0, 64, 128], 128), ([0, 63, 64, 129, 130], 130), ([5, 9, 9, 40], 50),
    ([0, 0, 1, 1, 300, 300, 333, 900], 900), ([3, 700, 701, 1400], 1500), ([-5, 20, 999], 64), ([0, 50, 50, 60], 64), ([0, 10], 300), ([200, 200], 200)])
def test_packed(sw, starts, T, t):
    """Empty sequences, single tokens, rows before the first and after the last sequence, starts out of range."""
    check(sw, Case(t, len(starts) - 1, T, 2, 1, 48, 64, starts=starts, seed=T))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", [5, 100, 700])
def test_rows_outside_of_sequences_are_zero(sw, T, t):
    c = Case(t, 2, T + 9, 2, 1, 32, 32, starts=[4, 4 + T // 2, 4 + T], states=False, seed=T)
    q, k, v, do, g = c.on_gpu("q", "k", "v", "do", "g")
    nan = lambda x: torch.full_like(x, float("nan"))
    o = sw.sw_linear_attention(q, k, v, g, starts=c.cu(), out=nan(do))
    grads = sw.sw_linear_attention_backward(do, q, k, v, g, starts=c.cu(), out=(nan(q), nan(k), nan(v)))
    for x in (o, *grads):
        assert torch.isfinite(x).all() and not x[:4].any() and not x[4 + T:].any() and x[4:4 + T].any()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", [1, 40, 64, 200, 600])
def test_decays_at_the_ends(sw, T, t):
    """No decay at all, everything before a token forgotten (exp underflows; -infinity), very strong and very weak decays."""
    g = torch.tensor([0.0, -float("inf"), -200.0, -20.0, -1e-6, -3.0])
    check(sw, Case(t, 1, T, 6, 3, 32, 48, seed=T, log_decay=g))


@pytest.mark.parametrize("t", TYPES)
def test_scales_and_magnitudes(sw, t):
    """Pair products and states beyond what half holds under results that it holds, and small values."""
    c = Case(t, 1, 300, 2, 2, 64, 64, seed=1, log_decay=torch.tensor([0.0, -0.01]), scale=1e-4)
    c.q, c.k = (c.q.float() * 40).to(c.q.dtype), (c.k.float() * 40).to(c.k.dtype)
    check(sw, c)
    c = Case(t, 1, 300, 2, 2, 64, 64, seed=2, scale=3.0)
    c.v = (c.v.float() * 2.0 ** -6).to(c.v.dtype)
    c.state = c.state * 2.0 ** -6
    check(sw, c)
    check(sw, Case(t, 1, 90, 2, 2, 64, 64, seed=3, scale=0.0))
    check(sw, Case(t, 1, 90, 2, 2, 64, 64, seed=3, scale=-0.3))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", [1, 50, 130, 700])
def test_strides(sw, T, t):
    """q, k and v out of one fused projection at odd offsets, heads before tokens, outputs into wider rows."""
    c = Case(t, 2, T, 4, 2, 40, 24, seed=T)
    q, k, v, do, g, s0, df = c.on_gpu("q", "k", "v", "do", "g", "state", "d_final")
    final, ds = torch.empty_like(s0), torch.empty_like(s0)
    want = sw.sw_linear_attention(q, k, v, g, state=s0, final_state=final)
    dwant = sw.sw_linear_attention_backward(do, q, k, v, g, state=s0, d_final_state=df, d_state=ds)

    def views(fill):
        fused = torch.full((2, T, 3 + 4 * 40 + 2 * 40 + 2 * 24), fill, dtype=q.dtype, device="cuda")
        cut = lambda at, h, d: fused[:, :, at:at + h * d].unflatten(-1, (h, d))
        return fused, [cut(3, 4, 40), cut(163, 2, 40), cut(243, 2, 24)]

    fused, (fq, fk, fv) = views(0.0)
    fq.copy_(q), fk.copy_(k), fv.copy_(v)
    swapped = do.transpose(1, 2).contiguous().transpose(1, 2)
    f2, ds2 = torch.empty_like(s0), torch.empty_like(s0)
    wide = torch.full((2, T, 4, 30), 7.0, dtype=q.dtype, device="cuda")
    o = sw.sw_linear_attention(fq, fk, fv, g, state=s0, final_state=f2, out=wide[..., 2:26])
    assert torch.equal(o, want) and torch.equal(f2, final) and torch.all(wide[..., :2] == 7.0) and torch.all(wide[..., 26:] == 7.0)
    grads, outs = views(7.0)
    got = sw.sw_linear_attention_backward(swapped, fq, fk, fv, g, state=s0, d_final_state=df, d_state=ds2, out=outs)
    assert all(torch.equal(a, b) for a, b in zip(got, dwant)) and torch.equal(ds2, ds) and torch.all(grads[..., :3] == 7.0)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", [1, 64, 300])
def test_keys_and_values_of_all_tokens_alike(sw, T, t):
    """Broadcast inputs (a stride of zero)."""
    c = Case(t, 1, T, 2, 2, 32, 32, seed=T, states=False)
    c.k, c.v = c.k[:, :1].expand(-1, T, -1, -1), c.v[:, :, :1].expand(-1, -1, 2, -1)
    check(sw, c)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", [7, 150, 700])
def test_slots_and_states_in_place(sw, T, t):
    c = Case(t, 4, T, 2, 1, 32, 48, starts=[0, T // 3, T // 3, T - 1, T], seed=T)
    q, k, v, g, s0 = c.on_gpu("q", "k", "v", "g", "state")
    final = torch.empty_like(s0)
    want = sw.sw_linear_attention(q, k, v, g, starts=c.cu(), state=s0, final_state=final)
    cache = torch.full((7, *s0.shape[1:]), 5.0, device="cuda")
    slots = torch.tensor([6, 0, 3, 2], dtype=torch.int32).cuda()
    cache[slots.long()] = s0
    o = sw.sw_linear_attention(q, k, v, g, starts=c.cu(), state=cache, final_state=cache, slots=slots)
    assert torch.equal(o, want) and torch.equal(cache[slots.long()], final) and torch.all(cache[torch.tensor([1, 4, 5]).cuda()] == 5.0)
    # entries out of range: from zero, and not kept
    cache[slots.long()] = s0
    before = cache.clone()
    out = torch.tensor([-1, 7, 3, 1 << 30], dtype=torch.int32).cuda()
    o = sw.sw_linear_attention(q, k, v, g, starts=c.cu(), state=cache, final_state=cache, slots=out)
    zero = torch.zeros_like(s0)
    zero[2] = s0[2]
    assert torch.equal(o, sw.sw_linear_attention(q, k, v, g, starts=c.cu(), state=zero))
    before[3] = final[2]
    assert torch.equal(cache, before)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", [9, 100, 260, 900])
def test_prompt_in_parts(sw, T, t):
    """A prompt in two calls, the second from the first one's states, is the prompt in one call; its last token by the step call too."""
    c = Case(t, 2, T, 2, 2, 64, 32, seed=T)
    q, k, v, g, s0 = c.on_gpu("q", "k", "v", "g", "state")
    (ro, rf), (ao, af) = c.forward(), c.forward(True)
    state, cut = s0.clone(), T // 3
    parts = [sw.sw_linear_attention(q[:, a:b], k[:, a:b], v[:, a:b], g, state=state, final_state=state) for a, b in ((0, cut), (cut, T - 1))]
    parts.append(sw.sw_linear_attention_step(q[:, -1], k[:, -1], v[:, -1], g, state)[:, None])
    near(torch.cat(parts, 1), ro, ao, t, "o")
    near_state(state, rf, af, t, "state")


def nonfinite_equal(got, want):
    got = got.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    return torch.isfinite(want)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,at", [(1, 0), (40, 7), (100, 70), (130, 129), (700, 65), (700, 400)])
@pytest.mark.parametrize("which,value", [("q", math.inf), ("k", math.nan), ("k", math.inf), ("v", -math.inf), ("v", math.nan)])
def test_nonfinite_values_reach_later_tokens_only(sw, T, at, which, value, t):
    """An infinity or a NaN in one token's row of one head: earlier tokens, other heads and other sequences keep their values, and what it
    reaches is what the recurrence makes of it."""
    c = Case(t, 2, T, 2, 2, 32, 48, seed=T, states=False, log_decay=torch.tensor([-0.02, -0.5]))
    clean, _ = c.forward()
    _, mag = c.forward(), c.forward(True)[0]
    getattr(c, which)[1, at, 0, 5] = value
    ro, rf = c.forward()
    q, k, v, g = c.on_gpu("q", "k", "v", "g")
    final = torch.empty(2, 2, 32, 48, device="cuda")
    o = sw.sw_linear_attention(q, k, v, g, final_state=final)
    fine = nonfinite_equal(o, ro)
    assert fine[0].all() and fine[1, :at].all() and fine[:, :, 1].all()
    e = torch.finfo(TYPES[t]).eps / 2
    assert torch.all(((o.cpu().double() - ro).abs() <= e * clean.abs() + (256 * U if t == "f32" else 2 * e) * mag + TINY[t])[fine])
    nonfinite_equal(final, rf)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,at", [(1, 0), (100, 70), (700, 400)])
@pytest.mark.parametrize("which", ["do", "q", "k", "v"])
def test_nonfinite_gradients(sw, T, at, which, t):
    c = Case(t, 1, T, 2, 2, 32, 48, seed=T, states=False, log_decay=torch.tensor([-0.02, -0.5]))
    getattr(c, which)[0, at, 1, 3] = math.inf
    q, k, v, do, g = c.on_gpu("q", "k", "v", "do", "g")
    for got, want in zip(sw.sw_linear_attention_backward(do, q, k, v, g), c.backward()):
        assert nonfinite_equal(got, want)[:, :, 0].all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,H,Hk,dk,dv", [(1, 1, 1, 1, 1), (1, 16, 16, 128, 128), (3, 4, 2, 64, 64), (2, 6, 1, 48, 80), (5, 2, 2, 33, 7), (1, 2, 2, 256, 256),
                                          (70, 3, 3, 32, 16), (2, 4, 4, 100, 36), (9, 2, 1, 17, 130), (4, 1, 1, 200, 3)])
def test_single_tokens(sw, B, H, Hk, dk, dv, t):
    c = Case(t, B, 1, H, Hk, dk, dv, seed=dk + dv)
    q, k, v, g = c.on_gpu("q", "k", "v", "g")
    (ro, rf), (ao, af) = c.forward(), c.forward(True)
    state = c.state.cuda()
    o = sw.sw_linear_attention_step(q[:, 0], k[:, 0], v[:, 0], g, state, scale=c.scale)
    near(o[:, None], ro, ao, t, "o")
    near_state(state, rf, af, "f32", "state")
    # slots, unused rows, strided rows and a strided output
    n = B + 3
    cache = torch.full((n, H, dk, dv), 5.0, device="cuda")
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(B))[:B]
    cache[slots.cuda()] = c.state.cuda()
    used = torch.ones(B, dtype=torch.bool)
    used[B // 2] = B == 1
    before = cache.clone()
    before[slots[used].cuda()] = state[used.cuda()]
    given = torch.where(used, slots, torch.tensor(-1 if B % 2 else n)).int().cuda()
    qkv = torch.zeros(B, H * dk + Hk * dk + Hk * dv + 1, dtype=q.dtype, device="cuda")[:, 1:]
    cut = lambda a, h, d: qkv[:, a:a + h * d].unflatten(-1, (h, d))
    fq, fk, fv = cut(0, H, dk), cut(H * dk, Hk, dk), cut((H + Hk) * dk, Hk, dv)
    fq.copy_(q[:, 0]), fk.copy_(k[:, 0]), fv.copy_(v[:, 0])
    out = torch.full((B, H, dv + 1), 7.0, dtype=q.dtype, device="cuda")
    got = sw.sw_linear_attention_step(fq, fk, fv, g, cache, given, c.scale, out=out[..., :dv])
    assert torch.equal(got[used.cuda()], o[used.cuda()]) and not got[~used.cuda()].any() and torch.all(out[..., dv] == 7.0)
    assert torch.equal(cache, before)


def test_offsets_beyond_32_bits(sw):
    """A cache of more than 2^31 values, and tokens 2 GiB apart."""
    H, d = 2, 64
    n = (1 << 31) // (H * d * d) + 40
    cache = torch.empty(n, H, d, d, device="cuda")
    c = Case("bf16", 2, 3, H, H, d, d, seed=4)
    q, k, v, g, s0 = c.on_gpu("q", "k", "v", "g", "state")
    slots = torch.tensor([n - 1, n // 2], dtype=torch.int32).cuda()
    cache[slots.long()] = s0
    stride = 1 << 30
    far = torch.empty(2 * stride + 2 * H * d, dtype=torch.bfloat16, device="cuda").as_strided((2, 3, H, d), (H * d, stride, d, 1))
    far.copy_(k)
    o = sw.sw_linear_attention(q[:, :2], far[:, :2], v[:, :2], g, state=cache, final_state=cache, slots=slots)
    last = sw.sw_linear_attention_step(q[:, 2], far[:, 2], v[:, 2], g, cache, slots)
    (ro, rf), (ao, af) = c.forward(), c.forward(True)
    near(torch.cat([o, last[:, None]], 1), ro, ao, "bf16", "o")
    near_state(cache[slots.long()], rf, af, "bf16", "state")


@pytest.mark.parametrize("T", [30, 600])
def test_another_stream_and_graph_replays(sw, T):
    c = Case("bf16", 2, T, 4, 2, 64, 64, seed=T)
    q, k, v, do, g, s0, df = c.on_gpu("q", "k", "v", "do", "g", "state", "d_final")
    final, ds, cache = torch.empty_like(s0), torch.empty_like(s0), s0.clone()

    def step(stream=None):
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            cache.copy_(s0)
        o = sw.sw_linear_attention(q, k, v, g, state=s0, final_state=final, stream=stream)
        grads = sw.sw_linear_attention_backward(do, q, k, v, g, state=s0, d_final_state=df, d_state=ds, stream=stream)
        return [o, *grads, sw.sw_linear_attention_step(q[:, 0], k[:, 0], v[:, 0], g, cache, stream=stream), final, ds, cache]

    want = [x.clone() for x in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        for x in (q, k, v, do, s0, df):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        assert (q.float() * 2).sum().isfinite().item()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_refusals(sw):
    q = torch.randn(2, 5, 4, 8, device="cuda")
    g = -torch.rand(4, device="cuda")
    s = torch.zeros(2, 4, 8, 8, device="cuda")
    A, Bk, S = sw.sw_linear_attention, sw.sw_linear_attention_backward, sw.sw_linear_attention_step
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for call in (lambda: A(q, q, q.bfloat16(), g), lambda: A(q, q[:, :4], q, g), lambda: A(q, q, q, g[:3]), lambda: A(q, q, q, g.double()),
                 lambda: A(q, q, q, g, state=s[:, :, :4]), lambda: A(q, q, q, g, state=s.bfloat16()), lambda: A(q, q, q, g, state=s, final_state=s[:1]),
                 lambda: A(q, q, q, g, slots=i32(0)), lambda: A(q, q, q, g, starts=i32(0, 5, 10)), lambda: A(q[0], q[0], q[0], g, starts=i32(0, 5).long()),
                 lambda: A(q.transpose(2, 3), q, q, g), lambda: A(q, q, q, g, out=q[:, :3]), lambda: Bk(q[..., :4], q, q, q, g),
                 lambda: Bk(q, q, q, q, g, d_final_state=s[:1]), lambda: S(q[:, 0], q[:, 0], q[:, 0], g, s[:, :3]), lambda: S(q, q, q, g, s)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: A(q, q, q, g, out=q), lambda: A(q, q, q, g, state=s[:1]), lambda: S(q[:, 0], q[:, 0], q[:, 0], g, s[:1]),
                 lambda: A(q[0], q[0], q[0], g, starts=i32(0)), lambda: A(q, q, q, g, scale=math.inf), lambda: Bk(q, q, q, q, g, out=(q, q, q))):
        with pytest.raises(sw.SwError):
            call()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,T,H,Hk,dk,dv", [(13, 70, 20, 20, 72, 100), (13, 33, 20, 10, 24, 128), (9, 65, 32, 8, 130, 70), (5, 20, 52, 52, 200, 130), (1, 1300, 32, 32, 16, 80),
                                            (2, 700, 30, 30, 80, 72)])
def test_many_heads_of_wide_values(sw, B, T, H, Hk, dk, dv, t):
    """Launches that fill the chip, on values (and keys) of more than 64 columns."""
    c = Case(t, B, T, H, Hk, dk, dv, seed=B + T)
    check(sw, c)


@pytest.mark.parametrize("t", TYPES)
def test_many_packed_heads_of_wide_values(sw, t):
    starts = [0, 0, 1, 130, 700, 701, 1000, 1490]
    check(sw, Case(t, len(starts) - 1, 1500, 30, 30, 24, 96, starts=starts, seed=7))
