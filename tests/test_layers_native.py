"""Layer norm and linear attention through the native short way of the binding: what the long way gives, the same bits and the same exceptions."""
import pytest

torch = pytest.importorskip("torch")

import paper_2310_05218_amd as sw  # noqa: E402
from paper_2310_05218_amd import binding  # noqa: E402


def calls(dev):
    g = torch.Generator().manual_seed(3)
    f = lambda *s: torch.randn(s, generator=g).to(dev)
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device=dev)
    x, w, b, dy = f(3, 5, 24), f(24), f(24), f(3, 5, 24)
    wide = f(7, 40)
    mean, rstd = x.mean(-1), x.std(-1)
    q, k, v, do, g4 = f(2, 70, 4, 16), f(2, 70, 2, 16), f(2, 70, 2, 24), f(2, 70, 4, 24), -f(4).abs()
    s0, s1 = f(2, 4, 16, 24), f(5, 4, 16, 24)
    fused = f(2, 70, 4 * 16 + 2 * 16 + 2 * 24)
    cut = lambda a, h, d: fused[:, :, a:a + h * d].unflatten(-1, (h, d))
    fq, fk, fv = cut(0, 4, 16), cut(64, 2, 16), cut(96, 2, 24)
    long = f(1, 900, 2, 32)
    N, NB, A, AB, S = sw.sw_layer_norm, sw.sw_layer_norm_backward, sw.sw_linear_attention, sw.sw_linear_attention_backward, sw.sw_linear_attention_step
    P = torch.nn.Parameter

    def with_state(call):
        """The call's outputs, and the states that it wrote."""
        def run():
            state = s1.clone()
            out = call(state)
            return (*(out if isinstance(out, tuple) else (out,)), state)
        return run

    token = q[:, 0], k[:, 0], v[:, 0], g4
    return {
        "norm": lambda: N(x, w, b), "norm stats": lambda: N(x, w, b, 1e-3, stats=True), "norm parameter": lambda: N(x, P(w), P(b)),
        "norm none": lambda: N(x, None, None, 1e-5, True), "norm bf16": lambda: N(x.bfloat16(), w, b), "norm rows": lambda: N(wide[:, 3:27], w, None),
        "norm one row": lambda: N(x[0, 0], w, b, stats=True), "norm turned": lambda: N(x.transpose(0, 1), w, b), "norm columns": lambda: N(x.transpose(1, 2), w),
        "norm every other": lambda: N(wide[::2, :24], w, b), "norm integer eps": lambda: N(x, w, b, 1), "norm negative eps": lambda: N(x, w, b, -1.0),
        "norm huge eps": lambda: N(x, w, b, 1e300), "norm none eps": lambda: N(x, w, b, None), "norm weight bf16": lambda: N(x, w.bfloat16()), "norm short": lambda: N(x, w[:8]),
        "norm double": lambda: N(x.double(), w), "norm empty": lambda: N(x[:0], w), "norm value": lambda: N(x[0, 0, 0], None), "norm no tensor": lambda: N(None, w),
        "norm back": lambda: NB(dy, x, w, mean, rstd), "norm back dx": lambda: NB(dy, x, w, mean, rstd, params=False),
        "norm back f16": lambda: NB(dy.half(), x.half(), None, mean, rstd), "norm back rows": lambda: NB(wide[:, :24], wide[:, 16:], w, wide[:, 0].contiguous(), wide[:, 1].contiguous()),
        "norm back types": lambda: NB(dy.half(), x, w, mean, rstd), "norm back shapes": lambda: NB(dy[:2], x, w, mean, rstd), "norm back none": lambda: NB(dy, x, w, None, rstd),
        "attention": lambda: A(q, k, v, g4), "attention scale": lambda: A(q, k, v, g4, 0.5), "attention integer scale": lambda: A(q, k, v, g4, 2),
        "attention bf16": lambda: A(q.bfloat16(), k.bfloat16(), v.bfloat16(), g4, state=s0), "attention segments": lambda: A(long, long, long, g4[:2].contiguous()),
        "attention strides": lambda: A(fq, fk, fv, g4), "attention packed": lambda: A(q[0], k[0], v[0], g4, starts=i(0, 9, 9, 70)),
        "attention states": with_state(lambda s: A(q, k, v, g4, state=s, final_state=s, slots=i(4, 1))),
        "attention final": with_state(lambda s: A(q, k, v, g4, final_state=s)), "attention few states": lambda: A(q, k, v, g4, state=s0[:1]),
        "attention infinite scale": lambda: A(q, k, v, g4, float("inf")), "attention mixed": lambda: A(q, k.half(), v, g4), "attention heads": lambda: A(q, k[:, :, :1], v, g4),
        "attention thirds": lambda: A(q[:, :, :3], k, v, g4[:3].contiguous()), "attention starts type": lambda: A(q[0], k[0], v[0], g4, starts=i(0, 70).long()),
        "attention starts short": lambda: A(q[0], k[0], v[0], g4, starts=i(0)), "attention empty": lambda: A(q[:, :0], k[:, :0], v[:, :0], g4),
        "attention decays": lambda: A(q, k, v, g4[:2]), "attention slots": lambda: A(q, k, v, g4, state=s1, slots=i(1)), "attention state type": lambda: A(q, k, v, g4, state=s0.half()),
        "attention two states": lambda: A(q, k, v, g4, state=s1, final_state=s0), "attention widths": lambda: A(q.transpose(2, 3), k, v, g4),
        "attention alias": lambda: A(q, k, v, g4, state=s1, final_state=s1[:]), "attention 3-d": lambda: A(q[0], k[0], v[0], g4),
        "back": lambda: AB(do, q, k, v, g4), "back states": with_state(lambda s: AB(do, q, k, v, g4, 0.3, state=s0, d_final_state=s1[:2].clone(), d_state=s[:2])),
        "back packed": lambda: AB(do[1], q[1], k[1], v[1], g4, starts=i(3, 60)), "back slots": lambda: AB(do, fq, fk, fv, g4, state=s1, slots=i(2, -1)),
        "back half": lambda: AB(do.half(), q.half(), k.half(), v.half(), g4), "back types": lambda: AB(do.half(), q, k, v, g4), "back widths": lambda: AB(q, q, k, v, g4),
        "back final": lambda: AB(do, q, k, v, g4, d_final_state=s1), "back segments": lambda: AB(long, long, long, long, g4[:2].contiguous()),
        "step": with_state(lambda s: S(*token, s[:2])), "step slots": with_state(lambda s: S(*token, s, i(3, -1), 0.7)), "step half": with_state(lambda s: S(*(t.half() for t in token[:3]), g4, s)),
        "step few": lambda: S(*token, s0[:1]), "step state": lambda: S(*token, s0[:, :, :3]), "step none": lambda: S(*token, None), "step 4-d": lambda: S(q, k, v, g4, s0),
        "step off the GPU": lambda: S(*token, s0.cpu()),
    }


def outcome(f):
    try:
        y = f()
        return tuple(None if t is None else (t.dtype, t.requires_grad, t.is_contiguous(), t.cpu()) for t in (y if isinstance(y, tuple) else (y,)))
    except Exception as e:
        return type(e), str(e)


def same(a, b):
    if isinstance(a, tuple) and isinstance(b, tuple):
        return len(a) == len(b) and all(same(x, y) for x, y in zip(a, b))
    return torch.equal(a, b) if torch.is_tensor(a) and torch.is_tensor(b) else a == b


def both_ways(monkeypatch, dev):
    binding._native(-1)         # (bound)
    assert binding._native.__name__ == "run", "the native module is not built"
    for name in calls(dev):
        short = outcome(calls(dev)[name])
        with monkeypatch.context() as m:
            m.setattr(binding, "_native", lambda *a: None)
            long = outcome(calls(dev)[name])
        assert same(short, long), f"{name}: {short} / {long}"


def test_off_the_gpu(monkeypatch):
    both_ways(monkeypatch, "cpu")


@pytest.mark.gpu
def test_on_the_gpu(monkeypatch):
    both_ways(monkeypatch, "cuda")


@pytest.mark.gpu
def test_plain_calls_are_taken():
    """The short way is the one that ordinary calls go."""
    binding._native(-1)
    x = torch.randn(4, 16, device="cuda")
    q, state, g = torch.randn(2, 8, 2, 16, device="cuda"), torch.zeros(2, 2, 16, 16, device="cuda"), torch.full((2,), -0.1, device="cuda")
    run = binding._native
    assert run(binding._LAYER_NORM, x, None, None, 1e-5, False).shape == x.shape
    assert len(run(binding._LAYER_NORM_BACKWARD, x, x, None, x[:, 0].contiguous(), x[:, 0].contiguous(), True)) == 3
    assert run(binding._ATTENTION, q, q, q, g, None, None, state, None, state).shape == q.shape
    assert len(run(binding._ATTENTION_BACKWARD, q, q, q, q, g, None, None, None, None, None, None)) == 3
    assert run(binding._ATTENTION_STEP, q[:, 0], q[:, 0], q[:, 0], g, None, state, None).shape == (2, 2, 16)
