"""Linear attention of tensors whose tokens lie more than 2^24 elements apart, which goes token by token: the cases and tolerances of near ones."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_linear_attention import TYPES, Case, near, near_state, nonfinite_equal, sw  # noqa: E402,F401

APART = (1 << 24) + 24


def far(x):
    """The same values, tokens APART elements from one to the next and batches between them."""
    *lead, T, H, d = x.shape
    B = lead[0] if lead else 1
    out = torch.empty((T - 1) * APART + B * H * d, dtype=x.dtype, device="cuda").as_strided((B, T, H, d), (H * d, APART, d, 1))
    out.copy_(x)
    return out if lead else out[0]


def calls(sw, c):
    q, k, v, do, g, s0, df = c.on_gpu("q", "k", "v", "do", "g", "state", "d_final")
    shape = (c.B, c.q.shape[-2], c.q.shape[-1], c.v.shape[-1])
    final, ds = (torch.full(shape, float("nan"), device="cuda") for _ in range(2))
    o = sw.sw_linear_attention(q, far(k), v, g, c.scale, starts=c.cu(), state=s0, final_state=final)
    assert sw.sw_last_kernel().startswith("attention_recurrent_kernel")
    grads = sw.sw_linear_attention_backward(do, q, k, far(v), g, c.scale, starts=c.cu(), state=s0, d_final_state=df, d_state=ds)
    return o, final, grads, ds


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,T,H,Hk,dk,dv,starts", [(1, 20, 2, 2, 48, 80, None), (2, 9, 4, 2, 33, 5, None), (1, 30, 2, 1, 136, 200, None), (1, 2, 1, 1, 1, 1, None),
                                                   (4, 30, 2, 1, 72, 100, [2, 2, 3, 20, 28]), (3, 25, 2, 2, 128, 64, [0, 0, 24, 25])])
def test_far_rows(sw, B, T, H, Hk, dk, dv, starts, t):  # noqa: F811
    c = Case(t, B, T, H, Hk, dk, dv, starts=starts, seed=T + dk)
    o, final, grads, ds = calls(sw, c)
    (ro, rf), (ao, af) = c.forward(), c.forward(True)
    near(o, ro, ao, t, "o")
    near_state(final, rf, af, t, "final_state")
    want, mag = c.backward(), c.backward(True)
    for x, y, a, n in zip(grads, want, mag, ("dq", "dk", "dv")):
        near(x, y, a, t, n)
    near_state(ds, want[3], mag[3], t, "d_state")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("dk,dv", [(48, 80), (65, 24), (136, 130), (64, 64)])
@pytest.mark.parametrize("which,value", [("v", math.inf), ("k", -math.inf), ("k", math.nan), ("do", math.inf), ("q", math.inf)])
def test_nonfinite_values(sw, which, value, dk, dv, t):  # noqa: F811
    """Among positive operands an infinity stays one: what the recurrence makes of it, whatever the widths."""
    c = Case(t, 1, 12, 2, 2, dk, dv, seed=dk, states=False)
    for n in ("q", "k", "v", "do"):
        getattr(c, n).abs_().add_(0.125)
    getattr(c, which)[0, 5, 1, 3] = value
    o, final, grads, ds = calls(sw, c)
    want, (ro, rf) = c.backward(), c.forward()
    for got, w in zip((o, final, *grads, ds), (ro, rf, *want)):
        nonfinite_equal(got, w)
