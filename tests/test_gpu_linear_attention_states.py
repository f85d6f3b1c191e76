"""States of linear attention at the ends of fp32's range: the cases and tolerances of ordinary ones."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_linear_attention import Case, check, near_state, nonfinite_equal, sw  # noqa: E402,F401


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,starts", [(1, 700, 6, None), (2, 400, 6, [0, 100, 400]), (8, 2000, 6, None)])
def test_large_states_fade_whole(sw, B, T, H, starts, t):  # noqa: F811
    """First states of 1e37 where a segment's decay is below 2^-126 or 2^-149: what is left of them is what the recurrence leaves."""
    c = Case(t, B, T, H, 3, 32, 32, starts=starts, seed=T, log_decay=torch.tensor([-0.35, -0.7, -1.0, -1.4, -2.0, -20.0]), scale=1.0)
    c.state, c.d_final = c.state.clamp(-2, 2) * 1e37, c.d_final.clamp(-2, 2) * 1e37
    check(sw, c)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [60, 700])
def test_infinite_states_stay(sw, T, t):  # noqa: F811
    """An infinity of the first state stays one however strong the decay, but where nothing is left of a state (0 times infinity, NaN)."""
    c = Case(t, 1, T, 4, 2, 32, 48, seed=T, log_decay=torch.tensor([-0.01, -1.4, -60.0, -math.inf]))
    c.q.abs_().add_(0.125)
    c.state[0, :, 3, 5] = math.inf
    q, k, v, g, s0 = c.on_gpu("q", "k", "v", "g", "state")
    final = torch.empty_like(s0)
    o = sw.sw_linear_attention(q, k, v, g, c.scale, state=s0, final_state=final)
    ro, rf = c.forward()
    nonfinite_equal(o, ro)
    nonfinite_equal(final, rf)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [1, 30, 64, 128, 700])
def test_large_states_beside_small_values(sw, T, t):  # noqa: F811
    """A state of 1e30 that values of 2^-20 are added to, and its gradient: finite, whatever the last chunk's own terms are."""
    c = Case(t, 1, T, 2, 1, 32, 48, seed=T, log_decay=torch.tensor([-0.001, -0.02]), scale=2.0 ** -100)
    c.v, c.do = (c.v.float() * 2.0 ** -20).to(c.v.dtype), (c.do.float() * 2.0 ** -20).to(c.do.dtype)
    c.state, c.d_final = c.state * 1e30, c.d_final * 1e30
    q, k, v, do, g, s0, df = c.on_gpu("q", "k", "v", "do", "g", "state", "d_final")
    final, ds = torch.empty_like(s0), torch.empty_like(s0)
    sw.sw_linear_attention(q, k, v, g, c.scale, state=s0, final_state=final)
    sw.sw_linear_attention_backward(do, q, k, v, g, c.scale, state=s0, d_final_state=df, d_state=ds)
    near_state(final, c.forward()[1], c.forward(True)[1], t, "final_state")
    near_state(ds, c.backward()[3], c.backward(True)[3], t, "d_state")
