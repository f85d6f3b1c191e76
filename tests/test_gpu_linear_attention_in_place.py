"""Gradients of linear attention whose d_state replaces d_final_state, against those with a buffer for each: the same bits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MANY = [0] + [b for i in range(150) for b in (i * 10 + 1, i * 10 + 10)] + [1500, 1900, 2500]     # 150 single tokens, as many of nine, a few long ones


@pytest.fixture(scope="module")
def sw():
    import paper_2310_05218_amd as _sw
    from paper_2310_05218_amd import binding

    assert torch.cuda.is_available(), "these tests need the GPU"
    binding.lib()            # fails loudly if the library is not built
    return _sw


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("bad", [False, True], ids=["finite", "infinity"])
@pytest.mark.parametrize("B,T,H,Hk,dk,dv,starts", [
    (2, 50, 2, 1, 32, 48, None), (16, 64, 16, 16, 256, 256, None), (16, 200, 16, 4, 256, 256, None), (64, 128, 16, 16, 128, 128, None),
    (40, 70, 16, 16, 64, 128, None), (2, 1100, 4, 4, 64, 64, None), (len(MANY) - 1, 2500, 8, 4, 128, 128, MANY), (len(MANY) - 1, 2500, 4, 4, 256, 200, MANY)])
def test_d_state_in_place(sw, B, T, H, Hk, dk, dv, starts, bad, t):
    """Launches that the chip holds at once and larger ones, one and several blocks of columns, whole sequences and segments."""
    r = torch.Generator(device="cuda").manual_seed(T + dk)
    n = lambda *s: torch.randn(s, generator=r, device="cuda")
    lead = (T,) if starts else (B, T)
    q, k, v, do = (n(*lead, h, d).to(TYPES[t]) for h, d in ((H, dk), (Hk, dk), (Hk, dv), (H, dv)))
    if bad:
        do[(0, T // 2)[len(lead) == 1:]][0, 1] = math.inf
        k[(B - 1, T - 1)[len(lead) == 1:]][0, 0] = math.nan
    g = torch.log1p(-torch.exp2(-torch.linspace(2, 8, H))).cuda()
    s0, df = n(B, H, dk, dv), n(B, H, dk, dv)
    at = torch.tensor(starts, dtype=torch.int32, device="cuda") if starts else None
    ds = torch.empty_like(df)
    want = sw.sw_linear_attention_backward(do, q, k, v, g, starts=at, state=s0, d_final_state=df, d_state=ds)
    for _ in range(3):
        both = df.clone()
        got = sw.sw_linear_attention_backward(do, q, k, v, g, starts=at, state=s0, d_final_state=both, d_state=both)
        bits = lambda x: x.view(torch.int16 if x.element_size() == 2 else torch.int32)
        for name, a, b in zip(("dq", "dk", "dv", "d_state"), (*got, both), (*want, ds)):
            assert torch.equal(bits(a.contiguous()), bits(b.contiguous())), name
