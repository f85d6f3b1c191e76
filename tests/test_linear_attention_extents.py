"""Linear attention's checks of extents at the ends of their types, on addresses that are never used."""
import pytest

from paper_2310_05218_amd import binding as B

FAR = 1 << 45


@pytest.fixture(scope="module")
def L():
    import os

    if not os.path.exists(B.LIB_PATH):
        from paper_2310_05218_amd import build
        build.build()
    return B.lib()


def strides(tokens, heads, width):
    return B.SwStrides(tokens * heads * width, heads * width, width)


@pytest.mark.parametrize("n_states", [100, (1 << 30) - 1, (1 << 31) - 1])
def test_as_many_states_as_an_int_counts(L, n_states):
    """Two entries of 64 x 64 each: fewer than 2^46 elements, so that what stops the call is the output, which lies among the states."""
    d = B.SwLinearAttentionDims(10, 1, 2, 2, 64, 64, n_states, B.SW_F32, 0.125)
    s = strides(10, 2, 64)
    call = lambda o: L.sw_linear_attention(FAR, FAR + 0x10000, FAR + 0x20000, o, FAR + 0x30000, 1 << 30, None, None, None, d, s, s, s, s, None, 0, None)
    back = lambda o: L.sw_linear_attention_backward(FAR, FAR + 0x10000, FAR + 0x20000, FAR + 0x30000, FAR + 0x40000, 1 << 30, None, o, FAR + 0x50000, FAR + 0x60000, None, None, None, d,
                                                    s, s, s, s, s, s, s, None, 0, None)
    inside = (1 << 30) + n_states * 2 * 64 * 64 * 4 - 0x10000
    assert call(inside) == back(inside) == B.SW_ERR_ALIAS
