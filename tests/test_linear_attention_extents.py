"""Linear attention's checks of extents at the ends of their types, and of gradients in one place, on addresses that are never used."""
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


@pytest.mark.parametrize("T,n,heads,packed", [(1 << 46, 1, 65535, 0), (1 << 46, 1, 65535, 1), (1 << 30, 100, 65535, 0), (1 << 44, 1, 1024, 0)])
def test_workspaces_of_rows_beyond_any_tensor(L, T, n, heads, packed):
    """Bytes that 64 bits do not count: 0, as for all invalid extents."""
    d = B.SwLinearAttentionDims(T, n, heads, 1, 256, 256, 0, B.SW_BF16, 1.0)
    assert L.sw_linear_attention_backward_workspace_bytes(d, packed) == L.sw_linear_attention_workspace_bytes(d, packed) == 0


@pytest.mark.parametrize("T,n,heads,packed", [(1 << 24, 1 << 14, 64, 1), (8192, 32, 64, 0)])
def test_workspaces_of_ordinary_rows(L, T, n, heads, packed):
    """Packed rows count once, whatever the number of sequences."""
    d = B.SwLinearAttentionDims(T, n, heads, 8, 128, 128, 0, B.SW_BF16, 1.0)
    rows = T if packed else T * n
    assert L.sw_linear_attention_backward_workspace_bytes(d, packed) >= 2 * rows * heads * 128 * 4


@pytest.mark.parametrize("same", ["qk", "qv", "kv"])
def test_gradients_in_one_place(L, same):
    d = B.SwLinearAttentionDims(10, 2, 4, 4, 16, 16, 0, B.SW_F32, 0.25)
    s = strides(10, 4, 16)
    at = {n: FAR + i * 0x100000 for i, n in enumerate("qkv")}
    at[same[1]] = at[same[0]]
    call = lambda g: L.sw_linear_attention_backward(1 << 40, (1 << 40) + 0x10000, (1 << 40) + 0x20000, (1 << 40) + 0x30000, 1 << 39, None, None, g["q"], g["k"], g["v"], None, None, None, d,
                                                    s, s, s, s, s, s, s, None, 0, None)
    assert call(at) == B.SW_ERR_ALIAS
