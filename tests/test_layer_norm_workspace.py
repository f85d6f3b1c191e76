"""Scratch memory of layer norm's backward pass: as many rows of sums as a launch writes, which is fewer for longer rows."""
import pytest

torch = pytest.importorskip("torch")            # (before the library is opened, which then has torch's runtime)

from paper_2310_05218_amd import binding as B  # noqa: E402


@pytest.fixture(scope="module")
def L():
    import os

    if not os.path.exists(B.LIB_PATH):
        from paper_2310_05218_amd import build
        build.build()
    return B.lib()


@pytest.mark.parametrize("rows,C,most", [(1, 64, 1), (3, 100, 3), (100000, 64, 1024), (100000, 4096, 512), (100000, 16384, 256), (100000, 16385, 64), (100000, 65536, 64), (7, 65536, 7),
                                         (1 << 40, 1 << 20, 64)])
def test_bytes(L, rows, C, most):
    """`most` rows of 2 C sums in fp32; rows of 16384 are the longest that registers hold (of 16-bit values)."""
    assert 0 < L.sw_layer_norm_backward_workspace_bytes(rows, C) <= (most * 2 * C * 4 + 15) // 16 * 16


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,C", [(1, 1), (5, 7), (3000, 5), (4100, 33), (2000, 64), (1500, 100), (1030, 255), (700, 999), (600, 1024), (600, 2048), (600, 4096), (300, 8192), (300, 8193),
                                    (300, 16384), (100, 16385), (70, 65536)])
def test_no_row_beyond(L, rows, C, t):
    dtype = getattr(torch, t)
    r = torch.Generator(device="cuda").manual_seed(C)
    x, dy = (torch.randn(rows, C, generator=r, device="cuda").to(dtype) for _ in range(2))
    mean, rstd = x.float().mean(1), x.float().var(1, unbiased=False).add_(1e-5).rsqrt_()
    need, guard = L.sw_layer_norm_backward_workspace_bytes(rows, C), 1 << 22
    work = torch.full((need // 4 + guard,), float("nan"), device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    kind = {"float32": B.SW_F32, "bfloat16": B.SW_BF16, "float16": B.SW_F16}[t]
    rc = L.sw_layer_norm_backward(dy.data_ptr(), x.data_ptr(), None, mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), rows, C, C, C, C, kind,
                                  work.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert rc == B.SW_OK
    assert work[need // 4:].isnan().all() and dw.isfinite().all() and db.isfinite().all()
    want = dy.double().sum(0)
    assert torch.all((db.double() - want).abs() <= 512 * 2.0 ** -24 * dy.double().abs().sum(0))
