"""The norm where a call's tensors are 256 MB or more together and go past the caches: every form with the residual at sizes where each of them does, and
the forms without it."""
import pytest
import torch

import test_gpu_norm as N

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rows,C,dtype,group", [(7501, 5120, BF, 128), (18803, 2048, BF, 0), (162_001, 128, FP, 128), (10_101, 2056, FP, 0)],
                         ids=["bf16_5120", "bf16_2048", "f32_128", "f32_2056"])
def test_with_the_residual(rows, C, dtype, group):
    size = 2 if dtype == BF else 4
    assert rows * C * (3 * size + 1) >= 256 << 20             # x, the residual, the sum and 8 bits: the least of the forms
    N.test_tensors_that_are_streamed(rows, C, dtype, group)


@pytest.mark.parametrize("rows,C,dtype,wtype", [(17_503, 5120, BF, BF), (44_003, 2048, BF, FP), (420_001, 128, FP, FP), (26_113, 2056, FP, BF)],
                         ids=["bf16_5120", "bf16_2048", "f32_128", "f32_2056"])
def test_without_the_residual(rows, C, dtype, wtype):
    import paper_2605_04569_amd as I
    assert rows * C * ((2 if dtype == BF else 4) + 1) >= 256 << 20
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, dy = (torch.randn((rows, C), generator=g, device="cuda").to(dtype) for _ in "xd")
    w = (1.0 + 0.3 * torch.randn(C, generator=g, device="cuda")).to(wtype)
    half = N.HALF[dtype]

    def within(got, want, tol, what):
        off = (got.double() - want).abs() - tol
        assert not torch.isnan(off).any() and float(off.max()) <= 0, (what, float(off.max()), int(off.argmax()))

    h = x.double()
    y = h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + 1e-6) * w.double()
    within(I.residual_rms_norm(x, w), y, y.abs() * (half + N.F32), "y")
    y8, s = I.residual_rms_norm_8bit(x, w)
    top = y.abs().amax(dim=1, keepdim=True) / 448.0
    within(s, top, top * N.F32, "scale")
    within(y8.double() * s.double(), y, y.abs() * (N.HALF[torch.float8_e4m3fn] + N.F32) + s.double() * 2.0 ** -10, "y8")
    rstd = (1.0 / torch.sqrt((h * h).mean(dim=1) + 1e-6)).float()
    n, u = h * rstd.double()[:, None], dy.double() * w.double()
    dx = I.isa_rms_norm_backward(x, None, w, rstd, dy, torch.empty_like(x))[0]
    dot = (u * n).mean(dim=1, keepdim=True)
    want = rstd.double()[:, None] * (u - n * dot)
    size = rstd.double()[:, None] * (u.abs() + n.abs() * (u * n).abs().mean(dim=1, keepdim=True))
    within(dx, want, size * N.F32 * (1 + half) + want.abs() * half, "dx")
