"""Cross attention where all scores of a row lie far from zero, on either side: a row with valid keys is never taken for one without.

All valid keys are alike, so that all weights are and the output is the mean of the valid values.  The scores are sums of equal products in fp32, the
same for every key: the weights differ by nothing, and their common factor cancels.  Bounds, with A the mean of |v|: S_k + 8 additions and divisions in
fp32 (2^-24 each) of A, and the output's rounding (bf16 2^-8, fp32 2^-24).  The log-sum-exp is the score and the logarithm of the number of keys: the
score's D products and additions and the conversions to base 2 and back, 2^-24 each of its size, and 2^-8 for bf16 weights, whose sum is of rounded
exponents past 2^15."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
SHAPES = [(2, 4, 2, 128, 1, 77), (2, 2, 1, 64, 3, 3000), (2, 2, 2, 128, 100, 90), (2, 2, 2, 64, 70, 3000), (2, 2, 1, 128, 40, 5000)]


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("kind", ["all", "mask"])
def test_rows_of_far_scores(shape, dtype, kind):
    import paper_2605_04569_amd as I
    B, H, Hkv, D, Sq, Sk = shape
    g = torch.Generator(device="cuda").manual_seed(Sk)
    v = torch.randn((B, Hkv, Sk, D), generator=g, device="cuda").to(dtype)
    ok = torch.ones((B, Sk), dtype=torch.bool, device="cuda")
    if kind == "mask":
        ok = torch.rand((B, Sk), generator=g, device="cuda") < 0.5
        ok[0, :Sk // 2], ok[0, -1] = False, True
        ok[1] = False                                          # an item without keys
    mask = ok if kind == "mask" else None
    count = ok.sum(dim=1).clamp_min(1).double()[:, None, None, None]
    vx = torch.where(ok[:, None, :, None], v, torch.zeros_like(v)).double().repeat_interleave(H // Hkv, dim=1)
    mean, size = vx.sum(dim=2, keepdim=True) / count, vx.abs().sum(dim=2, keepdim=True) / count
    half = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    for sign in (1.0, -1.0):
        for power in (0, 10, 20, 26, 29, 33, 40, 80, 99, 100, 105, 120):
            # scale q . k = sign 2^power
            a = 2.0 ** (power // 2)
            q = torch.full((B, H, Sq, D), sign * a, device="cuda").to(dtype)
            k = torch.full((B, Hkv, Sk, D), 2.0 ** power / a, device="cuda").to(dtype)
            out, lse = torch.empty_like(q), torch.empty((B, H, Sq), device="cuda")
            I.isa_cross_attention(q, k, v, out, key_mask=mask, scale=1.0 / D, lse=lse)
            assert torch.equal(I.cross_attention(q, k, v, key_mask=mask, scale=1.0 / D).nan_to_num(nan=7.0), out.nan_to_num(nan=7.0))
            nan = torch.isnan(out)
            if kind == "mask":
                assert not out[1].any() and not nan[1].any() and (lse[1] == -math.inf).all(), (sign, power)
            if dtype == FP or power <= 29:
                assert not nan.any(), (sign, power)
            off = (out.double() - mean).abs() - ((Sk + 8) * 2.0 ** -24 * size + half * (mean.abs() + Sk * 2.0 ** -24 * size))
            assert (nan | (off <= 0)).all(), (sign, power, float(off[~nan].max()))
            assert (nan.all(dim=3) == nan.any(dim=3)).all() and torch.equal(torch.isnan(lse), nan.any(dim=3)), (sign, power)
            want = sign * 2.0 ** power + torch.log(count[:, :, :, 0])
            want = want.expand(B, H, Sq)
            tol = (D + 16) * 2.0 ** -24 * 2.0 ** power + 2.0 ** -8 + (Sk + 8) * 2.0 ** -24
            live = ~nan.any(dim=3) & ok.any(dim=1)[:, None, None]
            assert ((lse.double() - want).abs()[live] <= tol).all(), (sign, power)
