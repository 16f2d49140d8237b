"""Infinities and NaN in gradients and queries: what cross attention promises to be zero (gradients of keys and values that are not valid, everything
of queries without a valid key) is zero whatever they meet, and rows and batch items that have none keep their bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
SHAPES = [  # B, H, Hkv, D, Sq, Sk: one part and several, one row tile and several, an end inside a tile
    (3, 4, 2, 128, 70, 90), (3, 2, 1, 64, 33, 300), (3, 2, 2, 128, 1, 700), (3, 4, 4, 64, 600, 130), (3, 10, 2, 128, 900, 200), (3, 64, 8, 64, 520, 70),
]


def _masks(kind, Sk):
    """The first batch item has keys, the second none, the third all or some."""
    lens = mask = None
    if "lens" in kind:
        lens = torch.tensor([Sk * 2 // 3 + 1, 0, Sk], dtype=torch.int32, device="cuda")
    if "mask" in kind:
        g = torch.Generator().manual_seed(5)
        mask = torch.rand((3, Sk), generator=g) < 0.6
        mask[0, 0], mask[1], mask[2, 0] = True, False, True
        mask = mask.cuda()
    ok = torch.ones((3, Sk), dtype=torch.bool, device="cuda")
    if lens is not None:
        ok &= torch.arange(Sk, device="cuda")[None] < lens[:, None]
    if mask is not None:
        ok &= mask
    return lens, mask, ok


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("kind", ["lens", "mask", "lens mask"])
def test_zeros_stay_zeros(shape, dtype, kind):
    import paper_2605_04569_amd as I
    B, H, Hkv, D, Sq, Sk = shape
    g = torch.Generator(device="cuda").manual_seed(Sk)
    q, d = (torch.randn((B, H, Sq, D), generator=g, device="cuda").to(dtype) for _ in "qd")
    k, v = (torch.randn((B, Hkv, Sk, D), generator=g, device="cuda").to(dtype) for _ in "kv")
    lens, mask, ok = _masks(kind, Sk)
    dead = ~ok[:, None, :, None].expand_as(k)
    none = ~ok.any(dim=1)

    def run(q, d):
        one = [t.detach().clone().requires_grad_(True) for t in (q, k, v)]
        out = I.cross_attention(*one, kv_len=lens, key_mask=mask)
        return [out.detach(), *torch.autograd.grad(out, one, d)]

    clean = run(q, d)
    rows = torch.zeros((B, H, Sq, 1), dtype=torch.bool, device="cuda")
    rows[0, 0, Sq // 2] = rows[0, 0, 0] = True                # of an item with keys: its other rows and the items beside it keep their bits
    rows[1] = True                                            # of the item without any: all rows
    for which in ("d_out", "q"):
        for bad in (float("inf"), float("-inf"), float("nan")):
            worse = torch.where(rows, torch.full_like(q, bad), q if which == "q" else d)
            out, dq, dk, dv = run(worse, d) if which == "q" else run(q, worse)
            assert not dk[dead].any() and not dv[dead].any(), (which, bad)
            assert not out[none].any() and not dq[none].any(), (which, bad)
            assert torch.equal(out.masked_fill(rows, 0), clean[0].masked_fill(rows, 0)), (which, bad)
            assert torch.equal(dq.masked_fill(rows, 0), clean[1].masked_fill(rows, 0)), (which, bad)
            assert torch.equal(dk[2], clean[2][2]) and torch.equal(dv[2], clean[3][2]), (which, bad)
            # and it is not hidden where it belongs: a row with keys has no gradient, nor have the keys that it looks at
            assert not torch.isfinite(dq[0, 0, Sq // 2]).all()
            assert not torch.isfinite(dk[0, 0][ok[0]]).all() and not torch.isfinite(dv[0, 0][ok[0]]).all()
