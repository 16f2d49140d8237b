"""The bf16 training pass where a workgroup of dq takes several row tiles, one after the other, through one sequence of key tiles (large problems of 128
channels), and forward and backward passes over long sequences of key tiles: against the formulas in 64 bits, with the bounds of test_gpu_cross."""
import pytest
import torch

from test_gpu_cross import BF, _inputs, _reference, _valid, _within

pytestmark = pytest.mark.gpu


def _parts(wgs, units, places=256):
    """cross_bwd.hip's parts of the keys (dq, 128 channels): those with the shortest rounds."""
    cost = {p: -(-wgs * p // places) * (-(-units // p) + (4 if p > 1 else 0)) for p in range(1, min(units, 64) + 1) if p == 1 or wgs * p <= 2048}
    return min(cost, key=lambda p: (cost[p], p))


def _row_tiles_of_a_workgroup(bh, tiles, places=256):
    """Its choice of row tiles to a workgroup of one part: the fewest within 5 % of the shortest rounds over one workgroup a compute unit."""
    cost = lambda c: -(-bh * -(-tiles // c) // places) * (c + 0.5)  # noqa: E731
    most = min(tiles, 32)
    best = min(cost(c) for c in range(1, most + 1))
    return next(c for c in range(1, most + 1) if c == most or cost(c) <= 1.05 * best)


# B, H, Hkv, Sq, Sk, kind, row tiles of a workgroup: one key tile, several with an end inside one, a length of zero among them, a mask that
# leaves an item empty, more keys than the bits of 64 tiles cover; the last workgroup of a head has fewer row tiles, the last row tile fewer rows
CASES = [
    (2, 10, 5, 2330, 50, "all", 2), (2, 10, 5, 2330, 64, "lens", 2), (2, 9, 3, 2500, 201, "lens", 2), (2, 9, 3, 2500, 333, "mask empty", 2),
    (3, 8, 2, 3500, 130, "lens mask", 3), (3, 9, 3, 6000, 2100, "mask", 6), (2, 10, 5, 9490, 100, "mask", 6), (1, 9, 9, 7000, 2300, "lens", 2),
    (1, 9, 9, 7000, 2300, "all", 2), (1, 9, 9, 7000, 2300, "mask", 2), (3, 9, 3, 6700, 2100, "lens mask", 6),
]


def _check(q, k, v, d, lens, mask, ok, D):
    import paper_2605_04569_amd as I
    (out, out_tol), _, grads = _reference(q, k, v, d, ok, D ** -0.5, BF)
    one = [t.detach().requires_grad_(True) for t in (q, k, v)]
    got = I.cross_attention(*one, kv_len=lens, key_mask=mask)
    _within(got, out, out_tol, "out", 2.0 ** -7)
    dq, dk, dv = torch.autograd.grad(got, one, d)
    for name, g, (want, tol) in zip(("dq", "dk", "dv"), (dq, dk, dv), grads):
        _within(g, want, tol, name, 2.0 ** -7)
    dead = ~ok[:, None, :, None].expand_as(k)
    assert not dk[dead].any() and not dv[dead].any()
    assert not dq[~ok.any(dim=1)].any()
    return dq, dk, dv


def _some(kind, B, Sk):
    lens = mask = None
    g = torch.Generator().manual_seed(Sk)
    if "lens" in kind:
        lens = torch.tensor([(Sk * 3) // 4 + 1, 0, Sk][:B], dtype=torch.int32, device="cuda")
    if "mask" in kind:
        mask = torch.rand((B, Sk), generator=g) < 0.7
        if "empty" in kind:
            mask[-1] = False
        mask = mask.cuda()
    return lens, mask, _valid(B, Sk, lens, mask)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)).replace(" ", "_"))
def test_several_row_tiles_a_workgroup(case):
    B, H, Hkv, Sq, Sk, kind, chunk = case
    tiles = -(-H // Hkv * Sq // 128)
    assert _parts(B * Hkv * tiles, -(-Sk // 64)) == 1 and _row_tiles_of_a_workgroup(B * Hkv, tiles) == chunk > 1
    assert torch.cuda.get_device_properties(0).multi_processor_count == 256
    q, k, v, d = _inputs(B, H, Hkv, 128, Sq, Sk, BF, Sk)
    lens, mask, ok = _some(kind, B, Sk)
    first = _check(q, k, v, d, lens, mask, ok, 128)
    import paper_2605_04569_amd as I
    one = [t.detach().requires_grad_(True) for t in (q, k, v)]
    for _ in range(3):                                        # the same bits, whatever else the chip does
        for a, b in zip(torch.autograd.grad(I.cross_attention(*one, kv_len=lens, key_mask=mask), one, d), first):
            assert torch.equal(a, b)


@pytest.mark.parametrize("D,kind", [(64, "mask"), (64, "lens mask"), (64, "all"), (128, "lens")])
def test_long_sequences_of_key_tiles(D, kind):
    """Workgroups that take some thousand keys themselves, and parts of them."""
    B, H, Hkv, Sq, Sk = (3, 6, 3, 4000, 2177) if kind != "lens" else (3, 9, 3, 2000, 4500)
    q, k, v, d = _inputs(B, H, Hkv, D, Sq, Sk, BF, D + 1, layout="heads")
    lens, mask, ok = _some(kind, B, Sk)
    _check(q, k, v, d, lens, mask, ok, D)
