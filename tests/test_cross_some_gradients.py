"""Training calls of cross attention where not every input wants a gradient (cached or frozen states): the launch for dk and dv is left out where neither
is wanted, and the gradients that are wanted are those of the full call, bit for bit."""
import ctypes as C
import itertools

import pytest
import torch

import paper_2605_04569_amd as I
from paper_2605_04569_amd import binding as B


def test_the_backward_call_is_asked_for_what_is_wanted(monkeypatch):
    asked = []

    def forward(q, k, v, out, kv_len=None, key_mask=None, scale=None, lse=None, workspace=None):
        return out.zero_()

    def backward(q, k, v, out, lse, d_out, dq, dk, dv, kv_len=None, key_mask=None, scale=None, workspace=None):
        asked.append((dk is not None, dv is not None))
        for t in (dq, dk, dv):
            if t is not None:
                t.zero_()

    monkeypatch.setattr(B, "isa_cross_attention", forward)
    monkeypatch.setattr(B, "isa_cross_attention_backward", backward)
    for want in itertools.product((False, True), repeat=3):
        if not any(want):
            continue
        ts = [torch.randn(1, 2, n, 64, requires_grad=w) for n, w in zip((3, 5, 5), want)]
        I.cross_attention(*ts).sum().backward()
        assert asked.pop() == (want[1] or want[2],) * 2
        assert [t.grad is not None for t in ts] == list(want)


def test_states_alone_may_be_left_out():
    S = B._CStrides
    # strides of gradients that are not asked for are not looked at
    p = B._CCross(2, 4, 2, 64, 10, 20, 0, 0.125, *[S(*s) for s in ((2560, 640, 64), (0, 0, 64), (0, 0, 64), (2560, 640, 64), (2560, 640, 64), (2560, 640, 64),
                                                                 (0, 0, 64), (0, 0, 64))])
    a = [C.c_void_p(4096 * (i + 1)) for i in range(9)]
    call = lambda dq, dk, dv, n: I.lib().isa_cross_attention_backward(  # noqa: E731
        C.byref(p), a[0], a[1], a[2], None, None, 0, a[3], a[4], a[5], dq, dk, dv, a[8], n, None)
    assert call(a[6], None, None, 0) == -6                    # everything but the workspace is accepted
    assert call(None, None, None, 0) == -1
    assert call(a[6], a[7], None, 0) == -2 and call(a[6], None, a[7], 0) == -2
    p.dk = p.dv = S(2560, 1280, 64)
    assert call(a[6], a[7], None, 0) == -1 and call(a[6], None, a[7], 0) == -1
    q, k = torch.zeros(1, 2, 5, 64), torch.zeros(1, 2, 7, 64)
    with pytest.raises(ValueError, match="together"):
        I.isa_cross_attention_backward(q, k, k, q, q[..., 0], q, q.clone(), k.clone(), None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 4, 2, 128, 70, 90), (1, 2, 1, 64, 1, 700), (2, 4, 2, 64, 600, 130), (1, 2, 2, 128, 2000, 0), (1, 2, 2, 128, 0, 9)],
                         ids=lambda s: "x".join(map(str, s)))
def test_every_subset_has_the_bits_of_the_whole(shape, dtype):
    B_, H, Hkv, D, Sq, Sk = shape
    g = torch.Generator(device="cuda").manual_seed(Sk)
    q, d = (torch.randn((B_, H, Sq, D), generator=g, device="cuda").to(dtype) for _ in "qd")
    k, v = (torch.randn((1, Hkv, Sk, D), generator=g, device="cuda").to(dtype).expand(B_, Hkv, Sk, D) for _ in "kv")      # shared by the batch
    lens = torch.full((B_,), max(Sk - 3, 0), dtype=torch.int32, device="cuda")

    def run(want):
        ts = [t.detach().requires_grad_(w) for t, w in zip((q, k, v), want)]
        out = I.cross_attention(*ts, kv_len=lens)
        return dict(zip([i for i in range(3) if want[i]], torch.autograd.grad(out, [t for t in ts if t.requires_grad], d)))

    whole = run((True,) * 3)
    for want in itertools.product((False, True), repeat=3):
        if any(want):
            for i, t in run(want).items():
                assert torch.equal(t, whole[i]), (want, i)
