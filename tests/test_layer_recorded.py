"""Calls that torch records or differentiates without requires_grad: a trace of cross attention and the norm has to hold the call, and
forward-mode derivatives are refused instead of being lost.  No GPU: the library's calls are replaced by copies between raw addresses, which
torch sees as little as the library's kernels."""
import ctypes

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

import paper_2605_04569_amd as I
from paper_2605_04569_amd import binding as B


def _copy(to, of):
    assert to.is_contiguous() and of.is_contiguous() and to.numel() * to.element_size() <= of.numel() * of.element_size()
    ctypes.memmove(to.data_ptr(), of.data_ptr(), to.numel() * to.element_size())


@pytest.fixture(autouse=True)
def stand_ins(monkeypatch):
    def cross(q, k, v, out, kv_len=None, key_mask=None, scale=None, lse=None, workspace=None):
        assert type(scale) is float
        _copy(out, q)
        if lse is not None:
            lse.zero_()
        return out

    def norm(x, weight, y, residual=None, h=None, rstd=None, eps=1e-6):
        _copy(y, x)
        if h is not None:
            _copy(h, residual)
        return y

    def eight(x, weight, y8, scales, residual=None, h=None, eps=1e-6, group=0):
        _copy(y8, x)
        _copy(scales, x)
        if h is not None:
            _copy(h, residual)
        return y8, scales

    monkeypatch.setattr(B, "isa_cross_attention", cross)
    monkeypatch.setattr(B, "isa_rms_norm", norm)
    monkeypatch.setattr(B, "isa_rms_norm_8bit", eight)


def _tensors(seed, n):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((1, 2, 5, 64), generator=g) for _ in range(n)]


def _tuple(x):
    return x if isinstance(x, tuple) else (x,)


CALLS = [
    ("cross", 3, lambda q, k, v: I.cross_attention(q, k, v)),
    ("cross module", 3, lambda q, k, v: I.CrossAttention(0.25)(q, k, v)),
    ("norm", 1, lambda x: I.residual_rms_norm(x)),
    ("norm residual", 2, lambda x, r: I.residual_rms_norm(x, torch.ones(64), r)),
    ("norm 8 bits", 2, lambda x, r: I.residual_rms_norm_8bit(x, torch.ones(64), r)),
]


@pytest.mark.filterwarnings("ignore")
@pytest.mark.parametrize("name,n,call", CALLS, ids=[c[0] for c in CALLS])
@pytest.mark.parametrize("grad", [False, True])
def test_a_trace_holds_the_call(name, n, call, grad):
    with torch.set_grad_enabled(grad):
        traced = torch.jit.trace(call, tuple(_tensors(0, n)), check_trace=False)
        for seed in (1, 2):
            new = _tensors(seed, n)
            junk = [torch.full_like(t, 7.0) for t in new]     # memory that is given back, for outputs that nothing would write
            del junk
            got, want = _tuple(traced(*new)), _tuple(call(*new))
            assert len(got) == len(want)
            for a, b in zip(got, want):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), name


@pytest.mark.parametrize("name,n,call", CALLS, ids=[c[0] for c in CALLS])
def test_forward_mode_is_refused(name, n, call):
    ts = _tensors(3, n)
    with forward_ad.dual_level():
        for i in range(n):
            dual = [forward_ad.make_dual(t, torch.ones_like(t)) if j == i else t for j, t in enumerate(ts)]
            with pytest.raises(NotImplementedError):
                call(*dual)
        call(*ts)                                             # nothing is carried along: an ordinary call
    call(*ts)


def test_ordinary_calls_take_the_short_way(monkeypatch):
    """Without gradients, a trace or a forward-mode level no autograd function is entered."""
    from paper_2605_04569_amd import cross, norm
    for cls in (cross._CrossAttentionFunction, norm._ResidualRMSNormFunction, norm._ResidualRMSNorm8Function):
        monkeypatch.setattr(cls, "apply", None)
    for _, n, call in CALLS:
        call(*_tensors(4, n))
    with torch.no_grad():
        I.residual_rms_norm(_tensors(4, 1)[0].requires_grad_(True))
