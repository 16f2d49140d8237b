"""Which tensors of lengths cross_attention takes, and that each means what it holds."""
import pytest
import torch

import paper_2605_04569_amd as I


@pytest.mark.parametrize("dtype", [torch.bool, torch.complex64, torch.float32, torch.float64, torch.bfloat16, torch.uint64], ids=str)
def test_lengths_that_are_no_whole_numbers_are_refused(dtype):
    q, k = torch.zeros(2, 4, 5, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 7, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="whole numbers"):
        I.cross_attention(q, k, k, kv_len=torch.zeros(2, dtype=dtype))


@pytest.mark.parametrize("dtype", [torch.int8, torch.uint8, torch.int16, torch.uint16, torch.int32, torch.uint32, torch.int64], ids=str)
def test_lengths_on_the_host_are_refused_for_their_place(dtype):
    q, k = torch.zeros(2, 4, 5, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 7, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the GPU"):
        I.cross_attention(q, k, k, kv_len=torch.zeros(2, dtype=dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.int8, torch.uint8, torch.int16, torch.uint16, torch.int32, torch.uint32, torch.int64], ids=str)
def test_lengths_of_every_type(dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn((4, 2, n, 64), generator=g, device="cuda").bfloat16() for n in (5, 90))
    top = 1 << 60 if dtype == torch.int64 else torch.iinfo(dtype).max
    lens = torch.tensor([7, 90, 0, top], dtype=torch.int64)
    want = I.cross_attention(q, k, k, kv_len=lens.clamp(0, 90).int().cuda())
    assert torch.equal(I.cross_attention(q, k, k, kv_len=lens.to(dtype).cuda()), want)
