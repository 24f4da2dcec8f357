"""Activations in 8 bits: codes and scales equal the definition's, bit for bit, and what they stand for."""
import math

import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import check, half_step, kept64, least, to_8_bits

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]


def values(M, K, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((M, K), generator=g, device="cuda") * torch.exp(3 * torch.randn((M, 1), generator=g, device="cuda"))).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", [(1, 1), (1, 7), (3, 8), (1, 127), (5, 128), (2, 129), (17, 136), (4, 250), (33, 264), (1, 4096), (300, 1000), (1025, 1288), (7, 11008)])
def test_codes_scales_and_back(M, K, dtype):
    x = values(M, K, dtype, seed=M * K)
    codes, scales = fbq.act8_pack(x)
    want, want_scales = to_8_bits(x)
    assert torch.equal(scales, want_scales) and torch.equal(codes, want)
    back = fbq.act8_unpack(codes, scales, dtype)
    exact = kept64(codes, scales)
    # code * scale: one rounding in single precision, one to the type
    check(back, exact, exact.abs() * (half_step(dtype) + 2.0**-23) + least(dtype), "x")
    step = scales.double().repeat_interleave(128, 1)[:, :K]
    check(back, x.double(), step * (0.5 + 128 * 2.0**-22) + exact.abs() * half_step(dtype) + least(dtype), "x")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [256, 250])
def test_groups_of_zeros_ties_and_what_is_not_finite(K, dtype):
    x = values(6, K, dtype, seed=1)
    x[0] = 0
    x[1, :128] = 0
    x[2, 3] = math.inf
    x[3, 130] = math.nan
    x[4, 128:] = -0.0
    x[5, :128] = torch.arange(128, device="cuda").to(dtype) / 2         # 63.5 is 127 steps: every odd number is between two codes
    codes, scales = fbq.act8_pack(x)
    want, want_scales = to_8_bits(x)
    assert torch.equal(codes, want)
    assert torch.equal(scales.nan_to_num(-1.0), want_scales.nan_to_num(-1.0))
    assert bool(torch.isnan(scales[2, 0])) and bool(torch.isnan(scales[3, 1])) and int(torch.isnan(scales).sum()) == 2
    back = fbq.act8_unpack(codes, scales, dtype)
    assert bool(torch.isnan(back[2, :128]).all()) and bool(torch.isnan(back[3, 128:]).all()) and int(torch.isnan(back).sum()) == 128 + K - 128
    assert not bool(back[0].any()) and not bool(back[1, :128].any()) and not bool(back[4, 128:].any())


def test_smallest_and_largest_values():
    for dtype in TYPES:
        x = torch.zeros((2, 256), dtype=dtype, device="cuda")
        x[0, 0] = torch.finfo(dtype).smallest_normal
        x[0, 128] = torch.finfo(dtype).max
        x[1, 5] = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
        codes, scales = fbq.act8_pack(x)
        want, want_scales = to_8_bits(x)
        assert torch.equal(codes, want) and torch.equal(scales, want_scales)
        back = fbq.act8_unpack(codes, scales, dtype)
        assert bool(torch.isfinite(back).all())
        if dtype == torch.float16:                              # (bf16's smallest are below what is kept)
            assert back[0, 0] == x[0, 0] and back[1, 5] == x[1, 5]


def test_more_than_31_bits_of_elements():
    M, K = 262200, 8200                                         # 2.15e9
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
    x.view(-1)[:] = 1.0
    last = values(2, K, torch.bfloat16, seed=5)
    x[-2:] = last
    codes, scales = fbq.act8_pack(x)
    want, want_scales = to_8_bits(last)
    assert torch.equal(codes[-2:], want) and torch.equal(scales[-2:], want_scales)
    back = fbq.act8_unpack(codes, scales, torch.bfloat16)
    assert torch.equal(back[-2:], (want.float() * want_scales.repeat_interleave(128, 1)[:, :K]).to(torch.bfloat16))
    assert bool((back[M // 2] == 1).all())


def test_more_than_31_bits_of_single_elements():
    M, K = 70001, 30701                                         # 2.149e9, rows of no whole pieces
    codes = torch.zeros((M, K), dtype=torch.int8, device="cuda")
    scales = torch.ones((M, 240), dtype=torch.float32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(6)
    codes[-2:] = torch.randint(-127, 128, (2, K), generator=g, device="cuda").to(torch.int8)
    back = fbq.act8_unpack(codes, scales, torch.bfloat16)
    assert torch.equal(back[-2:], codes[-2:].to(torch.bfloat16)) and not bool(back[M // 2].any())
    again, _ = fbq.act8_pack(back)
    want, _ = to_8_bits(back[-2:])
    assert torch.equal(again[-2:], want)


def test_no_rows_and_views():
    codes, scales = fbq.act8_pack(torch.empty((0, 40), dtype=torch.float16, device="cuda"))
    assert codes.shape == (0, 40) and scales.shape == (0, 1) and fbq.act8_unpack(codes, scales, torch.float16).shape == (0, 40)
    x = values(4, 64, torch.float16, seed=2)
    with pytest.raises(ValueError):
        fbq.act8_pack(x[:, ::2])
    with pytest.raises(TypeError):
        fbq.act8_pack(x.float())
    with pytest.raises(fbq.FbqError):
        fbq.act8_pack(torch.empty(4 * 64 + 1, dtype=torch.float16, device="cuda")[1:].view(4, 64))     # two bytes past an aligned address
