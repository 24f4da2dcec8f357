"""Where the domain of the backward passes ends: the last sizes that the header names are taken, the next ones are not."""
import ctypes

import pytest
import torch

import paper_2501_16385_b200 as fbq

UNSUPPORTED, CUDA = -2, -4
P = [ctypes.c_void_p((i + 1) << 20) for i in range(16)]         # addresses that are never read: there is no device
LAST = 1 << 21


def linear_backward(M, N, K=128, rank=16):
    return fbq.lib().fbq_linear_backward(P[0], P[1], None, None, *P[2:7], *P[7:10], M, N, K, 128, 4, rank, 0, None)


def gated_backward(M, N, K=128, rank=16):
    return fbq.lib().fbq_gated_backward(P[0], P[1], P[2], P[3], None, None, *P[4:9], *P[9:12], M, N, K, 128, 4, rank, 0, 0, None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="with a device these would run on addresses that are none")
@pytest.mark.parametrize("M", [1, 768, 769, 1 << 22])
def test_taken(M):
    for N in ((1 << 20) - 16, 1 << 20, (1 << 20) + 16, LAST):
        assert linear_backward(M, N) == CUDA and gated_backward(M, N) == CUDA
    assert linear_backward(M, (1 << 20) + 8) == CUDA and linear_backward(M, 8, K=1 << 30) == CUDA


@pytest.mark.parametrize("M", [1, 768, 769])
def test_refused(M):
    assert linear_backward(M, LAST + 8) == UNSUPPORTED and gated_backward(M, LAST + 16) == UNSUPPORTED
    assert linear_backward(M, 8, K=(1 << 30) + 128) == UNSUPPORTED and linear_backward((1 << 22) + 1, 8) == UNSUPPORTED
