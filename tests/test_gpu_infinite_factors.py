"""Infinite activations and gradients where the rank is no whole block of the tensor-core kernels: t and s of the missing entries are zero, not
0 times infinity, so results are infinite or NaN exactly where the sum of products is."""
import math

import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer, branches

pytestmark = pytest.mark.gpu


def normal(M, K, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((M, K), generator=g, device="cuda") * scale).to(dtype)


def layer_of(N, K, rank, dtype):
    """All of A and B is positive: an infinite t or s adds an infinity of one sign."""
    layer = Layer(fbq, N, K, 4, rank, dtype, seed=3)
    layer.A, layer.B = layer.A.abs() + 0.01, layer.B.abs() + 0.01
    return layer


def infinite(w):
    """inf * w + inf for a column or row w of the weights."""
    return torch.where(w > 0, math.inf, math.nan)


def same(got, want):
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.double().nan_to_num(nan=0.0, posinf=1.0, neginf=-1.0),
                                                                            want.double().nan_to_num(nan=0.0, posinf=1.0, neginf=-1.0))


@pytest.mark.parametrize("M,N,K", [(40, 136, 256), (700, 264, 384), (900, 264, 384), (1500, 520, 256)])
@pytest.mark.parametrize("rank,dtype", [(8, torch.float16), (72, torch.bfloat16), (128, torch.float16)])
def test_gradient(M, N, K, rank, dtype):
    layer = layer_of(N, K, rank, dtype)
    dy, x = normal(M, N, dtype, 1, 0.1), normal(M, K, dtype, 2)
    clean = fbq.linear_backward(dy, x, *layer.tensors, 128, 4)[0]
    dy[1, 5] = math.inf
    dx = fbq.linear_backward(dy, x, *layer.tensors, 128, 4)[0]
    assert fbq.poll_status() == 0
    others = [m for m in range(M) if m != 1]
    assert torch.equal(dx[others], clean[others])
    assert same(dx[1], infinite(layer.W[5]))


@pytest.mark.parametrize("M", [5, 40, 200, 513])
@pytest.mark.parametrize("rank,dtype", [(16, torch.float16), (80, torch.bfloat16), (128, torch.float16)])
@pytest.mark.parametrize("save", [False, True])
def test_gated(M, rank, dtype, save):
    N, K = 272, 384
    layer = layer_of(N, K, rank, dtype)
    x = normal(M, K, dtype, 2)
    clean = fbq.gated(x, *layer.tensors, N, 128, 4, save=save)
    x[1, 5] = math.inf
    got = fbq.gated(x, *layer.tensors, N, 128, 4, save=save)
    assert fbq.poll_status() == 0
    others = [m for m in range(M) if m != 1]
    gate, up = branches(infinite(layer.W[:, 5])[None, :])
    want = (gate * up)[0]                                       # f(inf) = inf
    h, first = (got[0], clean[0]) if save else (got, clean)
    assert torch.equal(h[others], first[others]) and same(h[1], want)
    if save:
        assert bool(torch.isnan(got[2][1]).all()) and all(torch.equal(a[others], b[others]) for a, b in zip(got[1:], clean[1:]))


@pytest.mark.parametrize("M", [17, 100, 200, 700])
@pytest.mark.parametrize("rank,dtype", [(8, torch.float16), (72, torch.bfloat16), (128, torch.float16)])
def test_prompt(M, rank, dtype):
    N, K = 264, 384
    layer = layer_of(N, K, rank, dtype)
    x = normal(M, K, dtype, 2)
    clean = fbq.linear(x, *layer.tensors, N, 128, 4)
    x[1, 5] = math.inf
    y = fbq.linear(x, *layer.tensors, N, 128, 4)
    assert fbq.poll_status() == 0
    others = [m for m in range(M) if m != 1]
    assert torch.equal(y[others], clean[others]) and same(y[1], infinite(layer.W[:, 5]))
