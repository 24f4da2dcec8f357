"""The dequantised weights that the gated block and the backward passes multiply: s (q - z), rounded once to the activation type."""
import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer, check, hidden

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def ones_at(M, K, columns, dtype):
    x = torch.zeros((M, K), dtype=dtype, device="cuda")
    x[torch.arange(M, device="cuda"), columns] = 1.0
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [3, 4])
@pytest.mark.parametrize("M,N,K", [(1, 8, 128), (40, 136, 384), (264, 264, 256), (1000, 1000, 640)])
def test_gradient_of_one_output(M, N, K, bits, dtype):
    """dy with a single one: dx is that row of the weights as it is multiplied, for nothing is added to it and its rounding is the result's."""
    dt = TYPES[dtype]
    layer = Layer(fbq, N, K, bits, 0, dt, seed=M + bits)
    rows = torch.arange(M, device="cuda") * 7 % N
    dx = fbq.linear_backward(ones_at(M, N, rows, dt), None, *layer.tensors, 128, bits, want_factors=False)[0]
    assert torch.equal(dx, layer.W.to(dt)[rows])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [3, 4])
@pytest.mark.parametrize("M,N,save", [(30, 272, False), (30, 272, True), (300, 528, False), (700, 272, True), (600, 20016, False), (1000, 17600, False)])
def test_hidden_activations_of_one_input(M, N, save, bits, dtype):
    """x with a single one: the products are a column of the weights as it is multiplied, exactly."""
    dt, K = TYPES[dtype], 256
    layer = Layer(fbq, N, K, bits, 0, dt, seed=M + N)
    columns = torch.arange(M, device="cuda") * 5 % K
    got = fbq.gated(ones_at(M, K, columns, dt), *layer.tensors, N, 128, bits, save=save)
    p = layer.W.to(dt).double().t()[columns]
    h, size = hidden("silu", p, torch.zeros_like(p), dt)
    check(got[0] if save else got, h, size, "h")
