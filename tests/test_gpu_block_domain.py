"""The feed-forward block's calls at the far ends of what the header says they take: contractions beyond what a 16-bit copy of the weights has
room for."""
import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer, check, gate_gradients, hidden, kept64, layer_gradients, own_half, to_8_bits

pytestmark = pytest.mark.gpu


def normal(M, K, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((M, K), generator=g, device="cuda") * scale).to(dtype)


def close(got, want):
    """The bounds of every entry, and, as those of sums this long are wide, the whole: operands rounded once to 16 bits (2^-8 / sqrt(3) each at
    most: dp or dy, W, s or t, the result) whose errors add as in a norm."""
    for g, (w, size), what in zip(got, want, ("dx", "dA", "dB")):
        check(g, w, size, what)
        assert float((g.double() - w).norm() / w.norm()) < 2 * 2.0**-8 / 3**0.5, what


@pytest.mark.parametrize("M,rank", [(513, 16), (901, 0)])
def test_products_kept_of_a_deep_layer(M, rank):
    N, K, dt = 16, (1 << 20) + 128, torch.bfloat16
    layer = Layer(fbq, N, K, 4, rank, dt, seed=1, gated=True)
    x = normal(M, K, dt, 2, 2.0**-7)
    h, codes, scales = fbq.gated(x, *layer.tensors, N, 128, 4, save=True)
    assert fbq.poll_status() == 0
    # (block_utils' bound, a few rows at a time: x in 64 bits is 4 GB)
    for m in range(0, M, 128):
        rows = slice(m, min(M, m + 128))
        p, off = layer.products(x[rows])
        check(h[rows], *hidden("silu", p, off, dt), "h")
        step = scales[rows].double().repeat_interleave(128, 1)[:, :N]
        check(kept64(codes[rows], scales[rows]), p, off + step * (0.5 + 128 * 2.0**-22), "kept products")
    again = fbq.gated(x, *layer.tensors, N, 128, 4, save=True)
    assert all(torch.equal(a, b) for a, b in zip((h, codes, scales), again))


@pytest.mark.parametrize("M,N,rank", [(5, (1 << 20) + 8, 8), (40, 1 << 21, 16), (800, (1 << 20) + 8, 16), (769, 1 << 21, 0)])
def test_gradients_of_a_layer_of_many_rows(M, N, rank):
    K, dt = 128, torch.bfloat16
    layer = Layer(fbq, N, K, 4, rank, dt, seed=1)
    dy, x = normal(M, N, dt, 2, 0.1), normal(M, K, dt, 3)
    got = fbq.linear_backward(dy, x, *layer.tensors, 128, 4)
    assert fbq.poll_status() == 0
    zero = torch.zeros((1, 1), dtype=torch.float64, device="cuda")
    want = layer_gradients(layer, dy.double(), zero.expand(M, N), x.double(), zero.expand(M, K), None)
    close(got, want)


def test_gradients_of_a_gated_layer_of_many_rows():
    M, N, K, rank, dt = 20, (1 << 20) + 16, 128, 16, torch.float16
    layer = Layer(fbq, N, K, 4, rank, dt, seed=1, gated=True)
    dh, x, kept = normal(M, N // 2, dt, 2, 0.01), normal(M, K, dt, 3), to_8_bits(normal(M, N, torch.float32, 4))
    got = fbq.gated_backward(dh, kept, x, *layer.tensors, 128, 4)
    zero = torch.zeros((1, 1), dtype=torch.float64, device="cuda")
    want = layer_gradients(layer, *gate_gradients("silu", dh, *kept, dt), x.double(), zero.expand(M, K), own_half(N, rank))
    close(got, want)
