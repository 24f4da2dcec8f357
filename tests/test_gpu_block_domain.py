"""The feed-forward block's calls at the far ends of what the header says they take: contractions beyond what a 16-bit copy of the weights has
room for."""
import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer, check, hidden, kept64

pytestmark = pytest.mark.gpu


def normal(M, K, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((M, K), generator=g, device="cuda") * scale).to(dtype)


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
