"""The gate's derivative far from its bend, by its relative error."""
import math

import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import half_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fn", ["silu", "gelu"])
def test_slope_far_from_the_bend(fn):
    """dx = dh * up * f'(gate) alone: a gate row's weights are ones in every eighth column and zeros else, an up row's are zeros."""
    N, K = 16, 128
    codes = torch.zeros((N, K), dtype=torch.uint8, device="cuda")
    for j in range(8):
        codes[j, j::8] = 1
    layer = fbq.pack(codes, 4), torch.ones((N, 1), dtype=torch.float16, device="cuda"), torch.zeros((N, 1), dtype=torch.float16, device="cuda"), None, None
    v = torch.arange(-86.0, 87.0, device="cuda")
    v = v[v != 0]
    M = v.numel()
    scales = (v.abs() / 127)[:, None].contiguous()
    kept = torch.full((M, N), 127, dtype=torch.int8, device="cuda")
    kept[:, :8] = (v.sign() * 127).to(torch.int8)[:, None]
    dh = torch.ones((M, 8), dtype=torch.bfloat16, device="cuda")
    dx = fbq.gated_backward(dh, (kept, scales), None, *layer, 128, 4, fn=fn, want_factors=False)[0].double()
    size = scales.double() * 127
    gate = size * v.sign()[:, None]
    # f = v S(z): f' = S + v S (1 - S) z'
    c = 2 * math.sqrt(2 / math.pi)
    z, dz = (gate, torch.ones_like(gate)) if fn == "silu" else (c * (gate + 0.044715 * gate**3), c * (1 + 3 * 0.044715 * gate**2))
    want = size * (torch.sigmoid(z) + gate * torch.sigmoid(z) * torch.sigmoid(-z) * dz)
    # Relative error of the terms S and |v| S z', in units of 2^-23: z has the error of its argument (half a unit, three times that for a cube) and of two
    # products, an fma and two constants, 4 |z| in all; the exponential 2 + 1.173 |z| (CUDA's bound); the quotient 2, sums and products in single
    # precision 8.  Then one rounding to bf16.  S below 2^-126 may be taken for 0.
    terms = size * (1 + gate.abs() * dz)
    off = terms * torch.sigmoid(z) * (12 + 6 * z.abs()) * 2.0**-23 + terms * 2.0**-126
    bound = off + (want.abs() + off) * half_step(torch.bfloat16)
    assert bool(((dx - want).abs() <= bound).all()), (dx - want).abs().div(bound).max()
    far = gate[:, 0] < -32
    if fn == "silu":
        assert bool((dx[far] < 0).all())
    else:
        assert not bool(dx[far].any())
