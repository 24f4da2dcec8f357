"""A call that finds no memory for its scratch says so, and the calls after it are not told so again."""
import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer, to_8_bits
from test_gpu_memory_used_up import free_megabytes

pytestmark = pytest.mark.gpu


def test_small_calls_after_a_refused_one():
    M, N, K, dt = 776, 65536, 1024, torch.bfloat16              # 134 MB of weights in 16 bits
    layer = Layer(fbq, N, K, 4, 0, dt, seed=1)
    dy = torch.zeros((M, N), dtype=dt, device="cuda")
    x = torch.ones((8, 256), dtype=dt, device="cuda")
    small = Layer(fbq, 32, 256, 4, 16, dt, seed=2, gated=True)
    dh, kept = torch.ones((8, 16), dtype=dt, device="cuda"), to_8_bits(torch.ones((8, 32), device="cuda"))
    calls = [lambda: fbq.act8_pack(x), lambda: (fbq.act8_unpack(*fbq.act8_pack(x), dt),), lambda: fbq.gated_layer(small.tensors, small.tensors, 128, 4),
             lambda: fbq.gated_backward(dh, kept, x, *small.tensors, 128, 4), lambda: (fbq.dequant(*small.tensors[:3], 32, 256, 128, 4),), lambda: (x + 1,)]
    want = [call() for call in calls]
    with free_megabytes(fbq, 60):
        for call, w in zip(calls, want):
            with pytest.raises(fbq.FbqError) as refused:
                fbq.linear_backward(dy, None, *layer.tensors, 128, 4, want_factors=False)
            assert refused.value.code == -4
            got = call()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, w))


def test_no_memory_for_results_is_torchs_error():
    M, K, N, dt = 1024, 65536, 131072, torch.float16
    x = torch.zeros((4 * M, K), dtype=dt, device="cuda")        # 537 MB; its codes are 268
    layer = Layer(fbq, N, 256, 4, 0, dt, seed=1, gated=True)
    few = torch.zeros((M, 256), dtype=dt, device="cuda")        # 134 MB of h, 268 of y
    fbq.act8_pack(x[:8]), fbq.linear(few[:8], *layer.tensors, N, 128, 4)
    with free_megabytes(fbq, 50):
        for call in (lambda: fbq.act8_pack(x), lambda: fbq.gated(few, *layer.tensors, N, 128, 4), lambda: fbq.linear(few, *layer.tensors, N, 128, 4)):
            with pytest.raises(torch.OutOfMemoryError):
                call()
        assert bool((fbq.act8_pack(few[:4])[0] == 0).all())
