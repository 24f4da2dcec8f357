"""The first CUDA call of a host thread is one of the library's."""
import threading

import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer

pytestmark = pytest.mark.gpu


def in_a_thread(call):
    result = []

    def run():
        try:
            result.append(call())
        except Exception as e:                                  # (raised below, in the test's own thread)
            result.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    if isinstance(result[0], Exception):
        raise result[0]
    return result[0]


def test_calls_that_begin_with_a_tensor_map():
    N, K, dt = 528, 640, torch.float16
    layer = Layer(fbq, N, K, 4, 64, dt, seed=1, gated=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    for M in (1, 2, 5, 16, 40, 300, 1000):
        x, dy = torch.randn((M, K), generator=g, device="cuda").to(dt), torch.randn((M, N), generator=g, device="cuda").to(dt)
        codes, scales = fbq.act8_pack(dy)
        for call in (lambda: (fbq.linear(x, *layer.tensors, N, 128, 4),), lambda: (fbq.gated(x, *layer.tensors, N, 128, 4),),
                     lambda: fbq.gated(x, *layer.tensors, N, 128, 4, save=True), lambda: fbq.linear_backward(dy, x, *layer.tensors, 128, 4),
                     lambda: fbq.gated_backward(dy[:, : N // 2].contiguous(), (codes, scales), x, *layer.tensors, 128, 4)):
            want = call()                                       # (blocks of the results' sizes are there: the thread allocates nothing)
            torch.cuda.synchronize()
            want = [t.clone() for t in want]
            call()
            got = in_a_thread(call)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
