"""The stream argument without that stream being current: results are in memory of the stream that makes them, which neither what the
current stream still has to do nor a later tensor of it can reach."""
import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer, to_8_bits

pytestmark = pytest.mark.gpu
CYCLES = 200_000_000                                            # a tenth of a second


def normal(M, K, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((M, K), generator=g, device="cuda") * scale).to(dtype)


def act8_pack():
    x = normal(1000, 4104, torch.float16, 1)
    return lambda stream: fbq.act8_pack(x, stream=stream)


def act8_unpack():
    codes, scales = fbq.act8_pack(normal(1000, 4104, torch.float16, 2))
    return lambda stream: (fbq.act8_unpack(codes, scales, torch.bfloat16, stream=stream),)


def linear():
    layer, x = Layer(fbq, 4104, 512, 4, 32, torch.float16, seed=3), normal(1000, 512, torch.float16, 4)
    return lambda stream: (fbq.linear(x, *layer.tensors, 4104, 128, 4, stream=stream),)


def gated():
    layer, x = Layer(fbq, 4112, 512, 4, 32, torch.float16, seed=3, gated=True), normal(500, 512, torch.float16, 4)
    return lambda stream: fbq.gated(x, *layer.tensors, 4112, 128, 4, save=True, stream=stream)


def linear_backward():
    layer, dy, x = Layer(fbq, 520, 4096, 4, 64, torch.float16, seed=5), normal(500, 520, torch.float16, 6), normal(500, 4096, torch.float16, 7)
    return lambda stream: fbq.linear_backward(dy, x, *layer.tensors, 128, 4, stream=stream)


def gated_backward():
    layer, dh, x = Layer(fbq, 528, 4096, 4, 64, torch.float16, seed=5, gated=True), normal(500, 264, torch.float16, 6), normal(500, 4096, torch.float16, 7)
    kept = to_8_bits(normal(500, 528, torch.float32, 8))
    return lambda stream: fbq.gated_backward(dh, kept, x, *layer.tensors, 128, 4, stream=stream)


def gated_layer():
    gate, up = (Layer(fbq, 2056, 1024, 4, 64, torch.float16, seed=s) for s in (9, 10))
    return lambda stream: fbq.gated_layer(gate.tensors, up.tensors, 128, 4, stream=stream)


def pack():
    codes = torch.randint(0, 16, (2048, 4096), device="cuda", dtype=torch.int32).to(torch.uint8)
    return lambda stream: (fbq.pack(codes, 4, stream=stream),)


def unpack():
    q = fbq.pack(torch.randint(0, 8, (2048, 4096), device="cuda", dtype=torch.int32).to(torch.uint8), 3)
    return lambda stream: (fbq.unpack(q, 2048, 4096, 3, stream=stream),)


def dequant():
    layer = Layer(fbq, 1024, 2048, 4, 0, torch.float16, seed=11)
    return lambda stream: (fbq.dequant(*layer.tensors[:3], 1024, 2048, 128, 4, stream=stream),)


def quantize_feedback():
    W = normal(1024, 4096, torch.float32, 12, 0.05)
    return lambda stream: fbq.quantize_feedback(W, None, None, 128, 4, want_wf=True, stream=stream)


def gram():
    X = normal(256, 1024, torch.float32, 13)
    return lambda stream: (fbq.gram(X, stream=stream),)


CALLS = [act8_pack, act8_unpack, linear, gated, linear_backward, gated_backward, gated_layer, pack, unpack, dequant, quantize_feedback, gram]


@pytest.mark.parametrize("make", CALLS)
def test_the_current_stream_is_still_writing_what_it_has_freed(make):
    call, side = make(), torch.cuda.Stream()
    want = [t.clone() for t in call(None)]
    call(side)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = [torch.empty_like(t) for t in want]                  # blocks of the results' sizes
    torch.cuda._sleep(CYCLES)
    for t in held:
        t.view(torch.uint8).fill_(7)
    del held
    got = call(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("make", CALLS)
def test_results_that_are_dropped_while_their_stream_writes_them(make):
    call, side = make(), torch.cuda.Stream()
    want = [t.clone() for t in call(side)]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        torch.cuda._sleep(CYCLES)
    call(side)                                                  # dropped
    mine = [torch.full_like(t, 5) for t in want]
    torch.cuda.synchronize()
    assert all(bool((t == 5).all()) for t in mine)
