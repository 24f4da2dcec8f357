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
    """Results larger than the device, or than what is beside their input."""
    M, N, K, dt = 65536, 1 << 22, 128, torch.float16            # 275 GB of h, 550 of y
    layer = Layer(fbq, N, K, 4, 0, dt, seed=1, gated=True)
    x = torch.zeros((M, K), dtype=dt, device="cuda")
    for call in (lambda: fbq.gated(x, *layer.tensors, N, 128, 4), lambda: fbq.linear(x, *layer.tensors, N, 128, 4)):
        with pytest.raises(torch.OutOfMemoryError):
            call()
    torch.cuda.empty_cache()
    K = torch.cuda.mem_get_info()[0] // 10 * 7 // 2 // M // 16 * 16           # seven tenths of what is free; the codes are half of that
    wide = torch.empty((M, K), dtype=dt, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):
        fbq.act8_pack(wide)
    del wide
    torch.cuda.empty_cache()
    assert not bool(fbq.act8_pack(x)[0].any())


def fill(bytes_left):
    """Takes the device's memory but for less than 2 MB and `bytes_left`; what it returns holds it."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    kept, held = torch.empty(max(bytes_left, 1), dtype=torch.uint8, device="cuda"), []
    for size in (1 << 34, 1 << 30, 64 << 20, 10 << 20, 1 << 20):
        try:
            while True:
                held.append(torch.empty(size, dtype=torch.uint8, device="cuda"))
        except torch.OutOfMemoryError:
            pass
    del kept
    torch.cuda.empty_cache()
    return held


def test_counters_that_could_not_grow_are_there_for_the_next_call():
    """A prompt of very many tiles needs more counters than there is memory for; what the stream had is gone then, and the next call gets its own."""
    N, K, M, dt = 65536, 128, 131072, torch.float16             # 2.1 MB of counters
    layer = Layer(fbq, N, K, 4, 0, dt, seed=1)
    x, y = torch.ones((M, K), dtype=dt, device="cuda"), torch.empty((M, N), dtype=dt, device="cuda")
    few = torch.ones((100, K), dtype=dt, device="cuda")
    want = fbq.linear(few, *layer.tensors, N, 128, 4)
    fbq.release_workspaces()
    out = torch.empty_like(want)
    fbq.linear(few, *layer.tensors, N, 128, 4, y=out)           # the stream has counters for this
    held = fill(0)
    with pytest.raises(fbq.FbqError) as refused:
        fbq.linear(x, *layer.tensors, N, 128, 4, y=y)
    assert refused.value.code == -4
    del held
    torch.cuda.empty_cache()
    out.zero_()
    fbq.linear(few, *layer.tensors, N, 128, 4, y=out)
    torch.cuda.synchronize()
    assert fbq.poll_status() == 0 and torch.equal(out, want)
    fbq.linear(x, *layer.tensors, N, 128, 4, y=y)
    assert torch.allclose(y[-1].float(), want[0].float(), rtol=2.0**-10, atol=2.0**-10)      # (another kernel's order of summation: a rounding apart)


def test_staging_that_could_not_grow_is_there_for_the_next_call():
    N, K, dt = 1024, 8192, torch.float16
    layer = Layer(fbq, N, K, 4, 0, dt, seed=1)
    few, many = torch.ones((64, K), dtype=dt).pin_memory(), torch.ones((8192, K), dtype=dt).pin_memory()          # 1 and 134 MB
    y, ys = torch.empty((64, N), dtype=dt).pin_memory(), torch.empty((8192, N), dtype=dt).pin_memory()
    fbq.linear_hostio(few, *layer.tensors, y, N, 128, 4)
    torch.cuda.synchronize()
    want = y.clone()
    held = fill(60 << 20)
    with pytest.raises(fbq.FbqError) as refused:
        fbq.linear_hostio(many, *layer.tensors, ys, N, 128, 4)
    assert refused.value.code == -4
    y.zero_()
    fbq.linear_hostio(few, *layer.tensors, y, N, 128, 4)
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    del held
    torch.cuda.empty_cache()
    fbq.linear_hostio(many, *layer.tensors, ys, N, 128, 4)
    torch.cuda.synchronize()
    assert torch.allclose(ys[-1].float(), want[0].float(), rtol=2.0**-10, atol=2.0**-10) and fbq.poll_status() == 0
