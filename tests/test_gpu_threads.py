"""Calls of several host threads on one stream: a call that hands values from launch to launch through the stream's scratch gets its
own, whatever the other thread queues meanwhile."""
import threading

import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer, to_8_bits

pytestmark = pytest.mark.gpu


def normal(M, K, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((M, K), generator=g, device="cuda") * scale).to(dtype)


def gated(seed):
    layer = Layer(fbq, 528, 640, 4, 112, torch.float16, seed=1, gated=True)
    x = normal(96, 640, torch.float16, seed)
    return lambda: fbq.gated(x, *layer.tensors, 528, 128, 4, save=True)


def linear_backward(seed):
    layer = Layer(fbq, 520, 640, 3, 64, torch.bfloat16, seed=2)
    dy, x8 = normal(70, 520, torch.bfloat16, seed, 0.1), fbq.act8_pack(normal(70, 640, torch.bfloat16, seed + 1))
    return lambda: fbq.linear_backward(dy, x8, *layer.tensors, 128, 3)


def gated_backward(seed):
    layer = Layer(fbq, 528, 384, 4, 32, torch.float16, seed=3, gated=True)
    dh, x, kept = normal(800, 264, torch.float16, seed, 0.1), normal(800, 384, torch.float16, seed + 1), to_8_bits(normal(800, 528, torch.float32, seed + 2))
    return lambda: fbq.gated_backward(dh, kept, x, *layer.tensors, 128, 4)


def generic(seed):
    """A group that only the generic kernels take: t in a launch of its own."""
    g = torch.Generator(device="cuda").manual_seed(4)
    N, K, r = 256, 320, 24
    q = fbq.pack(torch.randint(0, 16, (N, K), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8), 4)
    s = (torch.rand((N, K // 64), generator=g, device="cuda") * 0.01).half()
    z = torch.full_like(s, 8.0)
    A, B, x = normal(r, K, torch.float16, 5, 0.1), normal(N, r, torch.float16, 6, 0.1), normal(12, K, torch.float16, seed)
    return lambda: (fbq.linear(x, q, s, z, A, B, N, 64, 4),)


def unfused(seed):
    A, B, x = normal(32, 512, torch.float16, 5, 0.1), normal(256, 32, torch.float16, 6, 0.1), normal(12, 512, torch.float16, seed)
    return lambda: (fbq.sub_branch_unfused(x, A, B, torch.zeros((12, 256), dtype=torch.float16, device="cuda")),)


def hostio(seed):
    """x by way of the stream's staging buffer, y straight into the caller's."""
    layer = Layer(fbq, 256, 512, 4, 16, torch.float16, seed=7)
    x, ys = normal(4, 512, torch.float16, seed).cpu().pin_memory(), [torch.empty((4, 256), dtype=torch.float16).pin_memory() for _ in range(64)]
    turn = iter(range(1 << 30))

    def call():
        return (fbq.linear_hostio(x, *layer.tensors, ys[next(turn) % 64], 256, 128, 4),)
    return call


@pytest.mark.parametrize("make", [gated, linear_backward, gated_backward, generic, unfused, hostio])
def test_two_threads_on_one_stream(make):
    calls = [make(100), make(200)]

    def finished(call):
        got = call()
        torch.cuda.synchronize()
        return [t.clone() for t in got]

    want = [finished(call) for call in calls]                   # (scratch is as large as it gets from here on)
    assert all(torch.equal(a, b) for call, w in zip(calls, want) for a, b in zip(finished(call), w))
    start, wrong, errors = threading.Barrier(len(calls)), [0] * len(calls), []

    def run(i):
        try:
            start.wait()
            for _ in range(12):
                got = [calls[i]() for _ in range(48)]
                torch.cuda.synchronize()
                wrong[i] += sum(not all(torch.equal(a, b) for a, b in zip(g, want[i])) for g in got)
        except Exception as e:                                  # (raised in the test's own thread below)
            errors.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and wrong == [0, 0], (errors, wrong)
    assert fbq.poll_status() == 0


def test_scratch_that_grows_under_two_threads():
    """Both threads make their stream's scratch larger and larger; nobody loses what the other is still using."""
    layer = Layer(fbq, 520, 384, 4, 16, torch.float16, seed=8)
    sizes = [8 * 2**i for i in range(8)]
    dys = {M: normal(M, 520, torch.float16, M, 0.1) for M in sizes}
    xs = {M: normal(M, 384, torch.float16, M + 1) for M in sizes}
    want = {M: fbq.linear_backward(dys[M], xs[M], *layer.tensors, 128, 4) for M in sizes}
    torch.cuda.synchronize()
    fbq.release_workspaces()
    start, results, errors = threading.Barrier(2), [[], []], []

    def run(i):
        try:
            start.wait()
            for M in sizes:
                results[i].append((M, fbq.linear_backward(dys[M], xs[M], *layer.tensors, 128, 4)))
        except Exception as e:
            errors.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for M, got in results[0] + results[1]:
        assert all(torch.equal(a, b) for a, b in zip(got, want[M])), M
