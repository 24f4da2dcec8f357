"""Batches of two host threads whose problems run on side streams: each batch starts behind its own stream's work and its stream goes on behind
the batch, whatever the other thread forks and joins meanwhile."""
import threading

import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer

pytestmark = pytest.mark.gpu


def test_two_threads_with_a_stream_each():
    N, K, n, rounds = 512, 1024, 3, 60
    layer = Layer(fbq, N, K, 4, 16, torch.float16, seed=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    sources = [torch.randn((rounds, n, 1, K), generator=g, device="cuda").half() for _ in range(2)]
    want = [torch.stack([fbq.linear(s[r, i], *layer.tensors, N, 128, 4) for r in range(rounds) for i in range(n)]).view(rounds, n, 1, N) for s in sources]
    streams, xs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros((n, 1, K), dtype=torch.float16, device="cuda") for _ in range(2)]
    ys = [torch.empty((n, 1, N), dtype=torch.float16, device="cuda") for _ in range(2)]
    results = [torch.empty((rounds, n, 1, N), dtype=torch.float16, device="cuda") for _ in range(2)]
    # the x of the problems are not one: each goes to a stream of its own
    batches = [fbq.make_batch([(xs[t][i], *layer.tensors, ys[t][i]) for i in range(n)]) for t in range(2)]
    for b in batches:
        fbq.linear_batch(None, 128, 4, batch=b)
    torch.cuda.synchronize()
    start, errors = threading.Barrier(2), []

    def run(t):
        try:
            start.wait()
            with torch.cuda.stream(streams[t]):
                for r in range(rounds):
                    torch.cuda._sleep(20_000 * (1 + (r + t) % 3))
                    xs[t].copy_(sources[t][r])
                    fbq.linear_batch(None, 128, 4, batch=batches[t])
                    results[t][r].copy_(ys[t])
        except Exception as e:                                  # (raised in the test's own thread below)
            errors.append(e)

    threads = [threading.Thread(target=run, args=(t,)) for t in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    assert [int((a != b).any(dim=(1, 2, 3)).sum()) for a, b in zip(results, want)] == [0, 0]
