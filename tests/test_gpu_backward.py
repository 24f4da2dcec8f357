"""Backward passes of an FBQuant linear and of the gated block, against the formulas and against differences in 64 bits."""
import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer, branches, check, f64, gate_gradients, kept64, layer_gradients, own_half, to_8_bits

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def normal(M, K, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((M, K), generator=g, device="cuda") * scale).to(dtype)


def x_of(kind, M, K, dtype, seed):
    """(what the call gets, x in 64 bits, how far the kernels' x is from it)"""
    x = normal(M, K, dtype, seed)
    if kind == "16 bits":
        return x, x.double(), torch.zeros_like(x, dtype=torch.float64)
    kept = fbq.act8_pack(x)
    x64 = kept64(*kept)
    return kept, x64, x64.abs() * (torch.finfo(dtype).eps / 2 + 2.0**-23) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def check_gradients(got, want, rank):
    assert len(want) == (3 if rank else 1)
    for g, (w, size), what in zip(got, want, ("dx", "dA", "dB")):
        check(g, w, size, what)
    assert rank or (got[1] is None and got[2] is None)


SHAPES = [
    # N, K, bits, rank, type
    (8, 128, 4, 0, "f16"),
    (16, 128, 3, 8, "bf16"),
    (136, 256, 4, 16, "f16"),
    (264, 384, 3, 64, "bf16"),
    (1000, 640, 4, 72, "f16"),
    (520, 2176, 3, 128, "f16"),
    (328, 1152, 4, 256, "bf16"),
]


@pytest.mark.parametrize("M", [1, 2, 15, 64, 65, 127, 129, 300, 497, 1000])
@pytest.mark.parametrize("N,K,bits,rank,dtype", SHAPES)
def test_linear(M, N, K, bits, rank, dtype):
    dt = TYPES[dtype]
    layer = Layer(fbq, N, K, bits, rank, dt, seed=N + M)
    dy = normal(M, N, dt, seed=M, scale=0.1)
    x, x64, off = x_of("8 bits" if M % 2 else "16 bits", M, K, dt, seed=K)
    got = fbq.linear_backward(dy, x, *layer.tensors, 128, bits)
    torch.cuda.synchronize()
    assert fbq.poll_status() == 0
    check_gradients(got, layer_gradients(layer, dy.double(), torch.zeros_like(dy, dtype=torch.float64), x64, off, None), rank)


@pytest.mark.parametrize("M", [1, 3, 16, 63, 130, 512, 700])
@pytest.mark.parametrize("N,K,bits,rank,dtype,fn", [
    (16, 128, 4, 0, "f16", "silu"),
    (48, 256, 3, 16, "bf16", "gelu"),
    (272, 384, 4, 32, "f16", "gelu"),
    (1040, 640, 3, 128, "bf16", "silu"),
    (400, 1152, 4, 256, "f16", "silu"),
])
def test_gated(M, N, K, bits, rank, dtype, fn):
    dt = TYPES[dtype]
    layer = Layer(fbq, N, K, bits, rank, dt, seed=N + M, gated=True)
    dh = normal(M, N // 2, dt, seed=M, scale=0.1)
    kept = to_8_bits(normal(M, N, torch.float32, seed=M + 1, scale=2.0))
    x, x64, off = x_of("16 bits" if M % 2 else "8 bits", M, K, dt, seed=K)
    got = fbq.gated_backward(dh, kept, x, *layer.tensors, 128, bits, fn=fn)
    assert fbq.poll_status() == 0
    dp, ddp = gate_gradients(fn, dh, *kept, dt)
    check_gradients(got, layer_gradients(layer, dp, ddp, x64, off, own_half(N, rank) if rank else None), rank)
    if rank:
        assert not bool((got[2] * ~own_half(N, rank)).any())


@pytest.mark.parametrize("M,N,K,bits,rank,dtype", [(2100, 4104, 2816, 4, 64, "bf16"), (1500, 1024, 6016, 3, 128, "f16"), (4097, 2056, 1280, 4, 200, "f16")])
def test_many_tiles(M, N, K, bits, rank, dtype):
    dt = TYPES[dtype]
    layer = Layer(fbq, N, K, bits, rank, dt, seed=1)
    dy, x = normal(M, N, dt, seed=2, scale=0.1), normal(M, K, dt, seed=3)
    got = fbq.linear_backward(dy, x, *layer.tensors, 128, bits)
    zero = torch.zeros((1, 1), dtype=torch.float64, device="cuda")
    check_gradients(got, layer_gradients(layer, dy.double(), zero.expand(M, N), x.double(), zero.expand(M, K), None), rank)


@pytest.mark.parametrize("M,rank", [(40, 16), (800, 16), (800, 0)])
def test_weights_in_several_launches(M, rank):
    """A layer whose 16-bit copy of the weights is beyond one launch's scratch: columns in parts (few tokens need no copy)."""
    N, K, bits, dt = 131072, 2304, 4, torch.bfloat16
    layer = Layer(fbq, N, K, bits, rank, dt, seed=1)
    dy, x = normal(M, N, dt, seed=2, scale=0.1), normal(M, K, dt, seed=3)
    got = fbq.linear_backward(dy, x, *layer.tensors, 128, bits)
    zero = torch.zeros((1, 1), dtype=torch.float64, device="cuda")
    check_gradients(got, layer_gradients(layer, dy.double(), zero.expand(M, N), x.double(), zero.expand(M, K), None), rank)


@pytest.mark.parametrize("M", [16, 33, 95, 112, 160, 176, 192, 193, 385, 768, 769])
@pytest.mark.parametrize("rank", [64, 128, 192, 256])
def test_tiles_of_tokens_and_blocks_of_the_rank(M, rank):
    """Every depth of the rings, odd and even numbers of the sub-branch's blocks, both sides of the sizes at which kernels change."""
    N, K, bits, dt = 1160, 640, 3 if rank > 128 else 4, torch.float16
    layer = Layer(fbq, N, K, bits, rank, dt, seed=M)
    dy, x = normal(M, N, dt, seed=2, scale=0.1), normal(M, K, dt, seed=3)
    got = fbq.linear_backward(dy, x, *layer.tensors, 128, bits)
    assert fbq.poll_status() == 0
    zero = torch.zeros((1, 1), dtype=torch.float64, device="cuda")
    check_gradients(got, layer_gradients(layer, dy.double(), zero.expand(M, N), x.double(), zero.expand(M, K), None), rank)


@pytest.mark.parametrize("M,N,K,rank", [(333, 20488, 256, 72), (60, 1032, 16640, 200), (1100, 12296, 384, 136)])
def test_long_contractions_of_the_thin_products(M, N, K, rank):
    """s and t whose contraction several clusters share."""
    dt = torch.bfloat16
    layer = Layer(fbq, N, K, 4, rank, dt, seed=M)
    dy, x = normal(M, N, dt, seed=2, scale=0.1), normal(M, K, dt, seed=3)
    got = fbq.linear_backward(dy, x, *layer.tensors, 128, 4)
    zero = torch.zeros((1, 1), dtype=torch.float64, device="cuda")
    check_gradients(got, layer_gradients(layer, dy.double(), zero.expand(M, N), x.double(), zero.expand(M, K), None), rank)


def test_parts_of_the_results():
    N, K, bits, rank, dt, M = 264, 384, 4, 64, torch.float16, 200
    layer = Layer(fbq, N, K, bits, rank, dt, seed=1)
    dy, x = normal(M, N, dt, seed=2, scale=0.1), normal(M, K, dt, seed=3)
    dx, dA, dB = fbq.linear_backward(dy, x, *layer.tensors, 128, bits)
    only = fbq.linear_backward(dy, None, *layer.tensors, 128, bits, want_factors=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    only = fbq.linear_backward(dy, x, *layer.tensors, 128, bits, want_dx=False)
    assert only[0] is None and torch.equal(only[1], dA) and torch.equal(only[2], dB)
    assert fbq.linear_backward(dy, None, *layer.tensors, 128, bits, want_dx=False, want_factors=False) == (None, None, None)


def test_no_tokens():
    layer = Layer(fbq, 32, 128, 4, 16, torch.float16, seed=1, gated=True)
    dh, x = torch.empty((0, 16), dtype=torch.float16, device="cuda"), torch.empty((0, 128), dtype=torch.float16, device="cuda")
    kept = (torch.empty((0, 32), dtype=torch.int8, device="cuda"), torch.empty((0, 1), dtype=torch.float32, device="cuda"))
    for dx, dA, dB in (fbq.gated_backward(dh, kept, x, *layer.tensors, 128, 4), fbq.linear_backward(dh.new_empty((0, 32)), x, *layer.tensors, 128, 4)):
        assert dx.shape == (0, 128) and not bool(dA.any()) and not bool(dB.any()) and dA.shape == (16, 128) and dB.shape == (32, 16)


def test_directional_differences_of_the_block():
    """<dx, v> + <dA, a> + <dB, b> is the slope of sum(dh * h(x + e v, A + e a, B + e b)), by differences of the forward pass in 64 bits."""
    M, N, K, bits, rank, dt = 96, 272, 384, 4, 32, torch.float16
    for fn in ("silu", "gelu"):
        layer = Layer(fbq, N, K, bits, rank, dt, seed=5, gated=True)
        x, dh = normal(M, K, dt, seed=6, scale=0.3), normal(M, N // 2, dt, seed=7, scale=0.1)
        h, *kept = fbq.gated(x, *layer.tensors, N, 128, bits, fn=fn, save=True)
        got = fbq.gated_backward(dh, kept, x, *layer.tensors, 128, bits, fn=fn)
        v, a, b = (normal(*s, torch.float64, seed=i) for i, s in enumerate(((M, K), (rank, K), (N, rank))))
        b = b * own_half(N, rank)

        def loss(e):
            X, A, B = x.double() + e * v, layer.A64 + e * a, layer.B64 + e * b
            gate, up = branches(X @ layer.W.t() + (X @ A.t()) @ B.t())
            return (dh.double() * f64(fn, gate)[0] * up).sum()

        e = 1e-5
        slope = float((loss(e) - loss(-e)) / (2 * e))
        terms = [(g.double() * d) for g, d in zip(got, (v, a, b))]
        found = float(sum(t.sum() for t in terms))
        # The products were kept to 1/254 of their group's largest, which for these is below 4.5 times the typical one: a relative 2 % of
        # an entry's dp at most, of random sign over M N entries; the formula's gradient of exact products is what differences give.
        scale = float(sum(t.square().sum() for t in terms)) ** 0.5
        assert abs(found - slope) <= 0.02 * 4 * scale, (fn, found, slope, scale)


def test_the_formula_by_differences():
    """The reference itself, in 64 bits: layer_gradients and gate_gradients against differences of every kind of entry."""
    M, N, K, rank, dt = 5, 32, 128, 16, torch.float16
    layer = Layer(fbq, N, K, 4, rank, dt, seed=8, gated=True)
    x, dh = normal(M, K, dt, seed=9, scale=0.3).double(), normal(M, N // 2, dt, seed=10).double()
    for fn in ("silu", "gelu"):
        p = x @ layer.W.t() + (x @ layer.A64.t()) @ layer.B64.t()
        gate, up = branches(p)
        f, df = f64(fn, gate)
        dp = torch.stack(((dh * up * df).view(M, -1, 8), (dh * f).view(M, -1, 8)), 2).view(M, N)
        zero = torch.zeros((1, 1), dtype=torch.float64, device="cuda")
        grads = [g for g, _ in layer_gradients(layer, dp, zero.expand(M, N), x, zero.expand(M, K), own_half(N, rank))]

        def loss(x, A, B):
            gate, up = branches(x @ layer.W.t() + (x @ A.t()) @ B.t())
            return float((dh * f64(fn, gate)[0] * up).sum())

        at = [x, layer.A64, layer.B64]
        for which, i, j in ((0, 0, 0), (0, 4, 127), (1, 0, 5), (1, 15, 100), (2, 0, 3), (2, 9, 12), (2, 31, 8)):
            e = 1e-6
            up_, down = [t.clone() for t in at], [t.clone() for t in at]
            up_[which][i, j] += e
            down[which][i, j] -= e
            slope = (loss(*up_) - loss(*down)) / (2 * e)
            # differences: error e^2 f''' (below 1e-10) and 2^-52 times the loss (below 100) over e
            assert abs(slope - float(grads[which][i, j])) < 1e-7, (fn, which, i, j)


def test_a_training_step_of_the_whole_block():
    """gated -> 8 bits -> down projection, and back: what a step of an adaptation runs, against 64 bits all through."""
    M, d, F, bits, r, dt = 260, 384, 528, 4, 16, torch.bfloat16
    gate, up = (Layer(fbq, F, d, bits, r, dt, seed=s) for s in (1, 2))
    down = Layer(fbq, d, F // 128 * 128, bits, 2 * r, dt, seed=3)
    F = down.K                                                  # (a layer's inputs come in groups of 128)
    gate, up = (Layer(fbq, F, d, bits, r, dt, seed=s) for s in (1, 2))
    whole = fbq.gated_layer(gate.tensors, up.tensors, 128, bits)
    x, dy = normal(M, d, dt, seed=4), normal(M, d, dt, seed=5, scale=0.1)
    # forward
    x8 = fbq.act8_pack(x)
    h, codes, scales = fbq.gated(x, *whole, 2 * F, 128, bits, save=True)
    h8 = fbq.act8_pack(h)
    fbq.linear(h, *down.tensors, d, 128, bits)
    # backward
    dh, dA_down, dB_down = fbq.linear_backward(dy, h8, *down.tensors, 128, bits)
    dx, dA, dB = fbq.gated_backward(dh, (codes, scales), x8, *whole, 128, bits)
    assert fbq.poll_status() == 0
    assert all(bool(torch.isfinite(t).all()) for t in (dh, dA_down, dB_down, dx, dA, dB))

    def rel(got, want):
        return float((got.double() - want).norm() / want.norm())

    x64, dy64 = x.double(), dy.double()
    pg = x64 @ gate.W.t() + x64 @ gate.A64.t() @ gate.B64.t()
    pu = x64 @ up.W.t() + x64 @ up.A64.t() @ up.B64.t()
    f, df = f64("silu", pg)
    h64 = f * pu
    dh64 = dy64 @ down.W + dy64 @ down.B64 @ down.A64
    dg, du = dh64 * pu * df, dh64 * f
    want_dx = dg @ gate.W + dg @ gate.B64 @ gate.A64 + du @ up.W + du @ up.B64 @ up.A64
    # Sums of hundreds of terms of random sign: relative errors of the operands add as they do in a norm.  bf16 operands and results 2^-8 / sqrt(3)
    # each, at most six of them in a row (h, dh, dp, W, s or t, the result): 0.55 %.  8 bits: a step is 1/127 of the largest of 128, below
    # 1/35 of a normal group's norm per entry, over sqrt(12): 0.8 %; products of two (gate and up) enter dp, and h's are wider (largest below 9
    # times the norm): 2 %.
    assert rel(h, h64) < 0.0055 and rel(dh, dh64) < 0.0055
    assert rel(dA_down, (dy64 @ down.B64).t() @ h64) < 0.026 and rel(dB_down, dy64.t() @ (h64 @ down.A64.t())) < 0.026
    assert rel(dx, want_dx) < 0.026
    assert rel(dA[:r], (dg @ gate.B64).t() @ x64) < 0.026 and rel(dA[r:], (du @ up.B64).t() @ x64) < 0.026
    v = dB.view(-1, 16, 2 * r)
    assert rel(v[:, :8, :r].reshape(F, r), dg.t() @ (x64 @ gate.A64.t())) < 0.026
    assert rel(v[:, 8:, r:].reshape(F, r), du.t() @ (x64 @ up.A64.t())) < 0.026


def test_same_bits_again_in_a_graph_and_on_another_stream():
    N, K, bits, rank, dt, M = 528, 512, 3, 64, torch.bfloat16, 333
    layer = Layer(fbq, N, K, bits, rank, dt, seed=1, gated=True)
    dh, x = normal(M, N // 2, dt, seed=2, scale=0.1), normal(M, K, dt, seed=3)
    kept = to_8_bits(normal(M, N, torch.float32, seed=4))
    first = fbq.gated_backward(dh, kept, x, *layer.tensors, 128, bits)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, fbq.gated_backward(dh, kept, x, *layer.tensors, 128, bits)))
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        with pytest.raises(fbq.FbqError) as refused:            # scratch of this stream would have to grow during the capture
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                fbq.gated_backward(dh, kept, x, *layer.tensors, 128, bits)
        assert refused.value.code == -2
        del graph
        fbq.gated_backward(dh, kept, x, *layer.tensors, 128, bits)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = fbq.gated_backward(dh, kept, x, *layer.tensors, 128, bits)
    dh.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    want = fbq.gated_backward(dh, kept, x, *layer.tensors, 128, bits)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    del graph


def test_calls_of_two_streams_at_once():
    N, K, bits, rank, dt, M = 1040, 1152, 4, 64, torch.float16, 700
    layer = Layer(fbq, N, K, bits, rank, dt, seed=1)
    pairs = [(normal(M, N, dt, seed=i, scale=0.1), normal(M, K, dt, seed=10 + i)) for i in range(2)]
    want = [fbq.linear_backward(dy, x, *layer.tensors, 128, bits) for dy, x in pairs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    got = [None, None]
    for _ in range(5):
        for i, (dy, x) in enumerate(pairs):
            with torch.cuda.stream(streams[i]):
                got[i] = fbq.linear_backward(dy, x, *layer.tensors, 128, bits)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_results_end_where_they_should():
    N, K, bits, rank, dt, M = 136, 256, 4, 16, torch.float16, 70
    layer = Layer(fbq, N, K, bits, rank, dt, seed=1)
    dy, x = normal(M, N, dt, seed=2, scale=0.1), normal(M, K, dt, seed=3)
    want = fbq.linear_backward(dy, x, *layer.tensors, 128, bits)
    import ctypes
    stores = [torch.full((t.numel() + 64,), 7.0, dtype=dt, device="cuda") for t in want]
    p = [ctypes.c_void_p(t.data_ptr()) for t in (dy, x)]
    w = [ctypes.c_void_p(t.data_ptr()) for t in layer.tensors]
    outs = [ctypes.c_void_p(s[32:].data_ptr()) for s in stores]
    code = fbq.lib().fbq_linear_backward(p[0], p[1], None, None, *w, *outs, M, N, K, 128, bits, rank, 0, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert code == 0
    for s, t in zip(stores, want):
        assert bool((s[:32] == 7).all()) and bool((s[-32:] == 7).all()) and torch.equal(s[32:-32], t.reshape(-1))


def test_a_wait_that_runs_out():
    """s that its tiles do not announce: the main tiles' bounded wait gives up and the status tells; the next call is fine."""
    N, K, bits, rank, dt, M = 264, 384, 4, 64, torch.float16, 900
    layer = Layer(fbq, N, K, bits, rank, dt, seed=1)
    dy, x = normal(M, N, dt, seed=2, scale=0.1), normal(M, K, dt, seed=3)
    want = fbq.linear_backward(dy, x, *layer.tensors, 128, bits)
    assert fbq.poll_status() == 0
    fbq.set_option("test_prefill_skip_flag", 1)
    fbq.set_option("prefill_flag_polls", 200)
    try:
        fbq.linear_backward(dy, x, *layer.tensors, 128, bits)
        assert fbq.poll_status() == -5
    finally:
        fbq.set_option("test_prefill_skip_flag", 0)
        fbq.set_option("prefill_flag_polls", 0)
    assert fbq.poll_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(want, fbq.linear_backward(dy, x, *layer.tensors, 128, bits)))
    assert fbq.poll_status() == 0
