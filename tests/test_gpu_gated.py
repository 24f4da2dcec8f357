"""The gated block h = f(gate) * up over a gated layer, against a plain implementation in 64 bits."""
import pytest
import torch

import paper_2501_16385_b200 as fbq
from block_utils import Layer, branches, check, f64, half_step, hidden, interleave, kept64, own_half

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def inputs(M, K, dtype, seed, outliers=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((M, K), generator=g, device="cuda")
    if outliers:
        x[:, torch.randperm(K, generator=g, device="cuda")[: K // 100 + 1]] *= 20
    return x.to(dtype)


# One token to a few tiles of tokens; rows of one granule, ragged tiles, more than one tile; every kernel that gates.
@pytest.mark.parametrize("M", [1, 2, 3, 8, 9, 16, 17, 77, 128, 129, 300, 500])
@pytest.mark.parametrize("N,K,bits,rank,dtype,fn", [
    (16, 128, 4, 0, "f16", "silu"),
    (48, 128, 3, 16, "bf16", "gelu"),
    (272, 640, 4, 32, "bf16", "silu"),
    (528, 384, 3, 64, "f16", "gelu"),
    (1040, 1152, 4, 128, "f16", "silu"),
    (400, 2176, 3, 128, "bf16", "silu"),
    (288, 256, 4, 192, "f16", "silu"),
    (144, 512, 3, 256, "bf16", "gelu"),
])
def test_hidden_activations(M, N, K, bits, rank, dtype, fn):
    dt = TYPES[dtype]
    layer = Layer(fbq, N, K, bits, rank, dt, seed=M + N, gated=True)
    x = inputs(M, K, dt, seed=N + K, outliers=M > 16)
    h = fbq.gated(x, *layer.tensors, N, 128, bits, fn=fn)
    torch.cuda.synchronize()
    assert fbq.poll_status() == 0
    check(h, *hidden(fn, *layer.products(x), dt), "h")


# More than three waves of tiles: the dense kernel gates.
@pytest.mark.parametrize("M,N,K,bits,rank,dtype", [(1000, 16 * 1100, 256, 4, 64, "bf16"), (2049, 8208, 384, 3, 128, "f16"), (700, 22016, 128, 4, 0, "f16")])
def test_prompts_of_many_tiles(M, N, K, bits, rank, dtype):
    dt = TYPES[dtype]
    layer = Layer(fbq, N, K, bits, rank, dt, seed=3, gated=True)
    x = inputs(M, K, dt, seed=4, outliers=True)
    h = fbq.gated(x, *layer.tensors, N, 128, bits)
    check(h, *hidden("silu", *layer.products(x), dt), "h")


@pytest.mark.parametrize("M", [1, 5, 16, 33, 257, 481, 1030])
@pytest.mark.parametrize("N,K,bits,rank,dtype,fn", [(16, 128, 3, 16, "f16", "gelu"), (144, 256, 4, 0, "bf16", "silu"), (656, 384, 4, 64, "f16", "silu"),
                                                    (4112, 512, 3, 128, "bf16", "gelu")])
def test_products_kept_in_8_bits(M, N, K, bits, rank, dtype, fn):
    dt = TYPES[dtype]
    layer = Layer(fbq, N, K, bits, rank, dt, seed=M, gated=True)
    x = inputs(M, K, dt, seed=7, outliers=True)
    h, codes, scales = fbq.gated(x, *layer.tensors, N, 128, bits, fn=fn, save=True)
    assert fbq.poll_status() == 0
    p, off = layer.products(x)
    check(h, *hidden(fn, p, off, dt), "h")
    assert codes.shape == (M, N) and scales.shape == (M, -(-N // 128))
    pad = torch.nn.functional.pad
    groups = pad(p.abs(), (0, -N % 128)).view(M, -1, 128)
    worst = pad(off, (0, -N % 128)).view(M, -1, 128).amax(2)
    # the scale is a 127th of the group's largest product, which is known to the largest bound of the group
    check(scales, groups.amax(2) / 127, worst / 127 + groups.amax(2) / 127 * 2.0**-23, "scales")
    # a code is the nearest multiple of the scale: half a scale off at most, and two roundings of products up to 127
    step = scales.double().repeat_interleave(128, 1)[:, :N]
    check(kept64(codes, scales), p, off + step * (0.5 + 128 * 2.0**-22), "kept products")
    assert int(codes.abs().max()) <= 127 and bool((pad(codes.abs().int(), (0, -N % 128)).view(M, -1, 128).amax(2) == 127).all())


@pytest.mark.parametrize("M", [16, 40, 95, 112, 160, 176, 192, 193, 400, 512, 513])
@pytest.mark.parametrize("rank", [16, 112, 192, 256])
def test_products_kept_by_tiles_of_tokens(M, rank):
    """Every depth of the rings, odd and even numbers of the sub-branch's blocks, both sides of the size at which kernels change."""
    N, K, bits, dt = 1168, 640, 3 if rank > 128 else 4, torch.bfloat16
    layer = Layer(fbq, N, K, bits, rank, dt, seed=M, gated=True)
    x = inputs(M, K, dt, seed=7)
    h, codes, scales = fbq.gated(x, *layer.tensors, N, 128, bits, save=True)
    assert fbq.poll_status() == 0
    p, off = layer.products(x)
    check(h, *hidden("silu", p, off, dt), "h")
    step = scales.double().repeat_interleave(128, 1)[:, :N]
    check(kept64(codes, scales), p, off + step * (0.5 + 128 * 2.0**-22), "kept products")


@pytest.mark.parametrize("M", [513, 900, 901])
def test_wide_layers_of_hundreds_of_tokens(M):
    """Both sides of the size at which the kernel of a wide layer changes."""
    N, K, bits, rank, dt = 20016, 256, 4, 32, torch.float16
    layer = Layer(fbq, N, K, bits, rank, dt, seed=M, gated=True)
    x = inputs(M, K, dt, seed=7)
    h, codes, scales = fbq.gated(x, *layer.tensors, N, 128, bits, save=True)
    p, off = layer.products(x)
    check(h, *hidden("silu", p, off, dt), "h")
    check(fbq.gated(x, *layer.tensors, N, 128, bits), *hidden("silu", p, off, dt), "h")
    step = scales.double().repeat_interleave(128, 1)[:, :N]
    check(kept64(codes, scales), p, off + step * (0.5 + 128 * 2.0**-22), "kept products")


@pytest.mark.parametrize("save", [False, True])
def test_weights_in_several_launches(save):
    """A layer whose 16-bit copy of the weights is beyond one launch's scratch: rows in parts."""
    M, N, K, bits, rank, dt = 700, 131072 + 144, 2176, 4, 16, torch.float16
    layer = Layer(fbq, N, K, bits, rank, dt, seed=1, gated=True)
    x = inputs(M, K, dt, seed=2)
    got = fbq.gated(x, *layer.tensors, N, 128, bits, save=save)
    p, off = layer.products(x)
    check(got[0] if save else got, *hidden("silu", p, off, dt), "h")
    if save:
        step = got[2].double().repeat_interleave(128, 1)[:, :N]
        check(kept64(*got[1:]), p, off + step * (0.5 + 128 * 2.0**-22), "kept products")


def test_scratch_does_not_grow_in_a_capture():
    N, K, bits, dt = 272, 256, 4, torch.float16
    layer = Layer(fbq, N, K, bits, 32, dt, seed=23, gated=True)
    for M in (50, 700):                                         # both kernels that keep products
        x = inputs(M, K, dt, seed=M)
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream), pytest.raises(fbq.FbqError) as refused:
            with torch.cuda.graph(graph, stream=stream):
                fbq.gated(x, *layer.tensors, N, 128, bits, save=True)
        assert refused.value.code == -2
        del graph
        with torch.cuda.stream(stream):
            h, *_ = fbq.gated(x, *layer.tensors, N, 128, bits, save=True)
        stream.synchronize()
        check(h, *hidden("silu", *layer.products(x), dt), "h")


@pytest.mark.parametrize("M", [2, 12, 200, 700])
def test_calls_of_two_streams_at_once(M):
    N, K, bits, dt = 1040, 1152, 4, torch.float16
    layer = Layer(fbq, N, K, bits, 32, dt, seed=24, gated=True)
    xs = [inputs(M, K, dt, seed=i) for i in range(2)]
    want = [fbq.gated(x, *layer.tensors, N, 128, bits, save=M >= 200) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [None, None]
    for _ in range(5):
        for i, x in enumerate(xs):
            with torch.cuda.stream(streams[i]):
                got[i] = fbq.gated(x, *layer.tensors, N, 128, bits, save=M >= 200)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w)) if M >= 200 else torch.equal(g, w)


@pytest.mark.parametrize("M", [1, 3, 40])
def test_a_gated_layer_is_an_ordinary_layer(M):
    """fbq_gated_layer's rows, checked through fbq.linear of the branches and of the whole, and h of it."""
    F, K, r, bits = 200, 384, 16, 3
    gate, up = (Layer(fbq, F, K, bits, r, torch.float16, seed=s) for s in (1, 2))
    whole = fbq.gated_layer(gate.tensors, up.tensors, 128, bits)
    q, s, z, A, B = whole
    assert torch.equal(A, torch.cat((gate.A, up.A)))
    assert torch.equal(s, interleave(gate.scales.t().contiguous(), up.scales.t().contiguous()).t())
    assert torch.equal(z, interleave(gate.zeros.t().contiguous(), up.zeros.t().contiguous()).t())
    codes = fbq.unpack(q, 2 * F, K, bits)
    assert torch.equal(codes, interleave(fbq.unpack(gate.qweight, F, K, bits).t().contiguous(), fbq.unpack(up.qweight, F, K, bits).t().contiguous()).t())
    assert torch.equal(B.view(-1, 16, 2 * r)[:, :8, :r].reshape(F, r), gate.B) and torch.equal(B.view(-1, 16, 2 * r)[:, 8:, r:].reshape(F, r), up.B)
    assert not bool((B * ~own_half(2 * F, 2 * r)).any())
    x = inputs(M, K, torch.float16, seed=9)
    h = fbq.gated(x, *whole, 2 * F, 128, bits)
    pg, dg = gate.products(x)
    pu, du = up.products(x)
    check(h, *hidden("silu", interleave(pg, pu), interleave(dg, du), torch.float16), "h")


def test_gated_layer_of_rank_0_and_a_rank_that_is_no_multiple_of_16():
    for r in (0, 8):
        gate, up = (Layer(fbq, 64, 256, 4, r, torch.bfloat16, seed=s) for s in (3, 4))
        whole = fbq.gated_layer(gate.tensors, up.tensors, 128, 4)
        x = inputs(20, 256, torch.bfloat16, seed=5)
        h = fbq.gated(x, *whole, 128, 128, 4)
        (pg, dg), (pu, du) = gate.products(x), up.products(x)
        check(h, *hidden("silu", interleave(pg, pu), interleave(dg, du), torch.bfloat16), "h")


@pytest.mark.parametrize("M", [1, 2, 4, 12, 100, 600])
def test_large_and_extreme_products(M):
    """Products far outside the gate's bend, of both signs: h is 0 or the product itself, never NaN."""
    N, K, dt = 512, 256, torch.bfloat16
    layer = Layer(fbq, N, K, 4, 0, dt, seed=11)
    x = (inputs(M, K, dt, seed=12).float() * 3000).to(dt)
    for fn in ("silu", "gelu"):
        h = fbq.gated(x, *layer.tensors, N, 128, 4, fn=fn)
        check(h, *hidden(fn, *layer.products(x), dt), "h")


@pytest.mark.parametrize("rank", [0, 32])
@pytest.mark.parametrize("M", [4, 16, 40, 700])
def test_infinite_x(M, rank):
    """An infinite x makes every product of its token infinite or NaN as the sum of products does, so h is what the gate makes of that;
    other tokens do not notice."""
    N, K, dt = 272, 384, torch.float16
    layer = Layer(fbq, N, K, 4, rank, dt, seed=13)
    layer.zeros += 0.5                                         # no weight is 0
    x = inputs(M, K, dt, seed=14)
    clean = fbq.gated(x, *layer.tensors, N, 128, 4)
    x[1, 5] = float("inf")
    h = fbq.gated(x, *layer.tensors, N, 128, 4)
    others = [m for m in range(M) if m != 1]
    assert torch.equal(h[others], clean[others])
    w = fbq.dequant(layer.qweight, layer.scales, layer.zeros, N, K, 128, 4)[:, 5].double()
    t = layer.A64[:, 5]
    # an infinite t has entries of both signs: their sum over the rank is NaN unless the entries of B make all of one sign
    terms = (torch.cat((w[:, None], layer.B64 * t.sign()[None, :]), 1) if rank else w[:, None]) * float("inf")
    p = terms.sum(1)[None, :]
    gate, up = branches(p)
    want = (f64("silu", gate)[0] * up)[0]
    assert torch.equal(torch.isnan(h[1]), torch.isnan(want.half()))
    finite = ~torch.isnan(want)
    assert torch.equal(h[1].double()[finite], want[finite])


@pytest.mark.parametrize("rank", [0, 32])
def test_infinite_x_of_two_tokens(rank):
    """The streaming kernel holds x in fixed point: a group with an infinite value is NaN, and so is all of its token, and no other."""
    N, K, dt = 272, 384, torch.float16
    layer = Layer(fbq, N, K, 4, rank, dt, seed=13)
    x = inputs(2, K, dt, seed=14)
    for call in (fbq.linear, fbq.gated):
        for bad in (float("inf"), float("-inf"), float("nan")):
            broken = x.clone()
            broken[1, 5] = bad
            out = call(broken, *layer.tensors, N, 128, 4)
            assert bool(torch.isnan(out[1]).all())
            p, off = layer.products(torch.stack((x[0], x[0])))   # (the other token's t has its own scale now)
            if call is fbq.linear:
                check(out[:1], p[:1], off[:1] + p[:1].abs() * half_step(dt) + 2.0**-24, "y")
            else:
                check(out[:1], *(v[:1] for v in hidden("silu", p, off, dt)), "h")


def test_rows_of_other_memory_are_left_alone():
    """h of every kernel ends at its last row and column."""
    N, K, bits = 272, 256, 4
    layer = Layer(fbq, N, K, bits, 32, torch.float16, seed=17, gated=True)
    for M in (1, 3, 21, 130):
        store = torch.full(((M + 2) * N // 2,), 7.0, dtype=torch.float16, device="cuda")
        h = store[N // 2: (M + 1) * N // 2].view(M, N // 2)
        fbq.gated(inputs(M, K, torch.float16, seed=M), *layer.tensors, N, 128, bits, h=h)
        torch.cuda.synchronize()
        assert bool((store[: N // 2] == 7).all()) and bool((store[(M + 1) * N // 2:] == 7).all()) and not bool((h == 7).all())


def test_options_that_choose_kernels():
    N, K, bits, dt = 272, 384, 3, torch.float16
    layer = Layer(fbq, N, K, bits, 32, dt, seed=18, gated=True)
    for name, value in (("gemv", 0), ("force_kernel", fbq.KERNEL_PREFILL), ("force_kernel", fbq.KERNEL_GENERIC), ("gemv_ctas", 4), ("prefill_pair", 1), ("pdl", 0)):
        before = fbq.get_option(name)
        fbq.set_option(name, value)
        try:
            for M in (1, 7, 200):
                x = inputs(M, K, dt, seed=M)
                check(fbq.gated(x, *layer.tensors, N, 128, bits), *hidden("silu", *layer.products(x), dt), "%s = %d, %d tokens" % (name, value, M))
        finally:
            fbq.set_option(name, before)


def test_same_bits_again():
    N, K, bits, dt = 2064, 1024, 4, torch.bfloat16
    layer = Layer(fbq, N, K, bits, 64, dt, seed=19, gated=True)
    for M in (1, 6, 50, 260):
        x = inputs(M, K, dt, seed=M)
        first = fbq.gated(x, *layer.tensors, N, 128, bits, save=True)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, fbq.gated(x, *layer.tensors, N, 128, bits, save=True)))
            assert torch.equal(fbq.gated(x, *layer.tensors, N, 128, bits), fbq.gated(x, *layer.tensors, N, 128, bits))


def test_in_a_graph_and_on_another_stream():
    N, K, bits, dt = 528, 512, 4, torch.float16
    layer = Layer(fbq, N, K, bits, 32, dt, seed=20, gated=True)
    stream = torch.cuda.Stream()
    for M in (1, 9, 40, 300):
        x = inputs(M, K, dt, seed=M)
        want = fbq.gated(x, *layer.tensors, N, 128, bits, save=True)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            fbq.gated(x, *layer.tensors, N, 128, bits, save=True)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                got = fbq.gated(x, *layer.tensors, N, 128, bits, save=True)
        fresh = inputs(M, K, dt, seed=M + 1)
        x.copy_(fresh)
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        want = fbq.gated(fresh, *layer.tensors, N, 128, bits, save=True)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        del graph


def test_no_tokens():
    layer = Layer(fbq, 32, 128, 4, 16, torch.float16, seed=21, gated=True)
    h, codes, scales = fbq.gated(torch.empty((0, 128), dtype=torch.float16, device="cuda"), *layer.tensors, 32, 128, 4, save=True)
    assert h.shape == (0, 16) and codes.shape == (0, 32) and scales.shape == (0, 1)


def test_half_step_of_the_types():
    assert half_step(torch.float16) == 2.0**-11 and half_step(torch.bfloat16) == 2.0**-8
