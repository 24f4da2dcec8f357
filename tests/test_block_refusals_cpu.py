"""What the calls of the feed-forward block refuse, and in what order: no GPU is needed to be told so."""
import ctypes

import pytest
import torch

import paper_2501_16385_b200 as fbq

BADARG, UNSUPPORTED, ALIGN, CUDA = -1, -2, -3, -4
# addresses that are never read: every call below is refused, or finds no device
P = [ctypes.c_void_p((i + 1) << 20) for i in range(16)]
ODD = ctypes.c_void_p((1 << 20) + 8)


def gated(M=4, N=32, K=128, group=128, bits=4, rank=16, gate=0, x=P[0], q=P[1], s=P[2], z=P[3], A=P[4], B=P[5], h=P[6], kept=None, scales=None):
    return fbq.lib().fbq_gated(x, q, s, z, A, B, h, kept, scales, M, N, K, group, bits, rank, gate, 0, None)


def linear_backward(M=4, N=32, K=128, group=128, bits=4, rank=16, dy=P[0], x=P[1], x8=None, x8s=None, q=P[2], s=P[3], z=P[4], A=P[5], B=P[6], dx=P[7], dA=P[8],
                    dB=P[9]):
    return fbq.lib().fbq_linear_backward(dy, x, x8, x8s, q, s, z, A, B, dx, dA, dB, M, N, K, group, bits, rank, 0, None)


def gated_backward(M=4, N=32, K=128, group=128, bits=4, rank=16, gate=1, dh=P[0], kept=P[1], kept_scales=P[2], x=P[3], x8=None, x8s=None, dx=P[9], dA=P[10], dB=P[11]):
    return fbq.lib().fbq_gated_backward(dh, kept, kept_scales, x, x8, x8s, *P[4:9], dx, dA, dB, M, N, K, group, bits, rank, gate, 0, None)


def gated_layer(F=16, K=128, group=128, bits=4, rank=8, first=P[0], A=P[13]):
    return fbq.lib().fbq_gated_layer(first, *P[1:13], A, P[14], F, K, group, bits, rank, None)


SHAPES = [
    (dict(bits=5), BADARG), (dict(bits=2), BADARG), (dict(K=100), BADARG), (dict(K=0), BADARG), (dict(N=0), BADARG), (dict(M=-1), BADARG), (dict(rank=-16), BADARG),
    (dict(group=64), UNSUPPORTED), (dict(K=192, group=64), UNSUPPORTED), (dict(N=24, rank=264), UNSUPPORTED), (dict(N=32, rank=272), UNSUPPORTED),
    (dict(M=(1 << 22) + 1), UNSUPPORTED),
]


@pytest.mark.parametrize("call", [gated, linear_backward, gated_backward])
@pytest.mark.parametrize("shape,code", SHAPES)
def test_shapes(call, shape, code):
    assert call(**shape) == code


def test_gated_domain():
    for call in (gated, gated_backward):
        assert call(N=24) == UNSUPPORTED and call(N=31) == BADARG and call(rank=8) == UNSUPPORTED and call(rank=9) == BADARG
        assert call(gate=2) == BADARG and call(gate=-1) == BADARG
    assert gated(N=(1 << 30) + 16) == UNSUPPORTED and gated(K=(1 << 30) + 128) == UNSUPPORTED
    assert linear_backward(N=12) == UNSUPPORTED and linear_backward(rank=4) == UNSUPPORTED
    assert linear_backward(N=1 << 22, K=128) == UNSUPPORTED                    # not even 256 columns of a 16-bit copy fit the scratch


def test_gated_pointers():
    for name in "xqszABh":
        assert gated(**{name: None}) == BADARG and gated(**{name: ODD}) == ALIGN
    assert gated(kept=P[7]) == BADARG and gated(scales=P[7]) == BADARG
    assert gated(kept=ODD, scales=P[7]) == ALIGN and gated(kept=P[7], scales=ODD) == ALIGN
    assert gated(M=0, x=None, h=None) == 0


def test_backward_pointers():
    for name in ("dy", "q", "s", "z", "A", "B"):
        assert linear_backward(**{name: None}) == BADARG and linear_backward(**{name: ODD}) == ALIGN
    for name in ("x", "dx", "dA", "dB"):
        assert linear_backward(**{name: ODD}) == ALIGN
    assert linear_backward(x=None) == BADARG                                   # the factors' gradients need x
    assert linear_backward(x8=P[10], x8s=P[11]) == BADARG                      # once, not twice
    assert linear_backward(x=None, x8=P[10]) == BADARG
    assert linear_backward(x=None, x8=ODD, x8s=P[11]) == ALIGN and linear_backward(x=None, x8=P[10], x8s=ODD) == ALIGN
    assert linear_backward(dA=None) == BADARG and linear_backward(dB=None) == BADARG
    assert linear_backward(x=None, dx=None, dA=None, dB=None) == 0             # nothing is wanted
    assert linear_backward(rank=0, x=None, A=None, B=None, dx=None, dA=None, dB=None) == 0
    for name in ("dh", "kept", "kept_scales"):
        assert gated_backward(**{name: None}) == BADARG and gated_backward(**{name: ODD}) == ALIGN
    assert gated_backward(x=None) == BADARG and gated_backward(dA=None) == BADARG
    assert linear_backward(M=0, rank=0, dy=None, x=None, dx=None) == 0


def test_layer_layout():
    assert gated_layer(F=0) == BADARG and gated_layer(F=12) == UNSUPPORTED and gated_layer(rank=4) == UNSUPPORTED and gated_layer(rank=136) == UNSUPPORTED
    assert gated_layer(bits=5) == BADARG and gated_layer(rank=-8) == BADARG and gated_layer(K=130) == BADARG and gated_layer(group=64) == UNSUPPORTED
    assert gated_layer(F=(1 << 30) + 8) == BADARG
    assert gated_layer(first=None) == BADARG and gated_layer(first=ODD) == ALIGN and gated_layer(A=None) == BADARG and gated_layer(A=ODD) == ALIGN


def test_8_bits():
    for call in (fbq.lib().fbq_act8_pack, fbq.lib().fbq_act8_unpack):
        assert call(P[0], P[1], P[2], -1, 4, 0, None) == BADARG and call(P[0], P[1], P[2], 4, 0, 0, None) == BADARG
        assert call(None, None, None, 0, 4, 0, None) == 0
        for i in range(3):
            for bad, code in ((None, BADARG), (ODD, ALIGN)):
                args = [P[0], P[1], P[2]]
                args[i] = bad
                assert call(*args, 4, 4, 0, None) == code


@pytest.mark.skipif(torch.cuda.is_available(), reason="with a device these would run on addresses that are none")
def test_without_a_device():
    assert gated() == CUDA and linear_backward() == CUDA and gated_backward() == CUDA and gated_layer() == CUDA
    assert fbq.lib().fbq_act8_pack(P[0], P[1], P[2], 4, 4, 0, None) == CUDA and fbq.lib().fbq_act8_unpack(P[0], P[1], P[2], 4, 4, 0, None) == CUDA


def test_names_of_gates():
    with pytest.raises(ValueError):
        fbq.gated(torch.zeros((1, 128), dtype=torch.float16), None, None, None, None, None, 32, 128, 4, fn="relu")


def test_tensors_that_are_not_on_a_device():
    x, layer = torch.zeros((1, 128), dtype=torch.float16), (torch.zeros(512, dtype=torch.int32), *(torch.zeros((32, 1), dtype=torch.float16) for _ in range(2)), None, None)
    with pytest.raises(ValueError):
        fbq.gated(x, *layer, 32, 128, 4)
    with pytest.raises(ValueError):
        fbq.act8_pack(x)
    with pytest.raises(ValueError):
        fbq.act8_unpack(torch.zeros((1, 4), dtype=torch.int8), torch.zeros((1, 1)), torch.float16)
    with pytest.raises(ValueError):
        fbq.linear_backward(torch.zeros((1, 32), dtype=torch.float16), x, *layer, 128, 4)
    with pytest.raises(TypeError):
        fbq.gated(x.float(), *layer, 32, 128, 4)
    with pytest.raises(TypeError):
        fbq.gated(None, *layer, 32, 128, 4)
    with pytest.raises(TypeError):
        fbq.act8_unpack(torch.zeros((1, 4), dtype=torch.int8), torch.zeros((1, 1)), torch.float32)
