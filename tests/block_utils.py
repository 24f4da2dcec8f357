"""Plain implementations in 64 bits of the feed-forward operators, and the bounds that their results are held to.

A bound counts, entry by entry, what the kernels round: `u` = half a step of the activation type, relative, for every
operand that is rounded to it (dequantised weights, t, s, dp) and for the result; and `acc(n)` for n products added in
single precision.  Sums of absolute values carry them through the products.
"""
from __future__ import annotations

import math

import torch

KEPT = 128


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def least(dtype) -> float:
    """Half a step between the type's smallest numbers: what a rounding is off by where it is not relative."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def acc(n: int) -> float:
    return n * 2.0**-23


class Layer:
    """Random layer on the device: packed tensors for the library, float64 W, A, B for the reference."""

    def __init__(self, fbq, N, K, bits, rank, dtype, seed, gated=False, ab=0.02):
        g = torch.Generator(device="cuda").manual_seed(seed)
        top = 1 << bits
        codes = torch.randint(0, top, (N, K), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
        self.qweight = fbq.pack(codes, bits)
        self.scales = (torch.rand((N, K // 128), generator=g, device="cuda") * 0.015 + 0.005).half()
        self.zeros = torch.randint(top // 2 - 2, top // 2 + 2, (N, K // 128), generator=g, device="cuda").half()
        self.A = self.B = None
        if rank:
            self.A = (torch.randn((rank, K), generator=g, device="cuda") * ab).to(dtype)
            self.B = (torch.randn((N, rank), generator=g, device="cuda") * ab).to(dtype)
            if gated:
                self.B = self.B * own_half(N, rank)
        self.N, self.K, self.bits, self.rank, self.dtype = N, K, bits, rank, dtype
        q = codes.double().view(N, K // 128, 128)
        self.W = ((q - self.zeros.double()[:, :, None]) * self.scales.double()[:, :, None]).view(N, K)
        self.A64 = self.A.double() if rank else torch.zeros((1, K), device="cuda", dtype=torch.float64)
        self.B64 = self.B.double() if rank else torch.zeros((N, 1), device="cuda", dtype=torch.float64)

    @property
    def tensors(self):
        return self.qweight, self.scales, self.zeros, self.A, self.B

    def products(self, x):
        """p = x.W^T + (x.A^T).B^T in 64 bits, and a bound on the error of the kernels' p."""
        x = x.double()
        p = x @ self.W.t() + (x @ self.A64.t()) @ self.B64.t()
        u = half_step(self.dtype)
        size = (x.abs() @ self.W.abs().t()) * (u + acc(self.K)) + (x.abs() @ self.A64.abs().t()) @ self.B64.abs().t() * (u + acc(self.K + self.rank))
        # decode kernels hold x to 2^-17 of the largest of its group of 128
        top = x.abs().view(x.shape[0], -1, 128).amax(2)
        size += (top @ self.W.abs().view(self.N, -1, 128).sum(2).t()) * 2.0**-17
        return p, size + least(self.dtype) * self.B64.abs().sum(1)


def own_half(N, rank):
    up = (torch.arange(N, device="cuda") // 8 % 2).bool()
    return (torch.arange(rank, device="cuda") >= rank // 2)[None, :] == up[:, None]


def f64(fn, v):
    """f and f' in 64 bits."""
    if fn == "silu":
        s = torch.sigmoid(v)
        return v * s, s + v * s * (1 - s)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (v + 0.044715 * v**3))
    return 0.5 * v * (1 + t), 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * c * (1 + 3 * 0.044715 * v * v)


def branches(p):
    v = p.view(p.shape[0], -1, 2, 8)
    return v[:, :, 0].reshape(p.shape[0], -1), v[:, :, 1].reshape(p.shape[0], -1)


def interleave(a, b):
    return torch.stack((a.view(a.shape[0], -1, 8), b.view(b.shape[0], -1, 8)), 2).view(a.shape[0], -1)


SLOPE = 1.13          # |f'| of SiLU (1.10) and GELU (1.129) is below this


def hidden(fn, p, dp, dtype):
    """h in 64 bits from p known to dp, and a bound on the kernels' error."""
    gate, up = branches(p)
    dg, du = branches(dp)
    f = f64(fn, gate)[0]
    h = f * up
    size = up.abs() * SLOPE * dg + (f.abs() + SLOPE * dg) * du
    # f itself: a few 2^-24, and |z| 2^-23 of it where the exponential's argument z is large (|z| < 100, else f is 0 or v)
    size += (h.abs() + size) * 128 * 2.0**-23
    return h, size + (h.abs() + size) * half_step(dtype) + least(dtype)


def kept64(codes, scales):
    return codes.double() * scales.double().repeat_interleave(KEPT, 1)[:, : codes.shape[1]]


def to_8_bits(v):
    """The 8-bit form by its definition, on a float32 tensor, IEEE single precision."""
    M, K = v.shape
    w = torch.nn.functional.pad(v.float(), (0, -K % KEPT)).view(M, -1, KEPT)
    top = w.abs().amax(2)
    n127 = torch.full_like(top, 127.0)
    some = torch.isfinite(top) & (top >= 2.0**-100)
    scales = torch.where(some, top / n127, torch.where(torch.isfinite(top), 0.0, math.nan))
    inverse = torch.where(some, n127 / top, 0.0)
    codes = torch.where(some[:, :, None], torch.round(w * inverse[:, :, None]), 0.0).to(torch.int8)
    return codes.view(M, -1)[:, :K].contiguous(), scales


def gate_gradients(fn, dh, codes, scales, dtype):
    """dp in 64 bits and a bound on the error of the rounded dp that the kernels multiply."""
    gate, up = branches(kept64(codes, scales))
    f, df = f64(fn, gate)
    dh = dh.double()
    dp = interleave(dh * up * df, dh * f)
    # the kept values are products in single precision, f and f' are off by some 2^-24 of 1 + |v|
    off = interleave(dh.abs() * up.abs() * (1 + gate.abs()), dh.abs() * (1 + gate.abs())) * 64 * 2.0**-24
    return dp, off + (dp.abs() + off) * half_step(dtype) + least(dtype)


def layer_gradients(layer, dy, ddy, x, dx_of_x, mask):
    """(dx, dA, dB) in 64 bits with bounds: dy is known to ddy, x to dx_of_x (0 where the kernels have it exactly)."""
    u, e = half_step(layer.dtype), least(layer.dtype)
    M = dy.shape[0]
    W, A, B, r = layer.W, layer.A64, layer.B64, layer.rank
    s, t = dy @ B, x @ A.t()
    # s and t as they are multiplied: sums in single precision, rounded once
    ds = ddy @ B.abs() + (dy.abs() @ B.abs()) * acc(layer.N)
    ds = ds + (s.abs() + ds) * u + e
    dt = dx_of_x @ A.abs().t() + (x.abs() @ A.abs().t()) * acc(layer.K)
    dt = dt + (t.abs() + dt) * u + e

    def rounded(v, size):
        return v, size + (v.abs() + size) * u + e

    ya, wa = dy.abs() + ddy, W.abs()
    dx = dy @ W + (s @ A if r else 0)
    size = ddy @ wa + (ya @ wa) * (u + acc(layer.N)) + ya.sum(1, keepdim=True) * e + (ds @ A.abs() + (s.abs() @ A.abs()) * acc(layer.N + r) if r else 0)
    out = [rounded(dx, size)]
    if r:
        xa = x.abs() + dx_of_x
        size = ds.t() @ xa + s.abs().t() @ dx_of_x + (s.abs().t() @ xa) * acc(M)
        out.append(rounded(s.t() @ x, size))
        size = ya.t() @ dt + ddy.t() @ t.abs() + (ya.t() @ t.abs()) * acc(M)
        dB = dy.t() @ t
        if mask is not None:
            dB, size = dB * mask, size * mask
        out.append(rounded(dB, size))
    return out


def check(got, want, size, what):
    bad = (got.double() - want).abs() > size
    n = int(bad.sum())
    assert n == 0, "%s: %d of %d entries beyond their bound, worst %.2f of it" % (
        what, n, bad.numel(), float(((got.double() - want).abs() / size.clamp_min(1e-300)).max()))
    assert bool(torch.isfinite(got.double()).all()), what + " is not finite"
