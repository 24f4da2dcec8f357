"""Cases for timing the operators of a quantised feed-forward block: the gated block, its backward pass, the backward
pass of a linear, and activations kept in 8 bits between the two passes.

A gated layer is an FBQuant layer of N = 2 F rows that holds both projections of a gated feed-forward block, eight rows
of the gate, eight of the up projection, and so on; A has the gate's r rows and then those of the up projection, and a row of B
holds its own branch's r values in that branch's half and zeros in the other.  With p = x.dequant(Q,s,z)^T + (x.A^T).B^T,

    h[m][8i + j] = f(p[m][16i + j]) * p[m][16i + 8 + j],   j = 0..7,   f = SiLU or GELU (tanh form)

Sizes are those of Llama-2-7B and -13B layers, as in the benchmark, and prompts and training sequences of other lengths.
"""
import math

import torch

own = False

GROUP = 128
KEPT = 128          # values that share a scale when activations are kept in 8 bits


def listed():
    return [
        # Serving one request: both projections of a 7B block for a single token.
        dict(name="gated, 1 token", kind="gated", d=4096, ff=11008, tokens=1, bits=4, rank=64, dtype="f16", fn="silu", save=False),
        # A few requests together, on the wider model.
        dict(name="gated, 8 tokens", kind="gated", d=5120, ff=13824, tokens=8, bits=3, rank=32, dtype="bf16", fn="silu", save=False),
        # A short prompt of odd length; the other activation.
        dict(name="gated, 77 tokens", kind="gated", d=4096, ff=11008, tokens=77, bits=3, rank=64, dtype="f16", fn="gelu", save=False),
        # The usual prompt.
        dict(name="gated, 1024 tokens", kind="gated", d=4096, ff=11008, tokens=1024, bits=4, rank=64, dtype="bf16", fn="silu", save=False),
        # The forward pass of a training step on the wider model: the pre-activations are kept in 8 bits.
        dict(name="gated, 4000 tokens, kept", kind="gated", d=5120, ff=13824, tokens=4000, bits=4, rank=64, dtype="bf16", fn="silu", save=True),
        # The backward pass for a short sequence of odd length, x kept as it was.
        dict(name="gated backward, 333 tokens", kind="gated_backward", d=4096, ff=11008, tokens=333, bits=4, rank=64, dtype="bf16", fn="silu", x8=False),
        # The same for two sequences of 2048, x kept in 8 bits.
        dict(name="gated backward, 4096 tokens", kind="gated_backward", d=4096, ff=11008, tokens=4096, bits=3, rank=64, dtype="f16", fn="silu", x8=True),
        # A small projection's backward pass, few tokens: what an adaptation on short samples runs.
        dict(name="linear backward, 61 tokens", kind="linear_backward", n=4096, k=4096, tokens=61, bits=3, rank=16, dtype="f16", x8=False),
        # The down projection's, one sequence of 1024.
        dict(name="linear backward, 1024 tokens", kind="linear_backward", n=4096, k=11008, tokens=1024, bits=4, rank=64, dtype="bf16", x8=False),
        # The wider model's, two sequences of 2048, input kept in 8 bits.
        dict(name="linear backward, 4096 tokens", kind="linear_backward", n=5120, k=13824, tokens=4096, bits=4, rank=128, dtype="bf16", x8=True),
        # Activations to 8 bits and back: one token (the smallest call), and the input of a down projection for two sequences.
        dict(name="8 bits, 1 token", kind="act8", k=4096, tokens=1, dtype="f16"),
        dict(name="8 bits, 4096 tokens", kind="act8", k=11008, tokens=4096, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["gated", "gated", "gated", "gated_backward", "gated_backward", "linear_backward", "linear_backward", "act8"])
    dtype = rng.choice(("f16", "bf16"))
    if kind == "act8":
        return dict(kind=kind, k=_log(rng, 100, 11008), tokens=_log(rng, 1, 4096), dtype=dtype)
    case = dict(kind=kind, bits=rng.choice((3, 4)), dtype=dtype)
    if kind == "linear_backward":
        return dict(case, n=8 * _log(rng, 64, 1728), k=GROUP * _log(rng, 6, 40), rank=rng.choice((0, 16, 32, 48, 64, 128)), tokens=_log(rng, 1, 4096),
                    x8=rng.random() < 0.5)
    d = GROUP * rng.randint(10, 40 if kind == "gated" else 32)
    ff = min(13824 if kind == "gated" else 11008, 8 * int(round(d * rng.uniform(2.2, 3.6) / 8)))
    case = dict(case, d=d, ff=ff, rank=rng.choice((0, 8, 16, 32, 64, 128)), fn=rng.choice(("silu", "silu", "gelu")))
    if kind == "gated_backward":
        return dict(case, tokens=_log(rng, 1, 4096), x8=rng.random() < 0.5)
    save = rng.random() < 0.4
    return dict(case, tokens=_log(rng, 1, 4000), save=save)


# ---- inputs --------------------------------------------------------------------------------------------------
def _act(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _sizes(case):
    """Rows, columns and rank of the layer as the calls see it."""
    if case["kind"] == "linear_backward":
        return case["n"], case["k"], case["rank"]
    return 2 * case["ff"], case["d"], 2 * case["rank"]


def _layer(case, g):
    """(qweight, scales, zeros, A, B).  Random words are random codes in both packed formats."""
    N, K, r = _sizes(case)
    G, bits, act = K // GROUP, case["bits"], _act(case)
    qweight = torch.randint(-2**31, 2**31, (N * K // 32 * bits,), dtype=torch.int32, device="cuda", generator=g)
    scales = (torch.rand((N, G), device="cuda", generator=g) * 0.015 + 0.005).half()
    lo, hi = (6, 10) if bits == 4 else (2, 6)
    zeros = torch.randint(lo, hi, (N, G), device="cuda", generator=g).half()
    if r == 0:
        return qweight, scales, zeros, None, None
    A = (torch.randn((r, K), device="cuda", generator=g) * 0.02).to(act)
    B = (torch.randn((N, r), device="cuda", generator=g) * 0.02).to(act)
    if case["kind"] != "linear_backward":
        B = B * _own_half(N, r)
    return qweight, scales, zeros, A, B


def _own_half(N, r):
    """[N][r]: whether a place of B belongs to the branch of its row."""
    up = (torch.arange(N, device="cuda") // 8 % 2).bool()
    return (torch.arange(r, device="cuda") >= r // 2)[None, :] == up[:, None]


def _activations(case, K, g):
    """x ~ N(0, 1); more than a few tokens carry the outlier channels of real activations (1 % of them, 20 times as large)."""
    x = torch.randn((case["tokens"], K), device="cuda", generator=g)
    if case["tokens"] > 16:
        x[:, torch.randperm(K, device="cuda", generator=g)[: max(1, K // 100)]] *= 20.0
    return x.to(_act(case))


def _to_8_bits(v):
    """int8 codes [M][K] and one float32 scale per KEPT columns of a row: scale = max|v| / 127, code = rint(v * (127 / max|v|))."""
    M, K = v.shape
    pad = -K % KEPT
    w = torch.nn.functional.pad(v.float(), (0, pad)).view(M, -1, KEPT)
    top = w.abs().amax(2)
    all127 = torch.full_like(top, 127.0)
    some = top >= 2.0**-100
    scales = torch.where(some, top / all127, torch.zeros_like(top))
    inverse = torch.where(some, all127 / top, torch.zeros_like(top))
    codes = torch.round(w * inverse[:, :, None]).to(torch.int8)
    return codes.view(M, -1)[:, :K].contiguous(), scales


def _from_8_bits(codes, scales):
    return codes.float() * scales.repeat_interleave(KEPT, 1)[:, : codes.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]
    state = dict(case=case, kind=kind)
    if kind == "act8":
        state["x"] = _activations(case, case["k"], g)
        return state
    N, K, r = _sizes(case)
    state["layer"] = _layer(case, g)
    state["x"] = _activations(case, K, g)
    if kind == "gated":
        return state
    # gradients of a loss that has been scaled into the range of 16-bit types
    F = N if kind == "linear_backward" else N // 2
    state["dy"] = (torch.randn((case["tokens"], F), device="cuda", generator=g) * 0.05).to(_act(case))
    if kind == "gated_backward":
        state["kept"] = _to_8_bits(torch.randn((case["tokens"], N), device="cuda", generator=g) * 2.0)
    if case["x8"]:
        state["x"] = _to_8_bits(state["x"])
    return state


# ---- the framework's calls -----------------------------------------------------------------------------------
def _run_own(state):
    import paper_2501_16385_b200 as fbq
    case, kind = state["case"], state["kind"]
    if kind == "act8":
        codes, scales = fbq.act8_pack(state["x"])
        return [fbq.act8_unpack(codes, scales, _act(case)), scales]
    qweight, scales, zeros, A, B = state["layer"]
    if kind == "gated":
        N = scales.shape[0]
        if not case["save"]:
            return [fbq.gated(state["x"], qweight, scales, zeros, A, B, N, GROUP, case["bits"], fn=case["fn"])]
        h, codes, kept = fbq.gated(state["x"], qweight, scales, zeros, A, B, N, GROUP, case["bits"], fn=case["fn"], save=True)
        return [h, fbq.act8_unpack(codes, kept, _act(case))]
    if kind == "gated_backward":
        grads = fbq.gated_backward(state["dy"], state["kept"], state["x"], qweight, scales, zeros, A, B, GROUP, case["bits"], fn=case["fn"])
    else:
        grads = fbq.linear_backward(state["dy"], state["x"], qweight, scales, zeros, A, B, GROUP, case["bits"])
    return [t for t in grads if t is not None]


# ---- the plain form, in 32 bits ------------------------------------------------------------------------------
def _codes(qweight, N, K, bits):
    """Codes [N][K]: eight per word of four bits each; of three bits, 32 in three words (ten in a word's two halves, the
    last two in the halves' highest bits)."""
    if bits == 4:
        at = torch.arange(0, 32, 4, dtype=torch.int32, device=qweight.device)
        return (qweight.view(N, K // 8, 1) >> at & 15).view(N, K)
    w = qweight.view(N, K // 32, 3, 1)
    low = w >> torch.arange(0, 15, 3, dtype=torch.int32, device=w.device) & 7
    high = w >> torch.arange(16, 31, 3, dtype=torch.int32, device=w.device) & 7
    ten = torch.cat((low, high), 3).view(N, K // 32, 30)
    weight = torch.tensor([1, 2, 4], dtype=torch.int32, device=w.device)
    c30 = ((w[..., 0] >> 15 & 1) * weight).sum(2, keepdim=True)
    c31 = ((w[..., 0] >> 31 & 1) * weight).sum(2, keepdim=True)
    return torch.cat((ten, c30.int(), c31.int()), 2).view(N, K)


def _dense(layer, bits):
    """Dequantised weights plus sub-branch, float32 [N][K]."""
    qweight, scales, zeros, A, B = layer
    N, G = scales.shape
    q = _codes(qweight, N, G * GROUP, bits).view(N, G, GROUP).float()
    W = ((q - zeros.float()[:, :, None]) * scales.float()[:, :, None]).view(N, G * GROUP)
    return W


def _forward(x, layer, bits):
    A, B = layer[3:]
    p = x.float() @ _dense(layer, bits).t()
    return p if A is None else p + (x.float() @ A.float().t()) @ B.float().t()


_GELU = math.sqrt(2.0 / math.pi)


def _gate(fn, v):
    """f(v) and its derivative."""
    if fn == "silu":
        s = torch.sigmoid(v)
        return v * s, s * (1.0 + v * (1.0 - s))
    t = torch.tanh(_GELU * (v + 0.044715 * v * v * v))
    return 0.5 * v * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * v * (1.0 - t * t) * _GELU * (1.0 + 3 * 0.044715 * v * v)


def _halves(p):
    """The gate's and the up projection's columns of [M][2F]."""
    v = p.view(p.shape[0], -1, 2, 8)
    return v[:, :, 0].reshape(p.shape[0], -1), v[:, :, 1].reshape(p.shape[0], -1)


def _interleaved(a, b):
    return torch.stack((a.view(a.shape[0], -1, 8), b.view(b.shape[0], -1, 8)), 2).view(a.shape[0], -1)


def _gradients(dy, x, layer, bits, act, mask):
    """(dx, dA, dB) of a layer for the gradient dy [M][N], in 32 bits, rounded once."""
    A, B = layer[3:]
    dx = dy @ _dense(layer, bits)
    if A is None:
        return [dx.to(act)]
    A, B = A.float(), B.float()
    s, t = dy @ B, x @ A.t()
    dB = dy.t() @ t
    return [(dx + s @ A).to(act), (s.t() @ x).to(act), (dB * mask if mask is not None else dB).to(act)]


def _run_plain(state):
    case, kind = state["case"], state["kind"]
    act = _act(case)
    if kind == "act8":
        codes, scales = _to_8_bits(state["x"])
        return [_from_8_bits(codes, scales).to(act), scales]
    layer, bits = state["layer"], case["bits"]
    if kind == "gated":
        p = _forward(state["x"], layer, bits)
        gate, up = _halves(p)
        h = (_gate(case["fn"], gate)[0] * up).to(act)
        return [h, _from_8_bits(*_to_8_bits(p)).to(act)] if case["save"] else [h]
    x = _from_8_bits(*state["x"]) if case["x8"] else state["x"].float()
    dy = state["dy"].float()
    if kind == "linear_backward":
        return _gradients(dy, x, layer, bits, act, None)
    gate, up = _halves(_from_8_bits(*state["kept"]))
    f, df = _gate(case["fn"], gate)
    mask = _own_half(*layer[4].shape) if layer[4] is not None else None
    return _gradients(_interleaved(dy * up * df, dy * f), x, layer, bits, act, mask)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    kind, M = case["kind"], case["tokens"]
    if kind == "act8":
        # to 8 bits: 2 bytes read, 1 written; back: 1 read, 2 written; the scales written, then read
        return {"bytes": M * (6 * case["k"] + 8 * (-(-case["k"] // KEPT))), "flops": 4 * M * case["k"]}
    N, K, r = _sizes(case)
    weights = N * K * case["bits"] / 8 + 4 * N * (K // GROUP) + 2 * r * (N + K)
    # a branch of a gated layer has half of A's rows and half of B's columns
    branch = r * K + (r * N if kind == "linear_backward" else r * N / 2)
    if kind == "gated":
        kept = M * (N + 4 * (-(-N // KEPT))) if case["save"] else 0
        # (the unpacking of what was kept: read once more, written in 16 bits)
        return {"bytes": weights + 2 * M * K + M * N + kept * 2 + (2 * M * N if case["save"] else 0), "flops": 2 * M * N * K + 2 * M * branch}
    F = N if kind == "linear_backward" else N // 2
    x_bytes = M * (K + 4 * (K // KEPT)) if case["x8"] else 2 * M * K
    kept = M * (N + 4 * (-(-N // KEPT))) if kind == "gated_backward" else 0
    # dx = dy.W + (dy.B).A; t = x.A^T; dA = (dy.B)^T.x; dB = dy^T.t
    return {"bytes": weights + 2 * M * F + kept + x_bytes + 2 * M * K + 2 * r * (N + K), "flops": 2 * M * N * K + 6 * M * branch}


# ---- the definition, in 64 bits --------------------------------------------------------------------------------
def _weights64(layer, bits):
    qweight, scales, zeros = layer[:3]
    N, G = scales.shape
    K = G * GROUP
    words = qweight.long() & 0xFFFFFFFF
    q = torch.empty((N, K), dtype=torch.float64, device=words.device)
    if bits == 4:
        words = words.view(N, -1)
        for i in range(8):
            q[:, i::8] = words.bitwise_right_shift(4 * i).bitwise_and(15).double()
    else:
        words = words.view(N, -1, 3)
        for c in range(30):
            word, place = divmod(c, 10)
            q[:, c::32] = words[:, :, word].bitwise_right_shift(3 * place if place < 5 else 1 + 3 * place).bitwise_and(7).double()
        for c, place in ((30, 15), (31, 31)):
            q[:, c::32] = sum((words[:, :, i].bitwise_right_shift(place).bitwise_and(1) << i) for i in range(3)).double()
    q = q.view(N, G, GROUP)
    q -= zeros.double().unsqueeze(2)
    q *= scales.double().unsqueeze(2)
    return q.view(N, K)


def _kept64(codes, scales):
    M, K = codes.shape
    out = codes.double()
    for i in range(scales.shape[1]):
        out[:, i * KEPT: (i + 1) * KEPT] *= scales[:, i: i + 1].double()
    return out


def _f64(fn, v):
    if fn == "silu":
        return v / (1.0 + torch.exp(-v))
    return 0.5 * v * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (v + 0.044715 * v**3)))


def _df64(fn, v):
    if fn == "silu":
        e = torch.exp(-v.abs())
        s = torch.where(v >= 0, 1.0 / (1.0 + e), e / (1.0 + e))
        return s + v * s * (1.0 - s)
    u = (2.0 / math.pi) ** 0.5 * (v + 0.044715 * v**3)
    return 0.5 * (1.0 + torch.tanh(u)) + 0.5 * v / torch.cosh(u.clamp(-300, 300)) ** 2 * (2.0 / math.pi) ** 0.5 * (1.0 + 0.134145 * v * v)


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "act8":
        x = state["x"].double()
        M, K = x.shape
        out, scales = torch.zeros_like(x), []
        for k in range(0, K, KEPT):
            v = x[:, k: k + KEPT]
            step = v.abs().amax(1, keepdim=True) / 127.0
            out[:, k: k + KEPT] = torch.where(step > 0, torch.round(v / step.clamp_min(1e-300)) * step, torch.zeros_like(v))
            scales.append(step)
        return [out, torch.cat(scales, 1)]
    layer = state["layer"]
    W = _weights64(layer, case["bits"])
    A, B = (None, None) if layer[3] is None else (layer[3].double(), layer[4].double())
    if kind == "gated":
        x = state["x"].double()
        p = x @ W.t()
        if A is not None:
            p += (x @ A.t()) @ B.t()
        v = p.view(p.shape[0], -1, 16)
        h = (_f64(case["fn"], v[:, :, :8]) * v[:, :, 8:]).reshape(p.shape[0], -1)
        # What is kept is a value's nearest multiple of its group's step; which of two neighbours that is turns on the value's last
        # bits, so what is kept has no value of its own in 64 bits.
        return [h, None] if case["save"] else [h]
    x = _kept64(*state["x"]) if case["x8"] else state["x"].double()
    dy = state["dy"].double()
    if kind == "gated_backward":
        v = _kept64(*state["kept"]).view(dy.shape[0], -1, 16)
        d = dy.view(dy.shape[0], -1, 8)
        dy = torch.cat((d * v[:, :, 8:] * _df64(case["fn"], v[:, :, :8]), d * _f64(case["fn"], v[:, :, :8])), 2).reshape(dy.shape[0], -1)
    dx = dy @ W
    if A is None:
        return [dx]
    dx += (dy @ B) @ A
    dA, dB = (dy @ B).t() @ x, dy.t() @ (x @ A.t())
    if kind == "gated_backward":
        r = A.shape[0] // 2
        v = dB.view(-1, 16, 2 * r)
        v[:, :8, r:] = 0.0
        v[:, 8:, :r] = 0.0
    return [dx, dA, dB]
