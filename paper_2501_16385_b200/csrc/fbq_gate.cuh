// The gate of a feed-forward block, and the 8-bit form in which activations are kept for the backward pass.
#pragma once

#include "fbq_common.cuh"

namespace fbq {

// A gated layer's rows are eight of the gate, eight of the up projection, and so on; row n belongs to the up projection where
// n & kGateUp.  Rows of both branches then sit beside each other wherever a kernel keeps its sums: eight rows apart in an MMA
// fragment of 16 rows (the same lane), eight lanes apart in tensor memory.
constexpr int kGateUp = 8;

// f(v) = v S(z), S the logistic function: z = v (SiLU), or 2 sqrt(2/pi) (v + 0.044715 v^3), which makes 0.5 v (1 + tanh(z / 2)) of it
// (GELU).  Errors are a few 2^-24 of f, and for z < -1 of |z| 2^-23 of it: far below the rounding of a 16-bit output; below z = -87, where f is under 2^-119, it is 0.
constexpr float kGelu1 = 1.5957691216057308f, kGelu3 = 0.07135481282143484f;     // 2 sqrt(2/pi), times 0.044715
__device__ __forceinline__ float gate_arg(int fn, float v) { return fn == FBQ_GATE_GELU ? v * fmaf(kGelu3, v * v, kGelu1) : v; }
__device__ __forceinline__ float gate_value(int fn, float v) { return __fdividef(v, 1.f + __expf(-gate_arg(fn, v))); }
// f(v) and f'(v) = S + v S (1 - S) z'.  Above v = 32 the second term is below the last place of S in single precision for both functions (1 - S <= e^-32,
// times v z'), and it is left out: GELU's z' and an f that is infinite would make NaN of it.  Below -32 it is the larger one of SiLU's, |v| times S, and GELU has neither: S is 0, and
// z' may be infinite.
__device__ __forceinline__ void gate_both(int fn, float v, float &f, float &df)
{
    const float s = __fdividef(1.f, 1.f + __expf(-gate_arg(fn, v)));
    const float dz = fn == FBQ_GATE_GELU ? fmaf(3.f * kGelu3, v * v, kGelu1) : 1.f;
    f = v * s;
    df = (fn == FBQ_GATE_GELU ? fabsf(v) : v) > 32.f ? s : fmaf(f * (1.f - s), dz, s);
}

// Eight bits: kKeptGroup consecutive columns of a row share a scale.  scale = max|v| / 127, code = rint(v * (127 / max|v|)), each step
// one IEEE operation in single precision.  A group whose largest |v| is below 2^-100 is kept as zeros (127 / max|v| stays finite), a
// group that holds an Inf or a NaN as NaN: codes 0, scale NaN.  `top`: the largest |v|, as bits (which order like the values, NaN last).
constexpr int kKeptGroup = 128;
__device__ __forceinline__ void kept_scale(uint32_t top, float &scale, float &inverse)
{
    const float a = __uint_as_float(top);
    const bool some = a >= 7.888609052210118e-31f && top < 0x7F800000u;
    scale = some ? __fdiv_rn(a, 127.f) : (top < 0x7F800000u ? 0.f : __uint_as_float(0x7FFFFFFFu));
    inverse = some ? __fdiv_rn(127.f, a) : 0.f;
}
// The code as a byte.  Adding 1.5 2^23 rounds to a whole number, ties to even, and leaves it in the low bits (a conversion runs at a quarter
// of the rate).
__device__ __forceinline__ uint32_t kept_code(float v, float inverse)
{
    return inverse != 0.f ? __float_as_uint(__fadd_rn(__fmul_rn(v, inverse), 12582912.f)) & 0xFFu : 0u;
}

// A chunk of sums in tensor memory's layout, lane = row of the gated layer, v[j] = token j of 32: the lanes of a pair (eight apart) swap
// halves of their tokens, so that each gates sixteen.  out: where this warp's 16 columns of h of token 0 begin, tokens 64 columns apart.
template <typename T> __device__ __forceinline__ void gate_chunk(int fn, const uint32_t (&v)[32], T *out)
{
    const int lane = threadIdx.x & 31;
    const bool up = (lane & kGateUp) != 0;
    T *dst = out + (up ? 16 * 64 : 0) + (lane >> 4) * kGateUp + (lane & (kGateUp - 1));
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const float got = __uint_as_float(__shfl_xor_sync(0xffffffffu, up ? v[j] : v[16 + j], kGateUp));
        const float mine = __uint_as_float(up ? v[16 + j] : v[j]);
        dst[j * 64] = ActTraits<T>::from_float(gate_value(fn, up ? got : mine) * (up ? mine : got));
    }
}

}  // namespace fbq
