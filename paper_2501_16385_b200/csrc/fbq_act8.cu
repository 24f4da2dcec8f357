// Activations in 8 bits: the form in which a training step keeps them between its passes, and what the gated block's backward
// pass makes of it.  All three kernels are bound by memory: one pass, 16 bytes a lane and access where rows allow.
#include "fbq_common.cuh"
#include "fbq_dequant.cuh"
#include "fbq_gate.cuh"

namespace fbq {
namespace {

constexpr int kThr = 256;
constexpr int kLanes = 16, kEach = kKeptGroup / kLanes;       // lanes of a group, values of a lane

template <typename T> __device__ __forceinline__ float2 unpair(uint32_t v);
template <> __device__ __forceinline__ float2 unpair<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }
template <> __device__ __forceinline__ float2 unpair<__nv_bfloat16>(uint32_t v)
{
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}

// Sixteen lanes take a group: the largest |v| crosses lanes once, codes and values do not.  WIDE: rows of whole units of eight.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThr) pack_kernel(const T *__restrict__ x, int8_t *__restrict__ codes, float *__restrict__ scales, long long groups, int K, int G)
{
    const long long at = (long long)blockIdx.x * (kThr / kLanes) + threadIdx.x / kLanes;
    const int l = threadIdx.x % kLanes;
    const bool on = at < groups;
    const long long m = on ? at / G : 0;
    const int g = on ? (int)(at - m * G) : 0, k = g * kKeptGroup + l * kEach, n = on ? min(kEach, K - k) : 0;     // n <= 0: nothing
    const T *src = x + m * K + k;
    float v[kEach] = {};
    if (WIDE) {
        if (n > 0) {
            const uint4 w = __ldg(reinterpret_cast<const uint4 *>(src));
            const float2 a = unpair<T>(w.x), b = unpair<T>(w.y), c = unpair<T>(w.z), d = unpair<T>(w.w);
            v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (i < n) v[i] = ActTraits<T>::to_float(src[i]);
    }
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < kEach; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
#pragma unroll
    for (int o = 1; o < kLanes; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    float scale, inverse;
    kept_scale(top, scale, inverse);
    if (on && l == 0) scales[at] = scale;
    int8_t *dst = codes + m * K + k;
    if (WIDE) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < kEach; ++i) w[i / 4] |= ((uint32_t)kept_code(v[i], inverse) & 0xFFu) << (8 * (i % 4));
        if (n > 0) *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (i < n) dst[i] = (int8_t)kept_code(v[i], inverse);
    }
}

__device__ __forceinline__ float byte_to_float(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

// A lane turns EACH codes of a row (16, 8 or 1; K a multiple of it): code * scale, rounded once.
template <typename T, int EACH>
__global__ void __launch_bounds__(kThr) unpack_kernel(const int8_t *__restrict__ codes, const float *__restrict__ scales, T *__restrict__ x, long long units, int K, int G)
{
    const long long at = (long long)blockIdx.x * kThr + threadIdx.x;
    if (at >= units) return;
    const int per = K / EACH;
    const long long m = at / per;
    const int k = (int)(at - m * per) * EACH;
    const float s = __ldg(scales + m * G + k / kKeptGroup);
    if constexpr (EACH == 1) {
        x[at] = ActTraits<T>::from_float((float)codes[at] * s);
    } else {
        uint32_t w[EACH / 4], o[EACH / 2];
        if constexpr (EACH == 16) {
            const uint4 q = __ldg(reinterpret_cast<const uint4 *>(codes + at * EACH));
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else {
            const uint2 q = __ldg(reinterpret_cast<const uint2 *>(codes + at * EACH));
            w[0] = q.x; w[1] = q.y;
        }
#pragma unroll
        for (int i = 0; i < EACH / 2; ++i) o[i] = P2<T>::pack(byte_to_float(w[i / 2], 2 * i % 4) * s, byte_to_float(w[i / 2], 2 * i % 4 + 1) * s);
#pragma unroll
        for (int i = 0; i < EACH / 8; ++i) reinterpret_cast<uint4 *>(x + at * EACH)[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
    }
}

// dp of the gated block: p[16i + j] the gate's, p[16i + 8 + j] the up projection's value that met in h[8i + j], both as they were kept:
// dp_gate = dh p_up f'(p_gate), dp_up = dh f(p_gate), rounded once (they are operands of tensor-core products next).  A lane
// takes eight columns of h.
template <typename T>
__global__ void __launch_bounds__(kThr) gate_grad_kernel(const T *__restrict__ dh, const int8_t *__restrict__ codes, const float *__restrict__ scales, T *__restrict__ dp,
                                                         long long units, int per, int G, int fn)
{
    const long long at = (long long)blockIdx.x * kThr + threadIdx.x;
    if (at >= units) return;
    const long long m = at / per;
    const float s = __ldg(scales + m * G + (int)(at - m * per) / (kKeptGroup / 16));
    const uint4 q = __ldg(reinterpret_cast<const uint4 *>(codes) + at), d = __ldg(reinterpret_cast<const uint4 *>(dh) + at);
    const uint32_t gate[2] = {q.x, q.y}, up[2] = {q.z, q.w}, dd[4] = {d.x, d.y, d.z, d.w};
    uint32_t og[4], ou[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 e = unpair<T>(dd[i]);
        float f0, f1, df0, df1;
        gate_both(fn, byte_to_float(gate[i / 2], 2 * i % 4) * s, f0, df0);
        gate_both(fn, byte_to_float(gate[i / 2], 2 * i % 4 + 1) * s, f1, df1);
        og[i] = P2<T>::pack(e.x * (byte_to_float(up[i / 2], 2 * i % 4) * s) * df0, e.y * (byte_to_float(up[i / 2], 2 * i % 4 + 1) * s) * df1);
        ou[i] = P2<T>::pack(e.x * f0, e.y * f1);
    }
    uint4 *dst = reinterpret_cast<uint4 *>(dp) + 2 * at;
    dst[0] = make_uint4(og[0], og[1], og[2], og[3]);
    dst[1] = make_uint4(ou[0], ou[1], ou[2], ou[3]);
}

// Rows of `units` pieces of P: eight of the gate, eight of the up projection, and so on.  `half` > 0: a row of the result has twice the
// pieces, its own in its branch's half, zeros in the other.
template <typename P>
__global__ void __launch_bounds__(kThr) interleave_kernel(const P *__restrict__ gate, const P *__restrict__ up, P *__restrict__ out, long long total, int units, int padded)
{
    const long long at = (long long)blockIdx.x * kThr + threadIdx.x;
    if (at >= total) return;
    const int wide = padded ? 2 * units : units;
    const long long n = at / wide, row = n / (2 * kGateUp) * kGateUp + n % kGateUp;
    int u = (int)(at - n * wide);
    const bool is_up = (n & kGateUp) != 0;
    if (padded) {
        if ((u >= units) != is_up) {
            out[at] = P{};
            return;
        }
        if (is_up) u -= units;
    }
    out[at] = (is_up ? up : gate)[row * units + u];
}

unsigned blocks_for(long long n, int per) { return (unsigned)((n + per - 1) / per); }
// Grids have 31 bits.
bool fits(long long n, int per) { return n <= (long long)per * 0x7FFFFFFF; }

template <typename T> cudaError_t pack(const void *x, int8_t *codes, float *scales, int M, int K, cudaStream_t s)
{
    const int G = (K + kKeptGroup - 1) / kKeptGroup;
    const long long groups = (long long)M * G;
    if (!fits(groups, kThr / kLanes)) return cudaErrorInvalidConfiguration;
    const unsigned grid = blocks_for(groups, kThr / kLanes);
    if (K % kEach == 0) pack_kernel<T, true><<<grid, kThr, 0, s>>>(static_cast<const T *>(x), codes, scales, groups, K, G);
    else pack_kernel<T, false><<<grid, kThr, 0, s>>>(static_cast<const T *>(x), codes, scales, groups, K, G);
    return cudaGetLastError();
}
template <typename T, int EACH> cudaError_t unpack_by(const int8_t *codes, const float *scales, void *x, int M, int K, cudaStream_t s)
{
    const long long units = (long long)M * (K / EACH);
    if (!fits(units, kThr)) return cudaErrorInvalidConfiguration;
    unpack_kernel<T, EACH><<<blocks_for(units, kThr), kThr, 0, s>>>(codes, scales, static_cast<T *>(x), units, K, (K + kKeptGroup - 1) / kKeptGroup);
    return cudaGetLastError();
}
template <typename T> cudaError_t unpack(const int8_t *codes, const float *scales, void *x, int M, int K, cudaStream_t s)
{
    if (K % 16 == 0) return unpack_by<T, 16>(codes, scales, x, M, K, s);
    if (K % 8 == 0) return unpack_by<T, 8>(codes, scales, x, M, K, s);
    return unpack_by<T, 1>(codes, scales, x, M, K, s);
}

}  // namespace

cudaError_t launch_act8_pack(const void *x, int8_t *codes, float *scales, int M, int K, bool bf16, cudaStream_t s)
{
    return bf16 ? pack<__nv_bfloat16>(x, codes, scales, M, K, s) : pack<__half>(x, codes, scales, M, K, s);
}
cudaError_t launch_act8_unpack(const int8_t *codes, const float *scales, void *x, int M, int K, bool bf16, cudaStream_t s)
{
    return bf16 ? unpack<__nv_bfloat16>(codes, scales, x, M, K, s) : unpack<__half>(codes, scales, x, M, K, s);
}

cudaError_t launch_gate_grad(const void *dh, const int8_t *codes, const float *scales, void *dp, int M, int N, int fn, bool bf16, cudaStream_t s)
{
    const int per = N / 16, G = (N + kKeptGroup - 1) / kKeptGroup;
    const long long units = (long long)M * per;
    if (!fits(units, kThr)) return cudaErrorInvalidConfiguration;
    if (bf16)
        gate_grad_kernel<__nv_bfloat16><<<blocks_for(units, kThr), kThr, 0, s>>>(static_cast<const __nv_bfloat16 *>(dh), codes, scales, static_cast<__nv_bfloat16 *>(dp),
                                                                                 units, per, G, fn);
    else
        gate_grad_kernel<__half><<<blocks_for(units, kThr), kThr, 0, s>>>(static_cast<const __half *>(dh), codes, scales, static_cast<__half *>(dp), units, per, G, fn);
    return cudaGetLastError();
}

// Rows of `bytes` bytes each, F of either branch, in pieces of 16, 4 or 2 bytes.
cudaError_t launch_interleave(const void *gate, const void *up, void *out, int F, size_t bytes, bool padded, cudaStream_t s)
{
    auto go = [&](auto piece) {
        using P = decltype(piece);
        const int units = (int)(bytes / sizeof(P));
        const long long total = 2ll * F * (padded ? 2 : 1) * units;
        if (!fits(total, kThr)) return cudaErrorInvalidConfiguration;
        interleave_kernel<P><<<blocks_for(total, kThr), kThr, 0, s>>>(static_cast<const P *>(gate), static_cast<const P *>(up), static_cast<P *>(out), total, units, padded);
        return cudaGetLastError();
    };
    if (bytes % 16 == 0) return go(uint4{});
    if (bytes % 4 == 0) return go(uint32_t{});
    return go((unsigned short)0);
}

}  // namespace fbq
