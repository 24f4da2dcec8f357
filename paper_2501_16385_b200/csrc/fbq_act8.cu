// Activations in 8 bits: the form in which a training step keeps them between its passes, and what the gated block's backward
// pass makes of it.  All three kernels are bound by memory: one pass, 16 bytes a lane and access where rows allow, the lanes of a kernel with
// two accesses each on their way, places in 32 bits where they fit (a division of 64 bits takes as long as the rest of a lane's work).
// 4096 x 11008 bf16: pack 27.5 us (135 MB, 4.9 TB/s), unpack 27 (5.0 TB/s); dp of the gated block, 4096 x 22016, 67 us
// (361 MB, 5.4 TB/s).  Rows of no whole pieces of eight (11004, 11007; a layer's are always whole) go value by value: 78 and 111 us.
#include "fbq_common.cuh"
#include "fbq_dequant.cuh"
#include "fbq_gate.cuh"

namespace fbq {
namespace {

constexpr int kThr = 256;
constexpr int kTwice = 2;                                    // groups, or units, of a lane, a block's width apart

template <typename T> __device__ __forceinline__ float2 unpair(uint32_t v);
template <> __device__ __forceinline__ float2 unpair<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }
template <> __device__ __forceinline__ float2 unpair<__nv_bfloat16>(uint32_t v)
{
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}

// One group, 128 / EACH lanes: this lane's n values (WIDE: in `raw`, zeros where there are none).
template <typename T, int EACH, bool WIDE>
__device__ __forceinline__ void pack_group(const T *src, const uint4 (&raw)[EACH / 8], int8_t *dst, float *scale_at, int n, bool first)
{
    float v[EACH] = {};
    if (WIDE) {
#pragma unroll
        for (int i = 0; i < EACH / 8; ++i) {
            const float2 a = unpair<T>(raw[i].x), b = unpair<T>(raw[i].y), c = unpair<T>(raw[i].z), d = unpair<T>(raw[i].w);
            v[8 * i] = a.x; v[8 * i + 1] = a.y; v[8 * i + 2] = b.x; v[8 * i + 3] = b.y; v[8 * i + 4] = c.x; v[8 * i + 5] = c.y; v[8 * i + 6] = d.x; v[8 * i + 7] = d.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < n) v[i] = ActTraits<T>::to_float(src[i]);
    }
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < EACH; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
#pragma unroll
    for (int o = 1; o < kKeptGroup / EACH; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    float scale, inverse;
    kept_scale(top, scale, inverse);
    if (first) *scale_at = scale;
    if (WIDE) {
        uint32_t w[EACH / 4] = {};
#pragma unroll
        for (int i = 0; i < EACH; ++i) w[i / 4] |= kept_code(v[i], inverse) << (8 * (i % 4));
        if (n <= 0) return;
        if constexpr (EACH == 16) *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < n) dst[i] = (int8_t)kept_code(v[i], inverse);
    }
}

// 128 / EACH lanes take a group: the largest |v| crosses lanes once, codes and values do not.  WIDE: rows of whole units of EACH.  (Sixteen values a lane
// share the scale's two divisions and take three steps across lanes: 27.5 us for 4096 x 11008; eight 33 for 4096 x 11000.)
template <typename T, int EACH, bool WIDE, typename I>
__global__ void __launch_bounds__(kThr) pack_kernel(const T *__restrict__ x, int8_t *__restrict__ codes, float *__restrict__ scales, I groups, int K, int G)
{
    constexpr int LANES = kKeptGroup / EACH;
    const int l = threadIdx.x % LANES;
    I at[kTwice];
    int n[kTwice];                                               // <= 0: nothing
    size_t to[kTwice];
    uint4 raw[kTwice][EACH / 8];
#pragma unroll
    for (int j = 0; j < kTwice; ++j) {
        at[j] = ((I)blockIdx.x * kTwice + j) * (kThr / LANES) + threadIdx.x / LANES;
        const I m = at[j] < groups ? at[j] / G : 0;
        const int k = (int)(at[j] < groups ? at[j] - m * G : 0) * kKeptGroup + l * EACH;
        n[j] = at[j] < groups ? min(EACH, K - k) : 0;
        to[j] = (size_t)m * K + k;
#pragma unroll
        for (int i = 0; i < EACH / 8; ++i)
            if (WIDE) raw[j][i] = n[j] > 0 ? __ldg(reinterpret_cast<const uint4 *>(x + to[j]) + i) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int j = 0; j < kTwice; ++j) pack_group<T, EACH, WIDE>(x + to[j], raw[j], codes + to[j], scales + at[j], n[j], at[j] < groups && l == 0);
}

__device__ __forceinline__ float byte_to_float(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

// A lane turns EACH codes of a row (16, 8 or 1; K a multiple of it): code * scale, rounded once.
template <typename T, int EACH, typename I>
__global__ void __launch_bounds__(kThr) unpack_kernel(const int8_t *__restrict__ codes, const float *__restrict__ scales, T *__restrict__ x, I units, int K, int G)
{
    const I per = K / EACH;
    I at[kTwice];
    float s[kTwice];
    uint32_t w[kTwice][EACH / 4 + 1];
#pragma unroll
    for (int j = 0; j < kTwice; ++j) {
        at[j] = ((I)blockIdx.x * kTwice + j) * kThr + threadIdx.x;
        if (at[j] >= units) continue;
        const I m = at[j] / per;
        s[j] = __ldg(scales + (size_t)m * G + (int)(at[j] - m * per) * EACH / kKeptGroup);
        const int8_t *src = codes + (size_t)at[j] * EACH;
        if constexpr (EACH == 16) {
            const uint4 q = __ldg(reinterpret_cast<const uint4 *>(src));
            w[j][0] = q.x; w[j][1] = q.y; w[j][2] = q.z; w[j][3] = q.w;
        } else if constexpr (EACH == 8) {
            const uint2 q = __ldg(reinterpret_cast<const uint2 *>(src));
            w[j][0] = q.x; w[j][1] = q.y;
        } else {
            w[j][0] = (uint8_t)*src;
        }
    }
#pragma unroll
    for (int j = 0; j < kTwice; ++j) {
        if (at[j] >= units) continue;
        T *dst = x + (size_t)at[j] * EACH;
        if constexpr (EACH == 1) {
            *dst = ActTraits<T>::from_float(byte_to_float(w[j][0], 0) * s[j]);
        } else {
            uint32_t o[EACH / 2];
#pragma unroll
            for (int i = 0; i < EACH / 2; ++i) o[i] = P2<T>::pack(byte_to_float(w[j][i / 2], 2 * i % 4) * s[j], byte_to_float(w[j][i / 2], 2 * i % 4 + 1) * s[j]);
#pragma unroll
            for (int i = 0; i < EACH / 8; ++i) reinterpret_cast<uint4 *>(dst)[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        }
    }
}

// dp of the gated block: p[16i + j] the gate's, p[16i + 8 + j] the up projection's value that met in h[8i + j], both as they were kept:
// dp_gate = dh p_up f'(p_gate), dp_up = dh f(p_gate), rounded once (they are operands of tensor-core products next).  A lane
// takes eight columns of h.
template <typename T, typename I>
__global__ void __launch_bounds__(kThr) gate_grad_kernel(const T *__restrict__ dh, const int8_t *__restrict__ codes, const float *__restrict__ scales, T *__restrict__ dp,
                                                         I units, I per, int G, int fn)
{
    I at[kTwice];
    float s[kTwice];
    uint4 q[kTwice], d[kTwice];
#pragma unroll
    for (int j = 0; j < kTwice; ++j) {
        at[j] = ((I)blockIdx.x * kTwice + j) * kThr + threadIdx.x;
        if (at[j] >= units) continue;
        const I m = at[j] / per;
        s[j] = __ldg(scales + (size_t)m * G + (int)(at[j] - m * per) / (kKeptGroup / 16));
        q[j] = __ldg(reinterpret_cast<const uint4 *>(codes) + at[j]);
        d[j] = __ldg(reinterpret_cast<const uint4 *>(dh) + at[j]);
    }
#pragma unroll
    for (int j = 0; j < kTwice; ++j) {
        if (at[j] >= units) continue;
        const uint32_t gate[2] = {q[j].x, q[j].y}, up[2] = {q[j].z, q[j].w}, dd[4] = {d[j].x, d[j].y, d[j].z, d[j].w};
        uint32_t og[4], ou[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 e = unpair<T>(dd[i]);
            float f0, f1, df0, df1;
            gate_both(fn, byte_to_float(gate[i / 2], 2 * i % 4) * s[j], f0, df0);
            gate_both(fn, byte_to_float(gate[i / 2], 2 * i % 4 + 1) * s[j], f1, df1);
            og[i] = P2<T>::pack(e.x * (byte_to_float(up[i / 2], 2 * i % 4) * s[j]) * df0, e.y * (byte_to_float(up[i / 2], 2 * i % 4 + 1) * s[j]) * df1);
            ou[i] = P2<T>::pack(e.x * f0, e.y * f1);
        }
        uint4 *dst = reinterpret_cast<uint4 *>(dp) + 2 * (size_t)at[j];
        dst[0] = make_uint4(og[0], og[1], og[2], og[3]);
        dst[1] = make_uint4(ou[0], ou[1], ou[2], ou[3]);
    }
}

// Rows of `units` pieces of P: eight of the gate, eight of the up projection, and so on.  `padded`: a row of the result has twice the
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

int groups_of(int K) { return (K - 1) / kKeptGroup + 1; }          // (K + 127 may be beyond 31 bits)
unsigned blocks_for(long long n, int per) { return (unsigned)((n + per - 1) / per); }
// Grids have 31 bits.
bool fits(long long n, int per) { return n <= (long long)per * 0x7FFFFFFF; }

// A launch whose status is its own (the runtime's last error may be another call's).
template <typename... P, typename... A> cudaError_t launch(void (*kern)(P...), unsigned grid, cudaStream_t s, A... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThr);
    cfg.stream = s;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}
// `go` with the number of units in 32 bits where they and what a block may count beyond them fit, else in 64.
template <typename F> cudaError_t by_size(long long units, int per_block, F go)
{
    if (!fits(units, per_block)) return cudaErrorInvalidConfiguration;
    const unsigned grid = blocks_for(units, per_block);
    return units < (1ll << 31) ? go((unsigned)units, grid) : go(units, grid);
}
template <typename T, int EACH, bool WIDE> cudaError_t pack_by(const void *x, int8_t *codes, float *scales, int M, int K, cudaStream_t s)
{
    const int G = groups_of(K);
    return by_size((long long)M * G, kTwice * (kThr * EACH / kKeptGroup), [&](auto groups, unsigned grid) {
        return launch(pack_kernel<T, EACH, WIDE, decltype(groups)>, grid, s, static_cast<const T *>(x), codes, scales, groups, K, G);
    });
}
template <typename T> cudaError_t pack(const void *x, int8_t *codes, float *scales, int M, int K, cudaStream_t s)
{
    if (K % 16 == 0) return pack_by<T, 16, true>(x, codes, scales, M, K, s);
    if (K % 8 == 0) return pack_by<T, 8, true>(x, codes, scales, M, K, s);
    return pack_by<T, 8, false>(x, codes, scales, M, K, s);
}
template <typename T, int EACH> cudaError_t unpack_by(const int8_t *codes, const float *scales, void *x, int M, int K, cudaStream_t s)
{
    return by_size((long long)M * (K / EACH), kTwice * kThr, [&](auto units, unsigned grid) {
        return launch(unpack_kernel<T, EACH, decltype(units)>, grid, s, codes, scales, static_cast<T *>(x), units, K, groups_of(K));
    });
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
    const int per = N / 16, G = groups_of(N);
    return by_size((long long)M * per, kTwice * kThr, [&](auto units, unsigned grid) {
        using I = decltype(units);
        auto go = [&](auto type) {
            using T = decltype(type);
            return launch(gate_grad_kernel<T, I>, grid, s, static_cast<const T *>(dh), codes, scales, static_cast<T *>(dp), units, per, G, fn);
        };
        return bf16 ? go(__nv_bfloat16{}) : go(__half{});
    });
}

// Rows of `bytes` bytes each, F of either branch, in pieces of 16, 4 or 2 bytes.
cudaError_t launch_interleave(const void *gate, const void *up, void *out, int F, size_t bytes, bool padded, cudaStream_t s)
{
    auto go = [&](auto piece) {
        using P = decltype(piece);
        const int units = (int)(bytes / sizeof(P));
        const long long total = 2ll * F * (padded ? 2 : 1) * units;
        if (!fits(total, kThr)) return cudaErrorInvalidConfiguration;
        return launch(interleave_kernel<P>, blocks_for(total, kThr), s, static_cast<const P *>(gate), static_cast<const P *>(up), static_cast<P *>(out), total, units, padded);
    };
    if (bytes % 16 == 0) return go(uint4{});
    if (bytes % 4 == 0) return go(uint32_t{});
    return go((unsigned short)0);
}

}  // namespace fbq
