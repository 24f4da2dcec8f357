// Gradients of the sub-branch's factors, sm_100a:  dA = s^T.x [rank][K],  dB = dy^T.t [N][rank],  s = dy.B and t = x.A^T from the launch
// before (fbq_dense.cu, rounded to the activation type there: they are tensor-core operands).
//
// Both are D[c][j] = sum_m Q[m][c] P[m][j]: Q wide (x or dy), P narrow (s or t), the contraction over tokens, which are the rows of both as
// they lie.  A CTA takes 128 columns of Q and all of P's: tcgen05.mma 128 x rank x 16 with both operands MN-major, straight from TMA
// boxes of 64 columns x 64 tokens; nothing is transposed.  Q is read once, P (1 MB at 4096 tokens) stays in L2.  What bounds it is the
// stream of Q, so two CTAs share an SM and each keeps its stages of 24 to 48 KB in flight: 4096 tokens of x [4096] and dy [22016] at rank 128 take 43 us
// (214 MB, 5.0 TB/s), 1024 of 11008 and 4096 at rank 64 10 and 3.5 for the sums (31 MB, most of it still in L2).
// Few columns (or a bound on CTAs) leave SMs idle, so the tokens are cut into S slices; their fp32 sums go through scratch and a second
// launch adds them in order (results do not depend on timing; no counter has to be cleared after a launch that was given up).
#include <algorithm>

#include "fbq_common.cuh"
#include "fbq_dequant.cuh"
#include "fbq_gate.cuh"
#include "fbq_maps.h"
#include "fbq_umma.cuh"

namespace fbq {
namespace {
using namespace ptx;

constexpr int kCols = 128;                       // columns of Q of a tile: the MMA's rows
constexpr int kTok = 64;                         // tokens of a stage
constexpr uint32_t kBox = 64u * kTok * 2u;       // 64 columns x kTok tokens
constexpr int kMostStages = 4;
constexpr int kThreads = 192;                    // copies, MMAs, four epilogue warps
constexpr size_t kSmemMost = 110 * 1024;         // two CTAs per SM
constexpr int kLeastBlocks = 4;                  // stages' worth of tokens of a slice, at least

struct FactorParams {
    void *dA, *dB;
    float *part;              // [slice][tile][rank_pad][kCols], or none: one slice
    int *status;
    int M, N, K, rank, rank_pad, gated;
    int tiles_x, tiles;       // tiles of x (dA), of both
    int slices, blocks;       // blocks of kTok tokens, of all slices
    int stages;
    uint32_t tmem_cols;
};

// Sums of column c (of the tile's 128), entries j0 ... j0 + 7 of the rank, to dA or dB.  Of a gated layer's B the half that is not the
// row's own holds zeros that are no parameters: their gradient is left at zero.
template <typename T> __device__ __forceinline__ void store8(const FactorParams &p, int tile, int c, int j0, const float (&v)[8])
{
    if (j0 >= p.rank) return;                                    // (rank is a multiple of 8)
    if (tile < p.tiles_x) {
        const int k = tile * kCols + c;
        unsigned short *dst = static_cast<unsigned short *>(p.dA) + (size_t)j0 * p.K + k;
        if (k < p.K)
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[(size_t)i * p.K] = to_bits16<T>(v[i]);
    } else {
        const int n = (tile - p.tiles_x) * kCols + c;
        if (n >= p.N) return;
        uint4 w = make_uint4(P2<T>::pack(v[0], v[1]), P2<T>::pack(v[2], v[3]), P2<T>::pack(v[4], v[5]), P2<T>::pack(v[6], v[7]));
        if (p.gated && (j0 >= p.rank / 2) != ((n & kGateUp) != 0)) w = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4 *>(static_cast<unsigned short *>(p.dB) + (size_t)n * p.rank + j0) = w;
    }
}

// xmap: x [M][K], dymap: dy [M][N], smap, tmap: s, t [M][rank_pad]; all boxes 64 columns x 64 tokens, 128-byte swizzle.
template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
factor_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap dymap, const __grid_constant__ CUtensorMap smap,
              const __grid_constant__ CUtensorMap tmap, const FactorParams p)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ uint64_t bars[2 * kMostStages + 1];
    __shared__ uint32_t tmem_slot;
    const uint32_t sbase = (smem_u32(smem) + 1023u) & ~1023u, full0 = smem_u32(bars), empty0 = full0 + 8u * kMostStages, done = empty0 + 8u * kMostStages;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tile = (int)blockIdx.x % p.tiles, slice = (int)blockIdx.x / p.tiles;
    const bool of_x = tile < p.tiles_x;
    const int col = (of_x ? tile : tile - p.tiles_x) * kCols;
    const int b0 = (int)((long long)p.blocks * slice / p.slices), b1 = (int)((long long)p.blocks * (slice + 1) / p.slices);
    const int np = p.rank_pad / 64, stages = p.stages;
    const uint32_t stage_bytes = (uint32_t)(2 + np) * kBox;

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(full0 + 8u * i, 1);
            mbar_init(empty0 + 8u * i, 1);
        }
        mbar_init(done, 1);
        fence_barrier_init();
        prefetch_tensormap(of_x ? &xmap : &dymap);
        prefetch_tensormap(of_x ? &smap : &tmap);
    }
    if (warp == 1) umma::tmem_alloc<1>(smem_u32(&tmem_slot), p.tmem_cols);
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    const uint32_t tmem = tmem_slot;
    pdl_wait();
    bool ok = true;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, phase = 1u;
#pragma unroll 1
            for (int b = b0; b < b1; ++b) {
                if (b - b0 >= stages && !mbar_wait(empty0 + 8u * s, phase)) { ok = false; break; }
                const uint32_t bar = full0 + 8u * s, dst = sbase + s * stage_bytes;
                mbar_expect_tx(bar, stage_bytes);
                for (int i = 0; i < 2; ++i) tma_load_2d(dst + i * kBox, of_x ? &xmap : &dymap, col + 64 * i, b * kTok, bar);
                for (int i = 0; i < np; ++i) tma_load_2d(dst + (2 + i) * kBox, of_x ? &smap : &tmap, 64 * i, b * kTok, bar);
                if (++s == (uint32_t)stages) { s = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        // (the whole warp walks the loop, one elected lane issues: operands stay in uniform registers)
        const uint32_t idesc = umma::idesc_f16(P2<T>::kFmt, kCols, (uint32_t)p.rank_pad) | umma::kIdescMnA | umma::kIdescMnB;
        const uint64_t qd0 = umma::desc_mn128(sbase, kBox), pd0 = umma::desc_mn128(sbase + 2 * kBox, kBox);
        uint32_t s = 0, phase = 0;
#pragma unroll 1
        for (int b = b0; b < b1 && ok; ++b) {
            ok = __all_sync(0xffffffffu, mbar_wait(full0 + 8u * s, phase));
            umma::fence_after();
            if (ok && umma::elect_one()) {
                const uint64_t qd = qd0 + s * (stage_bytes >> 4), pd = pd0 + s * (stage_bytes >> 4);
#pragma unroll
                for (int j = 0; j < kTok / 16; ++j) umma::mma(tmem, qd + j * (2048u >> 4), pd + j * (2048u >> 4), idesc, b > b0 || j > 0);
                umma::commit(empty0 + 8u * s);
                if (b + 1 == b1) umma::commit(done);
            }
            __syncwarp();
            if (++s == (uint32_t)stages) { s = 0; phase ^= 1u; }
        }
    } else {
        // lane = column of Q, column of tensor memory = entry of the rank
        const int q = warp & 3, c = 32 * q + lane;
        ok = mbar_wait_idle(done, 0u);
        ok = __all_sync(0xffffffffu, ok);
        if (ok) {
            umma::fence_after();
#pragma unroll 1
            for (int j = 0; j < p.rank; j += 32) {
                uint32_t v[32];
                umma::ld32(tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)j, v);
                umma::wait_ld();
                if (p.part) {
                    float *dst = p.part + (((size_t)slice * p.tiles + tile) * p.rank_pad + j) * kCols + c;
#pragma unroll
                    for (int i = 0; i < 32; ++i) __stcg(dst + i * kCols, __uint_as_float(v[i]));
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        float e[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) e[k] = __uint_as_float(v[i + k]);
                        store8<T>(p, tile, c, j + i, e);
                    }
                }
            }
        }
    }
    if (!ok) {
        atomicExch(p.status, (int)FBQ_ERR_TIMEOUT);
        for (int i = 0; i < 64; ++i) __nanosleep(1000);          // copies in flight land before the CTA leaves
    }
    umma::fence_before();
    __syncthreads();
    if (warp == 1) {
        umma::fence_after();
        umma::tmem_free<1>(tmem, p.tmem_cols);
    }
}

// The slices' sums, added in order: a thread per column of a tile and eight entries of the rank.
template <typename T> __global__ void __launch_bounds__(256) factor_add_kernel(const FactorParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    const int tile = blockIdx.x, c = threadIdx.x % kCols, j0 = ((int)blockIdx.y * 2 + (int)threadIdx.x / kCols) * 8;
    if (j0 >= p.rank) return;
    const float *src = p.part + ((size_t)tile * p.rank_pad + j0) * kCols + c;
    const size_t next = (size_t)p.tiles * p.rank_pad * kCols;
    float v[8] = {};
    for (int s = 0; s < p.slices; ++s, src += next)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += __ldcg(src + i * kCols);
    store8<T>(p, tile, c, j0, v);
}

// ---- host ----------------------------------------------------------------------------------------------------------
void plan(FactorParams &p)
{
    p.rank_pad = (p.rank + 63) / 64 * 64;
    p.tiles_x = (p.K + kCols - 1) / kCols;
    p.tiles = p.tiles_x + (p.N + kCols - 1) / kCols;
    p.blocks = (p.M + kTok - 1) / kTok;
    // as many slices as there is room for at once, two CTAs an SM
    p.slices = std::max(1, std::min(2 * sms_of_device() / p.tiles, p.blocks / kLeastBlocks));
    p.stages = (int)std::min<size_t>(kMostStages, kSmemMost / ((2 + p.rank_pad / 64) * kBox));
    p.tmem_cols = p.rank_pad <= 64 ? 64 : p.rank_pad <= 128 ? 128 : 256;
}

template <typename T> cudaError_t run(const void *dy, const void *x, const void *s16, const void *t16, FactorParams &p, bool pdl, cudaStream_t s, int *launches)
{
    const CUtensorMapDataType dt = CU_TENSOR_MAP_DATA_TYPE_UINT16;
    const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B;
    CUtensorMap xmap, dymap, smap, tmap;
    cudaError_t e;
    if ((e = encode_map(&xmap, matrix_map(x, dt, 2, p.K, p.M, 64, kTok, sw))) != cudaSuccess) return e;
    if ((e = encode_map(&dymap, matrix_map(dy, dt, 2, p.N, p.M, 64, kTok, sw))) != cudaSuccess) return e;
    if ((e = encode_map(&smap, matrix_map(s16, dt, 2, p.rank_pad, p.M, 64, kTok, sw))) != cudaSuccess) return e;
    if ((e = encode_map(&tmap, matrix_map(t16, dt, 2, p.rank_pad, p.M, 64, kTok, sw))) != cudaSuccess) return e;
    const size_t smem = (size_t)p.stages * (2 + p.rank_pad / 64) * kBox + 1024;
    auto kern = factor_kernel<T>;
    static PerDevice attr_set;
    if (!attr_set.there()) {
        if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kSmemMost + 1024))) != cudaSuccess) return e;
        attr_set.set();
    }
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 1 : 0;
    cfg.stream = s;
    cfg.gridDim = dim3((unsigned)(p.tiles * p.slices));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    if ((e = cudaLaunchKernelEx(&cfg, kern, xmap, dymap, smap, tmap, p)) != cudaSuccess) return e;
    ++*launches;
    if (!p.part) return e;
    cfg.gridDim = dim3((unsigned)p.tiles, (unsigned)((p.rank + 15) / 16));
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = 0;
    if ((e = cudaLaunchKernelEx(&cfg, factor_add_kernel<T>, p)) == cudaSuccess) ++*launches;
    return e;
}

}  // namespace

size_t factor_grad_scratch_bytes(int M, int N, int K, int rank)
{
    if (rank == 0) return 0;
    FactorParams p{};
    p.M = M; p.N = N; p.K = K; p.rank = rank;
    plan(p);
    return p.slices > 1 ? (size_t)p.slices * p.tiles * p.rank_pad * kCols * sizeof(float) : 0;
}

cudaError_t launch_factor_grads(const void *dy, const void *x, const void *s16, const void *t16, void *dA, void *dB, int M, int N, int K, int rank, bool gated,
                                bool bf16, void *scratch, int *status, bool pdl, cudaStream_t s, int *launches)
{
    FactorParams p{};
    p.dA = dA; p.dB = dB; p.status = status;
    p.M = M; p.N = N; p.K = K; p.rank = rank; p.gated = gated;
    plan(p);
    p.part = p.slices > 1 ? static_cast<float *>(scratch) : nullptr;
    return bf16 ? run<__nv_bfloat16>(dy, x, s16, t16, p, pdl, s, launches) : run<__half>(dy, x, s16, t16, p, pdl, s, launches);
}

}  // namespace fbq
