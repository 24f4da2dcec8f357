// The sub-branch's thin products for few hundred tokens, sm_100a:  t = x.A^T  and  s = dy.B,  [M][rank], rounded once to the activation
// type (they are tensor-core operands of the launch behind this one); entries up to the next multiple of 64 are zeros.
//
// Little arithmetic over long contractions, so what counts is how many SMs read: a cluster of CTAs takes a tile of tokens and up to 128
// entries of the rank and cuts the contraction (tcgen05.mma, the rank's entries are the rows, tokens the columns; A is K-major, B as
// it lies MN-major).  Each CTA puts its fp32 sums into its shared memory, and after one cluster barrier every CTA adds an equal share of the
// tokens from all of them, in order, through distributed shared memory.  Long contractions (22016 rows of B at 333 tokens: 22 us with one cluster a
// tile) are cut over several clusters as well, each with its fp32 sums, which a second launch adds in order and rounds.
#include <algorithm>

#include "fbq_common.cuh"
#include "fbq_dequant.cuh"
#include "fbq_maps.h"
#include "fbq_umma.cuh"

namespace fbq {
namespace {
using namespace ptx;

constexpr int kBK = 64, kRows = 128;
constexpr int kMostTok = 128, kStages = 3, kMostCluster = 8;
constexpr int kPer = 2;                          // blocks of a stage
constexpr uint32_t kABytes = kRows * kBK * 2u, kBox = kABytes / 2;
constexpr int kThreads = 192;
constexpr uint32_t kSmem = kStages * kPer * (kABytes + kMostTok * kBK * 2u) + 1024;
static_assert(kMostTok * kRows * 4u <= kSmem - 1024, "the sums take the stages' place");

struct ThinParams {
    void *t, *s;              // [M][rank_pad]
    int *status;
    int M, rank, rank_pad, a_rows;
    int tok, ntt, nrt;        // tokens of a tile, tiles, tiles of the rank
    int cuts_s, cuts_t;       // clusters that share a tile's contraction
    int n_first;              // clusters of the one of s and t whose take longer, before the other's
    bool s_first;
    float *part;              // [cut][M][rank_pad] of s, then of t, or none: no contraction is cut
    int blocks_t, blocks_s;   // of the contractions
};

__device__ __forceinline__ float ld_cluster(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
    return v;
}

// xmap: x [M][K], dymap: dy [M][N], boxes of tok rows x 64; amap: A [rank][K], boxes of a_rows x 64; bmap: B [N][rank], boxes of 64 x 64 (MN-major);
// all in the 128-byte swizzle.
template <typename T>
__global__ void __launch_bounds__(kThreads, 1)
thin_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap dymap, const __grid_constant__ CUtensorMap amap,
            const __grid_constant__ CUtensorMap bmap, const ThinParams p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * kStages + 1];
    __shared__ uint32_t tmem_slot;
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t sbase = smem_u32(smem), full0 = smem_u32(bars), empty0 = full0 + 8u * kStages, done = empty0 + 8u * kStages;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t cs, crank;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
    crank = cluster_ctarank();
    int cluster = (int)(blockIdx.x / cs);
    const bool first = cluster < p.n_first, of_s = first == p.s_first;
    if (!first) cluster -= p.n_first;
    const int cuts = of_s ? p.cuts_s : p.cuts_t, cut = cluster % cuts;
    cluster /= cuts;
    const int rt = cluster % p.nrt, m0 = cluster / p.nrt * p.tok, row0 = rt * kRows;
    const long long all = of_s ? p.blocks_s : p.blocks_t;
    const int shares = cuts * (int)cs, share = cut * (int)cs + (int)crank, b0 = (int)(all * share / shares), b1 = (int)(all * (share + 1) / shares);
    const int boxes = min(2, (p.rank_pad - row0) / 64);
    const uint32_t xbytes = (uint32_t)p.tok * (kBK * 2u), block_bytes = kABytes + xbytes, stage_bytes = kPer * block_bytes, abytes = of_s ? (uint32_t)boxes * kBox : (uint32_t)p.a_rows * (kBK * 2u);

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(full0 + 8u * i, 1);
            mbar_init(empty0 + 8u * i, 1);
        }
        mbar_init(done, 1);
        fence_barrier_init();
        prefetch_tensormap(of_s ? &dymap : &xmap);
        prefetch_tensormap(of_s ? &bmap : &amap);
    }
    if (warp == 1) umma::tmem_alloc<1>(smem_u32(&tmem_slot), 128u);
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    const uint32_t tmem = tmem_slot;
    pdl_wait();
    pdl_launch_dependents();
    bool ok = true;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, phase = 1u;
#pragma unroll 1
            for (int b = b0; b < b1; b += kPer) {
                if (b - b0 >= kPer * kStages && !mbar_wait(empty0 + 8u * s, phase)) { ok = false; break; }
                const uint32_t bar = full0 + 8u * s;
                const int n = min(kPer, b1 - b);
                mbar_expect_tx(bar, n * (abytes + xbytes));
                for (int k = 0; k < n; ++k) {
                    const uint32_t dst = sbase + s * stage_bytes + k * block_bytes;
                    if (of_s)
                        for (int i = 0; i < boxes; ++i) tma_load_2d(dst + i * kBox, &bmap, row0 + 64 * i, (b + k) * kBK, bar);
                    else
                        tma_load_2d(dst, &amap, (b + k) * kBK, row0, bar);
                    tma_load_2d(dst + kABytes, of_s ? &dymap : &xmap, (b + k) * kBK, m0, bar);
                }
                if (++s == kStages) { s = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        // (the whole warp walks the loop, one elected lane issues: operands stay in uniform registers)
        const uint32_t idesc = umma::idesc_f16(P2<T>::kFmt, kRows, (uint32_t)p.tok) | (of_s ? umma::kIdescMnA : 0u), astep = of_s ? 2048u >> 4 : 2u;
        const uint64_t ad0 = of_s ? umma::desc_mn128(sbase, kBox) : umma::desc_k128(sbase), xd0 = umma::desc_k128(sbase + kABytes);
        uint32_t s = 0, phase = 0;
#pragma unroll 1
        for (int b = b0; b < b1 && ok; b += kPer) {
            ok = __all_sync(0xffffffffu, mbar_wait(full0 + 8u * s, phase));
            umma::fence_after();
            if (ok && umma::elect_one()) {
                uint64_t ad = ad0 + s * (stage_bytes >> 4), xd = xd0 + s * (stage_bytes >> 4);
#pragma unroll
                for (int j = 0; j < kBK / 16; ++j) umma::mma(tmem, ad + astep * j, xd + 2 * j, idesc, b > b0 || j > 0);
                if (b + 1 < b1) {
                    ad += block_bytes >> 4;
                    xd += block_bytes >> 4;
#pragma unroll
                    for (int j = 0; j < kBK / 16; ++j) umma::mma(tmem, ad + astep * j, xd + 2 * j, idesc, 1u);
                }
                umma::commit(empty0 + 8u * s);
                if (b + kPer >= b1) umma::commit(done);
            }
            __syncwarp();
            if (++s == kStages) { s = 0; phase ^= 1u; }
        }
    } else {
        // sums [token][rank entry] into shared memory, where the operands were
        const int q = warp & 3, j = 32 * q + lane;
        float *sums = reinterpret_cast<float *>(smem) + j;
        ok = b0 == b1 || __all_sync(0xffffffffu, mbar_wait(done, 0u));
        if (ok) {
            umma::fence_after();
#pragma unroll 1
            for (int c = 0; c < p.tok; c += 16) {
                uint32_t v[16];
                umma::ld16(tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)c, v);
                umma::wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[(c + i) * kRows] = b1 > b0 ? __uint_as_float(v[i]) : 0.f;
            }
        }
    }
    if (!ok) {
        atomicExch(p.status, (int)FBQ_ERR_TIMEOUT);
        for (int i = 0; i < 64; ++i) __nanosleep(1000);          // copies in flight land before the CTA leaves
    }
    umma::fence_before();
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    const int width = min(kRows, p.rank_pad - row0);
    unsigned short *out = static_cast<unsigned short *>(of_s ? p.s : p.t);
    float *part = p.part + (size_t)((of_s ? 0 : p.cuts_s) + cut) * p.M * p.rank_pad;
    // this CTA's tokens are crank, crank + cs, ...; a thread has the loads of a sum on their way at once
    for (int e = threadIdx.x; e < (p.tok + (int)cs - 1) / (int)cs * kRows; e += kThreads) {
        const int c = e / kRows * (int)cs + (int)crank, j = e % kRows;
        if (c >= p.tok || m0 + c >= p.M || j >= width) continue;
        float w[kMostCluster], v = 0.f;
#pragma unroll
        for (uint32_t k = 0; k < kMostCluster; ++k) w[k] = k < cs ? ld_cluster(mapa_shared(sbase + (uint32_t)(c * kRows + j) * 4u, k)) : 0.f;
#pragma unroll
        for (int k = 0; k < kMostCluster; ++k) v += w[k];
        if (row0 + j >= p.rank) v = 0.f;                         // (an infinite x times the zeros of an entry that is not there)
        const size_t to = (size_t)(m0 + c) * p.rank_pad + row0 + j;
        if (p.part) part[to] = v;
        else out[to] = to_bits16<T>(v);
    }
    cluster_arrive();
    cluster_wait();                                              // nobody reads this CTA's sums any more
    if (warp == 1) {
        umma::fence_after();
        umma::tmem_free<1>(tmem, 128u);
    }
}

// s and t from the sums of their cuts, in order.
template <typename T> __global__ void __launch_bounds__(256) thin_add_kernel(const ThinParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    const bool of_s = blockIdx.y == 0 && p.s;
    const size_t n = (size_t)p.M * p.rank_pad, at = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= n) return;
    const float *src = p.part + (of_s ? 0 : p.cuts_s * n) + at;
    float v = 0.f;
#pragma unroll 4
    for (int c = 0; c < (of_s ? p.cuts_s : p.cuts_t); ++c) v += __ldcg(src + c * n);
    static_cast<unsigned short *>(of_s ? p.s : p.t)[at] = to_bits16<T>(v);
}

// The plan: CTAs of a cluster, tokens of a tile, and clusters that share a tile's contraction, such that what a CTA has to go through takes
// least.  It reads some 60 bytes a nanosecond (A or B once per tile of tokens) and spends 4 us besides; where clusters are more than the GPU
// holds at a time (one CTA per SM, and a cluster stays within one of the processing clusters) the longer ones go first and the others fill the
// gaps, half of one's time late.  Cuts cost a launch and their sums' way through L2.  Sum of both launches, us, rank 128, against cuts by powers of
// two and s always first: 22016 rows of B and 4096 of A at 100 tokens 18 -> 12, 700 24 -> 20, 4096 83 -> 60; 4096 and 11008 at 400 17.5 -> 14;
// tiles of 256 tokens in two stages 86 for the 77 of the first launch.
void plan(const ThinArgs &a, ThinParams &p, int *cluster)
{
    p.M = a.M;
    p.rank = a.rank;
    p.rank_pad = (a.rank + kBK - 1) / kBK * kBK;
    p.a_rows = std::min(kRows, p.rank_pad);
    p.nrt = (p.rank_pad + kRows - 1) / kRows;
    p.blocks_t = a.t ? (a.K + kBK - 1) / kBK : 0;
    p.blocks_s = a.s ? (a.N + kBK - 1) / kBK : 0;
    static const int resident[4] = {148, 74, 33, 15};
    double least = 1e30;
    const int most = std::max(p.blocks_t, p.blocks_s);
    for (int c = 0; (1 << c) <= kMostCluster; ++c) {
        const int cs = 1 << c;
        if (c > 0 && 2 * cs > most) break;
        for (int tok = 16; tok <= kMostTok; tok += 16) {
            const int ntt = (a.M + tok - 1) / tok, sets = ntt * p.nrt;
            if (tok > 16 && (a.M + tok - 17) / (tok - 16) == ntt) continue;          // (fewer tokens make as many tiles)
            auto piece = [&](int blocks, int cuts) { return (double)((blocks + cs * cuts - 1) / (cs * cuts)) * (kABytes + tok * kBK * 2) / 60e3 + 4.0; };
            for (int cut = 1; cut <= 8; ++cut) {
                // of s and t the longer contraction is cut more often
                const int cuts_s = p.blocks_s ? std::max(1, std::min(cut, cut * p.blocks_s / most)) : 0, cuts_t = p.blocks_t ? std::max(1, std::min(cut, cut * p.blocks_t / most)) : 0;
                const double of_s = cuts_s ? piece(p.blocks_s, cuts_s) : 0, of_t = cuts_t ? piece(p.blocks_t, cuts_t) : 0;
                const double longest = std::max(of_s, of_t), all = sets * (cuts_s * of_s + cuts_t * of_t);
                const double last = cuts_s && cuts_t ? std::min(of_s, of_t) : longest;
                const int count = sets * (cuts_s + cuts_t);
                const double cost = (count <= resident[c] ? longest + 3.0 : std::max(longest, all / resident[c] + last / 2)) + (cut > 1 ? 8.0 : 0.0);
                if (cost >= least) continue;
                least = cost;
                *cluster = cs;
                p.tok = tok;
                p.ntt = ntt;
                p.cuts_s = cuts_s;
                p.cuts_t = cuts_t;
                p.s_first = of_s >= of_t;
            }
        }
    }
}

// The last plan of this host thread is kept: it holds sizes, no addresses, and a step's calls ask for it twice each.
void plan_for(const ThinArgs &a, ThinParams &p, int *cluster)
{
    static thread_local int key[6] = {}, cs = 0;
    static thread_local ThinParams kept{};
    const int want[6] = {a.M, a.N, a.K, a.rank, a.t != nullptr, a.s != nullptr};
    if (cs == 0 || !std::equal(want, want + 6, key)) {
        kept = ThinParams{};
        plan(a, kept, &cs);
        std::copy(want, want + 6, key);
    }
    p = kept;
    *cluster = cs;
}

template <typename T> cudaError_t run(const ThinArgs &a, int *status, bool pdl, cudaStream_t s, int *launches)
{
    const CUtensorMapDataType dt = CU_TENSOR_MAP_DATA_TYPE_UINT16;
    const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B;
    ThinParams p{};
    int cs = 1;
    plan_for(a, p, &cs);
    p.t = a.t; p.s = a.s; p.status = status;
    p.part = p.cuts_s > 1 || p.cuts_t > 1 ? static_cast<float *>(a.part) : nullptr;
    p.n_first = p.ntt * p.nrt * (p.s_first ? p.cuts_s : p.cuts_t);
    const int clusters = p.ntt * p.nrt * (p.cuts_s + p.cuts_t);
    CUtensorMap xmap, dymap, amap, bmap;
    cudaError_t e;
    if (a.t) {
        if ((e = encode_map(&xmap, matrix_map(a.x, dt, 2, a.K, a.M, kBK, p.tok, sw))) != cudaSuccess) return e;
        if ((e = encode_map(&amap, matrix_map(a.A, dt, 2, a.K, a.rank, kBK, p.a_rows, sw))) != cudaSuccess) return e;
    }
    if (a.s) {
        if ((e = encode_map(&dymap, matrix_map(a.dy, dt, 2, a.N, a.M, kBK, p.tok, sw))) != cudaSuccess) return e;
        if ((e = encode_map(&bmap, matrix_map(a.B, dt, 2, a.rank, a.N, kBK, kBK, sw))) != cudaSuccess) return e;
    }
    if (!a.t) { xmap = dymap; amap = bmap; }
    if (!a.s) { dymap = xmap; bmap = amap; }
    auto kern = thin_kernel<T>;
    static PerDevice attr_set;
    if (!attr_set.there()) {
        if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem)) != cudaSuccess) return e;
        if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
        attr_set.set();
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * cs));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cs;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 2 : 1;
    if ((e = cudaLaunchKernelEx(&cfg, kern, xmap, dymap, amap, bmap, p)) != cudaSuccess) return e;
    ++*launches;
    if (!p.part) return e;
    cfg.gridDim = dim3((unsigned)(((size_t)p.M * p.rank_pad + 255) / 256), (unsigned)((a.s ? 1 : 0) + (a.t ? 1 : 0)));
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = 0;
    cfg.attrs = at + 1;
    cfg.numAttrs = pdl ? 1 : 0;
    if ((e = cudaLaunchKernelEx(&cfg, thin_add_kernel<T>, p)) == cudaSuccess) ++*launches;
    return e;
}

}  // namespace

size_t thin_part_bytes(const ThinArgs &a)
{
    ThinParams p{};
    int cs;
    plan_for(a, p, &cs);
    return p.cuts_s > 1 || p.cuts_t > 1 ? (size_t)(p.cuts_s + p.cuts_t) * p.M * p.rank_pad * sizeof(float) : 0;
}

cudaError_t launch_thin(const ThinArgs &a, int *status, bool pdl, cudaStream_t s, int *launches)
{
    return a.bf16 ? run<__nv_bfloat16>(a, status, pdl, s, launches) : run<__half>(a, status, pdl, s, launches);
}

}  // namespace fbq
