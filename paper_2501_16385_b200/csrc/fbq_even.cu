// The gated block and dx of a layer's backward pass for few hundred tokens, sm_100a: weights dequantised where they are multiplied, and
// the blocks of the contraction shared out evenly.
//
//   h = f(gate) * up,  p = x.dequant(Q,s,z)^T + t.B^T          (forward; t = x.A^T from the launch before, fbq_thin.cu)
//   dx = dy.dequant(Q,s,z) + s.A                               (Grad; s = dy.B from there)
//
// Up to a few hundred tokens a weight is used too seldom to be dequantised in a pass of its own (the dense kernel's 16-bit copy costs 4
// bytes a weight through L2 beside the half byte of its code), and tiles of 128 features are about as many as SMs, which leaves a second
// wave nearly empty.  So a CTA takes all tokens of a tile (up to 512: 128 lanes x 512 columns are the whole tensor memory), turns codes
// into the operand in shared memory, and the blocks of all tiles, in order, are cut into equal ranges, one per CTA:
//
//   warps 8-23   two groups of eight dequantise every other block, 32 codes a thread; codes come straight from global memory into registers,
//                three blocks ahead of their use (what is in flight needs no shared memory and no barrier)
//   warp 0       copies x (dy) by TMA, and both operands of the sub-branch's blocks
//   warp 1       issues tcgen05.mma 128 x tokens x 16
//   warps 4-7    epilogue: of a tile that several CTAs share all but one store their fp32 sums; the CTA that holds its first block owns it, adds the
//                others' in order of the contraction and writes the outputs
//
// A range ends with the tiles it owns and begins with the one it does not, so whoever waits for sums waits for what another CTA did
// first.  CTA b takes the range of gridDim - 1 - b: ranges behind one's own belong to CTAs with lower numbers, which start earlier, and
// wait only for lower numbers still; any number of resident CTAs makes progress.  The sub-branch's blocks are the owner's, at the end of a tile.
// Sums do not depend on timing.  Tags of finished sums carry the launch's number (as in fbq_dense.cu, with the same words): nothing is cleared.
// All waits are bounded.
//
// Forward, features are rows of W and the operand is K-major; Grad, features are its columns, a block is 64 rows x 128 columns, one group
// of each row, and the operand is MN-major: rows are written as they lie.
#include <algorithm>
#include <type_traits>

#include "fbq_common.cuh"
#include "fbq_dequant.cuh"
#include "fbq_gate.cuh"
#include "fbq_maps.h"
#include "fbq_umma.cuh"

namespace fbq {
namespace {
using namespace ptx;

constexpr int kBK = 64, kFeat = 128;
constexpr uint32_t kWBytes = kFeat * kBK * 2u, kBox = kWBytes / 2;
constexpr int kMostTok = 512, kMostStages = 8;
constexpr int kDqWarp = 8, kGroupWarps = 8, kThreads = (kDqWarp + 2 * kGroupWarps) * 32;
constexpr int kAhead = 3;                        // blocks of its own that a dequantising thread has requested
constexpr uint32_t kYBytes = 32u * 128u * 2u;    // staged part of an output tile: 32 tokens
constexpr uint32_t kFixed = 2 * kYBytes + 512 + 256;     // staging, largest |p|, barriers
constexpr uint32_t kSmemMost = 227 * 1024 - 1024;        // (the base is moved up to 1024 bytes)
constexpr int kTagEpoch = 0, kTagDone = 1, kTagFirst = 4;        // words of the tag scratch, shared with fbq_dense.cu

enum Mode { kGated, kKept, kGrad };

struct EvenParams {
    const uint32_t *qw;
    const __half *scales, *zeros;
    float *part;              // [CTA][tok][kFeat] sums of the tile that a range begins with and does not own
    uint32_t *tags;           // see above; a word per range
    float *kept_scales;
    int *status;
    int M, F, D, K;           // tokens, features, contraction, columns of W
    int tok, ntt, nkb, slab;  // tokens of a tile, token tiles, blocks of the contraction, of the sub-branch
    int stages, gate, kept_pitch;
    long long blocks;         // of all tiles
    uint32_t wait_looks;
    int test_skip_flag;
};

// The pieces of a CTA's range: blocks [kb0, kb1) of a tile, and whether the tile is its own.
struct Pieces {
    long long at, end;
    int nkb, tile, kb0, kb1;
    __device__ __forceinline__ Pieces(const EvenParams &p, int range) : at(p.blocks * range / gridDim.x), end(p.blocks * (range + 1) / gridDim.x), nkb(p.nkb) {}
    __device__ __forceinline__ bool next()
    {
        if (at >= end) return false;
        tile = (int)(at / nkb);
        kb0 = (int)(at - (long long)tile * nkb);
        kb1 = (int)min((long long)nkb, kb0 + (end - at));
        at += kb1 - kb0;
        return true;
    }
    __device__ __forceinline__ bool owner() const { return kb0 == 0; }
};
// The same block by block, the sub-branch's included (kb >= kb1).
struct Blocks {
    Pieces pc;
    int kb, last, slab;
    bool on;
    __device__ __forceinline__ Blocks(const EvenParams &p, int range) : pc(p, range), slab(p.slab) { open(); }
    __device__ __forceinline__ void open()
    {
        on = pc.next();
        kb = pc.kb0;
        last = pc.kb1 + (pc.owner() ? slab : 0);
    }
    __device__ __forceinline__ void step()
    {
        if (on && ++kb == last) open();
    }
};

__device__ __forceinline__ void store_release(uint32_t *p, uint32_t v) { asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory"); }
__device__ __forceinline__ uint32_t load_acquire(const uint32_t *p)
{
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, const uint32_t *v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t src, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(c0), "r"(c1), "r"(src) : "memory");
}
// Whole warp; bounded.
__device__ __forceinline__ bool wait_tag(const EvenParams &p, const uint32_t *word, uint32_t tag, volatile int *quit)
{
    const unsigned long long t0 = global_ns();
#pragma unroll 1
    for (uint32_t look = 1;; ++look) {
        if (__all_sync(0xffffffffu, load_acquire(word) == tag)) return true;
        const bool end = *quit || (p.wait_looks && look >= p.wait_looks) || ((look & 63u) == 0u && global_ns() - t0 > kWaitNs);
        if (__any_sync(0xffffffffu, end)) return false;
        __nanosleep(64);
    }
}

// A thread's 32 codes of a block, with their scale and zero point.
template <int BITS> struct Raw {
    uint32_t w[BITS == 4 ? 4 : 3];
    __half s, z;
};

template <int BITS, typename T, int MODE>
__device__ __forceinline__ bool dequantise(const EvenParams &p, int range, uint32_t sbase, uint32_t stage_bytes, uint32_t full0, uint32_t empty0, volatile int *quit)
{
    constexpr bool GRAD = MODE == kGrad;
    constexpr int NW = BITS == 4 ? 4 : 3;
    const int warp = (threadIdx.x >> 5) - kDqWarp, group = warp / kGroupWarps, lane = threadIdx.x & 31, tid = (int)(threadIdx.x - (kDqWarp + group * kGroupWarps) * 32);
    const int G = p.K / kGroupFast;
    // Forward: two lanes per row of 64 k.  Grad: four per row of 128 columns, so that any eight neighbouring lanes store to four rows and
    // both halves of a box's (different banks in the 128-byte swizzle).
    const int row = GRAD ? (warp % kGroupWarps) * 8 + ((lane >> 1) & 7) : tid >> 1, part = GRAD ? (lane >> 4) * 2 + (lane & 1) : tid & 1;
    const uint32_t dst = GRAD ? (uint32_t)(part >> 1) * kBox + (uint32_t)row * 128u : (uint32_t)row * 128u;
    const uint32_t chunk = (uint32_t)(part & 1) * 4u;
    auto load = [&](const Blocks &b, Raw<BITS> &r) {
        if (!b.on || b.kb >= b.pc.kb1) return;
        const int ft = b.pc.tile / p.ntt;
        const int n = GRAD ? b.kb * kBK + row : ft * kFeat + row, k = GRAD ? ft * kFeat + part * 32 : b.kb * kBK + part * 32;
        const bool in = n < (GRAD ? p.D : p.F);
        const uint32_t *src = p.qw + (in ? ((size_t)n * p.K + k) / 32 * NW : 0);
        if constexpr (BITS == 4) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(src));
            r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i) r.w[i] = __ldg(src + i);
        }
        const size_t g = in ? (size_t)n * G + k / kGroupFast : 0;
        r.s = in ? p.scales[g] : __half(0.f);                    // what lies outside is a row of zeros
        r.z = in ? p.zeros[g] : __half(0.f);
    };
    Blocks cur(p, range), ahead(p, range);
    uint32_t s = 0, phase = 1u;                                  // stage of `cur`, parity of its previous use
    bool first = true;
    auto skip = [&]() {
        if (++s == (uint32_t)p.stages) { s = 0; phase ^= 1u; first = false; }
    };
    if (group) {
        cur.step();
        ahead.step();
        skip();
    }
    Raw<BITS> r[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        load(ahead, r[i]);
        ahead.step();
        ahead.step();
    }
#pragma unroll 1
    for (;;) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (!cur.on) return true;
            const bool main = cur.kb < cur.pc.kb1;
            uint32_t out[16];
            if (main) {
                uint32_t d[16];
                Dequant<BITS, T>::run(r[i].w, __half2float(r[i].s), __half2float(r[i].z), d);
                natural_pairs<BITS>(d, out);
            }
            if (!__all_sync(0xffffffffu, first || umma::wait_cluster(empty0 + 8u * s, phase, quit))) return false;
            if (main) {
                const uint32_t at = sbase + s * stage_bytes + dst;
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) sts128(at + (((chunk + j) ^ ((uint32_t)row & 7u)) << 4), out + 4 * j);
                fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(full0 + 8u * s);
            load(ahead, r[i]);
            ahead.step();
            ahead.step();
            cur.step();
            cur.step();
            skip();
            skip();
        }
    }
}

// xmap: x (Grad: dy) [M][D], boxes of 64 x tok rows (tok / 2 above 256); tmap: t (s) [M][rank_pad], the same boxes; bmap: B [F][rank], boxes 64 x 128 rows
// (Grad: A [rank][F], 64 x 64, MN-major); all in the 128-byte swizzle.  ymap: h [M][F / 2], boxes of 16 rows x 64 columns (Grad: dx [M][F], x 128);
// cmap, Kept: codes [M][F], 16 rows x 128.
template <int BITS, typename T, int MODE>
__global__ void __launch_bounds__(kThreads, 1)
even_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap bmap,
            const __grid_constant__ CUtensorMap ymap, const __grid_constant__ CUtensorMap cmap, const EvenParams p)
{
    constexpr bool GRAD = MODE == kGrad;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t sbase = smem_u32(smem), stage_bytes = kWBytes + (uint32_t)p.tok * (kBK * 2u), y_off = (uint32_t)p.stages * stage_bytes;
    const uint32_t full0 = sbase + y_off + 2 * kYBytes + 512u, empty0 = full0 + 8u * kMostStages, accf0 = empty0 + 8u * kMostStages, acce0 = accf0 + 16u;
    float *amax = reinterpret_cast<float *>(smem + y_off + 2 * kYBytes);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + y_off + 2 * kYBytes + 512u + 16u * kMostStages + 32u);
    volatile int *quit = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, range = (int)(gridDim.x - 1 - blockIdx.x);
    const int halves = p.tok > 256 ? 2 : 1, cols = p.tok / halves;     // an MMA has 256 columns at most
    const int nbuf = halves == 1 ? 2 : 1;                               // accumulators in tensor memory

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) {
            mbar_init(full0 + 8u * i, 1 + kGroupWarps);
            mbar_init(empty0 + 8u * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(accf0 + 8u * i, 1);
            mbar_init(acce0 + 8u * i, 4);
        }
        *quit = 0;
        fence_barrier_init();
        prefetch_tensormap(&xmap);
        prefetch_tensormap(&ymap);
        if (p.slab) {
            prefetch_tensormap(&tmap);
            prefetch_tensormap(&bmap);
        }
    }
    if (warp == 1) umma::tmem_alloc<1>(smem_u32(tmem_slot), 512u);
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    uint32_t tag = 0;

    if (warp == 0) {
        // =================================================== copies
        if (lane == 0) {
            pdl_wait();                                          // (codes, scales and zero points are weights: the others do not wait)
            uint32_t s = 0, phase = 1u;
            bool first = true;
            const uint32_t xbytes = (uint32_t)p.tok * (kBK * 2u);
#pragma unroll 1
            for (Blocks b(p, range); b.on && ok; b.step()) {
                if (!first && !umma::wait_cluster(empty0 + 8u * s, phase, quit)) { ok = false; break; }
                const bool main = b.kb < b.pc.kb1;
                const int ft = b.pc.tile / p.ntt, m0 = (b.pc.tile - ft * p.ntt) * p.tok, c0 = (main ? b.kb : b.kb - b.pc.kb1) * kBK;
                const uint32_t bar = full0 + 8u * s, wt = sbase + s * stage_bytes, xt = wt + kWBytes;
                mbar_expect_tx(bar, main ? xbytes : xbytes + kWBytes);
                for (int h = 0; h < halves; ++h) tma_load_2d(xt + (uint32_t)(h * cols) * (kBK * 2u), main ? &xmap : &tmap, c0, m0 + h * cols, bar);
                if (!main) {
                    if (GRAD) {
                        for (int h = 0; h < 2; ++h) tma_load_2d(wt + h * kBox, &bmap, ft * kFeat + 64 * h, c0, bar);
                    } else {
                        tma_load_2d(wt, &bmap, c0, ft * kFeat, bar);
                    }
                }
                if (++s == (uint32_t)p.stages) { s = 0; phase ^= 1u; first = false; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // =================================================== MMAs
        if (lane == 0) {
            const uint32_t idesc = umma::idesc_f16(P2<T>::kFmt, kFeat, (uint32_t)cols) | (GRAD ? umma::kIdescMnA : 0u);
            const uint32_t wstep = GRAD ? 2048u >> 4 : 2u;
            uint32_t s = 0, phase = 0, it = 0;
#pragma unroll 1
            for (Pieces pc(p, range); ok && pc.next(); ++it) {
                const uint32_t buf = nbuf == 2 ? it & 1u : 0u, use = nbuf == 2 ? it >> 1 : it, d = tmem + buf * 256u;
                if (use > 0 && !umma::wait_cluster(acce0 + 8u * buf, (use - 1u) & 1u, quit)) { ok = false; break; }
                umma::fence_after();
                const int n = pc.kb1 - pc.kb0 + (pc.owner() ? p.slab : 0);
#pragma unroll 1
                for (int i = 0; i < n; ++i) {
                    if (!umma::wait_cluster(full0 + 8u * s, phase, quit)) { ok = false; break; }
                    umma::fence_after();
                    const uint32_t wt = sbase + s * stage_bytes;
                    const uint64_t wd = GRAD ? umma::desc_mn128(wt, kBox) : umma::desc_k128(wt), xd = umma::desc_k128(wt + kWBytes);
#pragma unroll
                    for (int j = 0; j < kBK / 16; ++j) {
                        umma::mma(d, wd + wstep * j, xd + 2 * j, idesc, i > 0 || j > 0);
                        if (halves == 2) umma::mma(d + (uint32_t)cols, wd + wstep * j, xd + 2 * j + (uint32_t)cols * (kBK * 2u >> 4), idesc, i > 0 || j > 0);
                    }
                    umma::commit(empty0 + 8u * s);
                    if (++s == (uint32_t)p.stages) { s = 0; phase ^= 1u; }
                }
                if (ok) umma::commit(accf0 + 8u * buf);
            }
        }
        __syncwarp();
    } else if (warp >= 4 && warp < kDqWarp) {
        // =================================================== epilogue: lane = feature, column = token
        pdl_wait();
        tag = load_acquire(p.tags + kTagEpoch) + 1u;
        const int wq = warp & 3;
        uint32_t it = 0, staged = 0;
#pragma unroll 1
        for (Pieces pc(p, range); ok && pc.next(); ++it) {
            const uint32_t buf = nbuf == 2 ? it & 1u : 0u, use = nbuf == 2 ? it >> 1 : it;
            ok = named_barrier_and(1, 128, umma::wait_cluster(accf0 + 8u * buf, use & 1u, quit));      // (four warps go on, or none)
            if (!ok) break;
            umma::fence_after();
            const uint32_t lanes = tmem + buf * 256u + ((uint32_t)(32 * wq) << 16);
            const int ft = pc.tile / p.ntt, m0 = (pc.tile - ft * p.ntt) * p.tok, m_end = min(p.M, m0 + p.tok), n = ft * kFeat + 32 * wq + lane;
            if (!pc.owner()) {
                float *dst = p.part + (size_t)range * p.tok * kFeat + 32 * wq + lane;
#pragma unroll 1
                for (int c = 0; c < m_end - m0; c += 32) {
                    uint32_t v[32];
                    umma::ld32(lanes + (uint32_t)c, v);
                    umma::wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (c + j < m_end - m0) __stcg(dst + (size_t)(c + j) * kFeat, __uint_as_float(v[j]));
                }
                umma::fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(acce0 + 8u * buf);
                __threadfence();
                named_barrier_sync(1, 128);
                if (threadIdx.x == 4 * 32 && !p.test_skip_flag) store_release(p.tags + kTagFirst + range, tag);
                continue;
            }
            // ranges behind this one that hold blocks of the tile
            const long long tile_end = (long long)(pc.tile + 1) * p.nkb;
            int others = 0;
            while (range + others + 1 < (int)gridDim.x && p.blocks * (range + others + 1) / gridDim.x < tile_end) ++others;
            for (int o = 1; o <= others && ok; ++o) ok = wait_tag(p, p.tags + kTagFirst + range + o, tag, quit);
            if (others) ok = named_barrier_and(1, 128, ok);
            if (!ok) break;
#pragma unroll 1
            for (int c = 0; c < p.tok; c += 32) {
                uint32_t v[32];
                umma::ld32(lanes + (uint32_t)c, v);
                umma::wait_ld();
                if (c + 32 >= p.tok) {                           // all of the accumulator is in registers
                    umma::fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acce0 + 8u * buf);
                }
                if (m0 + c >= p.M) continue;
#pragma unroll 1
                for (int o = 1; o <= others; ++o) {
                    const float *src = p.part + ((size_t)(range + o) * p.tok + c) * kFeat + 32 * wq + lane;
                    float e[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) e[j] = c + j < m_end - m0 ? __ldcg(src + (size_t)j * kFeat) : 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + e[j]);
                }
                const uint32_t at = y_off + (staged & 1u) * kYBytes;
                if (threadIdx.x == 4 * 32) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                if constexpr (MODE == kKept) {                   // the largest |p| of each token over this warp's rows, lane = token
                    uint32_t mine = 0u;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const uint32_t top = __reduce_max_sync(0xffffffffu, v[j] & 0x7FFFFFFFu);
                        if (lane == j) mine = top;
                    }
                    amax[32 * wq + lane] = __uint_as_float(mine);
                }
                named_barrier_sync(1, 128);                      // the buffer's last copy has been read
                if constexpr (GRAD) {
                    unsigned short *row = reinterpret_cast<unsigned short *>(smem + at) + 32 * wq + lane;
#pragma unroll
                    for (int j = 0; j < 32; ++j) row[j * 128] = to_bits16<T>(__uint_as_float(v[j]));
                } else {
                    gate_chunk<T>(p.gate, v, reinterpret_cast<T *>(smem + at) + 16 * wq);
                }
                if constexpr (MODE == kKept) {                   // a tile's 128 rows are the columns that share a scale
                    uint32_t top = 0u;
#pragma unroll
                    for (int w = 0; w < 4; ++w) top = max(top, __float_as_uint(amax[32 * w + lane]));
                    float scale, inverse;
                    kept_scale(top, scale, inverse);
                    if (wq == 0 && lane < m_end - (m0 + c)) p.kept_scales[(size_t)(m0 + c + lane) * p.kept_pitch + ft] = scale;
                    uint8_t *codes = smem + at + kYBytes / 2 + 32 * wq + lane;
#pragma unroll
                    for (int j = 0; j < 32; ++j) codes[j * 128] = (uint8_t)kept_code(__uint_as_float(v[j]), __shfl_sync(0xffffffffu, inverse, j));
                }
                fence_proxy_async();
                named_barrier_sync(1, 128);
                if (threadIdx.x == 4 * 32) {
                    const int n_first = n - lane, out = GRAD ? n_first : n_first / 2;
                    const bool both = c + 16 < p.tok && m0 + c + 16 < m_end;
                    tma_store_2d(&ymap, sbase + at, out, m0 + c);
                    if (both) tma_store_2d(&ymap, sbase + at + kYBytes / (GRAD ? 2 : 4), out, m0 + c + 16);
                    if (MODE == kKept) {
                        tma_store_2d(&cmap, sbase + at + kYBytes / 2, n_first, m0 + c);
                        if (both) tma_store_2d(&cmap, sbase + at + kYBytes / 2 + kYBytes / 4, n_first, m0 + c + 16);
                    }
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
                ++staged;
            }
        }
        if (threadIdx.x == 4 * 32) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else if (warp >= kDqWarp) {
        ok = dequantise<BITS, T, MODE>(p, range, sbase, stage_bytes, full0, empty0, quit);
    }
    if (!ok) {
        *quit = 1;
        atomicExch(p.status, (int)FBQ_ERR_TIMEOUT);
        for (int i = 0; i < 64; ++i) __nanosleep(1000);          // copies in flight land before the CTA leaves
    }
    umma::fence_before();
    __syncthreads();
    if (warp == 1) {
        umma::fence_after();
        umma::tmem_free<1>(tmem, 512u);
    }
    if (threadIdx.x == 4 * 32) {                                 // (this thread has waited for the launch before)
        __threadfence();
        if (atomicAdd(p.tags + kTagDone, 1u) == gridDim.x - 1) { // the last CTA: the next launch's tags are other ones
            p.tags[kTagDone] = 0;
            __threadfence();
            p.tags[kTagEpoch] = tag;
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------
int sms_of_device()
{
    static int n = 0;
    if (n == 0) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
    }
    return n;
}
// Tokens of a tile: all of them up to kMostTok, else equal parts.  Above 256 two MMAs share them, each a multiple of 16.
void token_tiles(int M, int *tok, int *ntt)
{
    *ntt = (M + kMostTok - 1) / kMostTok;
    const int m = (M + *ntt - 1) / *ntt;
    *tok = m <= 256 ? (m + 15) / 16 * 16 : (m + 31) / 32 * 32;
}
long long all_blocks(int ntt, int F, int D) { return (long long)((F + kFeat - 1) / kFeat) * ntt * ((D + kBK - 1) / kBK); }
int ctas_for(long long blocks) { return (int)std::min<long long>(sms_of_device(), blocks); }

template <int BITS, typename T, int MODE>
cudaError_t start(const CUtensorMap (&maps)[5], const EvenParams &p, bool pdl, cudaStream_t s)
{
    auto kern = even_kernel<BITS, T, MODE>;
    static bool attr_set = false;
    if (!attr_set) {
        if (const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost + 1024); e != cudaSuccess) return e;
        attr_set = true;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas_for(p.blocks));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)p.stages * (kWBytes + p.tok * (kBK * 2u)) + kFixed + 1024;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, maps[0], maps[1], maps[2], maps[3], maps[4], p);
}

}  // namespace

size_t even_part_bytes(int M, int F, int D)
{
    int tok, ntt;
    token_tiles(M, &tok, &ntt);
    return (size_t)ctas_for(all_blocks(ntt, F, D)) * tok * kFeat * sizeof(float);
}
size_t even_tags() { return (size_t)kTagFirst + sms_of_device(); }

cudaError_t launch_even(const EvenArgs &a, Workspace &ws, const PrefillTuning &tune, cudaStream_t s, int *launches)
{
    const bool grad = a.gate < 0;
    EvenParams p{};
    p.qw = a.qw; p.scales = a.scales; p.zeros = a.zeros;
    p.part = static_cast<float *>(a.part);
    p.tags = ws.tags;
    p.status = ws.counters + kCtrStatus;
    p.M = a.M; p.K = a.K;
    p.F = grad ? a.K : a.N;
    p.D = grad ? a.N : a.K;
    token_tiles(a.M, &p.tok, &p.ntt);
    p.nkb = (p.D + kBK - 1) / kBK;
    const int rank_pad = (a.rank + kBK - 1) / kBK * kBK;
    p.slab = rank_pad / kBK;
    p.stages = (int)std::min<uint32_t>(kMostStages, (kSmemMost - kFixed) / (kWBytes + p.tok * (kBK * 2u)));
    p.gate = a.gate;
    p.kept_scales = a.kept_scales;
    p.kept_pitch = (p.F + kKeptGroup - 1) / kKeptGroup;
    p.blocks = all_blocks(p.ntt, p.F, p.D);
    p.wait_looks = tune.flag_polls > 0 ? (uint32_t)tune.flag_polls : 0u;
    p.test_skip_flag = tune.test_skip_flag;
    const CUtensorMapDataType dt = CU_TENSOR_MAP_DATA_TYPE_UINT16;
    const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B, none = CU_TENSOR_MAP_SWIZZLE_NONE;
    const int box = p.tok > 256 ? p.tok / 2 : p.tok;
    CUtensorMap maps[5];
    cudaError_t e;
    if ((e = encode_map(&maps[0], matrix_map(a.x, dt, 2, p.D, a.M, kBK, box, sw))) != cudaSuccess) return e;
    maps[1] = maps[2] = maps[0];
    if (a.rank > 0) {
        if ((e = encode_map(&maps[1], matrix_map(a.thin, dt, 2, rank_pad, a.M, kBK, box, sw))) != cudaSuccess) return e;
        if ((e = cached_map(&maps[2], grad ? matrix_map(a.factor, dt, 2, a.K, a.rank, kBK, kBK, sw) : matrix_map(a.factor, dt, 2, a.rank, a.N, kBK, kFeat, sw))) !=
            cudaSuccess)
            return e;
    }
    if ((e = encode_map(&maps[3], grad ? matrix_map(a.y, dt, 2, a.K, a.M, 128, 16, none) : matrix_map(a.y, dt, 2, a.N / 2, a.M, 64, 16, none))) != cudaSuccess) return e;
    maps[4] = maps[3];
    if (a.kept && (e = encode_map(&maps[4], matrix_map(a.kept, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.N, a.M, 128, 16, none))) != cudaSuccess) return e;
    auto go = [&](auto mode) {
        constexpr int MODE = decltype(mode)::value;
        const bool pdl = tune.pdl != 0;
        return a.bits == 4 ? (a.bf16 ? start<4, __nv_bfloat16, MODE>(maps, p, pdl, s) : start<4, __half, MODE>(maps, p, pdl, s))
                           : (a.bf16 ? start<3, __nv_bfloat16, MODE>(maps, p, pdl, s) : start<3, __half, MODE>(maps, p, pdl, s));
    };
    e = grad ? go(std::integral_constant<int, kGrad>{}) : a.kept ? go(std::integral_constant<int, kKept>{}) : go(std::integral_constant<int, kGated>{});
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace fbq
