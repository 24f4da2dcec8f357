// The gated block and dx of a layer's backward pass for few hundred tokens, sm_100a: weights dequantised where they are multiplied, and
// the blocks of the contraction shared out evenly.
//
//   h = f(gate) * up,  p = x.dequant(Q,s,z)^T + t.B^T          (forward; t = x.A^T from the launch before, fbq_thin.cu)
//   dx = dy.dequant(Q,s,z) + s.A                               (Grad; s = dy.B from there)
//
// Up to a few hundred tokens a weight is used too seldom to be dequantised in a pass of its own (the dense kernel's 16-bit copy costs 4
// bytes a weight through L2 beside the half byte of its code), and tiles are fewer than SMs or fill a second wave badly.  So a CTA turns
// codes into the operand in shared memory, 256 features for up to 192 tokens (128 features would read x twice as often, 64 bytes a clock and SM:
// more than L2 gives all of them), and the pairs of blocks of all tiles, in order, are cut into equal ranges, one per CTA:
//
//   warps 2, 3   bring the packed codes of a pair of blocks, 2 x 128 rows x one quantisation group, by TMA, and their scales and zero points
//   warps 8-23   dequantise them, 64 codes a thread: eight warps for either half of the features, into two stages of the operands
//   warp 0       copies the tokens by TMA, and both operands of the sub-branch's blocks
//   warp 1       issues tcgen05.mma, 128 features x tokens x 16, for both halves
//   warps 4-7    epilogue: of a tile that several CTAs share all but one store their fp32 sums; the one that holds its first block owns it, adds the
//                others' in order of the contraction and writes the outputs
//
// A range ends with the tiles it owns and begins with the one it does not, so whoever waits for sums waits for what another CTA did
// first.  CTA b takes the last range but b: ranges behind one's own belong to CTAs with lower numbers, which start earlier, and
// wait only for lower numbers still; any number of resident CTAs makes progress.  The sub-branch's blocks are the owner's, at the end of a tile.
// Sums do not depend on timing.  Tags of finished sums carry the launch's number (as in fbq_dense.cu, with the same words): nothing is cleared.
// All waits are bounded.
//
// Forward, features are rows of W and the operand is K-major: a pair of blocks is one group of each row.  Grad, features are its columns,
// 128 of them one group; a pair of blocks is 128 rows of it, and the operand is MN-major: rows are written as they lie.
//
// (Pairs of CTAs with cta_group::2 and half the tokens each were built as well: the dequantising warps' fence towards the asynchronous proxy
// then took 1500 cycles instead of 150, 77 tokens of 4096 -> 2 x 11008 41 us.)
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

constexpr int kBK = 64, kHalf = 128, kFeat = 2 * kHalf;
constexpr uint32_t kHalfBytes = kHalf * kBK * 2u, kWBytes = 2 * kHalfBytes, kBox = kHalfBytes / 2;
constexpr int kMostTok = 192, kMostStages = 6;
constexpr int kDqWarp = 8, kGroupWarps = 8, kThreads = (kDqWarp + 2 * kGroupWarps) * 32;
constexpr int kRing = 2;                         // pairs of blocks whose codes and scales are there or on their way
constexpr uint32_t kCodeBytes = 128u * 64u, kSlotBytes = 2 * (kCodeBytes + 512u);      // codes of both halves (INT3: 48 of 64 bytes a row), scales and zero points
constexpr int kScaleAhead = 3;                   // pairs whose scales a loading warp has requested
constexpr uint32_t kYBytes = 32u * 128u * 2u;    // staged part of an output tile: 32 tokens
constexpr uint32_t kFixed = kRing * kSlotBytes + 2 * kYBytes + 512 + 256;     // ring, staging, largest |p|, barriers
constexpr uint32_t kSmemMost = 227 * 1024 - 1024;        // (the base is moved up to 1024 bytes)
constexpr int kTagEpoch = 0, kTagDone = 1, kTagFirst = 4;        // words of the tag scratch, shared with fbq_dense.cu

enum Mode { kGated, kKept, kGrad };

struct EvenParams {
    int ranges;
    const __half *scales, *zeros;
    float *part;              // [range][half][tok][kHalf] sums of the tile that a range begins with and does not own
    uint32_t *tags;           // see above; a word per range
    float *kept_scales;
    int *status;
    int M, F, D, K;           // tokens, features, contraction, columns of W
    int tok, ntt, nkp, slab;  // tokens of a tile, token tiles, pairs of blocks of the contraction, blocks of the sub-branch
    int stages, gate, kept_pitch;
    long long pairs;          // of all tiles
    uint32_t wait_looks;
    int test_skip_flag;
};

// The pieces of a CTA's range: pairs of blocks [kp0, kp1) of a tile, and whether the tile is its own.
struct Pieces {
    long long at, end;
    int nkp, tile, kp0, kp1;
    __device__ __forceinline__ Pieces(const EvenParams &p, int range) : at(p.pairs * range / p.ranges), end(p.pairs * (range + 1) / p.ranges), nkp(p.nkp) {}
    __device__ __forceinline__ bool next()
    {
        if (at >= end) return false;
        tile = (int)(at / nkp);
        kp0 = (int)(at - (long long)tile * nkp);
        kp1 = (int)min((long long)nkp, kp0 + (end - at));
        at += kp1 - kp0;
        return true;
    }
    __device__ __forceinline__ bool owner() const { return kp0 == 0; }
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

__device__ __forceinline__ uint32_t ldg_u16(const __half *p)
{
    uint32_t v;
    asm volatile("ld.global.nc.u16 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 lds_v2(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

// Warps 2 and 3: the ring.  Scales and zero points lie 2 bytes here and there (an instruction touches as many lines as it has lanes),
// so each is loaded once per row and pair, kScaleAhead pairs before it is stored.
template <int BITS, int MODE>
__device__ __forceinline__ bool load_codes(const EvenParams &p, const CUtensorMap *qmap, int range, uint32_t ring, uint32_t rfull0, uint32_t rempty0, volatile int *quit)
{
    constexpr bool GRAD = MODE == kGrad;
    constexpr uint32_t kWords = BITS == 4 ? 16 : 12;
    const int lane = threadIdx.x & 31, half = (int)(threadIdx.x >> 5) - 2, G = p.K / kGroupFast;
    struct Scales {
        uint32_t v[8];
        bool on;
    };
    Pieces ahead(p, range);
    int kp = 0;
    bool on = ahead.next();
    kp = ahead.kp0;
    auto request = [&](Scales &c) {
        c.on = on;
        if (!on) return;
        const int ft = 2 * (ahead.tile / p.ntt) + half, n0 = (GRAD ? kp : ft) * kHalf + lane, g = GRAD ? ft : kp, rows = g < G ? (GRAD ? p.D : p.F) : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t at = (size_t)(n0 + 32 * i) * G + g;
            c.v[2 * i] = c.v[2 * i + 1] = 0u;                    // what lies outside is a row of zeros
            if (n0 + 32 * i < rows) {
                c.v[2 * i] = ldg_u16(p.scales + at);
                c.v[2 * i + 1] = ldg_u16(p.zeros + at);
            }
        }
        if (++kp == ahead.kp1) {
            on = ahead.next();
            kp = ahead.kp0;
        }
    };
    Scales c[kScaleAhead];
#pragma unroll
    for (int i = 0; i < kScaleAhead; ++i) request(c[i]);
    Pieces cur(p, range);
    cur.next();
    int ck = cur.kp0;
    uint32_t slot = 0, phase = 1u;
    bool first = true;
#pragma unroll 1
    for (;;) {
#pragma unroll
        for (int i = 0; i < kScaleAhead; ++i) {
            if (!c[i].on) return true;
            if (!__all_sync(0xffffffffu, first || umma::wait(rempty0 + 8u * slot, phase, quit))) return false;
            const uint32_t dst = ring + slot * kSlotBytes, bar = rfull0 + 8u * slot;
            if (half == 0 && lane == 0) {
                const int ft = 2 * (cur.tile / p.ntt);
                mbar_expect_tx(bar, 2u * 128u * kWords * 4u);
                for (int h = 0; h < 2; ++h) tma_load_2d(dst + h * kCodeBytes, qmap, (GRAD ? ft + h : ck) * (int)kWords, (GRAD ? ck : ft + h) * kHalf, bar);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + 2 * kCodeBytes + (uint32_t)(128 * half + lane + 32 * k) * 4u), "r"(c[i].v[2 * k] | c[i].v[2 * k + 1] << 16)
                             : "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
            request(c[i]);
            if (++ck == cur.kp1) {
                cur.next();
                ck = cur.kp0;
            }
            if (++slot == kRing) { slot = 0; phase ^= 1u; first = false; }
        }
    }
}

template <int BITS, typename T, int MODE>
__device__ __forceinline__ bool dequantise(const EvenParams &p, int range, uint32_t sbase, uint32_t stage_bytes, uint32_t ring, uint32_t full0, uint32_t empty0,
                                           uint32_t rfull0, uint32_t rempty0, volatile int *quit)
{
    constexpr bool GRAD = MODE == kGrad;
    constexpr int NW = BITS == 4 ? 4 : 3;
    const int warp = (threadIdx.x >> 5) - kDqWarp, group = warp / kGroupWarps, w = warp % kGroupWarps, lane = threadIdx.x & 31;
    // A thread's row of the pair and its 64 of the row's 128 codes.  Forward those are the pair's block and the row the operand's; Grad the
    // row's half chooses the block and the codes a box of the operand.  Eight neighbouring lanes store to eight rows: different banks in the
    // 128-byte swizzle, as they load them from different banks (INT4: the 64-byte swizzle of the copy).
    const int row = 32 * (w & 3) + lane, part = w >> 2, blk = GRAD ? row >> 6 : part;
    const uint32_t r = GRAD ? row & 63 : row;
    const uint32_t dst = sbase + (uint32_t)group * kHalfBytes + (GRAD ? (uint32_t)part * kBox : 0u) + r * 128u + ((r & 7u) << 4);          // unit j: ^ (j << 4)
    const uint32_t src = BITS == 4 ? (uint32_t)row * 64u + ((((uint32_t)row >> 1) & 3u) << 4) : (uint32_t)row * 48u + (uint32_t)part * 24u;
    Pieces pc(p, range);
    uint32_t s = 0, use = 0;                                     // stage of the next block, times it has been used
    uint32_t q = 0;                                              // pairs so far
    const uint32_t stages = (uint32_t)p.stages;
    auto free_again = [&](uint32_t stage, uint32_t n) { return __all_sync(0xffffffffu, n == 0 || umma::wait(empty0 + 8u * stage, (n - 1u) & 1u, quit)) != 0; };
    while (pc.next()) {
        const int n = pc.kp1 - pc.kp0;
#pragma unroll 1
        for (int k = 0; k < n; ++k, ++q) {
            // the stage of this thread's block, and its use before this one (the sub-branch's blocks are waited for as well: a wait tells one
            // phase of a barrier from the next, not from the one after that)
            uint32_t st = s + (uint32_t)blk, u = use;
            if (st >= stages) {
                st -= stages;
                ++u;
            }
            {
                const uint32_t slot = q % kRing, at = ring + slot * kSlotBytes + (uint32_t)group * kCodeBytes;
                if (!__all_sync(0xffffffffu, umma::wait(rfull0 + 8u * slot, (q / kRing) & 1u, quit))) return false;
                uint32_t c[2 * NW];
                if constexpr (BITS == 4) {
                    const uint4 a = lds128(at + (src ^ (uint32_t)(part << 5))), b = lds128(at + (src ^ (uint32_t)(part << 5 | 16)));
                    c[0] = a.x; c[1] = a.y; c[2] = a.z; c[3] = a.w;
                    c[4] = b.x; c[5] = b.y; c[6] = b.z; c[7] = b.w;
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        const uint2 a = lds_v2(at + src + 8u * i);
                        c[2 * i] = a.x;
                        c[2 * i + 1] = a.y;
                    }
                }
                uint32_t sz;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(sz) : "r"(ring + slot * kSlotBytes + 2 * kCodeBytes + (uint32_t)(128 * group + row) * 4u) : "memory");
                const float fs = __half2float(__ushort_as_half((unsigned short)(sz & 0xFFFFu))), fz = __half2float(__ushort_as_half((unsigned short)(sz >> 16)));
                const uint32_t to = dst + st * stage_bytes;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t d[16], out[16];
                    Dequant<BITS, T>::run(c + NW * i, fs, fz, d);
                    natural_pairs<BITS>(d, out);
                    if (i == 0) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(rempty0 + 8u * slot);         // (this warp has its codes in registers)
                        if (!free_again(st, u)) return false;
                    }
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) sts128(to ^ ((4u * i + j) << 4), out + 4 * j);
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(full0 + 8u * st);
            }
            s += 2;
            if (s >= stages) {
                s -= stages;
                ++use;
            }
        }
        if (pc.owner()) {                                        // the sub-branch's stages are made by copies
            for (int k = 0; k < p.slab; ++k) {
                if (!free_again(s, use)) return false;
                if (++s == stages) {
                    s = 0;
                    ++use;
                }
            }
        }
    }
    return true;
}

// xmap: x (Grad: dy) [M][D], boxes of 64 x tok rows; tmap: t (s) [M][rank_pad], the same boxes; bmap: B [F][rank], boxes 64 x 128 rows
// (Grad: A [rank][F], 64 x 64, MN-major); all in the 128-byte swizzle.  ymap: h [M][F / 2], boxes of 16 rows x 64 columns (Grad: dx [M][F], x 128);
// cmap, Kept: codes [M][F], 16 rows x 128.  qmap: packed codes [rows of W][words], boxes of 128 rows x one group (INT4: 64-byte swizzle).
template <int BITS, typename T, int MODE>
__global__ void __launch_bounds__(kThreads, 1)
even_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap bmap,
            const __grid_constant__ CUtensorMap ymap, const __grid_constant__ CUtensorMap cmap, const __grid_constant__ CUtensorMap qmap, const EvenParams p)
{
    constexpr bool GRAD = MODE == kGrad;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t sbase = smem_u32(smem), stage_bytes = kWBytes + (uint32_t)p.tok * (kBK * 2u), y_off = (uint32_t)p.stages * stage_bytes;
    const uint32_t ring = sbase + y_off + 2 * kYBytes, bars = kRing * kSlotBytes + 512u;
    const uint32_t full0 = ring + bars, empty0 = full0 + 8u * kMostStages, accf0 = empty0 + 8u * kMostStages, acce0 = accf0 + 16u, rfull0 = acce0 + 16u,
                   rempty0 = rfull0 + 8u * kRing;
    float *amax = reinterpret_cast<float *>(smem + y_off + 2 * kYBytes + kRing * kSlotBytes);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + y_off + 2 * kYBytes + bars + 16u * kMostStages + 32u + 16u * kRing);
    volatile int *quit = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, range = p.ranges - 1 - (int)blockIdx.x;
    // accumulators in tensor memory: two of two halves where they fit
    const uint32_t wide = p.tok > 128 ? 256u : 128u;
    const int nbuf = p.tok > 128 ? 1 : 2;

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) {
            mbar_init(full0 + 8u * i, 1 + kGroupWarps);          // the copying lane, and four warps of either half
            mbar_init(empty0 + 8u * i, 1);
        }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(rfull0 + 8u * i, 3);                       // the copy's lane and both loading warps
            mbar_init(rempty0 + 8u * i, 2 * kGroupWarps);
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
        prefetch_tensormap(&qmap);
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
            for (Pieces pc(p, range); ok && pc.next();) {
                const int ft = pc.tile / p.ntt, m0 = (pc.tile - ft * p.ntt) * p.tok, main = 2 * (pc.kp1 - pc.kp0), n = main + (pc.owner() ? p.slab : 0);
#pragma unroll 1
                for (int i = 0; i < n; ++i) {
                    if (!first && !umma::wait(empty0 + 8u * s, phase, quit)) { ok = false; break; }
                    const bool mine = i < main;
                    const int c0 = (mine ? 2 * pc.kp0 + i : i - main) * kBK;
                    const uint32_t bar = full0 + 8u * s, wt = sbase + s * stage_bytes, xt = wt + kWBytes;
                    mbar_expect_tx(bar, mine ? xbytes : xbytes + kWBytes);
                    tma_load_2d(xt, mine ? &xmap : &tmap, c0, m0, bar);
                    if (!mine) {
                        if (GRAD) {
                            for (int h = 0; h < 4; ++h) tma_load_2d(wt + h * kBox, &bmap, ft * kFeat + 64 * h, c0, bar);
                        } else {
                            for (int h = 0; h < 2; ++h) tma_load_2d(wt + h * kHalfBytes, &bmap, c0, ft * kFeat + kHalf * h, bar);
                        }
                        for (int k = 0; k < kGroupWarps; ++k) mbar_arrive(bar);          // (for the warps that have nothing to make)
                    }
                    if (++s == (uint32_t)p.stages) { s = 0; phase ^= 1u; first = false; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // =================================================== MMAs
        // The whole warp walks the loop and one elected lane issues: the MMAs' operands stay in uniform registers.  Two blocks at a time.
        const uint32_t idesc = umma::idesc_f16(P2<T>::kFmt, kHalf, (uint32_t)p.tok) | (GRAD ? umma::kIdescMnA : 0u);
        const uint32_t wstep = GRAD ? 2048u >> 4 : 2u;
        const uint64_t wd0 = GRAD ? umma::desc_mn128(sbase, kBox) : umma::desc_k128(sbase), xd0 = umma::desc_k128(sbase + kWBytes);
        uint32_t s = 0, phase = 0, it = 0;
#pragma unroll 1
        for (Pieces pc(p, range); ok && pc.next(); ++it) {
            const uint32_t buf = nbuf == 2 ? it & 1u : 0u, use = nbuf == 2 ? it >> 1 : it, d = tmem + buf * 256u;
            ok = __all_sync(0xffffffffu, use == 0 || umma::wait(acce0 + 8u * buf, (use - 1u) & 1u, quit));
            const int n = 2 * (pc.kp1 - pc.kp0) + (pc.owner() ? p.slab : 0);
#pragma unroll 1
            for (int i = 0; i < n && ok; i += 2) {
                const bool two = i + 1 < n;
                const uint32_t s0 = s, s1 = s + 1 == (uint32_t)p.stages ? 0u : s + 1, ph0 = phase, ph1 = s1 ? phase : phase ^ 1u;
                ok = umma::wait(full0 + 8u * s0, ph0, quit);
                if (two) ok = umma::wait(full0 + 8u * s1, ph1, quit) && ok;
                ok = __all_sync(0xffffffffu, ok);
                umma::fence_after();
                if (ok && umma::elect_one()) {
                    auto block = [&](uint32_t stage, bool more) {
                        const uint64_t wd = wd0 + stage * (stage_bytes >> 4), xd = xd0 + stage * (stage_bytes >> 4);
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int j = 0; j < kBK / 16; ++j) umma::mma(d + h * wide, wd + h * (kHalfBytes >> 4) + wstep * j, xd + 2 * j, idesc, more || j > 0);
                        umma::commit(empty0 + 8u * stage);
                    };
                    block(s0, i > 0);
                    if (two) block(s1, true);
                    if (i + 2 >= n) umma::commit(accf0 + 8u * buf);
                }
                __syncwarp();
                s = two ? s1 : s0;
                phase = two ? ph1 : ph0;
                if (++s == (uint32_t)p.stages) { s = 0; phase ^= 1u; }
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
            ok = named_barrier_and(1, 128, umma::wait(accf0 + 8u * buf, use & 1u, quit));      // (four warps go on, or none)
            if (!ok) break;
            umma::fence_after();
            const int ft = pc.tile / p.ntt, m0 = (pc.tile - ft * p.ntt) * p.tok, m_end = min(p.M, m0 + p.tok);
            int others = 0;                                      // ranges behind this one that hold blocks of a tile of ours
            if (pc.owner()) {
                const long long tile_end = (long long)(pc.tile + 1) * p.nkp;
                while (range + others + 1 < p.ranges && p.pairs * (range + others + 1) / p.ranges < tile_end) ++others;
                for (int o = 1; o <= others && ok; ++o) ok = wait_tag(p, p.tags + kTagFirst + range + o, tag, quit);
                if (others) ok = named_barrier_and(1, 128, ok);
                if (!ok) break;
            }
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const uint32_t lanes = tmem + buf * 256u + h * wide + ((uint32_t)(32 * wq) << 16);
                const int n = ft * kFeat + h * kHalf + 32 * wq + lane;
                const size_t part_at = (size_t)(2 * range + h) * p.tok * kHalf + 32 * wq + lane;
#pragma unroll 1
                for (int c = 0; c < p.tok; c += 32) {
                    uint32_t v[32];
                    umma::ld32(lanes + (uint32_t)c, v);
                    umma::wait_ld();
                    if (h == 1 && c + 32 >= p.tok) {             // all of the accumulators is in registers
                        umma::fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(acce0 + 8u * buf);
                    }
                    if (m0 + c >= p.M) continue;
                    if (!pc.owner()) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (c + j < m_end - m0) __stcg(p.part + part_at + (size_t)(c + j) * kHalf, __uint_as_float(v[j]));
                        continue;
                    }
#pragma unroll 1
                    for (int o = 1; o <= others; ++o) {
                        const float *src = p.part + part_at + ((size_t)2 * o * p.tok + c) * kHalf;
                        float e[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) e[j] = c + j < m_end - m0 ? __ldcg(src + (size_t)j * kHalf) : 0.f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + e[j]);
                    }
                    const uint32_t at = y_off + (staged & 1u) * kYBytes;
                    if (threadIdx.x == 4 * 32) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                    if constexpr (MODE == kKept) {               // the largest |p| of each token over this warp's rows, lane = token
                        uint32_t mine = 0u;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const uint32_t top = __reduce_max_sync(0xffffffffu, v[j] & 0x7FFFFFFFu);
                            if (lane == j) mine = top;
                        }
                        amax[32 * wq + lane] = __uint_as_float(mine);
                    }
                    named_barrier_sync(1, 128);                  // the buffer's last copy has been read
                    if constexpr (GRAD) {
                        unsigned short *row = reinterpret_cast<unsigned short *>(smem + at) + 32 * wq + lane;
#pragma unroll
                        for (int j = 0; j < 32; ++j) row[j * 128] = to_bits16<T>(__uint_as_float(v[j]));
                    } else {
                        gate_chunk<T>(p.gate, v, reinterpret_cast<T *>(smem + at) + 16 * wq);
                    }
                    if constexpr (MODE == kKept) {               // a half's 128 rows are the columns that share a scale
                        uint32_t top = 0u;
#pragma unroll
                        for (int w = 0; w < 4; ++w) top = max(top, __float_as_uint(amax[32 * w + lane]));
                        float scale, inverse;
                        kept_scale(top, scale, inverse);
                        if (wq == 0 && n - lane < p.F && lane < m_end - (m0 + c)) p.kept_scales[(size_t)(m0 + c + lane) * p.kept_pitch + 2 * ft + h] = scale;
                        uint8_t *codes = smem + at + kYBytes / 2 + 32 * wq + lane;
#pragma unroll
                        for (int j = 0; j < 32; ++j) codes[j * 128] = (uint8_t)kept_code(__uint_as_float(v[j]), __shfl_sync(0xffffffffu, inverse, j));
                    }
                    fence_proxy_async();
                    named_barrier_sync(1, 128);
                    if (threadIdx.x == 4 * 32 && n < p.F) {
                        const int out = GRAD ? n : n / 2;        // (lane 0's n is the half's first)
                        const bool both = c + 16 < p.tok && m0 + c + 16 < m_end;
                        tma_store_2d(&ymap, sbase + at, out, m0 + c);
                        if (both) tma_store_2d(&ymap, sbase + at + kYBytes / (GRAD ? 2 : 4), out, m0 + c + 16);
                        if (MODE == kKept) {
                            tma_store_2d(&cmap, sbase + at + kYBytes / 2, n, m0 + c);
                            if (both) tma_store_2d(&cmap, sbase + at + kYBytes / 2 + kYBytes / 4, n, m0 + c + 16);
                        }
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                    ++staged;
                }
            }
            if (!pc.owner()) {
                __threadfence();
                named_barrier_sync(1, 128);
                if (threadIdx.x == 4 * 32 && !p.test_skip_flag) store_release(p.tags + kTagFirst + range, tag);
            }
        }
        if (threadIdx.x == 4 * 32) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else if (warp >= kDqWarp) {
        ok = dequantise<BITS, T, MODE>(p, range, sbase, stage_bytes, ring, full0, empty0, rfull0, rempty0, quit);
    } else {
        ok = load_codes<BITS, MODE>(p, &qmap, range, ring, rfull0, rempty0, quit);
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
// Tokens of a tile: all of them up to kMostTok, else equal parts, in sixteens.
void token_tiles(int M, int *tok, int *ntt)
{
    *ntt = (M + kMostTok - 1) / kMostTok;
    *tok = ((M + *ntt - 1) / *ntt + 15) / 16 * 16;
}
long long all_pairs(int ntt, int F, int D) { return (long long)((F + kFeat - 1) / kFeat) * ntt * ((D + 2 * kBK - 1) / (2 * kBK)); }
int ranges_for(long long pairs) { return (int)std::min<long long>(sms_of_device(), pairs); }

template <int BITS, typename T, int MODE>
cudaError_t start(const CUtensorMap (&maps)[6], const EvenParams &p, bool pdl, cudaStream_t s)
{
    auto kern = even_kernel<BITS, T, MODE>;
    static bool attr_set = false;
    if (!attr_set) {
        if (const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost + 1024); e != cudaSuccess) return e;
        attr_set = true;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)p.ranges);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)p.stages * (kWBytes + p.tok * (kBK * 2u)) + kFixed + 1024;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, maps[0], maps[1], maps[2], maps[3], maps[4], maps[5], p);
}

}  // namespace

size_t even_part_bytes(int M, int F, int D)
{
    int tok, ntt;
    token_tiles(M, &tok, &ntt);
    return (size_t)ranges_for(all_pairs(ntt, F, D)) * tok * kFeat * sizeof(float);
}
size_t even_tags() { return (size_t)kTagFirst + sms_of_device(); }

cudaError_t launch_even(const EvenArgs &a, Workspace &ws, const PrefillTuning &tune, cudaStream_t s, int *launches)
{
    const bool grad = a.gate < 0;
    EvenParams p{};
    p.scales = a.scales; p.zeros = a.zeros;
    p.part = static_cast<float *>(a.part);
    p.tags = ws.tags;
    p.status = ws.counters + kCtrStatus;
    p.M = a.M; p.K = a.K;
    p.F = grad ? a.K : a.N;
    p.D = grad ? a.N : a.K;
    token_tiles(a.M, &p.tok, &p.ntt);
    p.nkp = (p.D + 2 * kBK - 1) / (2 * kBK);
    const int rank_pad = (a.rank + kBK - 1) / kBK * kBK;
    p.slab = rank_pad / kBK;
    p.stages = (int)std::min<uint32_t>(kMostStages, (kSmemMost - kFixed) / (kWBytes + p.tok * (kBK * 2u)));
    p.gate = a.gate;
    p.kept_scales = a.kept_scales;
    p.kept_pitch = (p.F + kKeptGroup - 1) / kKeptGroup;
    p.pairs = all_pairs(p.ntt, p.F, p.D);
    p.ranges = ranges_for(p.pairs);
    p.wait_looks = tune.flag_polls > 0 ? (uint32_t)tune.flag_polls : 0u;
    p.test_skip_flag = tune.test_skip_flag;
    const CUtensorMapDataType dt = CU_TENSOR_MAP_DATA_TYPE_UINT16;
    const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B, none = CU_TENSOR_MAP_SWIZZLE_NONE;
    const int box = p.tok;
    CUtensorMap maps[6];
    cudaError_t e;
    const int words = a.bits == 4 ? 16 : 12;
    if ((e = cached_map(&maps[5], matrix_map(a.qw, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, (size_t)(a.K / kGroupFast) * words, a.N, words, 128,
                                             a.bits == 4 ? CU_TENSOR_MAP_SWIZZLE_64B : none))) != cudaSuccess)
        return e;
    if ((e = encode_map(&maps[0], matrix_map(a.x, dt, 2, p.D, a.M, kBK, box, sw))) != cudaSuccess) return e;
    maps[1] = maps[2] = maps[0];
    if (a.rank > 0) {
        if ((e = encode_map(&maps[1], matrix_map(a.thin, dt, 2, rank_pad, a.M, kBK, box, sw))) != cudaSuccess) return e;
        if ((e = cached_map(&maps[2], grad ? matrix_map(a.factor, dt, 2, a.K, a.rank, kBK, kBK, sw) : matrix_map(a.factor, dt, 2, a.rank, a.N, kBK, kHalf, sw))) !=
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
