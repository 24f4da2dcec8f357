// The gated block and dx of a layer's backward pass for few hundred tokens, sm_100a: weights dequantised where they are multiplied, and
// the blocks of the contraction shared out evenly.
//
//   h = f(gate) * up,  p = x.dequant(Q,s,z)^T + t.B^T          (forward; t = x.A^T from the launch before, fbq_thin.cu)
//   dx = dy.dequant(Q,s,z) + s.A                               (Grad; s = dy.B from there)
//
// Up to a few hundred tokens a weight is used too seldom to be dequantised in a pass of its own (the dense kernel's 16-bit copy costs 4
// bytes a weight through L2 beside the half byte of its code), and tiles are fewer than SMs or fill a second wave badly.  So a CTA turns
// codes into the operand on chip, 128 features for up to 192 tokens, and the pairs of blocks of all tiles, in order, are cut into equal
// ranges, one per CTA:
//
//   warp 2       copies the packed codes of a pair of blocks, 128 rows x one quantisation group, warp 3 their scales and zero points
//   warps 8-23   two groups of eight dequantise a pair in turn, half a row a thread, and copy the tokens' block by TMA as soon as its stage
//                is free, and both operands of the sub-branch's blocks
//   warp 1       issues tcgen05.mma 128 features x tokens x 16
//   warps 4-7    epilogue: a tile that is the range's own is written; of one that several ranges share each stores its fp32 sums
//
// and a second launch adds the shares of each such tile in order of the contraction, gates and writes it: nobody waits for another
// CTA, and the results do not depend on timing.  (The CTA with a tile's first blocks adding the others' took 35 of 48 us at 61 tokens of 4096 x 4096,
// where nine share a tile: one SM reads what nine have written.)  The sub-branch's blocks are done where the tile's first ones are.
// All waits are bounded.
//
// Forward, features are rows of W: a pair of blocks is one group of each row, and a thread's weights are a row of the operand, which goes to tensor
// memory as it is (128 lanes x 32 columns a block; the multiplication reads it there and not from shared memory).  Grad, features are W's
// columns, 128 of them one group; a pair of blocks is 128 rows of it, and the operand is MN-major in shared memory: rows are written as they lie.
//
// What bounds it: the chain of a pair, stage free -> operand written -> MMAs issued and done -> free, with the pairs that fit on their way: three at 77
// tokens (six stages), two at 333 (Grad, tiles of 176: four stages).  From the times of layers of different depths (rank 0, both launches) a pair takes 0.50 us
// at 77 tokens (INT3; 2048 to 16384 deep 23.7, 32.7, 52.3, 89.7), 990 cycles where its MMAs alone would take 320, and 0.78 us at 333 (5504 to 22016 deep 26.9,
// 40.9, 55.4, 70.6), 1530 cycles where they would take 700; beyond that, codes and dy larger than L2, 0.97.  What is in no pair, the launch, the first pair's way
// through the ring, the last one's epilogue and the adding launch, is 13 to 14 us of a call.  4096 -> 2 x 11008 at 77 tokens takes 30 us of a call's 39, 22016 -> 4096 (dx) at
// 333 tokens 66 of 107.  Of single things left out (for timing) none gives more than a
// tenth: dequantisation 8 %, three of four MMAs 9, x 1 (Grad 9), codes 1.  Earlier forms, us of the two calls: a warp that copies all of x, whose 40
// instructions a block each wait their turn among 24 warps, 42.9 and 105; four groups of four warps, 128 codes a thread, 41.5 and 98; operands in shared
// memory forward too, 41 and -; one block per look of the MMA warp, 43.5 and 98; 256 features a CTA, one and a half pairs on their way, 38 for the kernel
// alone; pairs of CTAs with cta_group::2, slower still (the dequantising warps' fence towards the asynchronous proxy).
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
constexpr int kMostTok = 192, kMostStages = 8;
constexpr int kDqWarp = 8, kGroups = 2, kGroupWarps = 8, kMakers = kGroupWarps / 2, kThreads = (kDqWarp + kGroups * kGroupWarps) * 32;
constexpr int kRing = 4;                         // pairs of blocks whose codes and scales are there or on their way
constexpr uint32_t kCodeBytes = 128u * 64u, kSlotBytes = kCodeBytes + 512u;      // codes (INT3: 48 of 64 bytes a row), scales and zero points
static_assert(kMostStages <= 8, "");
constexpr int kFree = 32;                        // blocks whose stages' being free is told apart: more than the groups' pairs and their sub-branch's blocks (see `dequantise`)
static_assert(kGroups * (2 + kMaxRank / kBK) <= kFree, "");
constexpr int kScaleAhead = 3;                   // pairs whose scales a loading warp has requested
constexpr uint32_t kYBytes = 32u * 128u * 2u;    // staged part of an output tile: 32 tokens
constexpr uint32_t kFixed = kRing * kSlotBytes + 2 * kYBytes + 512 + 512;     // ring, staging, largest |p|, barriers
constexpr uint32_t kSmemMost = 227 * 1024 - 1024;        // (the base is moved up to 1024 bytes)
enum Mode { kGated, kKept, kGrad };

struct EvenParams {
    int ranges;
    const uint8_t *qw;
    const __half *scales, *zeros;
    float *part;              // [2 range + whether it holds the tile's first block][tok][kFeat]: a range has at most two shares
    float *kept_scales;
    int *status;
    int M, F, D, K;           // tokens, features, contraction, columns of W
    int tok, ntt, nkp, slab;  // tokens of a tile, token tiles, pairs of blocks of the contraction, blocks of the sub-branch
    int stages, gate, kept_pitch;
    uint32_t acc;             // columns of an accumulator; forward the weights' operands are behind two of them
    long long pairs;          // of all tiles
    void *y;                  // of the adding launch: h or dx, codes
    int8_t *kept;
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
    __device__ __forceinline__ bool whole() const { return kp0 == 0 && kp1 == nkp; }
};

__device__ __forceinline__ void sts128(uint32_t addr, const uint32_t *v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ uint32_t ldg_u16(const __half *p)
{
    uint32_t v;
    asm volatile("ld.global.nc.u16 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

// Where a ring's pair begins: row n0 of W, group g.  A warp alone runs on its instructions' latencies, some 500 cycles for a hundred of them, and a
// pair has that long: what changes from pair to pair is a step, the rest is worked out once per piece.
template <int MODE> struct Walk {
    Pieces pc;
    int kp, n0, g;
    bool on, opened;
    __device__ __forceinline__ Walk(const EvenParams &p, int range) : pc(p, range) { open(p); }
    __device__ __forceinline__ void open(const EvenParams &p)
    {
        on = pc.next();
        opened = true;
        const int ft = pc.tile / p.ntt;
        kp = pc.kp0;
        n0 = (MODE == kGrad ? kp : ft) * 128;
        g = MODE == kGrad ? ft : kp;
    }
    __device__ __forceinline__ void step(const EvenParams &p)
    {
        opened = false;
        if (MODE == kGrad) n0 += 128;
        else ++g;
        if (++kp == pc.kp1) open(p);
    }
};

// Warp 2: codes, 16 bytes a lane and copy, neighbouring lanes' along a row; they count on the slot's barrier when they have arrived.
template <int BITS, int MODE>
__device__ __forceinline__ bool load_codes(const EvenParams &p, int range, uint32_t ring, uint32_t rfull0, uint32_t rempty0, volatile int *quit)
{
    constexpr int kChunks = BITS == 4 ? 4 : 3, kCopies = 4 * kChunks;        // 16-byte pieces of a row's group, copies of a lane
    constexpr int kTurn = BITS == 4 ? 1 : 3, kTurnRows = 32 * kTurn / kChunks;          // copies after which the lane's piece is the same one, rows on
    const int lane = threadIdx.x & 31, G = p.K / kGroupFast, rows_all = MODE == kGrad ? p.D : p.F;
    const size_t row_bytes = (size_t)G * kChunks * 16, turn_bytes = (size_t)kTurnRows * row_bytes;
    const ptrdiff_t step = MODE == kGrad ? (ptrdiff_t)(128 * row_bytes) : kChunks * 16;
    int row[kTurn], piece[kTurn];
#pragma unroll
    for (int i = 0; i < kTurn; ++i) {
        row[i] = (lane + 32 * i) / kChunks;
        piece[i] = (lane + 32 * i) % kChunks;
    }
    // INT4: the 64-byte swizzle (rows are loaded by eight lanes at a time); the rows of further copies are multiples of eight on
    const uint32_t to0 = ring + (BITS == 4 ? (uint32_t)row[0] * 64u + (uint32_t)((piece[0] ^ ((row[0] >> 1) & 3)) << 4) : (uint32_t)lane * 16u);
    Walk<MODE> at(p, range);
    const uint8_t *src[kTurn];
    uint32_t slot = 0, phase = 1u;
    bool first = true;
#pragma unroll 1
    while (at.on) {
        if (at.opened) {
#pragma unroll
            for (int i = 0; i < kTurn; ++i) src[i] = p.qw + (size_t)at.n0 * row_bytes + (size_t)at.g * (kChunks * 16) + (size_t)row[i] * row_bytes + piece[i] * 16;
        }
        if (!__all_sync(0xffffffffu, first || umma::wait(rempty0 + 8u * slot, phase, quit))) return false;
        const uint32_t to = to0 + slot * kSlotBytes;
        const int last = rows_all - 1 - at.n0;                   // rows past it repeat it: their scales are 0
        if (last >= 127) {
            size_t more = 0;
#pragma unroll
            for (int k = 0; k < kCopies; ++k) {
                cp_async16(to + 512u * k, src[k % kTurn] + more);
                if (k % kTurn == kTurn - 1) more += turn_bytes;
            }
        } else {
#pragma unroll 1
            for (int k = 0; k < kCopies; ++k) {
                const int e = lane + 32 * k, n = e / kChunks;
                cp_async16(to + 512u * k, p.qw + (size_t)(at.n0 + min(n, last)) * row_bytes + (size_t)at.g * (kChunks * 16) + e % kChunks * 16);
            }
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(rfull0 + 8u * slot) : "memory");
        at.step(p);
#pragma unroll
        for (int i = 0; i < kTurn; ++i) src[i] += step;
        if (++slot == kRing) { slot = 0; phase ^= 1u; first = false; }
    }
    return true;
}

// Warp 3: scales and zero points.  They lie 2 bytes here and there (an instruction touches as many lines as it has lanes), so each is loaded
// once per row and pair, kScaleAhead pairs before it is stored.
template <int MODE>
__device__ __forceinline__ bool load_scales(const EvenParams &p, int range, uint32_t ring, uint32_t rfull0, uint32_t rempty0, volatile int *quit)
{
    const int lane = threadIdx.x & 31, G = p.K / kGroupFast, rows_all = MODE == kGrad ? p.D : p.F;
    const ptrdiff_t zero = p.zeros - p.scales, step = MODE == kGrad ? (ptrdiff_t)128 * G : 1, next = (ptrdiff_t)32 * G;
    struct Scales {
        uint32_t v[8];
        bool on;
    };
    Walk<MODE> at(p, range);
    const __half *src = p.scales;
    auto request = [&](Scales &c) {
        c.on = at.on;
        if (!at.on) return;
        if (at.opened) src = p.scales + (size_t)(at.n0 + lane) * G + at.g;
        const int left = rows_all - at.n0 - lane;
        const __half *q = src;
#pragma unroll
        for (int i = 0; i < 4; ++i, q += next) {
            c.v[2 * i] = c.v[2 * i + 1] = 0u;                    // what lies outside is a row of zeros, whatever its codes
            if (left > 32 * i) {
                c.v[2 * i] = ldg_u16(q);
                c.v[2 * i + 1] = ldg_u16(q + zero);
            }
        }
        at.step(p);
        src += step;
    };
    Scales c[kScaleAhead];
#pragma unroll
    for (int i = 0; i < kScaleAhead; ++i) request(c[i]);
    const uint32_t to0 = ring + kCodeBytes + (uint32_t)lane * 4u;
    uint32_t slot = 0, phase = 1u;
    bool first = true;
#pragma unroll 1
    for (;;) {
#pragma unroll
        for (int i = 0; i < kScaleAhead; ++i) {
            if (!c[i].on) return true;
            if (!__all_sync(0xffffffffu, first || umma::wait(rempty0 + 8u * slot, phase, quit))) return false;
            const uint32_t to = to0 + slot * kSlotBytes;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + 128u * k), "r"(c[i].v[2 * k] | c[i].v[2 * k + 1] << 16) : "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(rfull0 + 8u * slot);
            request(c[i]);
            if (++slot == kRing) { slot = 0; phase ^= 1u; first = false; }
        }
    }
}

// Warps 8-23.  A pair is one group's, half a row a thread; the first of a block's makers copies x of it.  The sub-branch's blocks are
// copied by the group whose turn comes next.
template <int BITS, typename T, int MODE>
__device__ __forceinline__ bool dequantise(const EvenParams &p, int range, const CUtensorMap *xmap, const CUtensorMap *tmap, const CUtensorMap *bmap, uint32_t tmem,
                                           uint32_t sbase, uint32_t stage_bytes, uint32_t ring, uint32_t full0, uint32_t free0, uint32_t rfull0, uint32_t rempty0,
                                           volatile int *quit)
{
    constexpr bool GRAD = MODE == kGrad;
    constexpr int NW = BITS == 4 ? 4 : 3;
    const int warp = (threadIdx.x >> 5) - kDqWarp, group = warp / kGroupWarps, w = warp % kGroupWarps, lane = threadIdx.x & 31;
    // A thread's half a row of the pair.  Forward the pair's blocks are the row's halves; Grad the row's half chooses the block and the codes' halves
    // are the operand's boxes.  Eight neighbouring lanes store to eight rows: different banks in the 128-byte swizzle, as they load them from
    // different banks (INT4: the 64-byte swizzle of the copy).
    const int q = w & 3, row = 32 * q + lane;
    const uint32_t half = (uint32_t)w >> 2, block = GRAD ? (uint32_t)q >> 1 : half;
    const bool copies = w == (GRAD ? 2 * (int)block : 4 * (int)block);
    const uint32_t r = row & 63;
    const uint32_t dst = sbase + half * kBox + r * 128u + ((r & 7u) << 4);   // Grad: unit j: ^ (j << 4)
    const uint32_t wcols = tmem + ((uint32_t)(32 * q) << 16) + 2u * p.acc;             // forward: of this warp's rows
    const uint32_t src = BITS == 4 ? (uint32_t)row * 64u + (((((uint32_t)row >> 1) & 3u) ^ (2u * half)) << 4) : (uint32_t)row * 48u + half * 24u;
    Pieces pc(p, range);
    uint32_t s = 0;                                              // stage of the next block
    uint32_t u = 0;                                              // blocks so far
    uint32_t slot = 0, rphase = 0;                               // of the ring
    int turn = 0;                                                // whose pair it is
    bool before = true;                                          // nothing of what the launch before wrote has been read
    const uint32_t stages = (uint32_t)p.stages, xbytes = (uint32_t)p.tok * (kBK * 2u);
    // A block's stage is free.  There is a barrier for each of kFree blocks in a row, not for each stage: a wait knows a phase only from its
    // neighbours, and a group looks at every other pair.  When it waits for block b it has seen b - kFree or a later one become free, and
    // b + kFree does not before b is written.
    auto free_stage = [&](uint32_t b) { return __all_sync(0xffffffffu, umma::wait(free0 + 8u * (b % kFree), (b / kFree) & 1u, quit)); };
    auto after_launch = [&]() {
        if (before) pdl_wait();
        before = false;
    };
    while (pc.next()) {
        const int n = pc.kp1 - pc.kp0, ft = pc.tile / p.ntt, m0 = (pc.tile - ft * p.ntt) * p.tok;
#pragma unroll 1
        for (int k = 0; k < n; ++k) {
            const uint32_t s1 = s + 1 == stages ? 0u : s + 1;    // the pair's second stage
            if (turn == group) {
                const uint32_t at = ring + slot * kSlotBytes;
                if (!__all_sync(0xffffffffu, umma::wait(rfull0 + 8u * slot, rphase, quit))) return false;
                uint32_t c[2 * NW];
                if constexpr (BITS == 4) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint4 a = lds128(at + (src ^ (uint32_t)(i << 4)));
                        c[4 * i] = a.x; c[4 * i + 1] = a.y; c[4 * i + 2] = a.z; c[4 * i + 3] = a.w;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(c[2 * i]), "=r"(c[2 * i + 1]) : "r"(at + src + 8u * i) : "memory");
                }
                uint32_t sz;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(sz) : "r"(at + kCodeBytes + (uint32_t)row * 4u) : "memory");
                const float fs = __half2float(__ushort_as_half((unsigned short)(sz & 0xFFFFu))), fz = __half2float(__ushort_as_half((unsigned short)(sz >> 16)));
                __syncwarp();
                if (lane == 0) mbar_arrive(rempty0 + 8u * slot);                 // (this warp has its codes in registers)
                // (in registers before the stage is waited for)
                uint32_t out[32];
                DequantNatural<BITS, T, true>::run(c, fs, fz, out);
                DequantNatural<BITS, T, true>::run(c + NW, fs, fz, out + 16);
                const uint32_t stage = block ? s1 : s;
                if (!free_stage(u + block)) return false;
                if (copies) {
                    after_launch();
                    if (umma::elect_one()) tma_load_2d(sbase + kWBytes + stage * stage_bytes, xmap, (2 * (pc.kp0 + k) + (int)block) * kBK, m0, full0 + 8u * stage);
                    __syncwarp();
                }
                if constexpr (GRAD) {
                    const uint32_t to = dst + stage * stage_bytes;
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) sts128(to ^ (j << 4), out + 4 * j);
                    fence_proxy_async();
                } else {
                    umma::fence_after();
                    umma::st32(wcols + 32u * stage, out);
                    umma::wait_st();
                    umma::fence_before();
                }
                __syncwarp();
                // (x's bytes may arrive before they are announced: a block is whole when its makers have arrived, too)
                if (lane == 0) {
                    if (copies) mbar_expect_tx(full0 + 8u * stage, xbytes);
                    else mbar_arrive(full0 + 8u * stage);
                }
            }
            u += 2;
            s = s1 + 1 == stages ? 0u : s1 + 1;
            if (++turn == kGroups) turn = 0;
            if (++slot == kRing) { slot = 0; rphase ^= 1u; }
        }
        for (int j = 0; pc.owner() && j < p.slab; ++j) {         // the sub-branch's blocks, whole copies
            if (turn == group && w == 0) {
                if (!free_stage(u)) return false;
                after_launch();
                if (umma::elect_one()) {
                    const uint32_t bar = full0 + 8u * s, wt = sbase + s * stage_bytes;
                    mbar_expect_tx(bar, xbytes + kWBytes);
                    for (int m = 1; m < kMakers; ++m) mbar_arrive(bar);              // (for the warps that have nothing to make)
                    tma_load_2d(wt + kWBytes, tmap, j * kBK, m0, bar);
                    if (GRAD) {
                        for (int h = 0; h < 2; ++h) tma_load_2d(wt + h * kBox, bmap, ft * kFeat + 64 * h, j * kBK, bar);
                    } else {
                        tma_load_2d(wt, bmap, j * kBK, ft * kFeat, bar);
                    }
                }
                __syncwarp();
            }
            ++u;
            if (++s == stages) s = 0;
        }
    }
    return true;
}

// xmap: x (Grad: dy) [M][D], boxes of 64 x tok rows; tmap: t (s) [M][rank_pad], the same boxes; bmap: B [F][rank], boxes 64 x 128 rows
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
    const uint32_t ring = sbase + y_off + 2 * kYBytes, bars = kRing * kSlotBytes + 512u;
    const uint32_t full0 = ring + bars, free0 = full0 + 8u * kMostStages, accf0 = free0 + 8u * kFree, acce0 = accf0 + 16u, rfull0 = acce0 + 16u,
                   rempty0 = rfull0 + 8u * kRing;
    float *amax = reinterpret_cast<float *>(smem + y_off + 2 * kYBytes + kRing * kSlotBytes);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + y_off + 2 * kYBytes + bars + 8u * kMostStages + 8u * kFree + 32u + 16u * kRing);
    volatile int *quit = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, range = (int)blockIdx.x;

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) mbar_init(full0 + 8u * i, kMakers);          // the warps that make a block
        for (int i = 0; i < kFree; ++i) mbar_init(free0 + 8u * i, 1);
        for (int i = 0; i < kRing; ++i) {
            mbar_init(rfull0 + 8u * i, 32 + 1);                  // every copying lane's codes, and the scales
            mbar_init(rempty0 + 8u * i, kGroupWarps);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(accf0 + 8u * i, 1);
            mbar_init(acce0 + 8u * i, 4);
        }
        *quit = 0;
        fence_barrier_init();
        for (int i = 0; i < p.stages; ++i) mbar_arrive(free0 + 8u * i);
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

    if (warp == 1) {
        // =================================================== MMAs
        // The whole warp walks the loop and one elected lane issues: the MMAs' operands stay in uniform registers.  Two blocks at a time.
        const uint32_t idesc = umma::idesc_f16(P2<T>::kFmt, kFeat, (uint32_t)p.tok) | (GRAD ? umma::kIdescMnA : 0u);
        const uint32_t wstep = GRAD ? 2048u >> 4 : 2u, wcols = tmem + 2u * p.acc;
        const uint64_t wd0 = GRAD ? umma::desc_mn128(sbase, kBox) : umma::desc_k128(sbase), xd0 = umma::desc_k128(sbase + kWBytes);
        uint32_t s = 0, phase = 0, it = 0, next = (uint32_t)p.stages;        // the block that the next one done makes room for
#pragma unroll 1
        for (Pieces pc(p, range); ok && pc.next(); ++it) {
            const uint32_t buf = it & 1u, use = it >> 1, d = tmem + buf * p.acc;
            ok = __all_sync(0xffffffffu, use == 0 || umma::wait(acce0 + 8u * buf, (use - 1u) & 1u, quit));
            const int own = 2 * (pc.kp1 - pc.kp0), n = own + (pc.owner() ? p.slab : 0);
#pragma unroll 1
            for (int i = 0; i < n && ok; i += 2) {
                const bool two = i + 1 < n;
                const uint32_t s0 = s, s1 = s + 1 == (uint32_t)p.stages ? 0u : s + 1, ph0 = phase, ph1 = s1 ? phase : phase ^ 1u;
                const uint32_t look = two && (lane & 1) ? s1 : s0;
                ok = __all_sync(0xffffffffu, umma::wait(full0 + 8u * look, two && (lane & 1) ? ph1 : ph0, quit));
                umma::fence_after();
                if (ok && umma::elect_one()) {
                    auto block = [&](uint32_t stage, uint32_t room, bool more) {
                        const uint64_t wd = wd0 + stage * (stage_bytes >> 4), xd = xd0 + stage * (stage_bytes >> 4);
#pragma unroll
                        for (int j = 0; j < kBK / 16; ++j) {
                            if (!GRAD && i < own) umma::mma_ts(d, wcols + 32u * stage + 8u * j, xd + 2 * j, idesc, more || j > 0);
                            else umma::mma(d, wd + wstep * j, xd + 2 * j, idesc, more || j > 0);
                        }
                        umma::commit(free0 + 8u * (room % kFree));
                    };
                    block(s0, next, i > 0);
                    if (two) block(s1, next + 1, true);
                    if (i + 2 >= n) umma::commit(accf0 + 8u * buf);
                }
                __syncwarp();
                next += two ? 2 : 1;
                s = two ? s1 : s0;
                phase = two ? ph1 : ph0;
                if (++s == (uint32_t)p.stages) { s = 0; phase ^= 1u; }
            }
        }
        __syncwarp();
    } else if (warp >= 4 && warp < kDqWarp) {
        // =================================================== epilogue: lane = feature, column = token
        pdl_wait();
        const int wq = warp & 3;
        uint32_t it = 0, staged = 0;
#pragma unroll 1
        for (Pieces pc(p, range); ok && pc.next(); ++it) {
            const uint32_t buf = it & 1u, use = it >> 1;
            ok = named_barrier_and(1, 128, umma::wait(accf0 + 8u * buf, use & 1u, quit));      // (four warps go on, or none)
            if (!ok) break;
            umma::fence_after();
            const int ft = pc.tile / p.ntt, m0 = (pc.tile - ft * p.ntt) * p.tok, m_end = min(p.M, m0 + p.tok);
            {
                const uint32_t lanes = tmem + buf * p.acc + ((uint32_t)(32 * wq) << 16);
                const int n = ft * kFeat + 32 * wq + lane;
                const size_t part_at = (size_t)(2 * range + pc.owner()) * p.tok * kFeat + 32 * wq + lane;
#pragma unroll 1
                for (int c = 0; c < p.tok; c += 32) {
                    uint32_t v[32];
                    umma::ld32(lanes + (uint32_t)c, v);
                    umma::wait_ld();
                    if (c + 32 >= p.tok) {                       // all of the accumulator is in registers
                        umma::fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(acce0 + 8u * buf);
                    }
                    if (m0 + c >= p.M) continue;
                    if (!pc.whole()) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (c + j < m_end - m0) __stcg(p.part + part_at + (size_t)(c + j) * kFeat, __uint_as_float(v[j]));
                        continue;
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
                    if constexpr (MODE == kKept) {               // a tile's 128 rows are the columns that share a scale
                        uint32_t top = 0u;
#pragma unroll
                        for (int w = 0; w < 4; ++w) top = max(top, __float_as_uint(amax[32 * w + lane]));
                        float scale, inverse;
                        kept_scale(top, scale, inverse);
                        if (wq == 0 && n - lane < p.F && lane < m_end - (m0 + c)) p.kept_scales[(size_t)(m0 + c + lane) * p.kept_pitch + ft] = scale;
                        uint8_t *codes = smem + at + kYBytes / 2 + 32 * wq + lane;
#pragma unroll
                        for (int j = 0; j < 32; ++j) codes[j * 128] = (uint8_t)kept_code(__uint_as_float(v[j]), __shfl_sync(0xffffffffu, inverse, j));
                    }
                    fence_proxy_async();
                    named_barrier_sync(1, 128);
                    if (threadIdx.x == 4 * 32 && n < p.F) {
                        const int out = GRAD ? n : n / 2;        // (lane 0's n is the tile's first)
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
        }
        if (threadIdx.x == 4 * 32) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else if (warp >= kDqWarp) {
        ok = dequantise<BITS, T, MODE>(p, range, &xmap, &tmap, &bmap, tmem, sbase, stage_bytes, ring, full0, free0, rfull0, rempty0, quit);
    } else if (warp == 2) {
        ok = load_codes<BITS, MODE>(p, range, ring, rfull0, rempty0, quit);
    } else if (warp == 3) {
        ok = load_scales<MODE>(p, range, ring, rfull0, rempty0, quit);
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
}

// The tiles that several ranges share: a block adds eight tokens of one, a thread per feature, in order of the ranges.
constexpr int kAddTok = 8;
template <typename T, int MODE> __global__ void __launch_bounds__(kFeat) add_kernel(const EvenParams p)
{
    __shared__ uint32_t tops[kFeat / 32][kAddTok];
    pdl_launch_dependents();
    pdl_wait();                                                  // (all blocks, so that this launch is not through before the one before it)
    const int tile = (int)blockIdx.x, c0 = (int)blockIdx.y * kAddTok, ft = tile / p.ntt, m0 = (tile - ft * p.ntt) * p.tok + c0, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int count = min(min(kAddTok, p.tok - c0), p.M - m0);
    // the ranges that hold the tile's first and last pair
    const long long first = (long long)tile * p.nkp, last = first + p.nkp - 1;
    const int r0 = (int)(((first + 1) * p.ranges - 1) / p.pairs), r1 = (int)(((last + 1) * p.ranges - 1) / p.pairs);
    if (r0 == r1 || count <= 0) return;
    const int n = ft * kFeat + (int)threadIdx.x;
    const float *src = p.part + (size_t)c0 * kFeat + threadIdx.x;
    const size_t slot = (size_t)p.tok * kFeat;
    float v[kAddTok];
#pragma unroll
    for (int j = 0; j < kAddTok; ++j) v[j] = j < count ? __ldcg(src + (2 * (size_t)r0 + 1) * slot + j * kFeat) : 0.f;
#pragma unroll 2
    for (int r = r0 + 1; r <= r1; ++r) {
        float e[kAddTok];
#pragma unroll
        for (int j = 0; j < kAddTok; ++j) e[j] = j < count ? __ldcg(src + 2 * (size_t)r * slot + j * kFeat) : 0.f;
#pragma unroll
        for (int j = 0; j < kAddTok; ++j) v[j] += e[j];
    }
    if constexpr (MODE == kKept) {
#pragma unroll
        for (int j = 0; j < kAddTok; ++j) {
            const uint32_t top = __reduce_max_sync(0xffffffffu, n < p.F ? __float_as_uint(v[j]) & 0x7FFFFFFFu : 0u);
            if (lane == 0) tops[warp][j] = top;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kAddTok; ++j) {
            const uint32_t *t = &tops[0][j];
            float scale, inverse;
            kept_scale(max(max(t[0], t[kAddTok]), max(t[2 * kAddTok], t[3 * kAddTok])), scale, inverse);
            if (j < count && n < p.F) {
                p.kept[(size_t)(m0 + j) * p.F + n] = (int8_t)kept_code(v[j], inverse);
                if (threadIdx.x == 0) p.kept_scales[(size_t)(m0 + j) * p.kept_pitch + n / kKeptGroup] = scale;
            }
        }
    }
    T *y = static_cast<T *>(p.y);
    if constexpr (MODE == kGrad) {
#pragma unroll
        for (int j = 0; j < kAddTok; ++j)
            if (j < count && n < p.F) y[(size_t)(m0 + j) * p.F + n] = ActTraits<T>::from_float(v[j]);
    } else {
        // lanes eight apart swap halves of their tokens, so that each gates four
        const bool up = (lane & kGateUp) != 0;
        const int col = ft * (kFeat / 2) + warp * 16 + (lane >> 4) * kGateUp + (lane & (kGateUp - 1));
#pragma unroll
        for (int j = 0; j < kAddTok / 2; ++j) {
            const float got = __shfl_xor_sync(0xffffffffu, up ? v[j] : v[j + kAddTok / 2], kGateUp), mine = up ? v[j + kAddTok / 2] : v[j];
            const int t = up ? j + kAddTok / 2 : j;
            if (t < count && n < p.F) y[(size_t)(m0 + t) * (p.F / 2) + col] = ActTraits<T>::from_float(gate_value(p.gate, up ? got : mine) * (up ? mine : got));
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------
// Tokens of a tile: all of them up to kMostTok, else equal parts, in sixteens.
void token_tiles(int M, int *tok, int *ntt)
{
    *ntt = (M + kMostTok - 1) / kMostTok;
    *tok = ((M + *ntt - 1) / *ntt + 15) / 16 * 16;
}
long long all_pairs(int ntt, int F, int D) { return (long long)((F + kFeat - 1) / kFeat) * ntt * ((D + 2 * kBK - 1) / (2 * kBK)); }
int ranges_for(long long pairs) { return (int)std::min<long long>(sms_of_device(), pairs); }

template <int BITS, typename T, int MODE>
cudaError_t start(const CUtensorMap (&maps)[5], const EvenParams &p, bool pdl, cudaStream_t s, int *launches)
{
    auto kern = even_kernel<BITS, T, MODE>;
    static PerDevice attr_set;
    if (!attr_set.there()) {
        if (const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost + 1024); e != cudaSuccess) return e;
        attr_set.set();
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
    if (const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, maps[0], maps[1], maps[2], maps[3], maps[4], p); e != cudaSuccess) return e;
    ++*launches;
    if (p.nkp == 1 || (p.pairs % p.ranges == 0 && p.pairs / p.ranges % p.nkp == 0)) return cudaSuccess;      // (every range is whole tiles)
    cfg.gridDim = dim3((unsigned)(p.pairs / p.nkp), (unsigned)((p.tok + kAddTok - 1) / kAddTok));
    cfg.blockDim = dim3(kFeat);
    cfg.dynamicSmemBytes = 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, add_kernel<T, MODE>, p);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace

size_t even_part_bytes(int M, int F, int D)
{
    int tok, ntt;
    token_tiles(M, &tok, &ntt);
    return (size_t)2 * ranges_for(all_pairs(ntt, F, D)) * tok * kFeat * sizeof(float);
}

cudaError_t launch_even(const EvenArgs &a, int *status, bool pdl, cudaStream_t s, int *launches)
{
    const bool grad = a.gate < 0;
    EvenParams p{};
    p.qw = reinterpret_cast<const uint8_t *>(a.qw);
    p.scales = a.scales; p.zeros = a.zeros;
    p.part = static_cast<float *>(a.part);
    p.status = status;
    p.M = a.M; p.K = a.K;
    p.F = grad ? a.K : a.N;
    p.D = grad ? a.N : a.K;
    token_tiles(a.M, &p.tok, &p.ntt);
    p.nkp = (p.D + 2 * kBK - 1) / (2 * kBK);
    const int rank_pad = (a.rank + kBK - 1) / kBK * kBK;
    p.slab = rank_pad / kBK;
    p.stages = (int)std::min<uint32_t>(kMostStages, (kSmemMost - kFixed) / (kWBytes + p.tok * (kBK * 2u)));
    p.acc = (uint32_t)(p.tok + 31) / 32 * 32;
    if (!grad) p.stages = std::min(p.stages, (int)((512u - 2u * p.acc) / 32u));
    p.gate = a.gate;
    p.kept_scales = a.kept_scales;
    p.kept_pitch = (p.F + kKeptGroup - 1) / kKeptGroup;
    p.pairs = all_pairs(p.ntt, p.F, p.D);
    p.ranges = ranges_for(p.pairs);
    p.y = a.y;
    p.kept = a.kept;
    const CUtensorMapDataType dt = CU_TENSOR_MAP_DATA_TYPE_UINT16;
    const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B, none = CU_TENSOR_MAP_SWIZZLE_NONE;
    const int box = p.tok;
    CUtensorMap maps[5];
    cudaError_t e;
    if ((e = encode_map(&maps[0], matrix_map(a.x, dt, 2, p.D, a.M, kBK, box, sw))) != cudaSuccess) return e;
    maps[1] = maps[2] = maps[0];
    if (a.rank > 0) {
        if ((e = encode_map(&maps[1], matrix_map(a.thin, dt, 2, rank_pad, a.M, kBK, box, sw))) != cudaSuccess) return e;
        if ((e = encode_map(&maps[2], grad ? matrix_map(a.factor, dt, 2, a.K, a.rank, kBK, kBK, sw) : matrix_map(a.factor, dt, 2, a.rank, a.N, kBK, kFeat, sw))) !=
            cudaSuccess)
            return e;
    }
    if ((e = encode_map(&maps[3], grad ? matrix_map(a.y, dt, 2, a.K, a.M, 128, 16, none) : matrix_map(a.y, dt, 2, a.N / 2, a.M, 64, 16, none))) != cudaSuccess) return e;
    maps[4] = maps[3];
    if (a.kept && (e = encode_map(&maps[4], matrix_map(a.kept, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.N, a.M, 128, 16, none))) != cudaSuccess) return e;
    auto go = [&](auto mode) {
        constexpr int MODE = decltype(mode)::value;
        return a.bits == 4 ? (a.bf16 ? start<4, __nv_bfloat16, MODE>(maps, p, pdl, s, launches) : start<4, __half, MODE>(maps, p, pdl, s, launches))
                           : (a.bf16 ? start<3, __nv_bfloat16, MODE>(maps, p, pdl, s, launches) : start<3, __half, MODE>(maps, p, pdl, s, launches));
    };
    e = grad ? go(std::integral_constant<int, kGrad>{}) : a.kept ? go(std::integral_constant<int, kKept>{}) : go(std::integral_constant<int, kGated>{});
    return e;
}

}  // namespace fbq
