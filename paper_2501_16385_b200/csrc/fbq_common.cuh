// Shared declarations of the CUDA sources of libfbq (sm_100a only).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/fbq.h"

namespace fbq {

constexpr int kGroupFast = 128;   // group size of the decode / prefill kernels (Section 5.1)
constexpr int kMaxRank = 256;
constexpr int kMostGradRows = 1 << 21;           // N of a backward pass
constexpr int kMostSide = 1 << 30;               // rows or columns of a layer, for calls that count whole tiles of them in 31 bits
constexpr int kDecodeMaxM = 16, kDecodePreferM = 6;

// What is set once on each device of the process, by its number: a kernel's attributes belong to the device that was current.
class PerDevice {
    std::atomic<unsigned long long> on{0};
    static unsigned long long bit()
    {
        int dev = 0;
        return cudaGetDevice(&dev) == cudaSuccess && dev < 64 ? 1ull << dev : 0ull;
    }

public:
    bool there() const { return (on.load(std::memory_order_relaxed) & bit()) != 0; }
    void set() { on.fetch_or(bit(), std::memory_order_relaxed); }
};

// SMs of the current device (a B200's where there is none to ask), asked for once on each.
inline int sms_of_device()
{
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 148;
    if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
    if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

// Activation-type helpers ---------------------------------------------------
template <typename T> struct ActTraits;
template <> struct ActTraits<__half> {
    using T2 = __half2;
    static __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }
};
template <> struct ActTraits<__nv_bfloat16> {
    using T2 = __nv_bfloat162;
    static __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
};

// Per-stream scratch space (device memory owned by the library).
struct Workspace {
    float *partial = nullptr;     // split-K partial sums  [SK][M][N]
    size_t partial_floats = 0;
    float *t = nullptr;           // down-projection t = x.A^T, [M][rank] fp32 (kept zero between calls)
    float *t_gen = nullptr;       // t of the generic path (no invariant), grows on demand
    float *tslots = nullptr;      // streaming decode kernel: partial sums of t, one encoded word per entry (all zero between calls)
    size_t tslots_floats = 0;
    size_t t_floats = 0, t_gen_floats = 0;
    int *counters = nullptr;      // [0]=t arrivals [1]=retired tiles [2]=status [3]=t ready [4]=parked; [8..] per tile
    size_t n_counters = 0;
    void *trace = nullptr;        // optional phase timestamps of the decode kernel (tuning aid)
    void *stage_x = nullptr;      // staging for the host-buffer entry point
    void *stage_y = nullptr;
    size_t stage_x_bytes = 0, stage_y_bytes = 0;
    void *w16 = nullptr;          // dequantised weights of the dense prefill kernel (no invariant)
    size_t w16_bytes = 0;
    uint32_t *tags = nullptr;     // its launch number and tags (starts at zero)
    size_t n_tags = 0;
    void *split = nullptr;        // the split kernel's launch number and words of t, which carry it (starts at zero)
    size_t split_bytes = 0;
    int gemv_ctas = 0;            // option of the stream (fbq_set_stream_option); outlives the buffers
    void *grad = nullptr;         // backward passes: x and dp in the activation type, s, t, partial sums (no invariant)
    size_t grad_bytes = 0;
    void *rec = nullptr;          // split operands of the Gram matrix and the reconstruction step (no invariant)
    size_t rec_bytes = 0;
};
constexpr int kCtrT = 0, kCtrDone = 1, kCtrStatus = 2;   // the decode kernel defines the rest

struct LinearArgs {
    const void *x;
    const uint32_t *qw;
    const __half *scales;
    const __half *zeros;
    const void *A;
    const void *B;
    void *y;
    int M, N, K, group, bits, rank;
    bool bf16;
    // The gated block: rows are eight of the gate, eight of the up projection, and so on, and y is h [M][N / 2].
    int gate = -1;                // fbq_gate, or -1: a plain linear
    int8_t *kept = nullptr;       // [M][N] codes and [M][ceil(N / 128)] scales of the products themselves, or none
    float *kept_scales = nullptr;
};

// Launchers implemented in the kernel files.  Each returns a cudaError_t from
// the launch and adds the number of kernels it launched to *launches.
cudaError_t launch_pack(const uint8_t *codes, uint32_t *qw, int N, int K, int bits, cudaStream_t s);
cudaError_t launch_unpack(const uint32_t *qw, uint8_t *codes, int N, int K, int bits, cudaStream_t s);
cudaError_t launch_act8_pack(const void *x, int8_t *codes, float *scales, int M, int K, bool bf16, cudaStream_t s);
cudaError_t launch_act8_unpack(const int8_t *codes, const float *scales, void *x, int M, int K, bool bf16, cudaStream_t s);
// dp [M][N] of the gated block from dh [M][N / 2] and p in 8 bits.
cudaError_t launch_gate_grad(const void *dh, const int8_t *codes, const float *scales, void *dp, int M, int N, int fn, bool bf16, cudaStream_t s);
cudaError_t launch_interleave(const void *gate, const void *up, void *out, int F, size_t bytes, bool padded, cudaStream_t s);
cudaError_t launch_dequant(const uint32_t *qw, const __half *sc, const __half *ze, float *W, int N,
                           int K, int group, int bits, cudaStream_t s);
cudaError_t launch_generic(const LinearArgs &a, Workspace &ws, cudaStream_t s, int *launches);
cudaError_t launch_sub_branch_unfused(const void *x, const void *A, const void *B, void *y, int M, int N, int K, int rank, bool bf16,
                                      Workspace &ws, cudaStream_t s, int *launches);
cudaError_t launch_quantize_feedback(const float *W, const void *A, const void *B, uint8_t *codes, __half *scales,
                                     __half *zeros, float *WF, float *Delta, int N, int K, int group, int bits, int rank,
                                     int ab_kind, cudaStream_t s);
size_t reconstruct_workspace_floats(int N, int K, int rank);
// Scratch of the two: about `budget` bytes at most, beyond what one slab of rows and the rank need.
size_t gram_scratch_bytes(int T, int K, size_t budget);
size_t reconstruct_scratch_bytes(int N, int K, int rank, size_t budget);
int run_gram(const float *X, float *H, int T, int K, size_t budget, void *scratch, int *status, bool pdl, cudaStream_t s, int *launches);
int run_reconstruct_step(const float *W, const float *H, float *A, float *B, float lr, float *loss, float *ws, int N, int K,
                         int group, int bits, int rank, size_t budget, void *scratch, int *status, bool pdl, cudaStream_t s,
                         int *launches);

struct DecodeTuning {
    int sk = 0, chunk = 0, depth = 0, max_ctas = 0, pdl = 1;
    int t_ctas = 1;  // 1: t = x.A^T comes from a few CTAs at the head of the grid (M <= 4, one K slice)
    int i8 = 1;      // 1: M <= 2 runs the form whose MMAs take the codes and x as 8-bit integers
};
// Returns cudaErrorInvalidConfiguration when no plan fits (caller falls back).
cudaError_t launch_decode(const LinearArgs &a, Workspace &ws, const DecodeTuning &tune,
                          cudaStream_t s, int *launches);
// Scratch the decode kernel needs for a shape (floats of partial sums, ints of counters).
void decode_workspace_need(const LinearArgs &a, const DecodeTuning &tune, size_t *partial_floats,
                           int *counters);

// The streaming decode kernel (fbq_gemv.cu), one and two tokens.
constexpr int kGemvMaxM = 2;
struct GemvTuning {
    int max_ctas = 0;          // 0: one main CTA per SM
    int pdl = 1;
    int poll_limit = 0;        // 0: default number of looks at the "t complete" counter
    int main_ctas = 0;         // > 0: this many main CTAs (a problem of a batch)
    int test_skip_arrive = 0;  // test switch: the t CTAs do not report their arrival (the wait for t must run out)
};
bool gemv_supported(const LinearArgs &a);
void gemv_workspace_need(const LinearArgs &a, const GemvTuning &tune, size_t *tpart_floats, int *counters);
cudaError_t launch_gemv(const LinearArgs &a, Workspace &ws, const GemvTuning &tune, cudaStream_t s, int *launches);

// Several problems of the streaming kernel in one launch: scratch, then launch.  false where they cannot share one (other
// forms, plans that do not fit): then they are launched one by one.
bool gemv_batch_need(const LinearArgs *a, int count, const GemvTuning &tune, size_t *tslots_floats, int *counters);
cudaError_t launch_gemv_batch(const LinearArgs *a, int count, Workspace &ws, const GemvTuning &tune, cudaStream_t s, int *launches);

// The split kernel (fbq_split.cu): the same domain of widths and ranks, up to kSplitMaxM tokens, one problem or several in
// one launch (cudaErrorInvalidConfiguration: no plan fits).  Scratch: Workspace::split, the status word of the counters.
constexpr int kSplitMaxM = 16;
constexpr int kSplitAnyK = 65536;     // up to eight tokens of this many inputs have a plan, with any N and rank
bool split_supported(const LinearArgs &a);
size_t split_scratch_bytes(const LinearArgs *a, int count);
bool split_plan_exists(const LinearArgs *a, int count, const GemvTuning &tune);
bool split_plan(const LinearArgs &a, const GemvTuning &tune, int *ctas, int *cluster);     // CTAs of the grid, of a cluster
cudaError_t launch_split(const LinearArgs *a, int count, Workspace &ws, const GemvTuning &tune, cudaStream_t s, int *launches);

int decode_batch_max();
bool decode_batch_need(const LinearArgs *a, int count, const int *ctas, const DecodeTuning &tune, size_t *partial_floats,
                       size_t *t_floats, int *counters);
cudaError_t launch_decode_batch(const LinearArgs *a, int count, const int *ctas, Workspace &ws, const DecodeTuning &tune,
                                cudaStream_t s, int *launches);
// The dense prefill kernel (fbq_dense.cu).
struct PrefillTuning {
    int pdl = 1;
    int flag_polls = 0;        // 0: waits for t end by time, else after this many looks
    int test_skip_flag = 0;    // test switch: t is not announced (the wait for it must run out)
};
// Backward pass of a layer: s = dy.B, dx = dy.W + s.A and t = x.A^T (fbq_dense.cu), dA = s^T.x and dB = dy^T.t (fbq_grad.cu).
struct GradArgs {
    const void *dy;               // [M][N]
    const void *x;                // [M][K], or none: no t
    const uint32_t *qw;
    const __half *scales, *zeros;
    const void *A, *B;
    void *dx;                     // [M][K] or none
    void *s16, *t16;              // scratch [M][rank rounded up to 64]: s and t in the activation type
    bool made;                    // they are there
    int M, N, K, bits, rank;
    bool bf16;
};
bool grad_thin_first(const GradArgs &a);        // s and t are better made by launch_thin
bool grad_dense_has_room(int N, int K);         // a tile's columns of W16 fit its scratch
bool grad_supported(int M, int N, int K, int group, int rank);
void grad_workspace_need(const GradArgs &a, size_t *w16_bytes, size_t *tags);
cudaError_t launch_grad(const GradArgs &a, Workspace &ws, const PrefillTuning &tune, cudaStream_t s, int *launches);
// The same for few hundred tokens, without a copy of the weights: t = x.A^T and s = dy.B (fbq_thin.cu; either may be left out), then dx, or h of a
// gated layer (fbq_even.cu).
struct ThinArgs {
    const void *x, *dy, *A, *B;
    void *t, *s;                  // [M][rank rounded up to 64] or none
    void *part;                   // thin_part_bytes of scratch
    int M, N, K, rank;
    bool bf16;
};
size_t thin_part_bytes(const ThinArgs &a);
cudaError_t launch_thin(const ThinArgs &a, int *status, bool pdl, cudaStream_t s, int *launches);
struct EvenArgs {
    const void *x;                // x [M][K], or dy [M][N]
    const uint32_t *qw;
    const __half *scales, *zeros;
    const void *factor, *thin;    // B and t, or A and s
    void *y;                      // h [M][N / 2], or dx [M][K]
    int8_t *kept;
    float *kept_scales;
    void *part;                   // even_part_bytes of scratch
    int M, N, K, bits, rank, gate;        // gate < 0: dx
    bool bf16;
};
size_t even_part_bytes(int M, int features, int depth);
cudaError_t launch_even(const EvenArgs &a, int *status, bool pdl, cudaStream_t s, int *launches);
size_t factor_grad_scratch_bytes(int M, int N, int K, int rank);
cudaError_t launch_factor_grads(const void *dy, const void *x, const void *s16, const void *t16, void *dA, void *dB, int M, int N, int K, int rank, bool gated,
                                bool bf16, void *scratch, int *status, bool pdl, cudaStream_t s, int *launches);

void dense_workspace_need(const LinearArgs &a, size_t *w16_bytes, size_t *tags, size_t *t_floats);
cudaError_t launch_dense(const LinearArgs &a, Workspace &ws, const PrefillTuning &tune, cudaStream_t s, int *launches);

bool prefill_supported(const LinearArgs &a);
bool dense_has_room(int N, int K);             // a tile's rows of W16 fit its scratch (fbq_dense.cu)
bool prefill_dense(const LinearArgs &a);       // the dense kernel is the faster one for this call (fbq_dense.cu)
void prefill_workspace_need(const LinearArgs &a, int *counters, size_t *t_floats, size_t *partial_floats);
// dense: by the dense kernel, whose scratch (dense_workspace_need) is there
cudaError_t launch_prefill(const LinearArgs &a, bool dense, Workspace &ws, cudaStream_t s, int *launches);

}  // namespace fbq
