// The vocabulary head's operators (gk_vocab_loss, gk_vocab_distill): what their translation
// units share.  Internal; the public interface is include/gk.h.
//
// A call works on the rows that count, in their order ("compact" rows, 0 .. n_valid - 1), so
// that rows left out cost nothing and nothing in them can reach a result.  n_valid is known on
// the device only: every kernel reads it there and the call never synchronises.
#pragma once

#include "gk_common.cuh"

namespace gk {

constexpr int kVocabTile = 128;        // columns of the vocabulary whose maximum and sum are kept together
constexpr int kVocabRowPad = 256;       // compact rows are padded to a multiple of this
constexpr int kVocabMaxPairs = 1024;    // largest K of gk_vocab_distill and gk_vocab_topk

// Device control block of one call.
struct VocabCtl {
    int n_valid;           // rows that count
    unsigned int status;   // GK_DEV_* flags
    float scale;           // brings the largest row coefficient to a power of two in the 16-bit type's range
    float inv_scale;
};

// Per compact row, written before the products that need it.
struct VocabRow {
    float lse2;     // log-sum-exp of the scaled logits, in units of log 2
    float coef;     // scale * g_n * Q_n / T: what multiplies p_nv
    float unit;     // scale * g_n / T: what multiplies q_nj
    float pad;
};

// One call's sizes and device pointers, passed to the kernels by value.
struct VocabCall {
    int64_t n, D, V;
    int64_t n_pad;              // n rounded up to kVocabRowPad
    int64_t Dp;                 // D rounded up to 64: row pitch of hc, and of wc where it is used
    int64_t ldh, ldw, lddh, lddw;
    int K;                      // pairs a row (1 for gk_vocab_loss)
    bool f16;                   // operands are fp16, else bf16
    float inv_T;
    float zscale;               // log2(e) / T
    const void* h;
    const void* w;
    void* dh;
    void* dw;
    // targets: a class per row, or pairs
    const int64_t* target;
    int64_t ignore_index;
    const int32_t* t_idx;
    const float* t_val;
    const float* t_lse;
    const float* row_grad;      // nullptr: 1 / n_valid
    float* loss;
    float* lse;
    // workspace
    VocabCtl* ctl;
    int32_t* row_of;            // compact row -> row
    int32_t* at_of;             // row -> compact row, -1 where left out
    float* q;                   // n x K teacher probabilities (distill), 0 for a pair left out
    float4* teacher;            // per row: Q, log-sum-exp L relative to a reference, the reference, and a whole
                                // number: 1 (indices strictly ascending, pairs left out at the end) + 2 (a pair counts)
    int32_t* cls;               // compact rows' classes (loss)
    unsigned* pairs_in;         // per (vocabulary tile, row): its pairs there, the first's number + 2^16 how many (distill)
    uint16_t* hc;               // n_pad x Dp compact rows of h
    uint16_t* wc;               // V x Dp copy of w where w itself cannot be the source of bulk copies, else nullptr
    float* zt;                  // n_pad x K raw logits at the targets
    float2* part;               // per (vocabulary tile, compact row): maximum (units of log 2), sum
    VocabRow* row;              // n_pad
    uint16_t* e;                // n_pad x vb: one piece's kept logits, then its logit gradients
    int64_t vb;                 // columns of a piece, a multiple of 256 (the pitch of e)
    float* dhp;                 // splits x n_pad x Dp partial sums of dh; nullptr: dh is stored by its product
    int splits;
};

// A call's launches (k_vocab_teacher's apart, which is a plain one): the kernel may be set up while the one before it
// in the stream ends, and waits for that with after_previous() before it reads or writes anything of the call.
template <class... Params, class... Args>
inline cudaError_t launch_next(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, Args&&... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Args&&>(args)...);
}

// T and what the kernels multiply by, 1 / T and log2(e) / T, are positive and finite.
inline bool temperature_ok(float T) { return T > 0.f && T < INFINITY && (float)(1.4426950408889634 / (double)T) < INFINITY; }

__host__ __device__ inline int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// The products (gk_vocab_gemm.cu).  v0, v1: the columns of the vocabulary [v0, v1).
// Logits of all compact rows: per tile of the vocabulary the maximum and the sum; keep: the
// logits go to e, as 16-bit codes of their distance from the tile's maximum.
int launch_vocab_logits(const VocabCall& c, int64_t v0, int64_t v1, bool keep, int sm_count, cudaStream_t st);
// The same product again with the rows' log-sum-exp known: e receives the logit gradients.
int launch_vocab_again(const VocabCall& c, int64_t v0, int64_t v1, int sm_count, cudaStream_t st);
// dw rows [v0, v1) = e^T hc / scale, and dh = e w[v0:v1] / scale, or its sums in fp32 in
// `splits` parts added to dhp (first: overwritten).
int launch_vocab_grads(const VocabCall& c, int64_t v0, int64_t v1, bool first, int sm_count, cudaStream_t st);
enum class DwRows { none, aligned, unaligned };     // dw's rows start and end on 16-byte boundaries, or not
int vocab_dh_splits(int64_t n, int64_t D, int64_t vb, DwRows dw, int sm_count);

#ifdef __CUDACC__

// The next kernel may be set up (it waits in the same way); then everything before in the stream is done
// and seen.
__device__ __forceinline__ void after_previous() {
    asm volatile("griddepcontrol.launch_dependents;\ngriddepcontrol.wait;" ::: "memory");
}

// What earlier kernels wrote, the caller's inputs among it, is read by ordinary loads after that: __ldg and its kin
// are for memory that nothing writes while the kernel is there, and may be moved ahead of the wait.  These two are
// for what is read once.
__device__ __forceinline__ uint4 load_once(const uint4* p) {
    uint4 x;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
    return x;
}
__device__ __forceinline__ float2 load_once(const float2* p) {
    float2 x;
    asm volatile("ld.global.cs.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "l"(p));
    return x;
}

__device__ __forceinline__ bool teacher_ascending(const float4& t) { return ((int)t.w & 1) != 0; }
__device__ __forceinline__ bool teacher_counts(const float4& t) { return ((int)t.w & 2) != 0; }

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The 16-bit code of a logit's distance d <= 0 from its tile's maximum, in units of log 2.  bf16: steps of 2^-9 over
// a range of 128, the exponents bf16 gradients can have.  fp16: steps of 2^-12 over the first 8 and of 1 / 1365.25
// over the next 24.  The last code stands for itself and more: 2^-32 (2.3e-10) of the tile's largest exponential is the
// least that an fp16 call's first piece tells from zero (fp16 gradients without a scale end at 6e-8).
template <bool F16>
__device__ __forceinline__ unsigned kept_code(float d) {
    // the bits of 2^23 + x hold x
    const float end = 8388608.f + 65535.f;
    float x = fminf(fmaf(d, F16 ? -4096.f : -512.f, 8388608.f), end);
    if constexpr (F16) x = fminf(x, fmaf(d, -1365.25f, 8388608.f + 21846.f));
    return __float_as_uint(x) & 0xffffu;
}
template <bool F16>
__device__ __forceinline__ float kept_distance(unsigned code) {      // -d
    const float x = __uint_as_float(0x4b000000u | code) - 8388608.f;
    if constexpr (F16) return fmaxf(x * (1.f / 4096.f), (x - 21846.f) * (1.f / 1365.25f));
    else return x * (1.f / 512.f);
}

// 16-bit storage <-> fp32, round to nearest even (F16: fp16, else bf16).
template <bool F16>
__device__ __forceinline__ float from16(uint16_t b) {
    if constexpr (F16) {
        float f;
        asm("cvt.f32.f16 %0, %1;" : "=f"(f) : "h"(b));
        return f;
    } else {
        return __uint_as_float((unsigned)b << 16);
    }
}
template <bool F16>
__device__ __forceinline__ uint16_t to16(float f) {
    uint16_t b;
    if constexpr (F16) asm("cvt.rn.f16.f32 %0, %1;" : "=h"(b) : "f"(f));
    else asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(b) : "f"(f));
    return b;
}
// two values in one word, lo in the lower half
template <bool F16>
__device__ __forceinline__ unsigned pack16(float lo, float hi) {
    unsigned r;
    if constexpr (F16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Joins (m, s) pairs of a running maximum and sum, in units of log 2.  A part without a term
// has m = -inf and s = 0, a part of nothing but NaN m = -inf and s = NaN.
__device__ __forceinline__ void join_max_sum(float& m, float& s, float m2, float s2) {
    const float top = fmaxf(m, m2);
    if (top == -INFINITY) {
        s += s2;
        return;
    }
    // a NaN sum stays NaN through the products; exp2(-inf) = 0 drops empty parts; a part at the
    // common maximum is taken as it is, also where that is +inf
    s = (m == top ? s : s * exp2_fast(m - top)) + (m2 == top ? s2 : s2 * exp2_fast(m2 - top));
    m = top;
}

#endif  // __CUDACC__

}  // namespace gk
