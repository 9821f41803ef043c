// Top logits of rows: what a teacher sends for distillation (include/gk.h: gk_vocab_topk).
// Simplest form: one CTA a row; radix select of the k-th largest value over four 8-bit digits, one
// pass over the row each, then one pass that writes the pairs in index order.
#include "gk_vocab.cuh"

namespace gk {

constexpr int kTopkThreads = 512;

template <int TYPE>
__device__ __forceinline__ float load_logit(const void* p, int64_t i) {
    if constexpr (TYPE == GK_TYPE_F32) return ((const float*)p)[i];
    else return from16<TYPE == GK_TYPE_F16>(((const uint16_t*)p)[i]);
}

// Unsigned key in the order of the values; -0 ties with +0, NaN is above +inf.
__device__ __forceinline__ unsigned order_key(float v) {
    if (v != v) return 0xffffffffu;
    const unsigned b = __float_as_uint(v == 0.f ? 0.f : v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Joins sums of exp((v - m) / T): the maximum stays in the logits' own unit, so that the types'
// largest and lowest values do not overflow.
__device__ __forceinline__ void join_raw(float& m, float& s, float m2, float s2, float zscale) {
    const float top = fmaxf(m, m2);
    if (top == -INFINITY) return;
    s = (m == top ? s : s * exp2_fast((m - top) * zscale)) + (m2 == top ? s2 : s2 * exp2_fast((m2 - top) * zscale));
    m = top;
}

template <int TYPE>
__global__ void __launch_bounds__(kTopkThreads) k_vocab_topk(const void* logits, int64_t ld, int64_t V, int K, float zscale, float inv_T,
                                                             int32_t* idx_out, float* val_out, float* lse_out) {
    __shared__ unsigned hist[256];
    __shared__ unsigned pick[2];
    __shared__ float sm[kTopkThreads / 32], ss[kTopkThreads / 32];
    __shared__ int wn[kTopkThreads / 32], we[kTopkThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const char* row = (const char*)logits + (int64_t)blockIdx.x * ld * (TYPE == GK_TYPE_F32 ? 4 : 2);
    unsigned prefix = 0, need = K;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kTopkThreads) hist[i] = 0;
        __syncthreads();
        for (int64_t i = tid; i < V; i += kTopkThreads) {
            const unsigned key = order_key(load_logit<TYPE>(row, i));
            if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            unsigned left = need;
            int b = 255;
            while (b > 0 && hist[b] < left) left -= hist[b--];
            pick[0] = (unsigned)b;
            pick[1] = left;
        }
        __syncthreads();
        prefix |= pick[0] << shift;
        need = pick[1];
    }
    // pairs above the k-th value, and the first `need` equal to it
    int taken = 0, equal = 0;
    float m = -INFINITY, s = 0.f;
    for (int64_t i0 = 0; i0 < V; i0 += kTopkThreads) {
        const int64_t i = i0 + tid;
        const float v = i < V ? load_logit<TYPE>(row, i) : -INFINITY;
        const unsigned key = i < V ? order_key(v) : 0u;
        if (i < V) {
            if (v != v) s = v;
            else if (v > -INFINITY) join_raw(m, s, v, 1.f, zscale);
        }
        const unsigned eq = __ballot_sync(0xffffffffu, i < V && key == prefix);
        if (lane == 0) we[wid] = __popc(eq);
        __syncthreads();
        int before = equal;
        for (int k = 0; k < kTopkThreads / 32; ++k) {
            if (k < wid) before += we[k];
            equal += we[k];
        }
        const bool on = i < V && (key > prefix || (key == prefix && before + __popc(eq & ((1u << lane) - 1u)) < (int)need));
        const unsigned sel = __ballot_sync(0xffffffffu, on);
        if (lane == 0) wn[wid] = __popc(sel);
        __syncthreads();
        int at = taken + __popc(sel & ((1u << lane) - 1u));
        for (int k = 0; k < kTopkThreads / 32; ++k) {
            if (k < wid) at += wn[k];
            taken += wn[k];
        }
        if (on) {
            idx_out[(int64_t)blockIdx.x * K + at] = (int32_t)i;
            val_out[(int64_t)blockIdx.x * K + at] = v;
        }
    }
    if (!lse_out) return;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        if (s != s || s2 != s2) s = NAN;
        else join_raw(m, s, m2, s2, zscale);
    }
    if (lane == 0) { sm[wid] = m; ss[wid] = s; }
    __syncthreads();
    if (tid == 0) {
        for (int k = 1; k < kTopkThreads / 32; ++k) {
            if (s != s || ss[k] != ss[k]) s = NAN;
            else join_raw(m, s, sm[k], ss[k], zscale);
        }
        lse_out[blockIdx.x] = m * inv_T + logf(s);
    }
}

}  // namespace gk

using namespace gk;

extern "C" int gk_vocab_topk(const void* logits, int64_t ld, int32_t dtype, int64_t n, int64_t V, int32_t k,
                             float temperature, int32_t* idx_out, float* val_out, float* lse_out, gk_stream_t stream) {
    if (n < 0 || V < 1 || V > 2147483647ll) return GK_ERR_SIZE;
    if (n > 2147483647ll) return GK_ERR_LIMIT;
    if (dtype != GK_TYPE_F32 && dtype != GK_TYPE_BF16 && dtype != GK_TYPE_F16) return GK_ERR_TYPE;
    if (n > 0 && (!logits || !idx_out || !val_out)) return GK_ERR_NULL;
    if (ld < V) return GK_ERR_STRIDE;
    if (((uintptr_t)logits & (dtype == GK_TYPE_F32 ? 3 : 1)) != 0) return GK_ERR_ALIGN;
    if (k < 1 || k > V || k > kVocabMaxPairs) return GK_ERR_K;
    if (!(temperature > 0.f) || !(temperature < INFINITY)) return GK_ERR_TEMPERATURE;
    if (n == 0) return GK_OK;
    cudaStream_t st = (cudaStream_t)stream;
    const float zscale = (float)(1.4426950408889634 / (double)temperature);
    const unsigned grid = (unsigned)n;
    switch (dtype) {
        case GK_TYPE_F32: k_vocab_topk<GK_TYPE_F32><<<grid, kTopkThreads, 0, st>>>(logits, ld, V, k, zscale, 1.f / temperature, idx_out, val_out, lse_out); break;
        case GK_TYPE_BF16: k_vocab_topk<GK_TYPE_BF16><<<grid, kTopkThreads, 0, st>>>(logits, ld, V, k, zscale, 1.f / temperature, idx_out, val_out, lse_out); break;
        default: k_vocab_topk<GK_TYPE_F16><<<grid, kTopkThreads, 0, st>>>(logits, ld, V, k, zscale, 1.f / temperature, idx_out, val_out, lse_out); break;
    }
    GK_CUDA_TRY(cudaGetLastError());
    note_launch();
    return GK_OK;
}
