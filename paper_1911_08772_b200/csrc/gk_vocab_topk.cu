// Top logits of rows: what a teacher sends for distillation (include/gk.h: gk_vocab_topk).
//
// One CTA a row, one pass over it.  The floor is the row's bytes: 4096 x 128000 bf16 are 1.05 GB, 160 us.
// A sample of the row, one 16-byte word in every few, gives a threshold that a little more than k
// elements are expected to reach; the pass takes the log-sum-exp with a running maximum and notes
// the 16-byte words with an element that reaches the threshold in shared memory, without a barrier; those
// words are then looked through.  The k largest of the elements found are exact whenever there are at least k and neither list overflowed; otherwise (values
// tied in thousands, or a row that the sample misses) the row is walked once more in chunks, the list
// being cut to its k largest whenever it is full, which needs no luck.
//
// The k-th largest key is found bit by bit from the highest bit in which the list's keys can differ,
// one count over the list and one barrier a bit.
#include "gk_vocab.cuh"

namespace gk {

// Unsigned key in the order of the values; -0 ties with +0, NaN is above +inf.
__device__ __forceinline__ unsigned order_key(float v) {
    if (v != v) return 0xffffffffu;
    const unsigned b = __float_as_uint(v == 0.f ? 0.f : v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);   // 0xffffffff: a NaN
}

// Sums of exp((v - m) / T) with the maximum in the logits' own unit, so that the types' largest and
// lowest values do not overflow.  What is subtracted is finite also where the maximum is not.
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : fminf(m, 3.402823466e38f); }
__device__ __forceinline__ void join_raw(float& m, float& s, float m2, float s2, float zscale) {
    const float top = fmaxf(m, m2);
    // an empty part has m = -inf and s = 0 (or NaN: it held nothing else)
    s = (m == top ? s : s * exp2_fast((m - top) * zscale)) + (m2 == top ? s2 : s2 * exp2_fast((m2 - top) * zscale));
    m = top;
}

template <int TYPE>
__device__ __forceinline__ float load_logit(const char* row, int64_t i) {
    if constexpr (TYPE == GK_TYPE_F32) return __ldg((const float*)row + i);
    else return from16<TYPE == GK_TYPE_F16>(__ldg((const uint16_t*)row + i));
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

template <int TYPE>
__device__ __forceinline__ void unpack(const uint4& x, float (&f)[TYPE == GK_TYPE_F32 ? 4 : 8]) {
    const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (TYPE == GK_TYPE_F32) f[i] = __uint_as_float(w[i]);
        else if constexpr (TYPE == GK_TYPE_BF16) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            f[2 * i] = from16<true>((uint16_t)w[i]);
            f[2 * i + 1] = from16<true>((uint16_t)(w[i] >> 16));
        }
    }
}

// Rows are served by 256 threads, five CTAs an SM, so that one row's selection runs under the
// others' streams; by 1024 threads where there are fewer rows than SMs.
template <int THREADS>
struct TopkShared {
    static constexpr int kCap = THREADS == 1024 ? 4096 : 3072;     // list entries
    unsigned key[kCap];
    int idx[kCap];
    int word[2048];   // noted words
    float m[THREADS / 32], s[THREADS / 32], sampled[THREADS / 32];
    int count;        // entries appended (may exceed the list)
    int words;        // words noted (may exceed their list)
    int bits[3];      // counts of three successive steps of a bit search
    int above;        // entries kept so far
};

// The largest t that at least `want` of the threads' keys reach, bit by bit from `bit` down, the bits
// above being t's; `reach` in: how many there are, out: how many reach t.  Stops early at
// exactly `want`.  Called by all threads, which agree on every argument but their keys.
template <int THREADS, class Count>
__device__ __forceinline__ unsigned bit_search(TopkShared<THREADS>& sh, unsigned t, int bit, int want, int& reach, const Count& count) {
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid < 3) sh.bits[tid] = 0;
    __syncthreads();
    for (int step = 0; bit >= 0 && reach != want; --bit, ++step) {
        const unsigned cand = t | 1u << bit;
        const int c = __reduce_add_sync(0xffffffffu, count(cand));
        if (lane == 0 && c) atomicAdd(&sh.bits[step % 3], c);
        if (tid == 0) sh.bits[(step + 1) % 3] = 0;      // read last two barriers ago
        __syncthreads();
        const int n = sh.bits[step % 3];
        if (n >= want) { t = cand; reach = n; }
    }
    __syncthreads();
    return t;
}

// Keeps the K largest of the list's `cnt` entries (cnt > K), ties to the lower index, in its first K
// places in no particular order; returns the K-th key without its lowest `drop` bits, which say no
// more than the others do (a 16-bit type's).  All keys lie between lo and hi; index_bits hold an index.
// A thread has OWN entries.
template <int THREADS, int OWN>
__device__ __noinline__ unsigned keep_largest(TopkShared<THREADS>& sh, int cnt, int K, unsigned lo, unsigned hi, int drop, int index_bits) {
    constexpr int kOwn = OWN;
    const int tid = threadIdx.x;
    // this thread's entries stay in registers; places past the list hold key 0, which no value has
    unsigned key[kOwn];
    int idx[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
        const int at = tid + j * THREADS;
        key[j] = at < cnt ? sh.key[at] >> drop : 0u;
        idx[j] = at < cnt ? sh.idx[at] : 0;
    }
    if (tid == 0) sh.above = 0;
    // the bits above those that differ are lo's
    lo >>= drop;
    hi >>= drop;
    const unsigned differ = lo ^ hi;
    const int bit = differ ? 31 - __clz(differ) : -1;
    const unsigned prefix = bit < 0 ? lo : bit == 31 ? 0u : lo >> (bit + 1) << (bit + 1);
    int reach = cnt;
    const unsigned t = bit_search<THREADS>(sh, prefix, bit, K, reach, [&](unsigned cand) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
            if (j * THREADS < cnt) c += key[j] >= cand;
        return c;
    });
    auto keep = [&](int j) {
        const int at = atomicAdd(&sh.above, 1);
        sh.key[at] = key[j] << drop;
        sh.idx[at] = idx[j];
    };
    // all that reach t where they are K; else those above t, and of those at t the lowest indices
    const bool all = reach == K;
#pragma unroll
    for (int j = 0; j < kOwn; ++j)
        if (key[j] > t || (all && key[j] == t)) keep(j);
    __syncthreads();
    if (all) return t;
    const int need = K - sh.above;
    int equal = reach - sh.above;
    const unsigned low = bit_search<THREADS>(sh, index_bits < 32 ? ~0u << index_bits : 0u, index_bits - 1, need, equal, [&](unsigned cand) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
            if (j * THREADS < cnt) c += key[j] == t && ~(unsigned)idx[j] >= cand;
        return c;
    });
#pragma unroll
    for (int j = 0; j < kOwn; ++j)
        if (key[j] == t && ~(unsigned)idx[j] >= low) keep(j);
    __syncthreads();
    return t;
}

template <int TYPE, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 1024 ? 1 : 5)
k_vocab_topk(const void* logits, int64_t ld, int64_t V, int K, float zscale, float inv_T, int32_t* idx_out, float* val_out, float* lse_out) {
    constexpr int kVec = TYPE == GK_TYPE_F32 ? 4 : 8, kSize = TYPE == GK_TYPE_F32 ? 4 : 2;
    constexpr int kCap = TopkShared<THREADS>::kCap;
    __shared__ TopkShared<THREADS> sh;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const char* row = (const char*)logits + (int64_t)blockIdx.x * ld * kSize;
    // elements before the first 16-byte boundary, whole words, the rest
    int64_t head = (16 - ((uintptr_t)row & 15)) % 16 / kSize;
    if (head > V) head = V;
    const int64_t words = (V - head) / kVec;
    const uint4* body = (const uint4*)(row + head * kSize);

    constexpr int kWords = 2048;
    // the low bits of a 16-bit type's keys follow from its sign
    constexpr int kDrop = TYPE == GK_TYPE_BF16 ? 16 : TYPE == GK_TYPE_F16 ? 13 : 0;
    const int index_bits = 32 - __clz((int)(V - 1) | 1);
    if (tid == 0) { sh.count = 0; sh.words = 0; }
    float tau = -INFINITY;
    if (V > kCap) {
        // The sample: up to four words a thread; of each thread the largest.  With x of the row's k
        // largest expected among the sampled elements, the (x + 4 sqrt(x) + 4)-th largest is taken:
        // about as many as k can hardly be above it.  Thread maxima stand for the elements: the
        // sample's largest are nearly always different threads'.
        const int per = words / THREADS >= 64 ? 4 : words / THREADS >= 16 ? 2 : 1;
        float top = -INFINITY;
        for (int j = 0; j < per; ++j) {
            const int64_t at = ((int64_t)j * THREADS + tid) * words / ((int64_t)per * THREADS);
            float f[kVec];
            unpack<TYPE>(__ldg(body + at), f);
#pragma unroll
            for (int i = 0; i < kVec; ++i) top = fmaxf(top, f[i]);
        }
        // the largest sampled element is where the log-sum-exp starts: few elements raise it
        float most = top;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (lane == 0) sh.sampled[wid] = most;
        const float x = (float)K * (float)(per * THREADS * kVec) / (float)V;
        const int r = min((int)(x + 4.f * sqrtf(x) + 4.f), THREADS / 2);
        const unsigned key = order_key(top);
        unsigned t = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const unsigned cand = t | 1u << bit;
            const int c = __syncthreads_count(key >= cand);
            if (c >= r) t = cand;
            if (c >= r && c <= r + r / 4) break;
        }
        tau = t == 0 ? -INFINITY : key_value(t);
        if (!(tau > -INFINITY)) tau = -INFINITY;   // below every value: the keys of -NaN
    }
    __syncthreads();

    float m = -INFINITY, s = 0.f;
    if (V > kCap)
        for (int k = 0; k < THREADS / 32; ++k) m = fmaxf(m, sh.sampled[k]);
    float ref = finite_ref(m);
    auto append = [&](float v, int64_t i) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < kCap) { sh.key[at] = order_key(v); sh.idx[at] = (int)i; }
    };
    auto raise = [&](float to) {
        if (to > m) {
            const float r = finite_ref(to);
            if (m > -INFINITY) s *= exp2_fast((ref - r) * zscale);   // else s is 0, or NaN from a NaN
            m = to;
            ref = r;
        }
    };
    auto single = [&](int64_t i) {
        const float v = load_logit<TYPE>(row, i);
        raise(v);
        s += exp2_fast((v - ref) * zscale);
        if (!(v < tau)) append(v, i);
    };
    uint64_t sums = pair(0.f, 0.f);
    auto word = [&](const uint4& x, int64_t at) {
        float f[kVec];
        unpack<TYPE>(x, f);
        float g = f[0];
#pragma unroll
        for (int i = 1; i < kVec; ++i) g = fmaxf(g, f[i]);
        if (g > m) {
            const float r = finite_ref(g), by = m > -INFINITY ? exp2_fast((ref - r) * zscale) : 1.f;   // else the sums are 0 or NaN
            s *= by;
            sums = mul2(sums, pair(by, by));
            m = g;
            ref = r;
        }
        const uint64_t less = pair(-ref, -ref), by = pair(zscale, zscale);
        uint64_t e[kVec / 2];
#pragma unroll
        for (int i = 0; i < kVec / 2; ++i) {
            float a, b;
            unpair(mul2(add2(pair(f[2 * i], f[2 * i + 1]), less), by), a, b);
            e[i] = pair(exp2_fast(a), exp2_fast(b));
        }
#pragma unroll
        for (int w = kVec / 4; w > 0; w /= 2)
#pragma unroll
            for (int i = 0; i < w; ++i) e[i] = add2(e[i], e[i + w]);
        sums = add2(sums, e[0]);
        if (!(g < tau)) {
            const int to = atomicAdd(&sh.words, 1);
            if (to < kWords) sh.word[to] = (int)at;
        }
    };
    if (tid < head) single(tid);
    if (tid < V - head - words * kVec) single(head + words * kVec + tid);
    int64_t at = tid;
    for (; at + 3 * THREADS < words; at += 4 * THREADS) {
        const uint4 a = __ldcs(body + at), b = __ldcs(body + at + THREADS), c = __ldcs(body + at + 2 * THREADS),
                    d = __ldcs(body + at + 3 * THREADS);
        word(a, at);
        word(b, at + THREADS);
        word(c, at + 2 * THREADS);
        word(d, at + 3 * THREADS);
    }
    for (; at < words; at += THREADS) word(__ldcs(body + at), at);

    {
        float a, b;
        unpair(sums, a, b);
        s += a + b;
    }
    // log-sum-exp and maximum of the row
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        join_raw(m, s, m2, s2, zscale);
    }
    if (lane == 0) { sh.m[wid] = m; sh.s[wid] = s; }
    __syncthreads();
    m = sh.m[0];
    s = sh.s[0];
    for (int k = 1; k < THREADS / 32; ++k) join_raw(m, s, sh.m[k], sh.s[k], zscale);
    if (lse_out && tid == 0) lse_out[blockIdx.x] = m * inv_T + logf(s);

    // The noted words' elements.  The pass compares a word's maximum, which knows nothing of NaN: a
    // row with one is taken in chunks.
    const int noted = sh.words;
    const bool whole = noted <= kWords && s == s;
    if (whole)
        for (int j = tid; j < noted; j += THREADS) {
            const int64_t w = sh.word[j];
            float f[kVec];
            unpack<TYPE>(__ldg(body + w), f);
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (!(f[i] < tau)) append(f[i], head + w * kVec + i);
        }
    __syncthreads();
    int cnt = sh.count;
    if (whole && cnt >= K && cnt <= kCap) {
        if (cnt > K) {
            if (cnt <= 2 * THREADS) keep_largest<THREADS, 2>(sh, cnt, K, order_key(tau), order_key(m), kDrop, index_bits);
            else keep_largest<THREADS, kCap / THREADS>(sh, cnt, K, order_key(tau), order_key(m), kDrop, index_bits);
        }
    } else {
        // The list overflowed or is short.  In chunks: after a cut only larger keys are appended,
        // for an equal one comes later in the row than all that are kept.
        constexpr int kEach = 2048 / THREADS, kChunk = kEach * THREADS;
        unsigned floor_key = 0;      // below every value's key
        __syncthreads();
        if (tid == 0) sh.count = 0;
        __syncthreads();
        for (int64_t i0 = 0; i0 < V; i0 += kChunk) {
            unsigned key[kEach];
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int64_t i = i0 + j * THREADS + tid;
                key[j] = i < V ? order_key(load_logit<TYPE>(row, i)) : 0u;
            }
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                if (key[j] > floor_key) {
                    const int to = atomicAdd(&sh.count, 1);
                    sh.key[to] = key[j];
                    sh.idx[to] = (int)(i0 + j * THREADS + tid);
                }
            __syncthreads();
            cnt = sh.count;
            if (cnt + kChunk > kCap || i0 + kChunk >= V) {
                if (cnt > K) {
                    floor_key = keep_largest<THREADS, kCap / THREADS>(sh, cnt, K, 0u, 0xffffffffu, 0, index_bits);
                    cnt = K;
                }
                if (tid == 0) sh.count = cnt;
            }
            __syncthreads();
        }
    }
    __syncthreads();
    // in the order of the indices
    for (int j = tid; j < K; j += THREADS) {
        const int i = sh.idx[j];
        int rank = 0;
        for (int e = 0; e < K; ++e) rank += sh.idx[e] < i;
        idx_out[(int64_t)blockIdx.x * K + rank] = i;
        val_out[(int64_t)blockIdx.x * K + rank] = load_logit<TYPE>(row, i);
    }
}

template <int TYPE>
static void launch_topk(const void* logits, int64_t ld, int64_t n, int64_t V, int k, float temperature, int32_t* idx_out,
                        float* val_out, float* lse_out, int sms, cudaStream_t st) {
    const float zscale = (float)(1.4426950408889634 / (double)temperature), inv_T = 1.f / temperature;
    if (n < sms) k_vocab_topk<TYPE, 1024><<<(unsigned)n, 1024, 0, st>>>(logits, ld, V, k, zscale, inv_T, idx_out, val_out, lse_out);
    else k_vocab_topk<TYPE, 256><<<(unsigned)n, 256, 0, st>>>(logits, ld, V, k, zscale, inv_T, idx_out, val_out, lse_out);
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
    int dev = 0, sms = 0;
    GK_CUDA_TRY(cudaGetDevice(&dev));
    GK_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    switch (dtype) {
        case GK_TYPE_F32: launch_topk<GK_TYPE_F32>(logits, ld, n, V, k, temperature, idx_out, val_out, lse_out, sms, st); break;
        case GK_TYPE_BF16: launch_topk<GK_TYPE_BF16>(logits, ld, n, V, k, temperature, idx_out, val_out, lse_out, sms, st); break;
        default: launch_topk<GK_TYPE_F16>(logits, ld, n, V, k, temperature, idx_out, val_out, lse_out, sms, st); break;
    }
    GK_CUDA_TRY(cudaGetLastError());
    note_launch();
    return GK_OK;
}
