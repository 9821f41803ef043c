// Top logits of rows: what a teacher sends for distillation (include/gk.h: gk_vocab_topk).
//
// One CTA a row, one pass over it.  The floor is the row's bytes: 4096 x 128000 bf16 are 1.05 GB, 160 us at the
// rate of a copy; the call takes 234 to 251.  Of 234 the stream with its exponentials takes 165, the noting of words 25,
// and 43 are selections that the other CTAs' streams do not hide (each of the three left out of a trial in turn).
// More CTAs an SM, with fewer registers for words in flight, took 270 to 410.
// Each warp streams a contiguous share of the row, four 16-byte words a thread at a time from four
// places of the share.  The first four are the sample: 32 or more places spread over the row, from which a
// threshold is taken that a little more than k elements are expected to reach.  The pass takes the
// log-sum-exp with a running maximum and notes the words with an element that reaches the threshold in
// shared memory, without a barrier; those words are then looked through.  The k largest of the elements found
// are exact whenever there are at least k and neither list overflowed; otherwise (values tied in
// thousands, or a row that the sample misses) the row is walked once more in chunks, the list being cut to its
// k largest whenever it is full, which needs no luck.
//
// The k-th largest key is found two bits at a time from the highest bit in which the keys can differ, with three
// counts over the list a step; by one warp where the list is short, so that no step needs a barrier.
#include "gk_words.cuh"

namespace gk {

// Sums of exp((v - m) / T) with the maximum in the logits' own unit, so that the types' largest and
// lowest values do not overflow.  What is subtracted is finite also where the maximum is not.
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : fminf(m, 3.402823466e38f); }
__device__ __forceinline__ void join_raw(float& m, float& s, float m2, float s2, float zscale) {
    const float top = fmaxf(m, m2);
    // an empty part has m = -inf and s = 0 (or NaN: it held nothing else)
    s = (m == top ? s : s * exp2_fast((m - top) * zscale)) + (m2 == top ? s2 : s2 * exp2_fast((m2 - top) * zscale));
    m = top;
}

// Rows are served by 256 threads, four CTAs an SM, so that one row's selection runs under the
// others' streams; by 1024 threads where there are fewer rows than SMs and the rows are long.
template <int THREADS>
struct TopkShared {
    static constexpr int kCap = (THREADS == 1024 ? 4 : 12) * THREADS;     // list entries
    static constexpr int kWords = 2048, kData = THREADS == 1024 ? 448 : 896;
    // the first of the noted words themselves: fetched again by number they cost 2000 x 100003 fp32 174 us, so 161
    uint4 data[kData];
    unsigned key[kCap];
    alignas(16) int idx[kCap];
    int word[kWords];           // noted words
    float m[THREADS / 32], s[THREADS / 32], sampled[THREADS / 32];
    float tau;
    int count;        // entries appended (may exceed the list)
    int words;        // words noted (may exceed their list)
    unsigned bits[2][THREADS / 32];   // the warps' counts of two successive steps of a search
    int above;        // entries kept so far
};

// The largest t that at least `want` of the threads' keys reach, two bits at a time from `bit` down, the
// bits above being t's; `reach` in: how many there are, out: how many reach t.  Stops early at between
// `want` and `most`.  count(a, b, c): how many of the thread's keys reach each, in tens of bits.
// Called by all threads, which agree on every argument but their keys.
template <int THREADS, class Count>
__device__ __forceinline__ unsigned bit_search(TopkShared<THREADS>& sh, unsigned t, int bit, int want, int most, int& reach,
                                               const Count& count) {
    constexpr int kWarps = THREADS / 32;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    for (int step = 0; bit >= 0 && reach > most; bit -= 2, ++step) {
        const int low = bit > 0 ? bit - 1 : 0;
        const unsigned c1 = t | 1u << low, c2 = t | 1u << bit, c3 = c2 | 1u << low;     // one candidate where one bit is left
        const unsigned c = __reduce_add_sync(0xffffffffu, count(c1, c2, c3));
        // (a step's counts are read before the next step's barrier, and written over after it)
        if (lane == 0) sh.bits[step & 1][wid] = c;
        __syncthreads();
        const unsigned all = lane < kWarps ? sh.bits[step & 1][lane] : 0u;
        const int n1 = (int)__reduce_add_sync(0xffffffffu, all & 1023), n2 = (int)__reduce_add_sync(0xffffffffu, all >> 10 & 1023),
                  n3 = (int)__reduce_add_sync(0xffffffffu, all >> 20);
        if (n3 >= want) { t = c3; reach = n3; }
        else if (n2 >= want) { t = c2; reach = n2; }
        else if (n1 >= want) { t = c1; reach = n1; }
    }
    return t;
}
__device__ __forceinline__ unsigned reaches(unsigned key, unsigned a, unsigned b, unsigned c) {
    return (key >= a ? 1u : 0u) + (key >= b ? 1u << 10 : 0u) + (key >= c ? 1u << 20 : 0u);
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
    __syncthreads();
    if (tid == 0) sh.above = 0;
    // the bits above those that differ are lo's
    lo >>= drop;
    hi >>= drop;
    const unsigned differ = lo ^ hi;
    const int bit = differ ? 31 - __clz(differ) : -1;
    const unsigned prefix = bit < 0 ? lo : bit == 31 ? 0u : lo >> (bit + 1) << (bit + 1);
    int reach = cnt;
    const unsigned t = bit_search<THREADS>(sh, prefix, bit, K, K, reach, [&](unsigned c1, unsigned c2, unsigned c3) {
        unsigned c = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
            if (j * THREADS < cnt) c += reaches(key[j], c1, c2, c3);
        return c;
    });
    auto keep = [&](int j) {
        const int at = atomicAdd(&sh.above, 1);
        sh.key[at] = key[j] << drop;
        sh.idx[at] = idx[j];
    };
    __syncthreads();
    // all that reach t where they are K; else those above t, and of those at t the lowest indices
    const bool all = reach == K;
#pragma unroll
    for (int j = 0; j < kOwn; ++j)
        if (key[j] > t || (all && key[j] == t)) keep(j);
    __syncthreads();
    if (all) return t;
    const int need = K - sh.above;
    int equal = reach - sh.above;
    const unsigned low = bit_search<THREADS>(sh, index_bits < 32 ? ~0u << index_bits : 0u, index_bits - 1, need, need, equal,
                                                 [&](unsigned c1, unsigned c2, unsigned c3) {
        unsigned c = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
            if (j * THREADS < cnt && key[j] == t) c += reaches(~(unsigned)idx[j], c1, c2, c3);
        return c;
    });
#pragma unroll
    for (int j = 0; j < kOwn; ++j)
        if (key[j] == t && ~(unsigned)idx[j] >= low) keep(j);
    __syncthreads();
    return t;
}

// The same search by one warp: no barriers, which with a few hundred keys cost more than the counting.
template <class Count>
__device__ __forceinline__ unsigned warp_search(unsigned t, int bit, int want, int most, int& reach, const Count& count) {
    for (; bit >= 0 && reach > most; bit -= 2) {
        const int low = bit > 0 ? bit - 1 : 0;
        const unsigned c1 = t | 1u << low, c2 = t | 1u << bit, c3 = c2 | 1u << low;
        const unsigned c = count(c1, c2, c3);
        const int n1 = (int)__reduce_add_sync(0xffffffffu, c & 1023), n2 = (int)__reduce_add_sync(0xffffffffu, c >> 10 & 1023),
                  n3 = (int)__reduce_add_sync(0xffffffffu, c >> 20);
        if (n3 >= want) { t = c3; reach = n3; }
        else if (n2 >= want) { t = c2; reach = n2; }
        else if (n1 >= want) { t = c1; reach = n1; }
    }
    return t;
}
constexpr int kFew = 768;      // keys that one warp counts faster than all of them with barriers

// keep_largest for up to kFew entries, by one warp, in the list's order.
template <int THREADS>
__device__ __forceinline__ void keep_few(TopkShared<THREADS>& sh, int cnt, int K, unsigned lo, unsigned hi, int drop, int index_bits) {
    const int lane = threadIdx.x & 31;
    lo >>= drop;
    hi >>= drop;
    const unsigned differ = lo ^ hi;
    const int bit = differ ? 31 - __clz(differ) : -1;
    const unsigned prefix = bit < 0 ? lo : bit == 31 ? 0u : lo >> (bit + 1) << (bit + 1);
    int reach = cnt;
    const unsigned t = warp_search(prefix, bit, K, K, reach, [&](unsigned c1, unsigned c2, unsigned c3) {
        unsigned c = 0;
#pragma unroll 4
        for (int j = lane; j < cnt; j += 32) c += reaches(sh.key[j] >> drop, c1, c2, c3);
        return c;
    });
    // those above t to the front, the indices of those at t to the word list
    int above = 0, equal = 0;
    for (int j0 = 0; j0 < cnt; j0 += 32) {
        const int j = j0 + lane;
        const unsigned key = j < cnt ? sh.key[j] : 0u;
        const int idx = j < cnt ? sh.idx[j] : 0;
        const unsigned up = __ballot_sync(0xffffffffu, key >> drop > t), at = __ballot_sync(0xffffffffu, key != 0 && key >> drop == t);
        const unsigned before = (1u << lane) - 1u;
        if (up >> lane & 1) sh.idx[above + __popc(up & before)] = idx;      // behind what has been read
        if (at >> lane & 1) sh.word[equal + __popc(at & before)] = idx;
        above += __popc(up);
        equal += __popc(at);
        __syncwarp();
    }
    // of those at t the lowest indices
    const int need = K - above;
    unsigned low = 0;
    if (equal > need) {
        if (equal <= 32) {
            // the need-th lowest is the one with need - 1 below it
            const int idx = lane < equal ? sh.word[lane] : 0x7fffffff;
            int rank = 0;
            for (int e = 0; e < equal; ++e) rank += __shfl_sync(0xffffffffu, idx, e) < idx;
            const unsigned is = __ballot_sync(0xffffffffu, lane < equal && rank == need - 1);
            low = ~(unsigned)__shfl_sync(0xffffffffu, idx, __ffs(is) - 1);
        } else {
            int n = equal;
            low = warp_search(index_bits < 32 ? ~0u << index_bits : 0u, index_bits - 1, need, need, n, [&](unsigned c1, unsigned c2, unsigned c3) {
                unsigned c = 0;
                for (int j = lane; j < equal; j += 32) c += reaches(~(unsigned)sh.word[j], c1, c2, c3);
                return c;
            });
        }
    }
    for (int j0 = 0; j0 < equal; j0 += 32) {
        const int j = j0 + lane;
        const int idx = j < equal ? sh.word[j] : 0;
        const unsigned on = __ballot_sync(0xffffffffu, j < equal && ~(unsigned)idx >= low);
        if (on >> lane & 1) sh.idx[above + __popc(on & ((1u << lane) - 1u))] = idx;
        above += __popc(on);
    }
}

template <int TYPE, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 1024 ? 1 : 4)
k_vocab_topk(const void* logits, int64_t ld, int64_t V, int K, float zscale, float inv_T, int32_t* idx_out, float* val_out, float* lse_out) {
    constexpr int kVec = TYPE == GK_TYPE_F32 ? 4 : 8, kSize = TYPE == GK_TYPE_F32 ? 4 : 2;
    constexpr int kCap = TopkShared<THREADS>::kCap;
    __shared__ TopkShared<THREADS> sh;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const char* row = (const char*)logits + (int64_t)blockIdx.x * ld * kSize;
    // elements before the first 16-byte boundary, whole words, the rest
    int64_t head = (16 - ((uintptr_t)row & 15)) % 16 / kSize;
    if (head > V) head = V;
    const int words = (int)((V - head) / kVec);
    const uint4* body = (const uint4*)(row + head * kSize);

    constexpr int kWords = TopkShared<THREADS>::kWords, kData = TopkShared<THREADS>::kData;
    // the low bits of a 16-bit type's keys follow from its sign
    constexpr int kDrop = TYPE == GK_TYPE_BF16 ? 16 : TYPE == GK_TYPE_F16 ? 13 : 0;
    const int index_bits = 32 - __clz((int)(V - 1) | 1);
    if (tid == 0) { sh.count = 0; sh.words = 0; }

    // Four words a thread at a time, from four places of the warp's share; the last THREADS words or fewer singly.
    // A CTA that has its SM for itself (1024 threads) sends for eight words before the threshold is known; with four
    // CTAs an SM that made the loop slower (4096 x 128000: 234 us, 312 so).
    constexpr int kWarps = THREADS / 32;
    constexpr bool kLone = THREADS == 1024;
    const int share = words / THREADS, quarter = (share + 3) / 4;   // in steps of 32 words
    const uint4* own = body + wid * share * 32 + lane;
    uint4 x[4], next[4];
    auto fetch = [&](uint4 (&to)[4], int q) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (q < quarter && q + i * quarter < share) to[i] = __ldcs(own + (q + i * quarter) * 32);
    };
    fetch(x, 0);
    if constexpr (kLone) fetch(next, 1);

    float tau = -INFINITY, m = -INFINITY, s = 0.f;
    if (V > kCap) {
        // The threshold.  With e of the row's k largest expected among the sample, the (e + 4 sqrt(e) + 4)-th largest
        // of it is taken: about as many as k can hardly be above it.  Where that is a small part of 256, the maxima of
        // 256 threads or groups of four stand for the elements; the sample's largest are nearly always different ones'.
        // (Elsewhere all but 16-bit types' fourth words count: a warp's count has to fit ten bits.)
        constexpr int kSample = TYPE == GK_TYPE_F32 ? 4 : 3;
        float top = -INFINITY;
        int steps = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i * quarter < share) {
                float f[kVec];
                unpack<TYPE>(x[i], f);
                ++steps;
#pragma unroll
                for (int e = 0; e < kVec; ++e) top = fmaxf(top, f[e]);
            }
        // the largest sampled element is where the log-sum-exp starts: few elements raise it
        float most = top;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (lane == 0) sh.sampled[wid] = most;
        if constexpr (THREADS == 1024) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        }
        if (tid % (THREADS / 256) == 0) sh.key[tid / (THREADS / 256)] = order_key(top);
        __syncthreads();
        m = lane < kWarps ? sh.sampled[lane] : -INFINITY;
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        m = __shfl_sync(0xffffffffu, m, 0);
        float e = (float)K * (float)(steps * THREADS * kVec) / (float)V;
        int r = (int)(e + 4.f * sqrtf(e) + 4.f);
        unsigned t = 0;
        if (r <= 64) {
            if (wid == 0) {
                // between the smallest and the largest of the maxima, which are kept in registers
                constexpr int kOwn = 256 / 32;
                unsigned key[kOwn], least = 0xffffffffu;
#pragma unroll
                for (int j = 0; j < kOwn; ++j) {
                    key[j] = sh.key[j * 32 + lane];
                    least = min(least, key[j]);
                }
                least = __reduce_min_sync(0xffffffffu, least);
                const unsigned differ = least ^ order_key(m);
                const int bit = differ ? 31 - __clz(differ) : -1;
                int reach = 256;
                t = warp_search(bit < 0 ? least : bit == 31 ? 0u : least >> (bit + 1) << (bit + 1), bit, r, r + r / 4, reach,
                                [&](unsigned c1, unsigned c2, unsigned c3) {
                    unsigned c = 0;
#pragma unroll
                    for (int j = 0; j < kOwn; ++j) c += reaches(key[j], c1, c2, c3);
                    return c;
                });
                if (lane == 0) sh.tau = t == 0 ? -INFINITY : key_value(t);
            }
            __syncthreads();
            tau = sh.tau;
        } else {
            steps = min(steps, kSample);
            int reach = steps * THREADS * kVec;
            e = (float)K * (float)reach / (float)V;
            r = (int)(e + 4.f * sqrtf(e) + 4.f);
            t = bit_search<THREADS>(sh, 0u, 31, r, r + r / 4, reach, [&](unsigned c1, unsigned c2, unsigned c3) {
                unsigned c = 0;
#pragma unroll
                for (int i = 0; i < kSample; ++i)
                    if (i * quarter < share) {
                        float f[kVec];
                        unpack<TYPE>(x[i], f);
#pragma unroll
                        for (int e = 0; e < kVec; ++e) c += reaches(order_key(f[e]), c1, c2, c3);
                    }
                return c;
            });
            tau = t == 0 ? -INFINITY : key_value(t);
        }
        if (!(tau > -INFINITY)) tau = -INFINITY;   // below every value: the keys of -NaN
    }
    __syncthreads();
    // The sums are of powers 2^(v zscale - ref), ref the maximum in that unit; what would overflow on the way
    // (values near the types' ends, infinities) shows in the sum and is taken again below.
    auto power_ref = [&](float v) { return v == -INFINITY ? 0.f : fmaxf(fminf(v, 1e37f), -1e37f) * zscale; };
    float ref = power_ref(m);
    auto append = [&](float v, int64_t i) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < kCap) { sh.key[at] = order_key(v); sh.idx[at] = (int)i; }
    };
    uint64_t sums = pair(0.f, 0.f);
    auto raise = [&](float to) {
        const float r = power_ref(to), by = m > -INFINITY ? exp2_fast(ref - r) : 1.f;   // else the sums are 0 or NaN
        s *= by;
        sums = mul2(sums, pair(by, by));
        m = to;
        ref = r;
    };
    auto single = [&](int64_t i) {
        const float v = load_logit<TYPE>(row, i);
        if (!(v < tau)) {
            append(v, i);
            if (v > m) raise(v);
        }
        s += exp2_fast(fmaf(v, zscale, -ref));
    };
    const uint64_t by = pair(zscale, zscale);
    auto word = [&](const uint4& x, int at) {
        float f[kVec];
        unpack<TYPE>(x, f);
        float g;
        if constexpr (kVec == 8) {
            g = max3(f[0], f[1], f[2]);
            g = max3(g, f[3], f[4]);
            g = fmaxf(max3(g, f[5], f[6]), f[7]);
        } else {
            g = fmaxf(max3(f[0], f[1], f[2]), f[3]);
        }
        if (!(g < tau)) {
            const int to = atomicAdd(&sh.words, 1);
            if (to < kWords) sh.word[to] = at;
            if (to < kData) sh.data[to] = x;
            if (g > m) raise(g);
        }
        const uint64_t less = pair(-ref, -ref);
        uint64_t e[kVec / 2];
#pragma unroll
        for (int i = 0; i < kVec / 2; ++i) {
            float a, b;
            unpair(fma2(pair(f[2 * i], f[2 * i + 1]), by, less), a, b);
            e[i] = pair(exp2_fast(a), exp2_fast(b));
        }
#pragma unroll
        for (int w = kVec / 4; w > 0; w /= 2)
#pragma unroll
            for (int i = 0; i < w; ++i) e[i] = add2(e[i], e[i + w]);
        sums = add2(sums, e[0]);
    };
    if (tid < head) single(tid);
    if (tid < V - head - (int64_t)words * kVec) single(head + (int64_t)words * kVec + tid);
    // the next words are on their way while four are looked at
    for (int q = 0; q < quarter; ++q) {
        if (!kLone || q > 0) fetch(next, q + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (q + i * quarter < share) word(x[i], (wid * share + q + i * quarter) * 32 + lane);
            x[i] = next[i];
        }
    }
    if (share * THREADS + tid < words) word(__ldcs(body + share * THREADS + tid), share * THREADS + tid);
    {
        float a, b;
        unpair(sums, a, b);
        s += a + b;
    }
    // log-sum-exp and maximum of the row
    auto join_lanes = [&](int from) {
#pragma unroll
        for (int o = from; o > 0; o >>= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
            join_raw(m, s, m2, s2, zscale);
        }
    };
    join_lanes(16);
    if (lane == 0) { sh.m[wid] = m; sh.s[wid] = s; }
    __syncthreads();
    auto join_warps = [&]() {
        m = lane < kWarps ? sh.m[lane] : -INFINITY;
        s = lane < kWarps ? sh.s[lane] : 0.f;
        join_lanes(kWarps / 2);
        m = __shfl_sync(0xffffffffu, m, 0);
        s = __shfl_sync(0xffffffffu, s, 0);
    };
    join_warps();
    if (!(s >= 0.5f && s < INFINITY) && !(m == -INFINITY && s == 0.f)) {
        // the maximum itself counts 1, so something overflowed (or is NaN): differences first, then the scale
        const float top = finite_ref(m);
        s = 0.f;
        for (int64_t i = tid; i < V; i += THREADS) s += exp2_fast((load_logit<TYPE>(row, i) - top) * zscale);
        join_lanes(16);
        __syncthreads();
        if (lane == 0) { sh.m[wid] = m; sh.s[wid] = s; }
        __syncthreads();
        join_warps();
    }
    if (lse_out && tid == 0) lse_out[blockIdx.x] = m * inv_T + logf(s);

    // The noted words' elements.  The pass compares a word's maximum, which knows nothing of NaN: a
    // row with one is taken in chunks.
    const int noted = sh.words;
    const bool whole = noted <= kWords && s == s;
    if (whole)
        for (int j = tid; j < noted; j += THREADS) {
            const int w = sh.word[j];
            float f[kVec];
            unpack<TYPE>(j < kData ? sh.data[j] : __ldg(body + w), f);
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (!(f[i] < tau)) append(f[i], head + (int64_t)w * kVec + i);
        }
    __syncthreads();
    int cnt = sh.count;
    if (whole && cnt >= K && cnt <= kCap) {
        if (cnt > K) {
            if (cnt <= kFew) {
                if (wid == 0) keep_few<THREADS>(sh, cnt, K, order_key(tau), order_key(m), kDrop, index_bits);
            } else keep_largest<THREADS, kCap / THREADS>(sh, cnt, K, order_key(tau), order_key(m), kDrop, index_bits);
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
    // In the order of the indices.
    auto emit = [&](int i, int rank) {
        idx_out[(int64_t)blockIdx.x * K + rank] = i;
        val_out[(int64_t)blockIdx.x * K + rank] = load_logit<TYPE>(row, i);
    };
    if (K <= 128) {
        // each against all; the list is filled up to a multiple of four with what is above them
        if (tid < 3) sh.idx[K + tid] = 0x7fffffff;
        __syncthreads();
        if (tid < K) {
            const int own_idx = sh.idx[tid];
            int rank = 0;
#pragma unroll 4
            for (int e = 0; e < K; e += 4) {
                const int4 i = *(const int4*)&sh.idx[e];
                rank += (i.x < own_idx) + (i.y < own_idx) + (i.z < own_idx) + (i.w < own_idx);
            }
            emit(own_idx, rank);
        }
    } else {
        // 256 stretches of the row: counted, the indices brought together by stretch (in sh.key), and each ranked in its own
        const unsigned stretch = (unsigned)((V + 255) / 256);
        int* count = sh.word;          // 256 counts, 256 starts, 256 places taken
        if (tid < 256) count[tid] = count[512 + tid] = 0;
        __syncthreads();
        for (int j = tid; j < K; j += THREADS) atomicAdd(&count[(unsigned)sh.idx[j] / stretch], 1);
        __syncthreads();
        if (wid == 0) {
            int before = 0;
            for (int j0 = 0; j0 < 256; j0 += 32) {
                const int n = count[j0 + lane];
                int incl = n;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const int v = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += v;
                }
                count[256 + j0 + lane] = before + incl - n;
                before += __shfl_sync(0xffffffffu, incl, 31);
            }
        }
        __syncthreads();
        for (int j = tid; j < K; j += THREADS) {
            const int b = (unsigned)sh.idx[j] / stretch;
            sh.key[count[256 + b] + atomicAdd(&count[512 + b], 1)] = (unsigned)sh.idx[j];
        }
        __syncthreads();
        for (int j = tid; j < K; j += THREADS) {
            const unsigned i = sh.key[j];
            const int from = count[256 + i / stretch], to = from + count[i / stretch];
            int rank = from;
            for (int e = from; e < to; ++e) rank += sh.key[e] < i;
            emit((int)i, rank);
        }
    }
}

template <int TYPE>
static void launch_topk(const void* logits, int64_t ld, int64_t n, int64_t V, int k, float temperature, int32_t* idx_out,
                        float* val_out, float* lse_out, int sms, cudaStream_t st) {
    const float zscale = (float)(1.4426950408889634 / (double)temperature), inv_T = 1.f / temperature;
    // 1024 threads a row while each row has an SM to itself and work for them: bf16 rows of 128000, 147 of them 24.6 us
    // (28.7 by 256 threads), 149 of them 35.8 (26.8), fp32 30.7 (38.9) and 45.1 (38.9); of rows of 16384 the two take
    // the same, 12 to 14 us.
    if (n < sms && V >= 16384) k_vocab_topk<TYPE, 1024><<<(unsigned)n, 1024, 0, st>>>(logits, ld, V, k, zscale, inv_T, idx_out, val_out, lse_out);
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
    if (off_boundary(dtype == GK_TYPE_F32 ? 4 : 2, logits) || off_boundary(4, idx_out, val_out, lse_out)) return GK_ERR_ALIGN;
    if (k < 1 || k > V || k > kVocabMaxPairs) return GK_ERR_K;
    if (!temperature_ok(temperature)) return GK_ERR_TEMPERATURE;
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
