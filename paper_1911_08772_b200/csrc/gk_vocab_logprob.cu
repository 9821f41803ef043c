// Log probabilities of given tokens with entropy, rank and the most probable tokens, and their gradient
// (include/gk.h: gk_vocab_logprob, gk_vocab_logprob_grad).
//
// Forward: one CTA a row, one pass.  With m the row's maximum so far and d = (z - m) / T in units of log 2, the
// pass sums S0 = 2^d and S1 = d 2^d; a larger maximum by b rescales S0 by 2^b and S1 to 2^b (S1 + b S0).  Then
//     lse = m / T + log S0,   entropy = log S0 - log(2) S1 / S0,
// two terms of one sign, as m is the maximum at the end, so that a small entropy keeps its digits.  The rank counts
// the elements before the token that are not below it, and those behind it that are above.
//
// Alternatives: a threshold from a sample of the row, which a little more than k elements are expected to be above;
// those are listed, and the place of each among them is counted, which sorts them.  Where fewer than k are above, the
// first elements equal to the threshold fill the list (rows whose mask leaves little); where that is not enough
// either, or the list is too short, the row is walked again in chunks and the list cut whenever it is full.
#include "gk_words.cuh"

namespace gk {

constexpr int kLogprobMaxTokens = 128, kLogprobMaxAlternatives = 128;
constexpr int kLpThreads = 256, kLpWarps = kLpThreads / 32;
constexpr int kLpList = 2048;       // entries of the list of alternatives
constexpr int kLpRanked = 512;      // as many as are sorted by counting; a longer list is cut first
constexpr float kLpFloor = -200.f;  // powers of two below this are zero in fp32, and their products with it too

struct LogprobCall {
    const char* logits;
    int64_t ld, n, V;
    const int64_t* token;
    int m, k;
    float T, zscale;      // zscale: log2(e) / T
    float* logp;
    int32_t* rank;
    float* entropy;
    float* lse;
    int32_t* idx;
    float* val;
};

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Maximum (as it is in the logits) and the two sums relative to it.
struct Sums {
    float m, s0, s1;
};
__device__ __forceinline__ float lp_ref(float m) { return m == -INFINITY ? 0.f : fminf(m, 3.402823466e38f); }
// What sums relative to m are multiplied by to be relative to `to` >= m, as a power of two.
__device__ __forceinline__ float lp_shift(float m, float to, float zscale) {
    return m == to ? 0.f : m == -INFINITY ? kLpFloor : fmaxf((m - lp_ref(to)) * zscale, kLpFloor);
}
__device__ __forceinline__ void lp_join(Sums& a, const Sums& b, float zscale) {
    const float top = fmaxf(a.m, b.m), da = lp_shift(a.m, top, zscale), db = lp_shift(b.m, top, zscale);
    const float ea = exp2_fast(da), eb = exp2_fast(db);      // one where the shift is nothing
    a.s1 = ea * fmaf(a.s0, da, a.s1) + eb * fmaf(b.s0, db, b.s1);
    a.s0 = ea * a.s0 + eb * b.s0;
    a.m = top;
}

struct LpShared {
    uint64_t list[kLpList];      // key of the value above, complement of the index below: all differ
    uint64_t best[kLogprobMaxAlternatives];
    float sample[kLpThreads];
    float m[kLpWarps], s0[kLpWarps], s1[kLpWarps];
    int above[kLpWarps];
    int count, any;
    float tau, first, top;
};
__device__ __forceinline__ uint64_t lp_entry(float v, int64_t i) { return (uint64_t)order_key(v) << 32 | (uint32_t)~(uint32_t)i; }

// The list of `cnt` entries cut to the k largest and at most kLpRanked - k more; returns a bound that all kept reach
// and that at least k do.  By all threads, which see `cnt` alike.
__device__ __noinline__ uint64_t lp_cut(LpShared& sh, int& cnt, int k) {
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    uint64_t own[kLpList / kLpThreads];
#pragma unroll
    for (int j = 0; j < kLpList / kLpThreads; ++j) own[j] = tid + j * kLpThreads < cnt ? sh.list[tid + j * kLpThreads] : 0;
    uint64_t t = 0;
    int reach = cnt;
    for (int bit = 63; bit >= 0 && reach > kLpRanked; --bit) {
        const uint64_t c = t | 1ull << bit;
        int n = 0;
#pragma unroll
        for (int j = 0; j < kLpList / kLpThreads; ++j) n += own[j] >= c;
        n = (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
        __syncthreads();
        if (lane == 0) sh.above[wid] = n;
        __syncthreads();
        n = 0;
#pragma unroll
        for (int w = 0; w < kLpWarps; ++w) n += sh.above[w];
        if (n >= k) { t = c; reach = n; }
    }
    __syncthreads();
    if (tid == 0) sh.count = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kLpList / kLpThreads; ++j)
        if (own[j] && own[j] >= t) sh.list[atomicAdd(&sh.count, 1)] = own[j];
    __syncthreads();
    cnt = sh.count;
    return t;
}

// The k largest of a row into sh.list, by walking it; cnt: how many came into the list, k at least.
template <int TYPE>
__device__ __noinline__ void lp_walk(LpShared& sh, const char* row, int64_t V, int k, int& cnt) {
    constexpr int kEach = 4, kChunk = kEach * kLpThreads;
    static_assert(kLpRanked + kChunk <= kLpList, "a chunk has to fit beside a cut list");
    const int tid = threadIdx.x;
    uint64_t least = 0;
    __syncthreads();
    if (tid == 0) sh.count = 0;
    __syncthreads();
    for (int64_t i0 = 0; i0 < V; i0 += kChunk) {
        float v[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int64_t i = i0 + j * kLpThreads + tid;
            v[j] = i < V ? load_logit<TYPE>(row, i) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int64_t i = i0 + j * kLpThreads + tid;
            const uint64_t e = lp_entry(v[j], i);
            if (i < V && e >= least) sh.list[atomicAdd(&sh.count, 1)] = e;
        }
        __syncthreads();
        cnt = sh.count;
        __syncthreads();
        if (cnt > kLpRanked) least = lp_cut(sh, cnt, k);
    }
}

template <int TYPE>
__global__ void __launch_bounds__(kLpThreads, 4) k_vocab_logprob(const LogprobCall c) {
    constexpr int kVec = TYPE == GK_TYPE_F32 ? 4 : 8, kSize = TYPE == GK_TYPE_F32 ? 4 : 2;
    __shared__ LpShared sh;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int64_t r = blockIdx.x, V = c.V;
    const char* row = c.logits + r * c.ld * kSize;
    // the given tokens
    const int64_t t = tid < c.m ? c.token[r * c.m + tid] : -1;
    const bool mine = t >= 0 && t < V;
    if (c.m > 0 && !__syncthreads_or(mine)) {
        if (tid < c.m && c.logp) c.logp[r * c.m + tid] = 0.f;
        if (tid == 0) {
            if (c.rank) c.rank[r] = -1;
            if (c.entropy) c.entropy[r] = 0.f;
            if (c.lse) c.lse[r] = 0.f;
        }
        if (tid < c.k) { c.idx[r * c.k + tid] = -1; c.val[r * c.k + tid] = 0.f; }
        return;
    }
    const float own = mine ? load_logit<TYPE>(row, t) : 0.f;
    if (tid == 0) {
        sh.count = 0;
        sh.first = own;
        sh.any = mine ? (int)t : -1;
    }
    // elements before the first 16-byte boundary, whole words, the rest
    int64_t head = (16 - ((uintptr_t)row & 15)) % 16 / kSize;
    if (head > V) head = V;
    const int words = (int)((V - head) / kVec);
    const int64_t rest = V - head - (int64_t)words * kVec;
    const uint4* body = (const uint4*)(row + head * kSize);
    // four words a thread at a time, from four places of the row
    const int steps = (words + kLpThreads - 1) / kLpThreads, quarter = (steps + 3) / 4;
    uint4 x[4];
    auto fetch = [&](int q) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int w = (q + i * quarter) * kLpThreads + tid;
            if (q + i * quarter < steps && w < words) x[i] = __ldcs(body + w);
        }
    };
    fetch(0);
    auto each = [&](int q, auto&& use) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int w = (q + i * quarter) * kLpThreads + tid;
            if (q + i * quarter < steps && w < words) use(x[i], w);
        }
    };
    // the first words are the sample: their maximum is where the sums start
    float top = -INFINITY;
    each(0, [&](const uint4& y, int) {
        float f[kVec];
        unpack<TYPE>(y, f);
#pragma unroll
        for (int e = 0; e < kVec; ++e) top = fmaxf(top, f[e]);
    });
    sh.sample[tid] = top;
    __syncthreads();
    const int first = sh.any;
    const float first_v = sh.first;
    float tau = INFINITY;
    if (c.k > 0) {
        // with e of the k largest expected in the sample, the (e + 4 sqrt(e) + 4)-th largest of the threads' maxima is
        // hardly among the row's k largest; where the sample is the row, the k + 1-th
        const float e = (float)c.k * fminf(1.f, 4.f * kLpThreads * kVec / (float)V);
        const int want = min(c.k + 1, (int)(e + 4.f * sqrtf(e) + 4.f));
        int above = 0, equal = 0;
        for (int j = 0; j < kLpThreads; ++j) {
            above += sh.sample[j] > top;
            equal += sh.sample[j] == top;
        }
        static_assert(kLogprobMaxAlternatives < kLpThreads, "the threshold is one of the threads' maxima");
        if (above < want && above + equal >= want) sh.tau = top;      // all who write write the same
        __syncthreads();
        tau = sh.tau;
    }
    Sums a = {top, 0.f, 0.f};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(0xffffffffu, a.m, o));
    float ref = lp_ref(a.m);
    uint64_t s0 = pair(0.f, 0.f), s1 = pair(0.f, 0.f);
    const uint64_t zscale2 = pair(c.zscale, c.zscale);
    int rank = 0;
    auto raise = [&](float to) {
        const float d = lp_shift(a.m, to, c.zscale), by = exp2_fast(d);
        const uint64_t by2 = pair(by, by);
        s1 = mul2(fma2(s0, pair(d, d), s1), by2);
        s0 = mul2(s0, by2);
        a.m = to;
        ref = lp_ref(to);
    };
    auto append = [&](float v, int64_t i) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < kLpList) sh.list[at] = lp_entry(v, i);
    };
    auto single = [&](int64_t i) {
        const float v = load_logit<TYPE>(row, i);
        if (v > a.m) raise(v);
        if (v > tau) append(v, i);
        if (first >= 0) rank += v > first_v || (v == first_v && i < first);
        const float d = max_nan((v - ref) * c.zscale, kLpFloor), e = exp2_fast(d);
        s0 = add2(s0, pair(e, 0.f));
        s1 = add2(s1, pair(e * d, 0.f));
    };
    auto word = [&](const uint4& y, int w) {
        float f[kVec];
        unpack<TYPE>(y, f);
        float g;
        if constexpr (kVec == 8) {
            g = max3(f[0], f[1], f[2]);
            g = max3(g, f[3], f[4]);
            g = fmaxf(max3(g, f[5], f[6]), f[7]);
        } else {
            g = fmaxf(max3(f[0], f[1], f[2]), f[3]);
        }
        if (g > a.m) raise(g);
        const int64_t i0 = head + (int64_t)w * kVec;
        if (g > tau) {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (f[e] > tau) append(f[e], i0 + e);
        }
        if (first >= 0 && g >= first_v) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) rank += f[e] > first_v || (f[e] == first_v && i0 + e < first);
        }
        const uint64_t less = pair(-ref, -ref);
#pragma unroll
        for (int e = 0; e < kVec; e += 2) {
            float d0, d1;
            unpair(mul2(add2(pair(f[e], f[e + 1]), less), zscale2), d0, d1);
            d0 = max_nan(d0, kLpFloor);
            d1 = max_nan(d1, kLpFloor);
            const uint64_t p = pair(exp2_fast(d0), exp2_fast(d1));
            s0 = add2(s0, p);
            s1 = fma2(p, pair(d0, d1), s1);
        }
    };
    if (tid < head) single(tid);
    if (tid < rest) single(V - rest + tid);
    for (int q = 0; q < quarter; ++q) {
        if (q > 0) fetch(q);
        each(q, word);
    }
    {
        float lo, hi;
        unpair(s0, lo, hi);
        a.s0 = lo + hi;
        unpair(s1, lo, hi);
        a.s1 = lo + hi;
    }
    // the row's sums
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Sums b;
        b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
        b.s0 = __shfl_xor_sync(0xffffffffu, a.s0, o);
        b.s1 = __shfl_xor_sync(0xffffffffu, a.s1, o);
        lp_join(a, b, c.zscale);
    }
    rank = (int)__reduce_add_sync(0xffffffffu, (unsigned)rank);
    if (lane == 0) {
        sh.m[wid] = a.m;
        sh.s0[wid] = a.s0;
        sh.s1[wid] = a.s1;
        sh.above[wid] = rank;
    }
    __syncthreads();
    a = {sh.m[0], sh.s0[0], sh.s1[0]};
    rank = sh.above[0];
#pragma unroll
    for (int w = 1; w < kLpWarps; ++w) {
        const Sums b = {sh.m[w], sh.s0[w], sh.s1[w]};
        lp_join(a, b, c.zscale);
        rank += sh.above[w];
    }
    const bool nan = a.s0 != a.s0, inf = a.m == INFINITY, none = a.m == -INFINITY && !nan;
    const float log_s0 = logf(a.s0);
    // the log probability of a logit
    auto logp_of = [&](float v) { return none ? -INFINITY : nan ? NAN : inf ? (v < INFINITY ? -INFINITY : NAN) : (v - a.m) / c.T - log_s0; };
    if (tid < c.m && c.logp) c.logp[r * c.m + tid] = mine ? logp_of(own) : 0.f;
    if (nan && c.rank && first >= 0) {
        // in the order that puts NaN above +inf
        const uint64_t mark = lp_entry(first_v, first);
        rank = 0;
        for (int64_t i = tid; i < V; i += kLpThreads) rank += lp_entry(load_logit<TYPE>(row, i), i) > mark;
        rank = (int)__reduce_add_sync(0xffffffffu, (unsigned)rank);
        __syncthreads();
        if (lane == 0) sh.above[wid] = rank;
        __syncthreads();
        rank = 0;
#pragma unroll
        for (int w = 0; w < kLpWarps; ++w) rank += sh.above[w];
    }
    if (tid == 0) {
        if (c.rank) c.rank[r] = first >= 0 ? rank : -1;
        if (c.entropy) c.entropy[r] = none ? 0.f : nan || inf ? NAN : log_s0 - 0.69314718f * (a.s1 / a.s0);
        if (c.lse) c.lse[r] = none ? -INFINITY : nan ? NAN : inf ? INFINITY : a.m / c.T + log_s0;
    }
    if (c.k == 0) return;
    // the alternatives
    int cnt = sh.count;
    __syncthreads();
    if (!nan && cnt < c.k) {
        // the first elements that equal the threshold
        for (int64_t i0 = 0; i0 < V && cnt < c.k; i0 += kLpThreads) {
            const int64_t i = i0 + tid;
            const float v = i < V ? load_logit<TYPE>(row, i) : 0.f;
            const bool is = i < V && v == tau;
            const unsigned ballot = __ballot_sync(0xffffffffu, is);
            __syncthreads();
            if (lane == 0) sh.above[wid] = __popc(ballot);
            __syncthreads();
            int at = cnt + __popc(ballot & ((1u << lane) - 1u));
#pragma unroll
            for (int w = 0; w < kLpWarps; ++w) {
                at += w < wid ? sh.above[w] : 0;
                cnt += sh.above[w];
            }
            if (is && at < c.k) sh.list[at] = lp_entry(v, i);
        }
        cnt = min(cnt, c.k);
        __syncthreads();
    }
    if (nan || cnt < c.k || cnt > kLpList) lp_walk<TYPE>(sh, row, V, c.k, cnt);
    if (cnt > kLpRanked) lp_cut(sh, cnt, c.k);
    // the place of each is how many are above it
    for (int j = tid; j < cnt; j += kLpThreads) {
        const uint64_t e = sh.list[j];
        int place = 0;
        for (int i = 0; i < cnt; ++i) place += sh.list[i] > e;
        if (place < c.k) sh.best[place] = e;
    }
    __syncthreads();
    if (tid < c.k) {
        const uint64_t e = sh.best[tid];
        const int i = (int)~(uint32_t)e;
        c.idx[r * c.k + tid] = i;
        c.val[r * c.k + tid] = logp_of(load_logit<TYPE>(row, i));
    }
}

struct LogprobGradCall {
    const char* logits;
    char* dz;
    int64_t ld, lddz, n, V;
    const int64_t* token;
    int m, pieces;
    float inv_T, inv_T_low;      // 1 / T in two parts
    const float* lse;
    const float* entropy;
    const float* a;
    const float* b;
    const float* c;
};

// A CTA a piece of a row of at most kWords words a thread, the logits read and their gradients written once.
//     dz = p (k0 + k1 log p),  k0 = (c - sum a - b entropy) / T,  k1 = -b / T,
// and a / T more at a token, which the CTA that has it writes again at the end.
template <int TYPE>
__global__ void __launch_bounds__(kLpThreads, 4) k_vocab_logprob_grad(const LogprobGradCall c) {
    constexpr int kVec = TYPE == GK_TYPE_F32 ? 4 : 8, kSize = TYPE == GK_TYPE_F32 ? 4 : 2, kWords = 4;
    __shared__ int64_t tokens[kLogprobMaxTokens];
    const int tid = threadIdx.x, lane = tid & 31;
    const int64_t V = c.V;
    for (int64_t job = blockIdx.x; job < c.n * c.pieces; job += gridDim.x) {
        const int64_t r = job / c.pieces;
        const int piece = (int)(job - r * c.pieces);
        const char* row = c.logits + r * c.ld * kSize;
        char* out = c.dz + r * c.lddz * kSize;
        // the piece's elements [v0, v1); words where both rows have the same 16-byte boundaries
        const bool apart = (((uintptr_t)row ^ (uintptr_t)out) & 15) != 0;
        int64_t head = (16 - ((uintptr_t)row & 15)) % 16 / kSize;
        if (head > V) head = V;
        const int64_t words = (V - head) / kVec;
        const int64_t w0 = words * piece / c.pieces, w1 = words * (piece + 1) / c.pieces;
        const int64_t v0 = piece == 0 ? 0 : head + w0 * kVec, v1 = piece == c.pieces - 1 ? V : head + w1 * kVec;
        uint4 x[kWords];
        if (!apart) {
#pragma unroll
            for (int j = 0; j < kWords; ++j)
                if (w0 + j * kLpThreads + tid < w1) x[j] = __ldcs((const uint4*)(row + head * kSize) + w0 + j * kLpThreads + tid);
        }
        const float lse = c.lse[r], b = c.b ? c.b[r] : 0.f;
        float k0 = c.c ? c.c[r] : 0.f;
        bool counts = c.m == 0, here = false;
        float sum = 0.f;
        for (int j0 = 0; j0 < c.m; j0 += 32) {
            const int64_t t = j0 + lane < c.m ? c.token[r * c.m + j0 + lane] : -1;
            const bool valid = t >= 0 && t < V;
            counts |= __any_sync(0xffffffffu, valid);
            here |= __any_sync(0xffffffffu, valid && t >= v0 && t < v1);
            if (valid && c.a) sum += c.a[r * c.m + j0 + lane];
            if (tid < 32 && j0 + lane < c.m) tokens[j0 + lane] = t;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        counts = counts && !(lse < -1e30f);      // else nothing is left, or masks of a type's lowest value alone
        k0 = (k0 - sum - (c.b ? b * c.entropy[r] : 0.f)) * c.inv_T;
        const float k1 = -b * c.inv_T;
        auto plain = [&](const char* p, int64_t i) {
            if constexpr (TYPE == GK_TYPE_F32) return ((const float*)p)[i];
            else return from16<TYPE == GK_TYPE_F16>(((const uint16_t*)p)[i]);
        };
        auto store = [&](int64_t i, float v) {
            if constexpr (TYPE == GK_TYPE_F32) ((float*)out)[i] = v;
            else ((uint16_t*)out)[i] = to16<TYPE == GK_TYPE_F16>(v);
        };
        // (a logit of -inf has a finite stand-in, and so has its log probability: both go into products with zero)
        auto grad = [&](float z) {
            z = max_nan(z, -3.402823466e38f);
            const float y = max_nan(fmaf(z, c.inv_T_low, fmaf(z, c.inv_T, -lse)), -1e30f);
            return counts ? exp2_fast(y * 1.44269504f) * fmaf(k1, y, k0) : 0.f;
        };
        here = here && counts && c.a;
        // a token's gradients are added up by the first of the threads that have it
        float at_token = 0.f;
        int64_t t = -1;
        if (here) {
            __syncthreads();
            if (tid < c.m) {
                t = tokens[tid];
                for (int j = 0; j < tid; ++j)
                    if (tokens[j] == t) t = -1;
                if (t < v0 || t >= v1) t = -1;
                if (t >= 0) {
                    float more = 0.f;
                    for (int j = tid; j < c.m; ++j)
                        if (tokens[j] == t) more += c.a[r * c.m + j];
                    at_token = fmaf(more, c.inv_T, grad(plain(row, t)));
                }
            }
            __syncthreads();      // read before it is written over, where dlogits are the logits
        }
        if (apart) {
            for (int64_t i = v0 + tid; i < v1; i += kLpThreads) store(i, grad(plain(row, i)));
        } else {
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
                if (w0 + j * kLpThreads + tid >= w1) break;
                float f[kVec];
                unpack<TYPE>(x[j], f);
#pragma unroll
                for (int e = 0; e < kVec; ++e) f[e] = grad(f[e]);
                uint4 y;
                if constexpr (TYPE == GK_TYPE_F32) {
                    y = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                } else {
                    constexpr bool F16 = TYPE == GK_TYPE_F16;
                    y = make_uint4(pack16<F16>(f[0], f[1]), pack16<F16>(f[2], f[3]), pack16<F16>(f[4], f[5]), pack16<F16>(f[6], f[7]));
                }
                __stcs((uint4*)(out + head * kSize) + w0 + j * kLpThreads + tid, y);
            }
            if (piece == 0 && tid < head) store(tid, grad(plain(row, tid)));
            const int64_t rest = V - head - words * kVec;
            if (piece == c.pieces - 1 && tid < rest) store(V - rest + tid, grad(plain(row, V - rest + tid)));
        }
        if (here) {
            __syncthreads();
            if (t >= 0) store(t, at_token);
            __syncthreads();
        }
    }
}

}  // namespace gk

using namespace gk;

static int check_rows(const void* logits, int64_t ld, int32_t dtype, int64_t n, int64_t V, const int64_t* token, int32_t m, float T) {
    if (n < 0 || V < 1 || V > 2147483647ll || m < 0) return GK_ERR_SIZE;
    if (n > 2147483647ll || m > kLogprobMaxTokens) return GK_ERR_LIMIT;
    if (dtype != GK_TYPE_F32 && dtype != GK_TYPE_BF16 && dtype != GK_TYPE_F16) return GK_ERR_TYPE;
    if (n > 0 && (!logits || (m > 0 && !token))) return GK_ERR_NULL;
    if (ld < V) return GK_ERR_STRIDE;
    if (((uintptr_t)logits & (dtype == GK_TYPE_F32 ? 3 : 1)) != 0) return GK_ERR_ALIGN;
    return temperature_ok(T) ? GK_OK : GK_ERR_TEMPERATURE;
}

extern "C" int gk_vocab_logprob(const void* logits, int64_t ld, int32_t dtype, int64_t n, int64_t V, const int64_t* token,
                                int32_t m, float temperature, int32_t k, float* logp_out, int32_t* rank_out,
                                float* entropy_out, float* lse_out, int32_t* idx_out, float* val_out, gk_stream_t stream) {
    const int rc = check_rows(logits, ld, dtype, n, V, token, m, temperature);
    if (rc != GK_OK) return rc;
    if (k < 0 || k > V || k > kLogprobMaxAlternatives) return GK_ERR_K;
    if (n > 0 && k > 0 && (!idx_out || !val_out)) return GK_ERR_NULL;
    if (n == 0) return GK_OK;
    const LogprobCall c = {(const char*)logits, ld, n, V, token, m, k, temperature, (float)(1.4426950408889634 / (double)temperature),
                           logp_out, rank_out, entropy_out, lse_out, idx_out, val_out};
    cudaStream_t st = (cudaStream_t)stream;
    switch (dtype) {
        case GK_TYPE_F32: k_vocab_logprob<GK_TYPE_F32><<<(unsigned)n, kLpThreads, 0, st>>>(c); break;
        case GK_TYPE_BF16: k_vocab_logprob<GK_TYPE_BF16><<<(unsigned)n, kLpThreads, 0, st>>>(c); break;
        default: k_vocab_logprob<GK_TYPE_F16><<<(unsigned)n, kLpThreads, 0, st>>>(c); break;
    }
    GK_CUDA_TRY(cudaGetLastError());
    note_launch();
    return GK_OK;
}

extern "C" int gk_vocab_logprob_grad(const void* logits, int64_t ld, int32_t dtype, int64_t n, int64_t V, const int64_t* token,
                                     int32_t m, float temperature, const float* lse, const float* entropy, const float* logp_grad,
                                     const float* entropy_grad, const float* lse_grad, void* dlogits, int64_t lddz,
                                     gk_stream_t stream) {
    const int rc = check_rows(logits, ld, dtype, n, V, token, m, temperature);
    if (rc != GK_OK) return rc;
    if (n > 0 && (!lse || !dlogits || (entropy_grad && !entropy))) return GK_ERR_NULL;
    if (lddz < V) return GK_ERR_STRIDE;
    const int64_t size = dtype == GK_TYPE_F32 ? 4 : 2;
    if (((uintptr_t)dlogits & (size - 1)) != 0) return GK_ERR_ALIGN;
    if (n == 0) return GK_OK;
    const uintptr_t z0 = (uintptr_t)logits, z1 = z0 + ((n - 1) * ld + V) * size, d0 = (uintptr_t)dlogits, d1 = d0 + ((n - 1) * lddz + V) * size;
    if (z0 < d1 && d0 < z1 && (z0 != d0 || (ld != lddz && n > 1))) return GK_ERR_ALIAS;
    const int64_t words = V / (16 / size);
    const double inv_T = 1.0 / (double)temperature;
    const int64_t pieces = words <= 4 * kLpThreads ? 1 : (words + 4 * kLpThreads - 1) / (4 * kLpThreads);
    const LogprobGradCall c = {(const char*)logits, (char*)dlogits, ld, lddz, n, V, token, m, (int)pieces, (float)inv_T,
                               (float)(inv_T - (double)(float)inv_T), lse, entropy, logp_grad, entropy_grad, lse_grad};
    const int64_t jobs = n * pieces;
    const unsigned grid = (unsigned)(jobs < (1 << 30) ? jobs : 1 << 30);
    cudaStream_t st = (cudaStream_t)stream;
    switch (dtype) {
        case GK_TYPE_F32: k_vocab_logprob_grad<GK_TYPE_F32><<<grid, kLpThreads, 0, st>>>(c); break;
        case GK_TYPE_BF16: k_vocab_logprob_grad<GK_TYPE_BF16><<<grid, kLpThreads, 0, st>>>(c); break;
        default: k_vocab_logprob_grad<GK_TYPE_F16><<<grid, kLpThreads, 0, st>>>(c); break;
    }
    GK_CUDA_TRY(cudaGetLastError());
    note_launch();
    return GK_OK;
}
