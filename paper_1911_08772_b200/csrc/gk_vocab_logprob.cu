// Log probabilities of given tokens with entropy, rank and the most probable tokens, and their gradient
// (include/gk.h: gk_vocab_logprob, gk_vocab_logprob_grad).
//
// Forward: one pass over a row, by a CTA or, where there are few rows, by the CTAs of a cluster.  With m about the row's
// maximum and d = (z - m) / T in units of log 2, threads sum S0 = 2^d and S1 = d 2^d; a larger m by b rescales S0 by
// 2^-b and S1 to 2^-b (S1 - b S0).  At the end, with the maximum itself,
//     lse = m / T + log S0,   entropy = log S0 - log(2) S1 / S0,
// two terms of one sign, so that a small entropy keeps its digits.  The rank counts the elements before the token that
// are not below it, and those behind it that are above.
//
// Alternatives: a threshold from a sample of the row, which a little more than k elements are expected to be above.
// Words that have some are noted; their elements are listed, and the place of each among them is counted, which sorts
// them.  Where fewer than k are above, the first elements equal to the threshold fill the list (rows whose mask leaves
// little); where that is not enough either, or the list is too short, the row is walked again in chunks, from a bound
// that the list gives, and the list cut whenever it is full.
#include <atomic>

#include "gk_words.cuh"

namespace gk {

constexpr int kLogprobMaxTokens = 128, kLogprobMaxAlternatives = 128;
constexpr float kLpFloor = -200.f;  // powers of two below this are zero in fp32, and their products with it too
constexpr int kLpQuad = 4;          // words a thread fetches together, from four places: the first are a sample of the row
constexpr int kLpParts = 8;         // CTAs a row at most (a cluster)
constexpr int kLpShort = 1500, kLpMiddle = 6000;      // words of a row that 64 threads take, and 128
constexpr float kLpSlack = 4.f;     // how far a logit may be above what the sums are relative to, in powers of two
// Exponents of rows' maxima up to this are kept to a sixteenth and better by one rounding; so are those down to twice
// its negative, the lowest that sums start from.
constexpr float kLpLargest = 1048576.f;

struct LogprobCall {
    const char* logits;
    int64_t ld, n, V;
    const int64_t* token;
    int m, k, parts;
    float inv_T, inv_T_low, zscale;      // 1 / T in two parts, log2(e) / T
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
// A value as a threshold for a word's elements, and the next smaller one: in both halves of a word for 16-bit types.
template <int TYPE>
__device__ __forceinline__ unsigned threshold_of(float v, bool below) {
    unsigned b = TYPE == GK_TYPE_F32 ? __float_as_uint(v) : to16<TYPE == GK_TYPE_F16>(v);
    const unsigned sign = TYPE == GK_TYPE_F32 ? 0x80000000u : 0x8000u;
    if (below) b = (b & ~sign) == 0 ? sign + 1u : b & sign ? b + 1u : b - 1u;
    return TYPE == GK_TYPE_F32 ? b : b << 16 | b;
}
// On the two halves of a word of 16-bit elements: all ones for above a threshold, maxima without regard to NaN, and
// with.
#define GK_HALVES(NAME, F16_OP, BF16_OP)                                                            \
    template <int TYPE>                                                                             \
    __device__ __forceinline__ unsigned NAME(unsigned a, unsigned b) {                              \
        unsigned r;                                                                                 \
        if constexpr (TYPE == GK_TYPE_F16) asm(F16_OP " %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));   \
        else asm(BF16_OP " %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));                                \
        return r;                                                                                   \
    }
GK_HALVES(above2, "set.gt.u32.f16x2", "set.gt.u32.bf16x2")
GK_HALVES(max2, "max.f16x2", "max.bf16x2")
GK_HALVES(max2_nan, "max.NaN.f16x2", "max.NaN.bf16x2")
#undef GK_HALVES
template <int TYPE>
__device__ __forceinline__ unsigned above(unsigned a, unsigned threshold) {
    if constexpr (TYPE == GK_TYPE_F32) {
        unsigned r;
        asm("set.gt.u32.f32 %0, %1, %2;" : "=r"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(threshold)));
        return r;
    } else {
        return above2<TYPE>(a, threshold);
    }
}
template <int TYPE>
__device__ __forceinline__ uint4 max2(const uint4& a, const uint4& b) {
    return make_uint4(max2<TYPE>(a.x, b.x), max2<TYPE>(a.y, b.y), max2<TYPE>(a.z, b.z), max2<TYPE>(a.w, b.w));
}
template <int TYPE>
__device__ __forceinline__ float max_of(const uint4& y) {      // a word's largest element, -inf for nothing but NaN
    if constexpr (TYPE == GK_TYPE_F32) {
        return fmaxf(max3(__uint_as_float(y.x), __uint_as_float(y.y), __uint_as_float(y.z)), fmaxf(__uint_as_float(y.w), -INFINITY));
    } else {
        const unsigned g = max2<TYPE>(max2<TYPE>(y.x, y.y), max2<TYPE>(y.z, y.w));
        return max3(from16<TYPE == GK_TYPE_F16>((uint16_t)g), from16<TYPE == GK_TYPE_F16>((uint16_t)(g >> 16)), -INFINITY);
    }
}
template <int TYPE>
__device__ __forceinline__ float max_of(const uint4 (&x)[kLpQuad]) {
    if constexpr (TYPE == GK_TYPE_F32) return fmaxf(max3(max_of<TYPE>(x[0]), max_of<TYPE>(x[1]), max_of<TYPE>(x[2])), max_of<TYPE>(x[3]));
    else return max_of<TYPE>(max2<TYPE>(max2<TYPE>(x[0], x[1]), max2<TYPE>(x[2], x[3])));
}
// What the sums take for anything lower, -inf among it: far enough below any maximum, or the row is taken again.  (A
// value of the type: -2^100 for fp32 and bf16.)
template <int TYPE>
constexpr float kLpLowest = TYPE == GK_TYPE_F16 ? -65504.f : -1267650600228229401496703205376.f;

// Maximum (as it is in the logits) and the two sums relative to it.
struct Sums {
    float m, s0, s1;
};
__device__ __forceinline__ float lp_ref(float m) { return m == -INFINITY ? 0.f : fminf(m, 3.402823466e38f); }
// Half of v - ref: within fp32 where the difference is not (a mask of the lowest value under logits of 1e31 and more).
__device__ __forceinline__ float lp_half(float v, float ref) { return fmaf(v, 0.5f, -0.5f * ref); }
// (v - ref) zscale, and kLpFloor at least.
__device__ __forceinline__ float lp_apart(float v, float ref, float zscale) { return 2.f * max_nan(lp_half(v, ref) * zscale, 0.5f * kLpFloor); }
// What sums relative to m are multiplied by to be relative to `to` >= m, as a power of two: nothing for +inf beside
// itself, the floor for -inf, whose sums are nothing.
__device__ __forceinline__ float lp_shift(float m, float to, float zscale) { return fminf(lp_apart(m, lp_ref(to), zscale), 0.f); }
__device__ __forceinline__ void lp_join(Sums& a, const Sums& b, float zscale) {
    const float top = fmaxf(a.m, b.m), da = lp_shift(a.m, top, zscale), db = lp_shift(b.m, top, zscale);
    const float ea = exp2_fast(da), eb = exp2_fast(db);      // one where the shift is nothing
    a.s1 = ea * fmaf(a.s0, da, a.s1) + eb * fmaf(b.s0, db, b.s1);
    a.s0 = ea * a.s0 + eb * b.s0;
    a.m = top;
}

// Barrier of a cluster's CTAs, and a value in the shared memory of one of them.
__device__ __forceinline__ void lp_cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
template <class T>
__device__ __forceinline__ T remote(const T& here, int cta) {
    uint64_t p;
    asm volatile("mapa.u64 %0, %1, %2;" : "=l"(p) : "l"(&here), "r"(cta));
    return *reinterpret_cast<const volatile T*>(p);
}

template <int NT>
struct LpShared {
    static constexpr int kCtas = 1024 / NT;                     // CTAs an SM
    static constexpr int kList = NT == 256 ? 1280 : NT == 128 ? 1024 : 512;      // entries of the list of alternatives
    static constexpr int kNotes = kList, kNoted = kList / 5 * 2;                 // words noted for it, the first with their contents
    static constexpr int kPlaced = NT == 64 ? 128 : 256;        // entries sorted by counting; a longer list is cut first
    static_assert(NT != 256 || kNoted * sizeof(uint4) >= kLpParts * kLogprobMaxAlternatives * sizeof(uint64_t), "all CTAs' alternatives");
    alignas(16) uint64_t list[kList];      // key of the value above, complement of the index below: all differ
    uint4 data[kNoted];                    // (before that the sample; SPLIT: at last all CTAs' alternatives)
    int note[kNotes];
    uint64_t best[kLogprobMaxAlternatives];      // SPLIT: this CTA's
    Sums sums[8];
    int above[8];
    int scratch[2][8];
    int notes, listed;      // (may exceed their lists)
    float tau;
    // what the other CTAs of a row read
    Sums part;
    int part_above;
};
__device__ __forceinline__ uint64_t lp_entry(float v, int64_t i) { return (uint64_t)order_key(v) << 32 | (uint32_t)~(uint32_t)i; }

// How many of all threads' n there are; `turn` alternates from call to call.
template <int NT>
__device__ __forceinline__ int lp_count(LpShared<NT>& sh, int n, int turn) {
    n = (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
    const int lane = threadIdx.x & 31;
    if (lane == 0) sh.scratch[turn & 1][threadIdx.x >> 5] = n;
    __syncthreads();
    return (int)__reduce_add_sync(0xffffffffu, lane < NT / 32 ? (unsigned)sh.scratch[turn & 1][lane] : 0u);
}
// The same, and how many of them are before this thread's (which is one or none).
template <int NT>
__device__ __forceinline__ int lp_count_before(LpShared<NT>& sh, bool on, int turn, int& before) {
    const unsigned ballot = __ballot_sync(0xffffffffu, on);
    const int all = lp_count(sh, on, turn);
    before = __popc(ballot & ((1u << (threadIdx.x & 31)) - 1u));
    for (int w = 0; w < (int)threadIdx.x / 32; ++w) before += sh.scratch[turn & 1][w];
    return all;
}

// The bit that a search for a bound starts with, all keys lying between lo and hi, and the bits above it.
__device__ __forceinline__ int lp_first_bit(unsigned lo, unsigned hi, uint64_t& t) {
    const unsigned differ = lo ^ hi;
    const int bit = differ ? 63 - __clz(differ) : 31;
    t = bit == 63 ? 0 : ((uint64_t)lo << 32) >> (bit + 1) << (bit + 1);
    return bit;
}

// The list of `cnt` entries, of keys between lo and hi, cut to between k and `most` >= k of the largest; returns a
// bound that all kept reach and no other.  All threads see `cnt` alike.
template <int NT>
__device__ __noinline__ uint64_t lp_cut(LpShared<NT>& sh, int& cnt, int k, int most, unsigned lo, unsigned hi) {
    const int tid = (int)threadIdx.x;
    uint64_t t;
    __syncthreads();
    int reach = cnt, turn = 0;
    for (int bit = lp_first_bit(lo, hi, t); bit >= 0 && reach > most; --bit) {
        const uint64_t c = t | 1ull << bit;
        int n = 0;
#pragma unroll 4
        for (int j = tid; j < cnt; j += NT) n += sh.list[j] >= c;
        n = lp_count(sh, n, turn++);
        if (n >= k) { t = c; reach = n; }
    }
    __syncthreads();
    // those that reach it to the front, behind what has been read
    int at = 0;
    for (int j0 = 0; j0 < cnt; j0 += NT) {
        const int j = j0 + tid;
        const uint64_t e = j < cnt ? sh.list[j] : 0;
        const bool on = j < cnt && e >= t;
        int before;
        const int all = lp_count_before(sh, on, turn++, before);
        if (on) sh.list[at + before] = e;
        at += all;
        __syncthreads();
    }
    cnt = at;
    return t;
}

// The k largest of the elements [v0, v1) of a row (all of them if they are fewer) into sh.list, by walking them; cnt:
// how many came into the list, k at least.  At least k elements reach `least`.  Eight elements a thread at a time where
// those that reach it fit the list; else one, and the list is cut when it is full.
template <int TYPE, int NT>
__device__ __noinline__ void lp_walk(LpShared<NT>& sh, const char* row, int64_t v0, int64_t v1, int k, uint64_t least, int& cnt) {
    constexpr int kList = LpShared<NT>::kList, kKept = kList - NT, kEach = 8;
    static_assert(kKept >= kLogprobMaxAlternatives, "a cut list holds all that are asked for");
    const int tid = (int)threadIdx.x;
    int turn = 0;
    cnt = 0;
    float next[kEach];
    auto fetch = [&](int64_t i0) {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (i0 + j * NT + tid < v1) next[j] = load_logit<TYPE>(row, i0 + j * NT + tid);
    };
    fetch(v0);
    __syncthreads();
    for (int64_t i0 = v0; i0 < v1; i0 += kEach * NT) {
        uint64_t e[kEach];
        int n = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int64_t i = i0 + j * NT + tid;
            e[j] = i < v1 ? lp_entry(next[j], i) : 0;
            n += i < v1 && e[j] >= least;
        }
        fetch(i0 + kEach * NT);
        n = lp_count(sh, n, turn++);
        if (n == 0) continue;
        const bool fits = cnt + n <= kList;
#pragma unroll 1
        for (int j = 0; j < kEach; ++j) {
            uint64_t own = e[0];
#pragma unroll
            for (int i = 1; i < kEach; ++i) own = i == j ? e[i] : own;
            int before;
            const bool on = own != 0 && own >= least;
            const int all = lp_count_before(sh, on, turn++, before);
            if (on) sh.list[cnt + before] = own;
            cnt += all;
            if (!fits && cnt > kKept) least = lp_cut(sh, cnt, k, kKept, 0u, ~0u);
        }
        if (cnt > kKept) least = lp_cut(sh, cnt, k, kKept, 0u, ~0u);
    }
    __syncthreads();
}

// The first elements that equal v into the list behind its `cnt` entries, until it has k.
template <int TYPE, int NT>
__device__ __noinline__ void lp_fill(LpShared<NT>& sh, const char* row, int64_t v0, int64_t v1, float v, int k, int& cnt) {
    const int tid = (int)threadIdx.x;
    int turn = 0;
    __syncthreads();
    for (int64_t i0 = v0; i0 < v1 && cnt < k; i0 += NT) {
        const int64_t i = i0 + tid;
        const bool is = i < v1 && load_logit<TYPE>(row, i) == v;
        int before;
        const int all = lp_count_before(sh, is, turn++, before);
        if (is && cnt + before < k) sh.list[cnt + before] = lp_entry(v, i);
        cnt += all;
    }
    cnt = min(cnt, k);
    __syncthreads();
}

// Sums joined with those of the lane that is o across.
__device__ __forceinline__ void lp_join_across(Sums& a, int o, float zscale) {
    Sums b;
    b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
    b.s0 = __shfl_xor_sync(0xffffffffu, a.s0, o);
    b.s1 = __shfl_xor_sync(0xffffffffu, a.s1, o);
    lp_join(a, b, zscale);
}
// (a join's last bit depends on which comes first: all take the first lane's)
__device__ __forceinline__ void lp_first_lanes(Sums& a) {
    a.m = __shfl_sync(0xffffffffu, a.m, 0);
    a.s0 = __shfl_sync(0xffffffffu, a.s0, 0);
    a.s1 = __shfl_sync(0xffffffffu, a.s1, 0);
}
// W warps' sums, those of a warp's threads relative to the same maximum, joined in one order.
template <int W>
__device__ __forceinline__ Sums lp_join_warps(const Sums (&part)[8], float zscale) {
    Sums a = part[threadIdx.x & (W - 1)];
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) lp_join_across(a, o, zscale);
    lp_first_lanes(a);
    return a;
}
__device__ __forceinline__ void lp_join_lanes(Sums& a) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a.s0 += __shfl_xor_sync(0xffffffffu, a.s0, o);
        a.s1 += __shfl_xor_sync(0xffffffffu, a.s1, o);
    }
}

// The sums of the elements [v0, v1) once more, without the shortcuts of the pass: differences first, then the scale.
template <int TYPE, int NT>
__device__ __noinline__ Sums lp_again(LpShared<NT>& sh, const char* row, int64_t v0, int64_t v1, float m, float zscale) {
    Sums a = {m, 0.f, 0.f};
    const float ref = lp_ref(m);
#pragma unroll 4
    for (int64_t i = v0 + (int)threadIdx.x; i < v1; i += NT) {
        const float d = lp_apart(load_logit<TYPE>(row, i), ref, zscale), e = exp2_fast(d);
        a.s0 += e;
        a.s1 = fmaf(e, d, a.s1);
    }
    lp_join_lanes(a);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.sums[threadIdx.x >> 5] = a;
    __syncthreads();
    return lp_join_warps<NT / 32>(sh.sums, zscale);
}

// Elements [v0, v1) that come before element `first` in the order that puts NaN above +inf.
template <int TYPE, int NT>
__device__ __noinline__ int lp_rank_again(LpShared<NT>& sh, const char* row, int64_t v0, int64_t v1, float first_v, int first) {
    const uint64_t mark = lp_entry(first_v, first);
    int rank = 0;
    for (int64_t i = v0 + (int)threadIdx.x; i < v1; i += NT) rank += lp_entry(load_logit<TYPE>(row, i), i) > mark;
    __syncthreads();
    return lp_count(sh, rank, 0);
}

// A row's results from its sums.
struct LpResult {
    float m, log_s0, inv_T, inv_T_low;
    bool nan, inf, none;
    __device__ __forceinline__ LpResult(const LogprobCall& c, const Sums& a)
        : m(a.m), log_s0(logf(a.s0)), inv_T(c.inv_T), inv_T_low(c.inv_T_low), nan(a.s0 != a.s0), inf(a.m == INFINITY), none(a.m == -INFINITY && a.s0 == a.s0) {}
    // (where the product leaves fp32's range, one with the second part of 1 / T may too, with either sign)
    __device__ __forceinline__ float scaled(float d) const {
        const float product = d * inv_T;
        return fabsf(product) < INFINITY ? fmaf(d, inv_T, d * inv_T_low) : product;
    }
    __device__ __forceinline__ float logp(float v) const { return none ? -INFINITY : nan ? NAN : inf ? (v < INFINITY ? -INFINITY : NAN) : 2.f * scaled(lp_half(v, m)) - log_s0; }
    __device__ __forceinline__ float lse() const { return none ? -INFINITY : nan ? NAN : inf ? INFINITY : scaled(m) + log_s0; }
    __device__ __forceinline__ float entropy(const Sums& a) const { return none ? 0.f : nan || inf ? NAN : log_s0 - 0.69314718f * __fdividef(a.s1, a.s0); }
};

// SPLIT: the CTAs of a cluster share a row.  LISTS: with alternatives.
// A thread keeps two times four words on their way, 64 KB an SM: 4096 x 128000 bf16 in 207 to 222 us (5 TB/s; the stream
// alone, without exponentials and rank, 190).  No unit is full (57 % of the issue slots, at nine instructions a logit, 55 %
// of the exponentials' unit and of DRAM): waiting bounds it, with 29 warps an SM there.  Two words a take 264, three
// fetches of four 244; rows through rings in shared memory 231 to 300.  With alternatives a row's own work shows, some
// 1000 instructions a warp: k = 20 256 us, k = 100 335; 2000 x 50001 fp16 with k = 20 70.  Few rows are a chain of
// latencies: 1 x 50001 fp32, k = 20, 9 us (11 where each CTA joined the others' sums and alternatives one part after the
// other), k = 0 5.4.
template <int TYPE, int NT, bool SPLIT, bool LISTS>
__global__ void __launch_bounds__(NT, SPLIT ? 2 : LpShared<NT>::kCtas) k_vocab_logprob(const LogprobCall c) {
    using Shared = LpShared<NT>;
    constexpr int kVec = TYPE == GK_TYPE_F32 ? 4 : 8, kSize = TYPE == GK_TYPE_F32 ? 4 : 2, kWarps = NT / 32;
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int parts = SPLIT ? c.parts : 1, part = SPLIT ? (int)(blockIdx.x % (unsigned)parts) : 0;
    const int64_t r = SPLIT ? blockIdx.x / (unsigned)parts : blockIdx.x;
    const char* row = c.logits + r * c.ld * kSize;
    // this CTA's share of the row: elements before its words and behind them, whole words
    const int V = (int)c.V, edge = min((int)((16 - ((uintptr_t)row & 15)) % 16) / kSize, V), all_words = (V - edge) / kVec;
    const int first_of = SPLIT ? (int)((int64_t)all_words * part / parts) : 0, words = (SPLIT ? (int)((int64_t)all_words * (part + 1) / parts) : all_words) - first_of;
    const int before = part == 0 ? edge : 0, behind = part == parts - 1 ? V - edge - all_words * kVec : 0;
    const int head = edge + first_of * kVec, v0 = head - before, v1 = head + words * kVec + behind;
    const uint4* own = (const uint4*)(row + edge * kSize) + first_of + tid;
    const int quarter = (words + NT * kLpQuad - 1) / (NT * kLpQuad), step = quarter * NT;
    // words past the end are -inf, which adds to nothing
    constexpr unsigned kNone = TYPE == GK_TYPE_F32 ? 0xff800000u : TYPE == GK_TYPE_F16 ? 0xfc00fc00u : 0xff80ff80u;
    auto fetch = [&](uint4 (&to)[kLpQuad], int q) {
        if (q >= quarter) return;
        const int w = q * NT;
        if (w + (kLpQuad - 1) * step + NT <= words) {
#pragma unroll
            for (int i = 0; i < kLpQuad; ++i) to[i] = __ldcs(own + w + i * step);
        } else {
#pragma unroll
            for (int i = 0; i < kLpQuad; ++i)
                to[i] = w + i * step + tid < words ? __ldcs(own + w + i * step) : make_uint4(kNone, kNone, kNone, kNone);
        }
    };
    uint4 x[kLpQuad], y[kLpQuad];
    fetch(x, 0);
    fetch(y, 1);
    // the given tokens
    bool any = false;
    for (int j = tid; j < c.m; j += NT) {
        const int64_t t = c.token[r * c.m + j];
        any |= t >= 0 && t < V;
    }
    const bool odd = lane < 16 ? lane < before : lane - 16 < behind;      // a warp's elements outside the words
    const int odd_at = !odd ? 0 : lane < 16 ? v0 + lane : v1 - behind + (lane - 16);      // (no sum past 2^31 on the way)
    const float odd_v = odd ? load_logit<TYPE>(row, odd_at) : -INFINITY;
    if (tid == 0) sh.notes = sh.listed = 0;
    if (!__syncthreads_or(any) && c.m > 0) {
        if (part == 0) {
            for (int j = tid; j < c.m && c.logp; j += NT) c.logp[r * c.m + j] = 0.f;
            for (int j = tid; j < c.k; j += NT) { c.idx[r * c.k + j] = -1; c.val[r * c.k + j] = 0.f; }
            if (tid == 0) {
                if (c.rank) c.rank[r] = -1;
                if (c.entropy) c.entropy[r] = 0.f;
                if (c.lse) c.lse[r] = 0.f;
            }
        }
        return;
    }
    // the first one's logit, by all
    const int64_t t0 = c.m > 0 ? c.token[r * c.m] : -1;
    const int first = t0 >= 0 && t0 < V ? (int)t0 : -1;
    const float first_v = first >= 0 ? load_logit<TYPE>(row, first) : 0.f;

    // the first words are the sample: their maximum is where the sums start
    float top = quarter > 0 ? max_of<TYPE>(x) : -INFINITY;
    float tau = INFINITY;
    if constexpr (LISTS) {
        // With e of the k largest expected in the sample, the (e + 4 sqrt(e) + 4)-th largest of 64 groups' or all
        // threads' maxima is hardly among the row's k largest; where the sample is all there is, the k + 8-th leaves room
        // for equal ones.
        const float e = (float)c.k * fminf(1.f, (float)(kLpQuad * NT * kVec) / (float)(v1 - v0));
        const int want = min(min(c.k + 8, NT), (int)(e + 4.f * sqrtf(e) + 4.f));
        const int count = NT > 64 && want <= 32 ? 64 : NT;
        float* sample = reinterpret_cast<float*>(sh.data);
        float mine = top;
        if (NT > 64 && count == 64) {
#pragma unroll
            for (int o = 1; o < NT / 64; o *= 2) mine = fmaxf(mine, __shfl_xor_sync(0xffffffffu, mine, o));
            if (lane % (NT / 64) == 0) sample[tid / (NT / 64)] = mine;
        } else {
            sample[tid] = mine;
        }
        __syncthreads();
        if (tid < count) {
            mine = sample[tid];
            int n = 0, reach = 0;
#pragma unroll 4
            for (int j = 0; j < count; j += 4) {
                const float4 s = *(const float4*)&sample[j];
                n += (s.x > mine) + (s.y > mine) + (s.z > mine) + (s.w > mine);
                reach += (s.x >= mine) + (s.y >= mine) + (s.z >= mine) + (s.w >= mine);
            }
            if (n < want && reach >= want) sh.tau = mine;      // all who write write the same
        }
        __syncthreads();
        tau = sh.tau;
    }
    // The powers' exponents are z log2(e) / T - ref, one rounding, ref the rounded exponent of about the maximum:
    // it is taken anew where a logit is kLpSlack powers of two above.  What it is off by is put right at the end.
    // It is never below -2 kLpLargest: of logits further down, as masks are, the rounding of their exponents, or the
    // bound kLpLowest, would leave any power of two.  So their powers are at most one, and nothing beside the row's.
    const float zscale = c.zscale;
    const uint64_t zscale2 = pair(zscale, zscale);
    float m = top, least_up = top;      // the largest so far, and what raises ref
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) least_up = fmaxf(least_up, __shfl_xor_sync(0xffffffffu, least_up, o));
    auto ref_of = [&](float v) { return v == -INFINITY ? 0.f : fminf(fmaxf(fmaxf(v, kLpLowest<TYPE>) * zscale, -2.f * kLpLargest), 1e30f); };
    float ref = ref_of(least_up);
    bool empty = least_up == -INFINITY;
    least_up += empty ? 0.f : kLpSlack / zscale;
    float stir = fminf(least_up, tau);      // what four words' largest element has to be above for them to be looked at
    uint64_t s0 = pair(0.f, 0.f), s1 = s0, less = pair(-ref, -ref);
    auto raise = [&](float to) {
        const float r2 = ref_of(to), d = empty ? kLpFloor : fmaxf(ref - r2, kLpFloor), by = exp2_fast(d);
        const uint64_t by2 = pair(by, by);
        s1 = mul2(fma2(s0, pair(d, d), s1), by2);
        s0 = mul2(s0, by2);
        ref = r2;
        empty = false;
        least_up = to + kLpSlack / zscale;
        stir = fminf(least_up, tau);
        less = pair(-ref, -ref);
    };
    // The rank: elements not below the token's before it, and above it behind it; by words, the token's own among those
    // behind until the end.
    const bool ranked = c.rank != nullptr && first >= 0;
    const int first_at = first - head, first_word = first_at >= 0 ? first_at / kVec : -1;      // (may be past the words)
    const unsigned th_behind = threshold_of<TYPE>(first_v, false), th_before = threshold_of<TYPE>(first_v, true);
    unsigned masks = 0;      // less the all-ones of elements above
    int rank = 0;
    auto count_masks = [&]() {
        if constexpr (TYPE == GK_TYPE_F32) {
            rank += (int)masks;
        } else {
            // 65536 (upper - lower) + lower
            const unsigned lower = masks & 0xffffu;
            rank += (int)(lower + (((masks >> 16) + lower) & 0xffffu));
        }
        masks = 0;
    };
    auto word = [&](const uint4& x, int w) {
        if (ranked) {
            const unsigned th = w < first_word ? th_before : th_behind;
            masks -= above<TYPE>(x.x, th) + above<TYPE>(x.y, th);
            masks -= above<TYPE>(x.z, th) + above<TYPE>(x.w, th);
        }
        float f[kVec];
        if constexpr (TYPE == GK_TYPE_F32) {
            unpack<TYPE>(x, f);
        } else {
            const unsigned n = threshold_of<TYPE>(kLpLowest<TYPE>, false);
            unpack<TYPE>(make_uint4(max2_nan<TYPE>(x.x, n), max2_nan<TYPE>(x.y, n), max2_nan<TYPE>(x.z, n), max2_nan<TYPE>(x.w, n)), f);
        }
#pragma unroll
        for (int e = 0; e < kVec; e += 2) {
            if constexpr (TYPE == GK_TYPE_F32) {
                f[e] = max_nan(f[e], kLpLowest<TYPE>);
                f[e + 1] = max_nan(f[e + 1], kLpLowest<TYPE>);
            }
            const uint64_t d = fma2(pair(f[e], f[e + 1]), zscale2, less);
            float d0, d1;
            unpair(d, d0, d1);
            const uint64_t p = pair(exp2_fast(d0), exp2_fast(d1));
            s0 = add2(s0, p);
            s1 = fma2(p, d, s1);
        }
    };
    auto quad = [&](const uint4 (&x)[kLpQuad], int q) {
        if (q >= quarter) return;
        const float g = max_of<TYPE>(x);
        m = fmaxf(m, g);
        if (g > stir) {
            if (g > least_up) raise(g);
            if (LISTS && g > tau) {
#pragma unroll
                for (int i = 0; i < kLpQuad; ++i)
                    if (max_of<TYPE>(x[i]) > tau) {
                        const int to = atomicAdd(&sh.notes, 1);
                        if (to < Shared::kNotes) sh.note[to] = q * NT + i * step + tid;
                        if (to < Shared::kNoted) sh.data[to] = x[i];
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < kLpQuad; ++i) word(x[i], q * NT + i * step + tid);
        if ((q & 2047) == 2047) count_masks();      // 2^15 of a half
    };
    // the next words are on their way while four are looked at
#pragma unroll 1
    for (int q = 0; q < quarter; q += 2) {
        quad(x, q);
        fetch(x, q + 2);
        quad(y, q + 1);
        fetch(y, q + 3);
    }
    count_masks();
    if (wid == 0 && odd) {
        m = fmaxf(m, odd_v);
        if (odd_v > least_up) raise(odd_v);
        if (LISTS && odd_v > tau) sh.list[atomicAdd(&sh.listed, 1)] = lp_entry(odd_v, odd_at);      // 32 at most, the first
        if (ranked) rank += odd_v > first_v || (odd_v == first_v && odd_at < first);
        const float d = max_nan(fmaf(odd_v, zscale, -ref), kLpFloor), e = exp2_fast(d);
        s0 = add2(s0, pair(e, 0.f));
        s1 = add2(s1, pair(e * d, 0.f));
    }
    // equal elements in the token's own word before it
    if (ranked && first_word >= 0 && first_word < words && tid < first_at % kVec)
        rank += load_logit<TYPE>(row, first - first_at % kVec + tid) == first_v;
    const int64_t token = tid < c.m ? c.token[r * c.m + tid] : -1;
    const bool mine = token >= 0 && token < V;
    const float own_v = tid == 0 ? first_v : mine ? load_logit<TYPE>(row, token) : 0.f;
    Sums a;
    {
        float lo, hi;
        unpair(s0, lo, hi);
        a.s0 = lo + hi;
        unpair(s1, lo, hi);
        a.s1 = lo + hi;
        // Relative to the warp's maximum itself, which is at or above what this thread's ref was taken from, and far
        // above where the thread met masked logits alone: their sums become nothing.  (A maximum that is too large for
        // this, or lower than ref can be, is that of a row that goes through lp_again, or of a warp that is nothing
        // beside the row's.)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        a.m = m;
        const float off = ref < kLpLargest && m > -INFINITY ? fminf(fmaxf(fmaf(m, zscale, -ref), -1.f), -kLpFloor) : 0.f;
        const float by = exp2_fast(-off);
        a.s1 = fmaf(-off, a.s0, a.s1) * by;
        a.s0 *= by;
        lp_join_lanes(a);
        rank = (int)__reduce_add_sync(0xffffffffu, (unsigned)rank);
        if (lane == 0) {
            sh.above[wid] = rank;
            sh.sums[wid] = a;
        }
    }
    __syncthreads();
    a = lp_join_warps<kWarps>(sh.sums, zscale);
    rank = (int)__reduce_add_sync(0xffffffffu, lane < kWarps ? (unsigned)sh.above[lane] : 0u);
    // Exponents that fp32 has no digits for, and infinities: differences first.  So too where s1 alone is NaN: at small
    // T the exponent of kLpLowest is -inf, its power 0.
    if ((a.m > -INFINITY && !(fabsf(a.m * zscale) < kLpLargest && (a.m - kLpLowest<TYPE>) * zscale > -kLpFloor)) || (a.s1 != a.s1 && a.s0 == a.s0))
        a = lp_again<TYPE>(sh, row, v0, v1, a.m, zscale);
    // (-inf and NaN have no next smaller value; where the token's logit is NaN, only one of a row's CTAs has it in its sums)
    if (ranked && (a.s0 != a.s0 || first_v == -INFINITY || first_v != first_v)) rank = lp_rank_again<TYPE>(sh, row, v0, v1, first_v, first);
    const int k = SPLIT ? min(c.k, v1 - v0) : c.k;      // of this CTA's elements
    int cnt = 0;
    if constexpr (LISTS) {
        // the list of what may be among the alternatives
        const int notes = sh.notes;
        const bool nan = a.s0 != a.s0;
        for (int j = tid; !nan && j < min(notes, Shared::kNotes); j += NT) {
            const int w = sh.note[j];
            float f[kVec];
            unpack<TYPE>(j < Shared::kNoted ? sh.data[j] : __ldg(own - tid + w), f);
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (f[e] > tau) {
                    const int to = atomicAdd(&sh.listed, 1);
                    if (to < Shared::kList) sh.list[to] = lp_entry(f[e], head + w * kVec + e);
                }
        }
        __syncthreads();
        cnt = sh.listed;
        const bool listed = !nan && notes <= Shared::kNotes && cnt <= Shared::kList;
        if (listed && cnt < k) lp_fill<TYPE>(sh, row, v0, v1, tau, k, cnt);
        const bool walked = !listed || cnt < k;
        if (walked) {
            // what there is of a list that is too long gives a bound
            uint64_t least = 0;
            cnt = min(cnt, Shared::kList);
            if (!nan && !listed && cnt >= k) least = lp_cut(sh, cnt, k, max(k, Shared::kPlaced / 2), order_key(tau), order_key(a.m));
            lp_walk<TYPE>(sh, row, v0, v1, k, least, cnt);
        }
        if (cnt > Shared::kPlaced)      // (a walk's list has NaN, or elements below tau where there were too few above)
            lp_cut(sh, cnt, k, max(k, Shared::kPlaced / 2), walked ? 0u : order_key(tau), walked ? ~0u : order_key(a.m));
    }
    // the place of each is how many are above it
    auto place_all = [&](auto&& put) {
        for (int j = tid; j < cnt; j += NT) {
            const uint64_t e = sh.list[j];
            int place = 0, i = 0;
#pragma unroll 2
            for (; i + 4 <= cnt; i += 4) {
                const ulonglong2 p = *(const ulonglong2*)&sh.list[i], q = *(const ulonglong2*)&sh.list[i + 2];
                place += (p.x > e) + (p.y > e) + (q.x > e) + (q.y > e);
            }
            for (; i < cnt; ++i) place += sh.list[i] > e;
            if (place < k) put(place, e);
        }
    };
    if constexpr (SPLIT) {
        if constexpr (LISTS) {
            if (tid >= k && tid < c.k) sh.best[tid] = 0;      // below all
            place_all([&](int place, uint64_t e) { sh.best[place] = e; });
        }
        if (tid == 0) {
            sh.part = a;
            sh.part_above = rank;
        }
        lp_cluster_barrier();
        // every warp joins all parts' sums, a lane each, in one order
        const int p = lane & (parts - 1);
        a = Sums{remote(sh.part.m, p), remote(sh.part.s0, p), remote(sh.part.s1, p)};
        rank = remote(sh.part_above, p);
        rank = (int)__reduce_add_sync(0xffffffffu, lane < parts ? (unsigned)rank : 0u);
        for (int o = parts / 2; o > 0; o >>= 1) lp_join_across(a, o, zscale);
        lp_first_lanes(a);
    }
    const LpResult result(c, a);
    if (part == 0) {
        if (c.logp && tid < c.m) c.logp[r * c.m + tid] = mine ? result.logp(own_v) : 0.f;
        for (int j = tid + NT; NT < kLogprobMaxTokens && c.logp && j < c.m; j += NT) {
            const int64_t t = c.token[r * c.m + j];
            c.logp[r * c.m + j] = t >= 0 && t < V ? result.logp(load_logit<TYPE>(row, t)) : 0.f;
        }
        if (tid == 0) {
            if (c.rank) c.rank[r] = first >= 0 ? rank : -1;
            if (c.entropy) c.entropy[r] = result.entropy(a);
            if (c.lse) c.lse[r] = result.lse();
        }
    }
    auto write = [&](int place, uint64_t e) {
        c.idx[r * c.k + place] = (int)~(uint32_t)e;
        c.val[r * c.k + place] = result.logp(key_value((unsigned)(e >> 32)));
    };
    if constexpr (!SPLIT) {
        if constexpr (LISTS) place_all(write);
    } else {
        // all parts' alternatives beside one another, and how many of each part are above each of this CTA's: a thread a part
        uint64_t* all = reinterpret_cast<uint64_t*>(sh.data);
        for (int j = tid; j < parts * c.k; j += NT) all[j] = remote(sh.best[j / parts], j & (parts - 1));
        __syncthreads();
        for (int j0 = 0; LISTS && j0 < parts * k; j0 += NT) {
            const int i = min((j0 + tid) / parts, k - 1), p = tid & (parts - 1);
            const uint64_t e = all[i * parts + part];
            int lo = 0, hi = c.k;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (all[mid * parts + p] > e) lo = mid + 1; else hi = mid;
            }
            for (int o = parts / 2; o > 0; o >>= 1) lo += __shfl_xor_sync(0xffffffffu, lo, o);
            if (p == 0 && j0 + tid < parts * k && lo < c.k) write(lo, e);
        }
        lp_cluster_barrier();      // the others have read what is here
    }
}

template <int TYPE, bool LISTS>
static cudaError_t launch_logprob(LogprobCall& c, int sms, cudaStream_t st) {
    const int64_t words = c.V / (TYPE == GK_TYPE_F32 ? 4 : 8);
    // CTAs a row: as many as there is room for (two an SM: 64 rows of 128000 bf16, 4 a row 13 us, 8 22), while each still
    // has four words for every thread (64 rows of 32000 bf16, 2 a row 9.1, 4 9.8; one row of 50001 fp32, 8 a row 8.6, 4 9.7)
    while (c.parts < kLpParts && c.n * c.parts * 2 <= 2 * sms && words >= 8 * c.parts * 256) c.parts *= 2;
    if (c.parts > 1) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)c.parts;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        cfg.stream = st;
        cfg.blockDim = dim3(256);
        cfg.gridDim = dim3((unsigned)(c.n * c.parts));
        return cudaLaunchKernelEx(&cfg, k_vocab_logprob<TYPE, 256, true, LISTS>, c);
    }
    // 4096 rows of 10000 bf16 with 10 alternatives: 51 us by 64 threads a row, 59 by 128, 76 by 256; of 32000: 106, 102
    // and 108; of 128000: 1000, 300 and 280 (few threads' samples are small, and their lists overflow).  Twice the
    // threads while there is room for them.
    int threads = words <= kLpShort && c.k <= 48 ? 64 : words <= kLpMiddle ? 128 : 256;
    while (threads < 256 && c.n * threads * 2 <= 1024ll * sms && words >= 4 * threads) threads *= 2;
    if (threads == 64) k_vocab_logprob<TYPE, 64, false, LISTS><<<(unsigned)c.n, 64, 0, st>>>(c);
    else if (threads == 128) k_vocab_logprob<TYPE, 128, false, LISTS><<<(unsigned)c.n, 128, 0, st>>>(c);
    else k_vocab_logprob<TYPE, 256, false, LISTS><<<(unsigned)c.n, 256, 0, st>>>(c);
    return cudaGetLastError();
}

struct LogprobGradCall {
    const char* logits;
    char* dz;
    int64_t ld, lddz, n, V;
    const int64_t* token;
    int m;
    float inv_T, inv_T_low;      // 1 / T in two parts
    const float* lse;
    const float* entropy;
    const float* a;
    const float* b;
    const float* c;
};
constexpr int kLgThreads = 256;

// A CTA a piece of a row (grid: pieces by rows), logits read and gradients written once, four words a thread at a time
// and four on their way.  Bounded by memory: 4096 x 128000 bf16, 2.1 GB, in 325 us, a copy's rate; with 30 % of the rows
// left out, which are written only, 299.  700 x 10000 fp32, 56 MB, in 12 us on the GPU; 33 x 1003 fp16 in 3.5.  Rows of
// other 16-byte boundaries than their logits' go element by element: 4096 x 128000 bf16 in 1.7 to 1.9 ms.
//     dz = p (k0 + k1 log p),  k0 = (c - sum a - b entropy) / T,  k1 = -b / T,
// and a / T more at a token, which the CTA that has it writes again at the end.
template <int TYPE>
__global__ void __launch_bounds__(kLgThreads, 4) k_vocab_logprob_grad(const LogprobGradCall c) {
    constexpr int kVec = TYPE == GK_TYPE_F32 ? 4 : 8, kSize = TYPE == GK_TYPE_F32 ? 4 : 2, kWords = 4;
    constexpr float kLowest = TYPE == GK_TYPE_F32 ? -3.402823466e38f : TYPE == GK_TYPE_BF16 ? -3.3895313892515355e38f : -65504.f;
    __shared__ int64_t tokens[kLogprobMaxTokens];
    const int tid = threadIdx.x, lane = tid & 31;
    const int V = (int)c.V;
    for (int64_t r = blockIdx.y; r < c.n; r += gridDim.y) {
        const char* row = c.logits + r * c.ld * kSize;
        char* out = c.dz + r * c.lddz * kSize;
        // the piece's elements [v0, v1); words where both rows have the same 16-byte boundaries
        const bool apart = (((uintptr_t)row ^ (uintptr_t)out) & 15) != 0;
        const int head = min((int)((16 - ((uintptr_t)row & 15)) % 16) / kSize, V), all = (V - head) / kVec;
        const int w0 = (int)((int64_t)all * blockIdx.x / gridDim.x), words = (int)((int64_t)all * (blockIdx.x + 1) / gridDim.x) - w0;
        const int v0 = blockIdx.x == 0 ? 0 : head + w0 * kVec, v1 = blockIdx.x == gridDim.x - 1 ? V : head + (w0 + words) * kVec;
        const int behind = v1 - (head + (w0 + words) * kVec);      // elements behind the words (sums past 2^31 are not formed)
        const uint4* from = (const uint4*)(row + head * kSize) + w0 + tid;
        uint4* to = (uint4*)(out + head * kSize) + w0 + tid;
        uint4 x[kWords], y[kWords];
        auto fetch = [&](uint4 (&x)[kWords], int w) {
            if (apart) return;
#pragma unroll
            for (int j = 0; j < kWords; ++j)
                if (w + j * kLgThreads + tid < words) x[j] = __ldcs(from + w + j * kLgThreads);
        };
        fetch(x, 0);
        const float lse = c.lse[r], b = c.b ? c.b[r] : 0.f, entropy = c.b ? c.entropy[r] : 0.f;
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
        fetch(y, kWords * kLgThreads);
        auto store = [&](int64_t i, float v) {
            if constexpr (TYPE == GK_TYPE_F32) ((float*)out)[i] = v;
            else ((uint16_t*)out)[i] = to16<TYPE == GK_TYPE_F16>(v);
        };
        counts = counts && !(lse < -1e30f);      // else nothing is left, or masks of a type's lowest value alone
        if (!counts) {
            if (apart) {
                for (int64_t i = (int64_t)v0 + tid; i < v1; i += kLgThreads) store(i, 0.f);
                continue;
            }
            for (int w = tid; w < words; w += kLgThreads) __stcs(to + w - tid, make_uint4(0, 0, 0, 0));
            if (tid < head - v0) store(v0 + tid, 0.f);
            if (tid < behind) store(v1 - behind + tid, 0.f);
            continue;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        k0 = lse < INFINITY ? (k0 - sum - b * entropy) * c.inv_T : NAN;      // a row without a log-sum-exp: NaN throughout
        const float k1 = -b * c.inv_T;
        auto plain = [&](int64_t i) {
            if constexpr (TYPE == GK_TYPE_F32) return ((const float*)row)[i];
            else return from16<TYPE == GK_TYPE_F16>(((const uint16_t*)row)[i]);
        };
        // (zero where the probability is, whatever factor it has: log p is -inf there, or times 1 / T past fp32)
        auto grad = [&](float z) {
            const float d = z == -INFINITY ? z : fmaf(z, c.inv_T_low, fmaf(z, c.inv_T, -lse)), p = exp2_fast(d * 1.44269504f);
            return p == 0.f && k0 == k0 ? 0.f : p * fmaf(k1, d, k0);
        };
        // A token's gradients are added up by the first of the threads that have it.
        here = here && c.a;
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
                    at_token = fmaf(more, c.inv_T, grad(plain(t)));
                }
            }
            __syncthreads();      // read before it is written over, where dlogits are the logits
        }
        if (apart) {
            for (int64_t i = (int64_t)v0 + tid; i < v1; i += kLgThreads) store(i, grad(plain(i)));
        } else {
            // One bound takes the place of all logits below it, -inf among them, where their probabilities are zero in fp32
            // and the bound's is too: 200 nats below the log-sum-exp, with room for its own rounding to 16 bits.  Where no
            // such value exists (fp16 at temperatures of hundreds), or the factor of its probability is past fp32 (twice it:
            // the rounding), element by element.
            const float bound = fmaxf(fmaf(-fabsf(lse), 0.0078125f, lse - 200.f) / c.inv_T, kLowest), below = fmaf(bound, c.inv_T, -lse);
            const bool paired = below <= -110.f && fmaf(fabsf(k1 * below), 2.f, fabsf(k0)) < INFINITY;
            const unsigned bound2 = threshold_of<TYPE>(bound, false);
            const uint64_t hi = pair(c.inv_T, c.inv_T), lo = pair(c.inv_T_low, c.inv_T_low), less = pair(-lse, -lse),
                           log2e = pair(1.44269504f, 1.44269504f), a0 = pair(k0, k0), a1 = pair(k1, k1);
            auto word = [&](const uint4& x) {
                float f[kVec];
                if (paired) {
                    if constexpr (TYPE == GK_TYPE_F32) {
                        unpack<TYPE>(x, f);
#pragma unroll
                        for (int e = 0; e < kVec; ++e) f[e] = max_nan(f[e], bound);
                    } else {
                        unpack<TYPE>(make_uint4(max2_nan<TYPE>(x.x, bound2), max2_nan<TYPE>(x.y, bound2), max2_nan<TYPE>(x.z, bound2), max2_nan<TYPE>(x.w, bound2)), f);
                    }
#pragma unroll
                    for (int e = 0; e < kVec; e += 2) {
                        const uint64_t z = pair(f[e], f[e + 1]), d = fma2(z, lo, fma2(z, hi, less));
                        float d0, d1;
                        unpair(mul2(d, log2e), d0, d1);
                        unpair(mul2(pair(exp2_fast(d0), exp2_fast(d1)), fma2(a1, d, a0)), f[e], f[e + 1]);
                    }
                } else {
                    unpack<TYPE>(x, f);
#pragma unroll 1
                    for (int e = 0; e < kVec; ++e) {
                        const float g = grad(f[0]);      // (turned round, so that the code is there once)
#pragma unroll
                        for (int i = 0; i + 1 < kVec; ++i) f[i] = f[i + 1];
                        f[kVec - 1] = g;
                    }
                }
                if constexpr (TYPE == GK_TYPE_F32) {
                    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                } else {
                    constexpr bool F16 = TYPE == GK_TYPE_F16;
                    return make_uint4(pack16<F16>(f[0], f[1]), pack16<F16>(f[2], f[3]), pack16<F16>(f[4], f[5]), pack16<F16>(f[6], f[7]));
                }
            };
            auto words_of = [&](const uint4 (&x)[kWords], int w) {
#pragma unroll
                for (int j = 0; j < kWords; ++j)
                    if (w + j * kLgThreads + tid < words) __stcs(to + w + j * kLgThreads, word(x[j]));
            };
            constexpr int kStep = kWords * kLgThreads;
#pragma unroll 1
            for (int w = 0; w < words; w += 2 * kStep) {
                words_of(x, w);
                fetch(x, w + 2 * kStep);
                words_of(y, w + kStep);
                fetch(y, w + 3 * kStep);
            }
            if (tid < head - v0) store(v0 + tid, grad(plain(v0 + tid)));
            if (tid < behind) store(v1 - behind + tid, grad(plain(v1 - behind + tid)));
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

// SMs of the current device, looked up once.
static cudaError_t sm_count(int& sms) {
    static std::atomic<int> known[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    sms = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
    if (sms > 0) return cudaSuccess;
    e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess && dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    return e;
}

static int check_rows(const void* logits, int64_t ld, int32_t dtype, int64_t n, int64_t V, const int64_t* token, int32_t m, float T) {
    if (n < 0 || V < 1 || V > 2147483647ll || m < 0) return GK_ERR_SIZE;
    if (n > 2147483647ll || m > kLogprobMaxTokens) return GK_ERR_LIMIT;
    if (dtype != GK_TYPE_F32 && dtype != GK_TYPE_BF16 && dtype != GK_TYPE_F16) return GK_ERR_TYPE;
    if (n > 0 && (!logits || (m > 0 && !token))) return GK_ERR_NULL;
    if (ld < V) return GK_ERR_STRIDE;
    if (off_boundary(dtype == GK_TYPE_F32 ? 4 : 2, logits) || off_boundary(8, token)) return GK_ERR_ALIGN;
    return temperature_ok(T) ? GK_OK : GK_ERR_TEMPERATURE;
}

extern "C" int gk_vocab_logprob(const void* logits, int64_t ld, int32_t dtype, int64_t n, int64_t V, const int64_t* token,
                                int32_t m, float temperature, int32_t k, float* logp_out, int32_t* rank_out,
                                float* entropy_out, float* lse_out, int32_t* idx_out, float* val_out, gk_stream_t stream) {
    const int rc = check_rows(logits, ld, dtype, n, V, token, m, temperature);
    if (rc != GK_OK) return rc;
    if (k < 0 || k > V || k > kLogprobMaxAlternatives) return GK_ERR_K;
    if (n > 0 && k > 0 && (!idx_out || !val_out)) return GK_ERR_NULL;
    if (off_boundary(4, logp_out, rank_out, entropy_out, lse_out, idx_out, val_out)) return GK_ERR_ALIGN;
    if (n == 0) return GK_OK;
    const double inv_T = 1.0 / (double)temperature;
    LogprobCall c = {(const char*)logits, ld, n, V, token, m, k, 1, (float)inv_T, (float)(inv_T - (double)(float)inv_T), (float)(1.4426950408889634 * inv_T),
                     logp_out, rank_out, entropy_out, lse_out, idx_out, val_out};
    int sms = 0;
    GK_CUDA_TRY(sm_count(sms));
    cudaError_t e;
    switch (dtype) {
#define GK_LAUNCH(TYPE) e = k > 0 ? launch_logprob<TYPE, true>(c, sms, (cudaStream_t)stream) : launch_logprob<TYPE, false>(c, sms, (cudaStream_t)stream)
        case GK_TYPE_F32: GK_LAUNCH(GK_TYPE_F32); break;
        case GK_TYPE_BF16: GK_LAUNCH(GK_TYPE_BF16); break;
        default: GK_LAUNCH(GK_TYPE_F16); break;
#undef GK_LAUNCH
    }
    if (e != cudaSuccess) return cuda_fail(e);
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
    if (off_boundary((unsigned)size, dlogits) || off_boundary(4, lse, entropy, logp_grad, entropy_grad, lse_grad)) return GK_ERR_ALIGN;
    if (n == 0) return GK_OK;
    const uintptr_t z0 = (uintptr_t)logits, z1 = z0 + ((n - 1) * ld + V) * size, d0 = (uintptr_t)dlogits, d1 = d0 + ((n - 1) * lddz + V) * size;
    if (z0 < d1 && d0 < z1 && (z0 != d0 || (ld != lddz && n > 1))) {
        // rows of one stride may lie between one another
        const int64_t apart = (int64_t)(((z0 < d0 ? d0 - z0 : z0 - d0) / size) % ld);
        if (ld != lddz || apart < V || ld - apart < V) return GK_ERR_ALIAS;
    }
    int sms = 0;
    GK_CUDA_TRY(sm_count(sms));
    // sixteen words a thread, fewer where there are not enough CTAs
    const int64_t words = V / (16 / size);
    int64_t pieces = (words + 16 * kLgThreads - 1) / (16 * kLgThreads);
    if (pieces < 1) pieces = 1;
    while (n * pieces < 4 * sms && words > 2 * kLgThreads * pieces) pieces *= 2;
    const double inv_T = 1.0 / (double)temperature;
    const LogprobGradCall c = {(const char*)logits, (char*)dlogits, ld, lddz, n, V, token, m, (float)inv_T,
                               (float)(inv_T - (double)(float)inv_T), lse, entropy, logp_grad, entropy_grad, lse_grad};
    const dim3 grid((unsigned)pieces, (unsigned)(n < 65535 ? n : 65535));
    cudaStream_t st = (cudaStream_t)stream;
    switch (dtype) {
        case GK_TYPE_F32: k_vocab_logprob_grad<GK_TYPE_F32><<<grid, kLgThreads, 0, st>>>(c); break;
        case GK_TYPE_BF16: k_vocab_logprob_grad<GK_TYPE_BF16><<<grid, kLgThreads, 0, st>>>(c); break;
        default: k_vocab_logprob_grad<GK_TYPE_F16><<<grid, kLgThreads, 0, st>>>(c); break;
    }
    GK_CUDA_TRY(cudaGetLastError());
    note_launch();
    return GK_OK;
}
