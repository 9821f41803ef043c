// The gradients of many tensors: their norm, and clipping them by it (include/gk.h: gk_grad_norm,
// gk_grad_clip).
//
// The work is cut into units of 16 KB of a tensor's gradients; a CTA has a contiguous stretch of all units, so
// that of each tensor it meets it has one contiguous span.  A long span is the whole CTA's; a short one is cut
// into pieces of 4 KB, a warp each.  Squares are added in fp32
// over 32 (fp32) or 64 (16-bit) elements and those sums in fp64; where such a sum says that squares left fp32's
// range, or is zero, the elements are squared again in fp64 (4e8 zeros in bf16: 178 us, random ones 122).  Sums are joined in a fixed order: threads, warps, CTAs.
// Bounded by memory, with eight words a thread (64 KB an SM) on their way: the norm of 1e9 bf16 in 400 tensors, 2 GB,
// takes 297 us (a copy's rate; two CTAs an SM with four words, double-buffered, 350), of 25.6 M fp32 in 161 tensors 26.
//
// Clipping is one cooperative kernel: squares, a barrier of the grid, and the scaling from the last unit back
// to the first, which meets in L2 what the squares read last.  4e8 elements of bf16 and fp32 into one fp32 vector: 3.0 GB
// in 551 us; 25.6 M fp32 in 161 tensors, from L2 the second time, 57; 269722 in 65, 8.6, most of it the barrier.  With the
// norm given, gradients are read once and no CTA waits: 423 us and, with nothing in L2 before, 46 (66 without it).
#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "gk_coop.cuh"
#include "gk_grad.cuh"
#include "gk_segmented.cuh"
#include "gk_words.cuh"

namespace gk {

constexpr int kGradThreads = 512, kGradWarps = kGradThreads / 32;
constexpr int kGradUnit = 16384;          // bytes of source in a unit
// Bytes of a span that is cut into pieces, a warp each, and of a piece.  The CTA's warps together take 64 KB in turns, the
// last of them only in part: the norms of 25.6 M fp32 in 161 tensors 20.1 us (spans beyond 64 KB so), 19.3 (128 KB),
// 19.2 (256 KB); of 1e9 bf16, where all spans are long, 312 against 322 in pieces.
constexpr int kGradSmall = 131072, kGradPiece = 4096;
constexpr int kGradParts = 32;            // sums of spans kept before they are joined

struct GradRec {
    const void* src;
    void* dst;
    int64_t n;              // elements
    unsigned first;         // units of the tensors before
    unsigned types;         // of src, and of dst in bits 8 and up
};
// The table travels as a kernel argument where it fits (a captured call then needs nothing of the host),
// else kernels with a part of it as their argument write it to the workspace first.
constexpr int kGradFew = 64, kGradMany = 1000;      // (and sizes between: an argument of 16 KB takes the host 4 us more)
template <int CAP>
struct GradTable {
    GradRec rec[CAP];
};

struct GradCall {
    const GradRec* table;   // nullptr: the kernel's argument
    int T;
    unsigned units;
    GradCtl* ctl;
    double* cta_sums;       // one a CTA
    double* span_sums;      // tensor + CTA: a CTA's span of a tensor
    float* norm_out;
    float* norms_out;
    const float* scale;
    const float* norm_in;
    float max_norm;
    unsigned extra;         // arrivals that the barrier expects beyond the grid's (test hook)
};

__device__ __forceinline__ double block_total(double v, double* smem) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    double r = 0.0;
#pragma unroll
    for (int i = 0; i < kGradWarps; ++i) r += smem[i];
    return r;
}

template <int TYPE>
struct Elem {
    static constexpr int size = TYPE == GK_TYPE_F32 ? 4 : 2, vec = 16 / size;
};
template <int TYPE>
__device__ __forceinline__ float load_elem(const char* p, int64_t i) {
    if constexpr (TYPE == GK_TYPE_F32) return ((const float*)p)[i];
    else return from16<TYPE == GK_TYPE_F16>(((const uint16_t*)p)[i]);
}
template <int TYPE>
__device__ __forceinline__ void store_elem(char* p, int64_t i, float v) {
    if constexpr (TYPE == GK_TYPE_F32) ((float*)p)[i] = v;
    else ((uint16_t*)p)[i] = to16<TYPE == GK_TYPE_F16>(v);
}

template <int TYPE>
__device__ __noinline__ double squares64(uint4 a, uint4 b, uint4 c, uint4 d) {
    double acc = 0.0;
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
        float f[Elem<TYPE>::vec];
        unpack<TYPE>(a, f);
        a = b;
        b = c;
        c = d;
#pragma unroll
        for (int e = 0; e < Elem<TYPE>::vec; ++e) acc = fma((double)f[e], (double)f[e], acc);
    }
    return acc;
}

// Sum of the squares of n elements at p, the part of thread tid of G.
template <int TYPE, int G>
__device__ __forceinline__ double squares(const char* p, int64_t n, int tid) {
    constexpr int kVec = Elem<TYPE>::vec, kSize = Elem<TYPE>::size, kWords = 8;
    int64_t head = (16 - ((uintptr_t)p & 15)) % 16 / kSize;
    if (head > n) head = n;
    const int64_t words = (n - head) / kVec;
    const uint4* own = (const uint4*)(p + head * kSize) + tid;
    double acc = 0.0;
#pragma unroll 1
    for (int64_t w0 = 0; w0 < words; w0 += kWords * G) {
        const int left = (int)(words - w0 < kWords * G ? words - w0 : kWords * G) - tid;
        uint4 x[kWords];
#pragma unroll
        for (int j = 0; j < kWords; ++j) x[j] = j * G < left ? own[w0 + j * G] : make_uint4(0, 0, 0, 0);
        float s = 0.f, t = 0.f;
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            float f[kVec];
            unpack<TYPE>(x[j], f);
#pragma unroll
            for (int e = 0; e < kVec; e += 2) {
                s = fmaf(f[e], f[e], s);
                t = fmaf(f[e + 1], f[e + 1], t);
            }
        }
        s += t;
        if (s > 7.9e-31f && s < INFINITY) {      // 2^-100: what lies below fp32's range is nothing beside it
            acc += (double)s;
        } else {
#pragma unroll
            for (int j = 0; j < kWords; j += 4) acc += squares64<TYPE>(x[j], x[j + 1], x[j + 2], x[j + 3]);
        }
    }
    // before the first 16-byte boundary and after the last
    const int64_t tail = n - head - words * kVec;
    if (tid < head) {
        const double v = (double)load_elem<TYPE>(p, tid);
        acc = fma(v, v, acc);
    }
    if (tid < tail) {
        const double v = (double)load_elem<TYPE>(p, n - tail + tid);
        acc = fma(v, v, acc);
    }
    return acc;
}
template <int G>
__device__ __noinline__ double squares(int type, const char* p, int64_t n, int tid) {
    switch (type) {
        case GK_TYPE_F32: return squares<GK_TYPE_F32, G>(p, n, tid);
        case GK_TYPE_BF16: return squares<GK_TYPE_BF16, G>(p, n, tid);
        default: return squares<GK_TYPE_F16, G>(p, n, tid);
    }
}

// The eight elements that begin `off` of a 16-byte word's elements into w.
template <int TYPE, int W>
__device__ __forceinline__ void shifted(unsigned (&w)[W], int off, float (&f)[8]) {
    if constexpr (TYPE == GK_TYPE_F32) {
#pragma unroll
        for (int i = 0; i + 1 < W; ++i) w[i] = off & 1 ? w[i + 1] : w[i];
#pragma unroll
        for (int i = 0; i + 2 < W; ++i) w[i] = off & 2 ? w[i + 2] : w[i];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[e]);
    } else {
#pragma unroll
        for (int i = 0; i + 2 < W; ++i) w[i] = off & 4 ? w[i + 2] : w[i];
#pragma unroll
        for (int i = 0; i + 1 < W; ++i) w[i] = off & 2 ? w[i + 1] : w[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = off & 1 ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
        unpack<TYPE>(make_uint4(w[0], w[1], w[2], w[3]), f);
    }
}

// dst = c src, n elements, from the last to the first, by thread tid of G.  A thread has eight elements at a time that
// begin on a boundary of 32 bytes (fp32) or 16 in dst; where they lie otherwise in src, they are cut out of the 16-byte
// words around them.
template <int SRC, int DST, int G>
__device__ __forceinline__ void scaled(const char* src, char* dst, int64_t n, float c, int tid) {
    constexpr int kS = Elem<SRC>::size, kD = Elem<DST>::size, kEach = SRC == GK_TYPE_F32 ? 2 : DST == GK_TYPE_F32 ? 4 : 8;
    constexpr int kLoads = SRC == GK_TYPE_F32 ? 3 : 2;      // words around eight elements
    // elements before the first boundary; eight more where the first words would begin before src
    int64_t head = (8 * kD - (int)((uintptr_t)dst & (8 * kD - 1))) % (8 * kD) / kD;
    const int off = (int)(((uintptr_t)src + head * kS) & 15) / kS;
    if (off > head) head += 8;
    // and no words end behind src
    const int64_t room = n - head + off - (off ? kLoads : kLoads - 1) * (16 / kS);
    int64_t groups = room < 0 ? 0 : room / 8 + 1;
    if (groups == 0) head = 0;
    const uint4* s = (const uint4*)(src + (head - off) * kS) + tid * (kS / 2);
    char* d = dst + (head + tid * 8) * kD;
    constexpr int kStep = kEach * G;
#pragma unroll 1
    for (int64_t g0 = (groups - 1) / kStep * kStep; groups > 0 && g0 >= 0; g0 -= kStep) {
        const int left = (int)(groups - g0 < kStep ? groups - g0 : kStep) - tid;
        const bool whole = groups - g0 >= kStep;
        const uint4* from = s + g0 * (kS / 2);
        char* to = d + g0 * 8 * kD;
        uint4 x[kEach][kLoads];
#pragma unroll
        for (int j = 0; j < kEach; ++j)
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                x[j][i] = j * G < left && (i + 1 < kLoads || off) ? from[j * G * (kS / 2) + i] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (j * G >= left) break;
            unsigned w[kLoads * 4];
            float f[8];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                w[4 * i] = x[j][i].x;
                w[4 * i + 1] = x[j][i].y;
                w[4 * i + 2] = x[j][i].z;
                w[4 * i + 3] = x[j][i].w;
            }
            shifted<SRC>(w, off, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= c;
            if constexpr (DST == GK_TYPE_F32) {
                float4* at = (float4*)(to + (int64_t)j * G * 32);
                if (SRC != GK_TYPE_F32 && whole) {
                    // two threads' 64 bytes as two times 32 (4e8 elements: 582 us without, 554 so; fp32's source no change)
                    const bool up = tid & 1;
                    float g[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) g[e] = __shfl_xor_sync(0xffffffffu, up ? f[e] : f[4 + e], 1);
                    at[up ? -1 : 0] = up ? make_float4(g[0], g[1], g[2], g[3]) : make_float4(f[0], f[1], f[2], f[3]);
                    at[up ? 1 : 2] = up ? make_float4(f[4], f[5], f[6], f[7]) : make_float4(g[0], g[1], g[2], g[3]);
                } else {
                    at[0] = make_float4(f[0], f[1], f[2], f[3]);
                    at[1] = make_float4(f[4], f[5], f[6], f[7]);
                }
            } else {
                constexpr bool F16 = DST == GK_TYPE_F16;
                *(uint4*)(to + (int64_t)j * G * 16) = make_uint4(pack16<F16>(f[0], f[1]), pack16<F16>(f[2], f[3]), pack16<F16>(f[4], f[5]), pack16<F16>(f[6], f[7]));
            }
        }
    }
    for (int64_t i = tid; i < head; i += G) store_elem<DST>(dst, i, c * load_elem<SRC>(src, i));
    for (int64_t i = head + groups * 8 + tid; i < n; i += G) store_elem<DST>(dst, i, c * load_elem<SRC>(src, i));
}
template <int G>
__device__ __noinline__ void scaled(unsigned types, const char* src, char* dst, int64_t n, float c, int tid) {
    switch (types) {
#define GK_PAIR(S, D) case (S | D << 8): scaled<S, D, G>(src, dst, n, c, tid); break;
        GK_PAIR(0, 0) GK_PAIR(0, 1) GK_PAIR(0, 2) GK_PAIR(1, 0) GK_PAIR(1, 1) GK_PAIR(1, 2) GK_PAIR(2, 0) GK_PAIR(2, 1)
        default: scaled<2, 2, G>(src, dst, n, c, tid); break;
#undef GK_PAIR
    }
}

// A CTA's stretch of units, and the tensor that it begins in.
__device__ __forceinline__ unsigned unit_of(unsigned units, unsigned b, unsigned G) { return (unsigned)((uint64_t)units * b / G); }
__device__ __forceinline__ int tensor_of(const GradRec* rec, int T, unsigned unit) {
    int lo = 0, hi = T - 1;      // the last tensor whose first unit is not behind `unit`: empty ones have none of their own
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (rec[mid].first <= unit) lo = mid; else hi = mid - 1;
    }
    return lo;
}
// Elements of tensor r in the units [u0, u1), which it has some of.
__device__ __forceinline__ void span_of(const GradRec& r, unsigned u0, unsigned u1, int64_t& from, int64_t& to) {
    const int each = (r.types & 255u) == GK_TYPE_F32 ? kGradUnit / 4 : kGradUnit / 2;
    from = u0 > r.first ? (int64_t)(u0 - r.first) * each : 0;
    to = (int64_t)(u1 - r.first) * each;
    if (to > r.n) to = r.n;
}

// Every thread: the square root of the CTAs' sums, in the order of the CTAs.
__device__ __forceinline__ double total_norm(const double* cta_sums, unsigned G, double* smem) {
    double v = 0.0;
    for (unsigned b = threadIdx.x; b < G; b += kGradThreads) v += __ldcg(&cta_sums[b]);
    v = warp_sum(v);
    return sqrt(block_total((threadIdx.x & 31) == 0 ? v : 0.0, smem));
}

// atomicInc that all before it is seen by whoever counts later.
__device__ __forceinline__ unsigned count_in(unsigned* counter, unsigned last) {
    unsigned before;
    asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(before) : "l"(counter), "r"(last) : "memory");
    return before;
}

// Arrive at the barrier and wait for all G arrivals; false where a CTA's bounded wait ran out before they were complete.
// All CTAs get the same answer: one gives up by a mark in the counter, made by compare-and-swap while arrivals are
// missing, and whoever looks later finds it.
constexpr unsigned kGradGivenUp = 0x80000000u;
__device__ __forceinline__ bool all_arrive(unsigned* arrived, unsigned G, int* flag) {
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        atomicAdd(arrived, 1u);
        const int limit = g_barrier_poll_limit;
        int polls = 0;
        unsigned v;
        while (true) {
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(arrived) : "memory");
            if (v >= G) break;      // complete, or marked
            if (++polls <= limit) __nanosleep(40);
            else if (atomicCAS(arrived, v, v | kGradGivenUp) == v) { v |= kGradGivenUp; break; }      // else one arrived: look again
        }
        *flag = v < kGradGivenUp;
    }
    __syncthreads();
    return *flag != 0;
}

template <bool CLIP, int CAP>
__global__ void __launch_bounds__(kGradThreads, 1) k_grad(const GradCall c, const __grid_constant__ GradTable<CAP> table) {
    __shared__ double smem[kGradWarps];
    __shared__ double part[kGradParts][kGradWarps];      // the warps' sums of spans that all take, and whose they are
    __shared__ int part_of[kGradParts];
    __shared__ int flag;
    const GradRec* rec = c.table ? c.table : table.rec;
    const unsigned G = gridDim.x, b = blockIdx.x;
    const unsigned u0 = unit_of(c.units, b, G), u1 = unit_of(c.units, b + 1, G);
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    int last = -1;      // the tensor that the stretch ends in
    if (!CLIP || !c.norm_in) {
        const bool each = !CLIP && c.norms_out;
        double all = 0.0;
        int little = 0, parts = 0;
        auto join_parts = [&]() {
            __syncthreads();
            if (tid < parts) {
                double v = 0.0;
#pragma unroll
                for (int w = 0; w < kGradWarps; ++w) v += part[tid][w];
                c.span_sums[part_of[tid] + b] = v;
            }
            parts = 0;
        };
        if (u0 < u1)
            for (int i = tensor_of(rec, c.T, u0); i < c.T && rec[i].first < u1; ++i) {
                const GradRec r = rec[i];
                int64_t from, to;
                span_of(r, u0, u1, from, to);
                if (from >= to) continue;
                last = i;
                const int type = (int)(r.types & 255u), size = type == GK_TYPE_F32 ? 4 : 2;
                const char* p = (const char*)r.src + from * size;
                // a small span is cut into pieces, a warp each
                const int64_t bytes = (to - from) * size, step = kGradPiece / size;
                const int pieces = bytes <= kGradSmall ? (int)((bytes + kGradPiece - 1) / kGradPiece) : 0;
                const int at = (wid - little) & (kGradWarps - 1);      // this warp's first
                little += pieces;
                if (pieces == 1 && at > 0) continue;
                double v = 0.0;
                for (int j = at; j < pieces; j += kGradWarps)
                    v += squares<32>(type, p + (int64_t)j * kGradPiece, min(step, to - from - j * step), lane);
                if (pieces == 0) v = squares<kGradThreads>(type, p, to - from, tid);
                all += v;
                if (!each) continue;
                v = warp_sum(v);
                if (pieces == 1) {
                    if (lane == 0) c.span_sums[i + b] = v;
                    continue;
                }
                if (lane == 0) part[parts][wid] = v;
                if (tid == 0) part_of[parts] = i;
                if (++parts == kGradParts) {
                    join_parts();
                    __syncthreads();
                }
            }
        if (each) join_parts();
        all = block_total(all, smem);
        if (tid == 0) c.cta_sums[b] = all;
    }
    if constexpr (!CLIP) {
        // the CTA that is done last joins the sums
        __syncthreads();
        if (tid == 0) flag = count_in(&c.ctl->done, G - 1) == G - 1;
        __syncthreads();
        if (!flag) return;
        const double norm = total_norm(c.cta_sums, G, smem);
        if (tid == 0) c.norm_out[0] = (float)norm;
        if (!c.norms_out) return;
        // a tensor's spans are those of the CTAs from its first unit's to its last's: up to eight by a thread, more by a warp
        auto spans_of = [&](int i, unsigned& b0, unsigned& b1) {
            const unsigned f = rec[i].first, l = i + 1 < c.T ? rec[i + 1].first - 1 : c.units - 1;
            b0 = (unsigned)((((uint64_t)f + 1) * G - 1) / c.units);
            b1 = (unsigned)((((uint64_t)l + 1) * G - 1) / c.units);
        };
        for (int i0 = 0; i0 < c.T; i0 += kGradThreads) {
            const int i = i0 + tid;
            unsigned b0 = 1, b1 = 0;
            if (i < c.T && rec[i].n > 0) spans_of(i, b0, b1);
            const bool lengthy = b1 >= b0 + 8 && b0 <= b1;
            if (i < c.T && !lengthy) {
                double v[8], sum = 0.0;
#pragma unroll
                for (unsigned j = 0; j < 8; ++j) v[j] = b0 + j <= b1 ? __ldcg(&c.span_sums[i + b0 + j]) : 0.0;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += v[j];
                c.norms_out[i] = (float)sqrt(sum);
            }
            for (unsigned more = __ballot_sync(0xffffffffu, lengthy); more; more &= more - 1) {
                const int l = __ffs(more) - 1, t = i0 + wid * 32 + l;
                const unsigned from = __shfl_sync(0xffffffffu, b0, l), to = __shfl_sync(0xffffffffu, b1, l);
                double v = 0.0;
                for (unsigned a = from + lane; a <= to; a += 32) v += __ldcg(&c.span_sums[t + a]);
                v = warp_sum(v);
                if (lane == 0) c.norms_out[t] = (float)sqrt(v);
            }
        }
    } else {
        const float scale = c.scale ? *c.scale : 1.f;      // (read before the barrier: norm_out may be its place)
        double norm;
        if (c.norm_in) {
            norm = (double)*c.norm_in;
        } else {
            const bool ok = all_arrive(&c.ctl->arrived, G + c.extra, &flag);
            if (tid == 0) {
                // whoever leaves last makes the counters ready for the next call
                if (atomicInc(&c.ctl->left, G - 1) == G - 1) c.ctl->arrived = 0;
            }
            if (!ok) {
                if (b == 0 && tid == 0) {
                    c.ctl->status = GK_DEV_TIMEOUT;
                    c.ctl->clipped = 0;
                    if (c.norm_out) c.norm_out[0] = NAN;
                }
                return;
            }
            norm = total_norm(c.cta_sums, G, smem) * fabs((double)scale);
        }
        // norms that are not finite in norm_out clip nothing: the caller sees them
        const bool clips = norm > (double)c.max_norm && (float)norm < INFINITY;
        const float by = clips ? (float)((double)scale * ((double)c.max_norm / norm)) : scale;
        if (b == 0 && tid == 0) {
            if (c.norm_out) c.norm_out[0] = (float)norm;
            c.ctl->status = GK_DEV_OK;
            c.ctl->clipped = clips;
        }
        if (u0 >= u1) return;
        if (last < 0) last = tensor_of(rec, c.T, u1 - 1);
        int little = 0;
        for (int i = last; i >= 0; --i) {
            const GradRec r = rec[i];
            if (r.n > 0 && !(by == 1.f && r.src == r.dst)) {
                int64_t from, to;
                span_of(r, u0, u1, from, to);
                const int64_t s = (r.types & 255u) == GK_TYPE_F32 ? 4 : 2, d = r.types >> 8 == GK_TYPE_F32 ? 4 : 2;
                const char* p = (const char*)r.src + from * s;
                char* q = (char*)r.dst + from * d;
                if ((to - from) * s > kGradSmall) {
                    scaled<kGradThreads>(r.types, p, q, to - from, by, tid);
                } else {
                    const int64_t step = kGradPiece / s;
                    const int pieces = (int)((to - from + step - 1) / step);
                    for (int j = (wid - little) & (kGradWarps - 1); j < pieces; j += kGradWarps)
                        scaled<32>(r.types, p + (int64_t)j * kGradPiece, q + j * step * d, min(step, to - from - j * step), by, lane);
                    little += pieces;
                }
            }
            if (r.first <= u0) break;
        }
    }
}

// A part of a long table into the workspace.
__global__ void k_grad_table(GradRec* to, int n, const __grid_constant__ GradTable<kGradMany> part) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) to[i] = part.rec[i];
}

size_t grad_scratch_bytes(int32_t S) {
    const size_t T = S > kGradMany ? S : kGradMany;
    return 256 + sizeof(double) * (kGradMaxCtas + kGradMaxCtas + T) + (S > kGradMany ? sizeof(GradRec) * (size_t)S : 0);
}

// CTAs of a device, 0 where it has no cooperative launch.
static int grad_grid(int dev, int sm_count, int* grid) {
    static std::mutex mu;
    static int known[64];
    if (dev < 0 || dev >= 64) return GK_ERR_LIMIT;
    std::lock_guard<std::mutex> lock(mu);
    if (!known[dev]) {
        int coop = 0, occ = 0;
        GK_CUDA_TRY(cudaDeviceGetAttribute(&coop, cudaDevAttrCooperativeLaunch, dev));
        if (!coop) return GK_ERR_LIMIT;
        GK_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, k_grad<true, kGradMany>, kGradThreads, 0));
        known[dev] = std::min(occ * sm_count, kGradMaxCtas);
    }
    *grid = known[dev];
    return *grid > 0 ? GK_OK : GK_ERR_LIMIT;
}

static bool known_type(int32_t t) { return t == GK_TYPE_F32 || t == GK_TYPE_BF16 || t == GK_TYPE_F16; }
static int type_size(int32_t t) { return t == GK_TYPE_F32 ? 4 : 2; }

// What both calls refuse of their lists.
static int check_list(const void* const* grads, const int32_t* types, const int64_t* sizes, int32_t T) {
    if (T < 0) return GK_ERR_SIZE;
    if (T > kMaxSegments) return GK_ERR_LIMIT;
    if (T > 0 && (!grads || !types || !sizes)) return GK_ERR_NULL;
    uint64_t units = 0;
    for (int32_t i = 0; i < T; ++i) {
        if (!known_type(types[i])) return GK_ERR_TYPE;
        if (sizes[i] < 0) return GK_ERR_SIZE;
        if (sizes[i] > (int64_t)1 << 44) return GK_ERR_LIMIT;
        if (sizes[i] > 0 && !grads[i]) return GK_ERR_NULL;
        if ((uintptr_t)grads[i] & (type_size(types[i]) - 1)) return GK_ERR_ALIGN;
        units += ((uint64_t)sizes[i] * type_size(types[i]) + kGradUnit - 1) / kGradUnit;
        if (units > 0xfffffffeull) return GK_ERR_LIMIT;
    }
    return GK_OK;
}

// Whether an output shares memory with another output or with an input that is not its own, the scalars among them.  (A
// norm may go where it was given, being the same number, or where the scale was, which all CTAs have read when they
// meet.)
static bool outputs_overlap(const void* const* grads, const int32_t* types, void* const* outs, const int32_t* out_types,
                            const int64_t* sizes, int32_t T, const float* scale, const float* norm_in, const float* norm_out) {
    using Range = std::pair<uintptr_t, uintptr_t>;
    std::vector<Range> in, out;
    in.reserve(T);
    out.reserve(T);
    for (int32_t i = 0; i < T; ++i) {
        if (sizes[i] == 0) continue;
        const uintptr_t a = (uintptr_t)grads[i], b = (uintptr_t)outs[i];
        out.emplace_back(b, b + sizes[i] * type_size(out_types[i]));
        if (a != b || types[i] != out_types[i]) in.emplace_back(a, a + sizes[i] * type_size(types[i]));
    }
    if (!std::is_sorted(out.begin(), out.end())) std::sort(out.begin(), out.end());
    if (!std::is_sorted(in.begin(), in.end())) std::sort(in.begin(), in.end());
    for (size_t i = 1; i < out.size(); ++i)
        if (out[i].first < out[i - 1].second) return true;
    // inputs may share memory with one another
    size_t o = 0;
    uintptr_t seen = 0;      // the furthest end of an input that starts before the output at hand
    for (const Range& r : out) {
        while (o < in.size() && in[o].first < r.second) seen = std::max(seen, in[o++].second);
        if (seen > r.first) return true;
    }
    // the scalars: in the last output that begins before their end, or, norm_out, in an input
    auto within = [&](const float* p) {
        const auto next = std::upper_bound(out.begin(), out.end(), Range((uintptr_t)p + sizeof(float) - 1, UINTPTR_MAX));
        return next != out.begin() && (uintptr_t)p < (next - 1)->second;
    };
    for (const float* p : {scale, norm_in, norm_out})
        if (p && within(p)) return true;
    for (size_t i = 0; norm_out && i < in.size() && in[i].first < (uintptr_t)norm_out + sizeof(float); ++i)
        if ((uintptr_t)norm_out < in[i].second) return true;
    return scale && norm_in && scale == norm_out;
}

template <bool CLIP, int CAP>
static cudaError_t launch_grad(const GradCall& c, const GradTable<CAP>& table, unsigned G, cudaStream_t st) {
    if (!CLIP || c.norm_in) {
        k_grad<CLIP, CAP><<<G, kGradThreads, 0, st>>>(c, table);
        return cudaGetLastError();
    }
    void* args[] = {(void*)&c, (void*)&table};
    return cudaLaunchCooperativeKernel((const void*)k_grad<CLIP, CAP>, dim3(G), dim3(kGradThreads), args, 0, st);
}

template <bool CLIP>
static int enqueue_grad(GradCall& c, const void* const* grads, const int32_t* types, void* const* outs,
                        const int32_t* out_types, const int64_t* sizes, cudaStream_t st) {
    Workspace* ws = nullptr;
    WorkspaceLock held;
    const int wrc = acquire_workspace(1, c.T > kGradMany ? c.T : 1, st, &ws, held);
    if (wrc != GK_OK) return wrc;
    int dev = 0, most = 0;
    GK_CUDA_TRY(cudaGetDevice(&dev));
    const int grc = grad_grid(dev, ws->sm_count, &most);
    if (grc != GK_OK) return grc;
    char* at = static_cast<char*>(ws->grad_block);
    c.ctl = reinterpret_cast<GradCtl*>(at);
    c.cta_sums = reinterpret_cast<double*>(at + 256);
    c.span_sums = c.cta_sums + kGradMaxCtas;
    // (the records before the sums' end by the workspace's own size, which may be for more tensors)
    GradRec* in_ws = reinterpret_cast<GradRec*>(c.span_sums + kGradMaxCtas + (ws->s_cap > kGradMany ? ws->s_cap : kGradMany));
    c.extra = host_knob(kKnobExtraArrivals) > 0 ? 1u : 0u;
    unsigned units = 0;
    auto record = [&](GradRec& r, int32_t i) {
        r.src = grads[i];
        r.dst = CLIP ? outs[i] : nullptr;
        r.n = sizes[i];
        r.first = units;
        r.types = (unsigned)types[i] | (CLIP ? (unsigned)out_types[i] << 8 : 0u);
        units += (unsigned)(((uint64_t)sizes[i] * type_size(types[i]) + kGradUnit - 1) / kGradUnit);
    };
    auto grid = [&]() { return std::min(std::max(units, 1u), (unsigned)most); };
    auto launch = [&](auto& table) -> cudaError_t {
        if (!c.table)
            for (int32_t i = 0; i < c.T; ++i) record(table.rec[i], i);
        c.units = units;
        return launch_grad<CLIP>(c, table, grid(), st);
    };
    if (c.T <= kGradFew) {
        GradTable<kGradFew> table;
        GK_CUDA_TRY(launch(table));
    } else if (c.T <= 2 * kGradFew) {
        GradTable<2 * kGradFew> table;
        GK_CUDA_TRY(launch(table));
    } else if (c.T <= 3 * kGradFew) {
        GradTable<3 * kGradFew> table;
        GK_CUDA_TRY(launch(table));
    } else if (c.T <= 6 * kGradFew) {
        GradTable<6 * kGradFew> table;
        GK_CUDA_TRY(launch(table));
    } else if (c.T <= kGradMany) {
        GradTable<kGradMany> table;
        GK_CUDA_TRY(launch(table));
    } else {
        GradTable<kGradMany> part;
        for (int32_t i = 0; i < c.T; i += kGradMany) {
            const int n = std::min(kGradMany, c.T - i);
            for (int j = 0; j < n; ++j) record(part.rec[j], i + j);
            k_grad_table<<<(n + 255) / 256, 256, 0, st>>>(in_ws + i, n, part);
            GK_CUDA_TRY(cudaGetLastError());
            note_launch();
        }
        c.table = in_ws;
        GradTable<kGradFew> none;
        GK_CUDA_TRY(launch(none));
    }
    note_launch();
    return GK_OK;
}

}  // namespace gk

using namespace gk;

extern "C" int gk_grad_norm(const void* const* grads, const int32_t* types, const int64_t* sizes, int32_t T,
                            float* norm_out, float* norms_out, gk_stream_t stream) {
    const int rc = check_list(grads, types, sizes, T);
    if (rc != GK_OK) return rc;
    if (!norm_out) return GK_ERR_NULL;
    if (off_boundary(4, norm_out, norms_out)) return GK_ERR_ALIGN;
    GradCall c = {};
    c.T = T;
    c.norm_out = norm_out;
    c.norms_out = norms_out;
    return enqueue_grad<false>(c, grads, types, nullptr, nullptr, sizes, (cudaStream_t)stream);
}

extern "C" int gk_grad_clip(const void* const* grads, const int32_t* types, void* const* outs, const int32_t* out_types,
                            const int64_t* sizes, int32_t T, float max_norm, const float* scale, const float* norm_in,
                            float* norm_out, gk_stream_t stream) try {
    const int rc = check_list(grads, types, sizes, T);
    if (rc != GK_OK) return rc;
    if (T > 0 && (!outs || !out_types)) return GK_ERR_NULL;
    if (!(max_norm > 0.f)) return GK_ERR_NORM;
    for (int32_t i = 0; i < T; ++i) {
        if (!known_type(out_types[i])) return GK_ERR_TYPE;
        if (sizes[i] > 0 && !outs[i]) return GK_ERR_NULL;
        if ((uintptr_t)outs[i] & (type_size(out_types[i]) - 1)) return GK_ERR_ALIGN;
    }
    if (off_boundary(4, scale, norm_in, norm_out)) return GK_ERR_ALIGN;
    if (outputs_overlap(grads, types, outs, out_types, sizes, T, scale, norm_in, norm_out)) return GK_ERR_ALIAS;
    GradCall c = {};
    c.T = T;
    c.max_norm = max_norm;
    c.scale = scale;
    c.norm_in = norm_in;
    c.norm_out = norm_out;
    return enqueue_grad<true>(c, grads, types, outs, out_types, sizes, (cudaStream_t)stream);
} catch (const std::bad_alloc&) {
    return GK_ERR_NOMEM;
}
