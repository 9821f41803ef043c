// The vocabulary head: softmax cross entropy and distillation from a teacher's top logits through
// z = h w^T, without keeping the logits, with their gradients (include/gk.h: gk_vocab_loss,
// gk_vocab_distill).  This file: the entry points, the workspace and the passes between the
// products; the products themselves are in gk_vocab_gemm.cu.
//
// With T the temperature, lse_n = log sum_v exp(z_nv / T), p_nv = exp(z_nv / T - lse_n):
//     loss_n = sum_j q_nj (log q_nj - z_n,i(n,j) / T + lse_n)      (q = 1 at the class: lse_n - z_n,t)
//     dz_nv  = (g_n / T) (Q_n p_nv - sum_{j: i(n,j) = v} q_nj),     Q_n = sum_j q_nj
//     dh = dz w,   dw = dz^T h.
//
// One call:
//   1. (distill) the teacher's probabilities; the rows that count, numbered in their order;
//   2. those rows of h copied together;
//   3. logits tile by tile, of which each row keeps the sums of the exponentials, and for the first
//      piece of the vocabulary (all of it where the budget allows) something of each logit in 16 bits;
//      the logits at the class or at the teacher's pairs as they pass;
//   4. the row's log-sum-exp from the tiles, loss;
//   5. per piece: the logit gradients in 16 bits (from what was kept, or from the product taken again),
//      then dw and dh as products with them.
// Kept between the steps is one piece, whose size the budget bounds whatever n and V are.
//
// What is kept of a logit is its distance from the largest of its 128 columns in fixed point.  For bf16 in steps
// of 2^-9 in the exponent of two: the exponential it stands for is then off by at most 2^-10 log 2 = 6.8e-4 of
// itself, where a bf16 exponential is off by up to 2^-9 = 2.0e-3, and a logit of 16 by 3e-2; the 65536 codes reach
// 2^-128, as bf16 itself does.  For fp16 the steps are 2^-12 (8.5e-5, against 4.9e-4) down to 2^-8 of the largest,
// and coarser (2.5e-4) to 2^-32, below which all count as that.  A pass over them makes the logit gradients: the one
// rounding to the operands' type that the products dw and dh need.  (Exponentials relative to a reference known
// beforehand, the logit at the target, could be the operand themselves, with the rows of h scaled for dw instead:
// that saved the pass, 5 to 7 % of a call, but rounds once more, and dw was off by 1.7 times what an exact dw
// rounded to bf16 is off by, where it now is by 1.3 times.)
#include <atomic>
#include <map>
#include <mutex>
#include <new>

#include "gk_vocab.cuh"

namespace gk {

constexpr float kLn2 = 0.69314718055994531f;
constexpr double kLog2e = 1.4426950408889634;

__device__ __forceinline__ float warp_sum_f(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max_f(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// ---------------------------------------------------------------------------
// 1. Teacher probabilities, one warp a row, and of rows in ascending order which pairs are in which tile of the
// vocabulary.
// ---------------------------------------------------------------------------
// `place`: the pairs' indices, those left out above all; `held`: how many, none where they do not ascend.
__device__ __forceinline__ void teacher_row(const VocabCall& c, int64_t r, int lane, int* place, int& held) {
    const int32_t* ti = c.t_idx + r * c.K;
    const float* tv = c.t_val + r * c.K;
    // the largest logit is taken off before the division by T, so that masks of the type's lowest
    // value do not overflow; with the teacher's own log-sum-exp there is nothing to take off
    float top = -INFINITY;
    bool any = false, ascending = true;
    for (int j = lane; j < c.K; j += 32) {
        const int32_t i = ti[j], before = j > 0 ? ti[j - 1] : -1;
        const float t = tv[j];
        const bool in = i >= 0 && i < c.V;
        if (in && t != -INFINITY) {
            any = true;
            top = fmaxf(top, t);
        }
        if (in && j > 0 && (before >= i || before < 0)) ascending = false;
        place[j] = in ? i : 0x7fffffff;
    }
    any = __any_sync(0xffffffffu, any);
    ascending = __all_sync(0xffffffffu, ascending);
    const float most = warp_max_f(top);
    float L;
    if (c.t_lse) {
        L = c.t_lse[r];
        top = 0.f;
    } else {
        top = most;
        float s = 0.f;
        for (int j = lane; j < c.K; j += 32)
            if (ti[j] >= 0 && ti[j] < c.V && tv[j] != -INFINITY) s += expf((tv[j] - top) * c.inv_T);
        L = logf(warp_sum_f(s));
    }
    float Q = 0.f;
    for (int j = lane; j < c.K; j += 32) {
        const bool on = ti[j] >= 0 && ti[j] < c.V && tv[j] != -INFINITY;
        const float q = on ? expf((tv[j] - top) * c.inv_T - L) : 0.f;
        c.q[r * c.K + j] = q;
        Q += q;
    }
    Q = warp_sum_f(Q);
    if (lane == 0) {
        held = ascending ? c.K : 0;
        c.teacher[r] = make_float4(Q, L, top, (float)((ascending ? 1 : 0) + (any ? 2 : 0)));
    }
}
__global__ void __launch_bounds__(256) k_vocab_teacher(VocabCall c) {
    __shared__ int place[8][kVocabMaxPairs + 1];      // (the odd pitch: eight rows at one place are in eight banks)
    __shared__ int held[8];
    after_previous();
    const int wid = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t r = (int64_t)blockIdx.x * 8 + wid;
    if (r < c.n) teacher_row(c, r, lane, place[wid], held[wid]);
    else if (lane == 0) held[wid] = 0;
    __syncthreads();
    // eight rows' entries of a tile are one 32-byte sector
    const int row = threadIdx.x & 7, n = held[row];
    const int64_t tiles = (c.V + kVocabTile - 1) / kVocabTile;
    for (int64_t t = threadIdx.x >> 3; t < tiles; t += 32) {
        const int from = (int)t * kVocabTile;
        int lo = 0, hi = n;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (place[row][mid] < from) lo = mid + 1;
            else hi = mid;
        }
        int end = lo;
        while (end < n && place[row][end] < from + kVocabTile) ++end;
        c.pairs_in[t * c.n_pad + (int64_t)blockIdx.x * 8 + row] = (unsigned)lo | (unsigned)(end - lo) << 16;
    }
}

// ---------------------------------------------------------------------------
// The rows that count, numbered in their order, and the scale that brings the gradients' largest row
// coefficient to 2 (bf16) or 2048 (fp16, whose smallest step is 2^-24: an entry 2^-34 of the largest is still
// held).  A row that has learned little has an entry of nearly its whole coefficient, and the rounding to 16 bits
// is finest, relative to the value, just below a power of two.  A coefficient that is not finite has no say in it:
// its own row of dh, and dw, are lost, the other rows of dh are not.
// ---------------------------------------------------------------------------

// Whether row r counts, and the magnitude of its gradient's coefficient (times T), 0 where that is not finite.
__device__ __forceinline__ bool row_counts(const VocabCall& c, int64_t r, float& g) {
    g = 0.f;
    if (r >= c.n) return false;
    bool on;
    float Q = 1.f;
    const float rg = c.row_grad ? c.row_grad[r] : 1.f;
    if (c.target) {
        const int64_t t = c.target[r];
        on = t != c.ignore_index && t >= 0 && t < c.V;
    } else {
        const float4 te = c.teacher[r];
        on = teacher_counts(te);
        Q = te.x;
    }
    if (on) {
        g = fabsf(Q * rg);
        if (!(g * c.inv_T < INFINITY)) g = 0.f;     // a NaN too
    }
    return on;
}
__device__ __forceinline__ void write_ctl(const VocabCall& c, int n_valid, float top) {
    if (!c.row_grad && n_valid > 0) top /= (float)n_valid;
    top *= c.inv_T;
    int e = 0;
    float part = 1.f;
    if (top > 0.f) part = frexpf(top, &e);   // top = part 2^e
    e = min(max((c.f16 ? 11 : 1) - e, -100), 100);
    c.ctl->n_valid = n_valid;
    c.ctl->status = 0;
    c.ctl->scale = ldexpf(1.f, e) / part;
    c.ctl->inv_scale = ldexpf(part, -e);
}

// By one CTA, 8192 rows at a time: all loads first, then one scan over the 256 counts of (32 rows).
__global__ void __launch_bounds__(1024) k_vocab_rows(VocabCall c) {
    constexpr int kEach = 8;
    __shared__ int count[kEach * 32], part[8];
    __shared__ float warp_g[32];
    after_previous();
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    int base = 0;
    float top = 0.f;
    for (int64_t r0 = 0; r0 < c.n; r0 += kEach * 1024) {
        unsigned ballot[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            float g;
            ballot[j] = row_counts(c, r0 + j * 1024 + tid, g);
            top = fmaxf(top, g);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) ballot[j] = __ballot_sync(0xffffffffu, ballot[j]);
        __syncthreads();
        if (lane == 0)
#pragma unroll
            for (int j = 0; j < kEach; ++j) count[j * 32 + wid] = __popc(ballot[j]);
        __syncthreads();
        int own = 0, incl = 0;
        if (tid < kEach * 32) {
            own = incl = count[tid];
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            if (lane == 31) part[wid] = incl;
        }
        __syncthreads();
        if (tid < kEach * 32) {
            int before = incl - own;
            for (int i = 0; i < wid; ++i) before += part[i];
            count[tid] = before;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int64_t r = r0 + j * 1024 + tid;
            if (ballot[j] >> lane & 1) {
                const int at = base + count[j * 32 + wid] + __popc(ballot[j] & ((1u << lane) - 1u));
                c.row_of[at] = (int32_t)r;
                c.at_of[r] = at;
            } else if (r < c.n) {
                c.at_of[r] = -1;
                c.loss[r] = 0.f;
                c.lse[r] = 0.f;
            }
        }
        for (int i = 0; i < kEach; ++i) base += part[i];
    }
    top = warp_max_f(top);
    if (lane == 0) warp_g[wid] = top;
    __syncthreads();
    if (tid == 0) {
        for (int i = 0; i < 32; ++i) top = fmaxf(top, warp_g[i]);
        write_ctl(c, base, top);
    }
}

// ---------------------------------------------------------------------------
// 2. Compact rows of h (padded with zeros to the pitch, and zero rows to a multiple of 256, which
// the products read), and where a teacher's pairs are in no order the logits at them, which the products
// do not deliver then.  One CTA a row.
// ---------------------------------------------------------------------------

// Eight values from 2-byte-aligned memory, zero from `left` on.
__device__ __forceinline__ uint4 load8(const uint16_t* p, int64_t left) {
    const uintptr_t a = (uintptr_t)p;
    if (left >= 8) {
        if ((a & 15) == 0) return *(const uint4*)p;
        if ((a & 7) == 0) {
            const uint2 x = *(const uint2*)p, y = *((const uint2*)p + 1);
            return make_uint4(x.x, x.y, y.x, y.y);
        }
        if ((a & 3) == 0) {
            const unsigned* q = (const unsigned*)p;
            return make_uint4(q[0], q[1], q[2], q[3]);
        }
    }
    unsigned v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0u;
    return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

// s plus eight products.
template <bool F16>
__device__ __forceinline__ float dot8(const uint4& x, const uint4& y, float s) {
    const unsigned xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        s = fmaf(from16<F16>((uint16_t)xs[q]), from16<F16>((uint16_t)ys[q]), s);
        s = fmaf(from16<F16>((uint16_t)(xs[q] >> 16)), from16<F16>((uint16_t)(ys[q] >> 16)), s);
    }
    return s;
}

// RANK (few rows): each CTA takes a row of the caller's and finds its number itself, by looking at all rows; one of
// them writes the control block.  1024 rows are 8 loads a thread, where a launch of its own costs 3 to 6 us; 2048 rows
// took 25 us so, and 17 by two launches.
// CTAs from n_pad on make the copy of w with rows that start and end on 16-byte boundaries, where w's own do not.
constexpr int64_t kRankRows = 1024;

template <bool F16, bool RANK>
__global__ void __launch_bounds__(128) k_vocab_gather(VocabCall c) {
    __shared__ int counts[2][4];
    __shared__ float tops[4];
    after_previous();
    const int tid = threadIdx.x, lane = tid & 31;
    if (blockIdx.x >= c.n_pad) {
        const int64_t words = c.Dp / 8, total = c.V * words, threads = (gridDim.x - c.n_pad) * 128;
        // (the loads of four words before their stores)
        for (int64_t i0 = (blockIdx.x - c.n_pad) * 128 + tid; i0 < total; i0 += 4 * threads) {
            uint4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t i = i0 + j * threads, v = i / words, k = (i - v * words) * 8;
                if (i < total) x[j] = load8((const uint16_t*)c.w + v * c.ldw + k, c.D - k);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i0 + j * threads < total) ((uint4*)c.wc)[i0 + j * threads] = x[j];
        }
        return;
    }
    int at = blockIdx.x, n_valid;
    int64_t r;
    bool left_out;
    if constexpr (RANK) {
        r = blockIdx.x;
        int before = 0, all = 0;
        float top = 0.f;
        bool mine = false;
#pragma unroll 4
        for (int64_t i = tid; i < c.n; i += 128) {
            float g;
            const bool on = row_counts(c, i, g);
            all += on;
            before += on && i < r;
            mine |= on && i == r;
            top = fmaxf(top, g);
        }
        all = __reduce_add_sync(0xffffffffu, all);
        before = __reduce_add_sync(0xffffffffu, before);
        top = warp_max_f(top);
        if (lane == 0) { counts[0][tid >> 5] = all; counts[1][tid >> 5] = before; tops[tid >> 5] = top; }
        left_out = !__syncthreads_or(mine) && r < c.n;
        n_valid = counts[0][0] + counts[0][1] + counts[0][2] + counts[0][3];
        at = counts[1][0] + counts[1][1] + counts[1][2] + counts[1][3];
        if (tid == 0) {
            if (r == 0) write_ctl(c, n_valid, fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
            if (left_out) {
                c.at_of[r] = -1;
                c.loss[r] = 0.f;
                c.lse[r] = 0.f;
            } else if (r < c.n) {
                c.row_of[at] = (int32_t)r;
                c.at_of[r] = at;
            }
        }
        // rows up to the padding are zero
        if (r >= n_valid && r < round_up(n_valid, kVocabRowPad))
            for (int64_t i = tid; i < c.Dp / 8; i += 128) ((uint4*)(c.hc + r * c.Dp))[i] = make_uint4(0, 0, 0, 0);
    } else {
        r = c.row_of[at < c.n ? at : 0];       // a row of the call where at < n_valid
        n_valid = c.ctl->n_valid;
        left_out = at < c.n && c.at_of[at] < 0;
    }
    if (c.dh && left_out) {
        uint16_t* out = (uint16_t*)c.dh + (int64_t)blockIdx.x * c.lddh;
        for (int64_t i = tid; i < c.D; i += 128) out[i] = 0;
    }
    uint16_t* to = c.hc + (int64_t)at * c.Dp;
    if constexpr (RANK) {
        if (left_out || r >= c.n) return;
    } else {
        if (at >= round_up(n_valid, kVocabRowPad)) return;
        if (at >= n_valid) {
            for (int64_t i = tid; i < c.Dp / 8; i += 128) ((uint4*)to)[i] = make_uint4(0, 0, 0, 0);
            return;
        }
    }
    const uint16_t* from = (const uint16_t*)c.h + r * c.ldh;
    const int64_t words = c.Dp / 8;
    for (int64_t i0 = tid; i0 < words; i0 += 4 * 128) {
        uint4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i0 + j * 128 < words) x[j] = load8(from + (i0 + j * 128) * 8, c.D - (i0 + j * 128) * 8);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i0 + j * 128 < words) ((uint4*)to)[i0 + j * 128] = x[j];
    }
    if (c.target) {
        if (tid == 0) c.cls[at] = (int32_t)c.target[r];
        return;
    }
    if (teacher_ascending(c.teacher[r])) return;
    __syncthreads();
    for (int j = tid >> 5; j < c.K; j += 4) {
        const int64_t v = c.t_idx[r * c.K + j];
        float s = 0.f;
        if (v >= 0 && v < c.V) {
            const uint16_t* wr = (const uint16_t*)c.w + v * c.ldw;
            for (int64_t b = lane; b < words; b += 32) s = dot8<F16>(((const uint4*)to)[b], load8(wr + b * 8, c.D - b * 8), s);
        }
        s = warp_sum_f(s);
        if (lane == 0) c.zt[(int64_t)at * c.K + j] = s;
    }
}

// ---------------------------------------------------------------------------
// 4. Log-sum-exp and loss.  A CTA takes 32 compact rows; its 32 warps share the tiles, a fixed order
// joins them, and each warp finishes a row.
// ---------------------------------------------------------------------------

// What a row's end needs besides its log-sum-exp; fetched while that is still being summed.
struct RowEnd {
    int64_t r;
    float g, z;      // its gradient's coefficient; with a class its raw logit
    float4 te;
};
__device__ __forceinline__ RowEnd fetch_end(const VocabCall& c, int64_t at, int64_t r, int n_valid) {
    RowEnd e;
    e.r = r;
    e.g = c.row_grad ? c.row_grad[r] : 1.f / (float)n_valid;
    e.z = c.target ? c.zt[at] : 0.f;
    e.te = c.target ? make_float4(1.f, 0.f, 0.f, 0.f) : c.teacher[r];
    return e;
}
// A row from its log-sum-exp, by one warp: its loss (write) and what the gradients need of it.
__device__ __forceinline__ VocabRow finish_row(const VocabCall& c, int64_t at, const RowEnd& e, float lse2, int lane, bool write) {
    if (write) {
        float loss;
        if (c.target) {
            loss = (lse2 - e.z * c.zscale) * kLn2;
        } else {
            float sum = 0.f;
            for (int j = lane; j < c.K; j += 32) {
                const float q = c.q[e.r * c.K + j];
                if (q > 0.f) sum += q * (((c.t_val[e.r * c.K + j] - e.te.z) * c.inv_T - e.te.y) + (lse2 - c.zt[at * c.K + j] * c.zscale) * kLn2);
                else if (q != q) sum = q;
            }
            loss = warp_sum_f(sum);
        }
        if (lane == 0) {
            c.loss[e.r] = loss;
            c.lse[e.r] = lse2 * kLn2;
        }
    }
    VocabRow out;
    out.unit = c.ctl->scale * (e.g * c.inv_T);
    out.lse2 = lse2;
    out.coef = out.unit * e.te.x;
    out.pad = 0.f;
    return out;
}

__global__ void __launch_bounds__(1024) k_vocab_rows_done(VocabCall c) {
    __shared__ float sm[32][33], ss[32][33];
    after_previous();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int64_t at0 = (int64_t)blockIdx.x * 32;
    const int n_valid = c.ctl->n_valid;
    if (at0 >= n_valid) return;
    const int64_t tiles = (c.V + kVocabTile - 1) / kVocabTile;
    // With 32 rows a lane is a row; with fewer, lanes of a row share its tiles (one row: 1024 loads at once).
    const int rows = (int)(n_valid - at0 < 32 ? n_valid - at0 : 32);
    const int pitch = rows > 16 ? 32 : rows > 8 ? 16 : rows > 4 ? 8 : rows > 2 ? 4 : rows;
    const int mine = lane % pitch, share = lane / pitch, shares = 32 / pitch;
    const int64_t at = at0 + wid;
    const int32_t r = at < n_valid ? c.row_of[at] : 0;
    float m = -INFINITY, s = 0.f;
    if (mine < rows) {
        const float2* p = c.part + at0 + mine;
#pragma unroll 4
        for (int64_t t = wid * shares + share; t < tiles; t += 32 * shares) {
            const float2 x = load_once(p + t * c.n_pad);
            join_max_sum(m, s, x.x, x.y);
        }
    }
    for (int o = pitch; o < 32; o *= 2) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        float ml = lane & o ? m2 : m, sl = lane & o ? s2 : s;
        join_max_sum(ml, sl, lane & o ? m : m2, lane & o ? s : s2);
        m = ml;
        s = sl;
    }
    sm[wid][lane] = m;
    ss[wid][lane] = s;
    RowEnd end = {};
    if (at < n_valid) end = fetch_end(c, at, r, n_valid);
    __syncthreads();
    if (at >= n_valid) return;
    m = sm[lane][wid];
    s = ss[lane][wid];
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        // both sides join in the order of their lanes
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        float ml = lane & o ? m2 : m, sl = lane & o ? s2 : s;
        join_max_sum(ml, sl, lane & o ? m : m2, lane & o ? s : s2);
        m = ml;
        s = sl;
    }
    const VocabRow out = finish_row(c, at, end, m + log2f(s), lane, true);
    if (lane == 0) c.row[at] = out;
}

// ---------------------------------------------------------------------------
// 5. The logit gradients of one piece.  The targets' entries are formed in fp32 from their own logits
// and written over, so that 1 - p loses nothing where p is near 1.
// ---------------------------------------------------------------------------
// A thread's pair: fetched before it is needed, written where its column is in [lo, hi).
struct Target {
    int64_t v;
    float z, q;
};
__device__ __forceinline__ Target fetch_target(const VocabCall& c, int64_t at, int64_t r, int j) {
    Target t = {-1, 0.f, 0.f};
    if (j < c.K) {
        t.v = c.target ? c.target[r] : (int64_t)c.t_idx[r * c.K + j];
        t.z = c.zt[at * c.K + j];
        t.q = c.target ? 1.f : c.q[r * c.K + j];
    }
    return t;
}
template <bool F16>
__device__ __forceinline__ void write_target(const VocabCall& c, int64_t at, int64_t r, const VocabRow& vr, bool distinct, Target t,
                                             int64_t lo, int64_t hi, int64_t v0) {
    if (t.v < lo || t.v >= hi) return;
    if (!distinct) {      // an index given more than once: each of its pairs writes the same sum
        t.q = 0.f;
        for (int i = 0; i < c.K; ++i)
            if (c.t_idx[r * c.K + i] == t.v) t.q += c.q[r * c.K + i];
    }
    const float p = exp2_fast(t.z * c.zscale - vr.lse2);
    c.e[at * c.vb + (t.v - v0)] = to16<F16>(fmaf(vr.coef, p, -(vr.unit * t.q)));
}

constexpr int64_t kOwnTiles = 128;   // tiles a CTA joins itself

// From the distances kept of the piece [v0, v1): e <- coef 2^(m_tile - lse - distance), in place, and zero
// for the rows up to the padding, which the product for dw sums over.  DONE (vocabularies of up to
// 128 tiles): each CTA joins the row's tiles itself, and the first of a row writes its loss, instead
// of a launch of its own before this one.  All of a thread's words are on their way before anything that they
// wait for is looked at.  Bound by memory: 4096 x 64000, 524 MB read and as many written, takes 174 us by itself,
// 6.0 TB/s.
template <bool DONE>
constexpr int kScaleWords = DONE ? 2 : 4;                                  // 16-byte words a thread
template <bool DONE>
constexpr int kGradCols = 256 * 8 * kScaleWords<DONE>;                     // columns a CTA

template <bool F16, bool DONE>
__global__ void __launch_bounds__(256) k_vocab_scale(VocabCall c, int64_t v0, int64_t v1) {
    __shared__ float sm[4], ss[4];
    after_previous();
    const int64_t at = blockIdx.x;
    const int64_t lo = v0 + (int64_t)blockIdx.y * kGradCols<DONE>;
    const int64_t hi = lo + kGradCols<DONE> < v1 ? lo + kGradCols<DONE> : v1;
    uint4* const mine = (uint4*)(c.e + at * c.vb + (lo - v0)) + threadIdx.x;
    const int left = (int)((hi - lo + 7) / 8) - (int)threadIdx.x;          // words from this thread's first on
    uint4 x[kScaleWords<DONE>];
    float top[kScaleWords<DONE>];
#pragma unroll
    for (int j = 0; j < kScaleWords<DONE>; ++j)
        if (j * 256 < left) {
            x[j] = load_once(mine + j * 256);
            top[j] = c.part[(lo + (j * 256 + threadIdx.x) * 8) / kVocabTile * c.n_pad + at].x;
        }
    const int n_valid = c.ctl->n_valid;
    const int64_t r = c.row_of[at < c.n ? at : 0];
    if (at >= round_up(n_valid, 64)) return;
    if (at >= n_valid) {
#pragma unroll
        for (int j = 0; j < kScaleWords<DONE>; ++j)
            if (j * 256 < left) mine[j * 256] = make_uint4(0, 0, 0, 0);
        return;
    }
    const bool distinct = c.target || teacher_ascending(c.teacher[r]);
    const Target first = fetch_target(c, at, r, threadIdx.x);
    VocabRow vr;
    if constexpr (DONE) {
        const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
        const int64_t tiles = (c.V + kVocabTile - 1) / kVocabTile;
        const RowEnd end = fetch_end(c, at, r, n_valid);
        float m = -INFINITY, s = 0.f;
        if (wid < 4) {
            if (tid < tiles) {
                const float2 x = c.part[tid * c.n_pad + at];
                m = x.x;
                s = x.y;
            }
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
                float ml = lane & o ? m2 : m, sl = lane & o ? s2 : s;
                join_max_sum(ml, sl, lane & o ? m : m2, lane & o ? s : s2);
                m = ml;
                s = sl;
            }
            if (lane == 0) { sm[wid] = m; ss[wid] = s; }
        }
        __syncthreads();
        m = sm[0];
        s = ss[0];
#pragma unroll
        for (int k = 1; k < 4; ++k) join_max_sum(m, s, sm[k], ss[k]);
        vr = finish_row(c, at, end, m + log2f(s), lane, blockIdx.y == 0 && wid == 0);
        if (blockIdx.y == 0 && tid == 0) c.row[at] = vr;
    } else {
        vr = c.row[at];
    }
#pragma unroll
    for (int j = 0; j < kScaleWords<DONE>; ++j)
        if (j * 256 < left) {
            const float base = top[j] - vr.lse2;
            unsigned xs[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
            for (int q = 0; q < 4; ++q)
                xs[q] = pack16<F16>(vr.coef * exp2_fast(base - kept_distance<F16>(xs[q] & 0xffffu)),
                                    vr.coef * exp2_fast(base - kept_distance<F16>(xs[q] >> 16)));
            mine[j * 256] = make_uint4(xs[0], xs[1], xs[2], xs[3]);
        }
    __syncthreads();
    write_target<F16>(c, at, r, vr, distinct, first, lo, hi, v0);
    for (int j = threadIdx.x + 256; j < c.K; j += 256) write_target<F16>(c, at, r, vr, distinct, fetch_target(c, at, r, j), lo, hi, v0);
}

// The product taken again has written the gradients; only the targets' entries are left.
template <bool F16>
__global__ void __launch_bounds__(128) k_vocab_targets(VocabCall c, int64_t v0, int64_t v1) {
    after_previous();
    const int64_t at = blockIdx.x;
    if (at >= c.ctl->n_valid) return;
    const int64_t r = c.row_of[at];
    const bool distinct = c.target || teacher_ascending(c.teacher[r]);
    for (int j = threadIdx.x; j < c.K; j += 128) write_target<F16>(c, at, r, c.row[at], distinct, fetch_target(c, at, r, j), v0, v1, v0);
}

// dh in the caller's rows from its parts' sums, added in their order.
template <bool F16>
__global__ void __launch_bounds__(256) k_vocab_finish_dh(VocabCall c) {
    after_previous();
    const int64_t at = blockIdx.x, i = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 2;
    if (at >= c.ctl->n_valid || i >= c.D) return;
    const float f = c.ctl->inv_scale;
    const float* from = c.dhp + at * c.Dp + i;
    const int64_t part = c.n_pad * c.Dp;
    float2 s = *(const float2*)from;
#pragma unroll 4
    for (int k = 1; k < c.splits; ++k) {
        const float2 x = *(const float2*)(from + k * part);
        s.x += x.x;
        s.y += x.y;
    }
    uint16_t* to = (uint16_t*)c.dh + (int64_t)c.row_of[at] * c.lddh + i;
    to[0] = to16<F16>(s.x * f);
    if (i + 1 < c.D) to[1] = to16<F16>(s.y * f);
}

// ---------------------------------------------------------------------------
// Workspace: one block per (device, stream), grown as calls need it.  A call holds its stream's block from the
// lookup to its last launch: a call is several launches over that block, so calls of two host threads on one
// stream must not mix theirs, and neither may replace the block under the other.
// ---------------------------------------------------------------------------
struct VocabWorkspace {
    std::mutex held;
    void* base = nullptr;
    size_t bytes = 0;
    int sm_count = 0;
    bool called = false;
};
static std::mutex g_vocab_mu;
static std::map<WorkspaceKey, VocabWorkspace> g_vocab_ws;      // (entries stay where they are)
static std::atomic<int64_t> g_vocab_budget{(int64_t)2 << 30};

static int64_t piece_columns(int64_t n_pad, int64_t V) {
    const int64_t fit = g_vocab_budget.load() / (2 * n_pad) / 256 * 256;
    const int64_t all = round_up(V, 256);
    return fit >= all ? all : fit < 256 ? 256 : fit;
}

// Lays the workspace out in `c` from `base` (nullptr: only the size is wanted).
static size_t lay_out(VocabCall& c, bool distill, bool copy_w, char* base) {
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* p = base ? base + at : nullptr;
        at = (at + bytes + 255) / 256 * 256;
        return p;
    };
    const size_t n = (size_t)c.n, np = (size_t)c.n_pad, K = (size_t)c.K;
    const size_t tiles = (size_t)((c.V + kVocabTile - 1) / kVocabTile);
    c.ctl = (VocabCtl*)take(sizeof(VocabCtl));
    c.row_of = (int32_t*)take(4 * n);
    c.at_of = (int32_t*)take(4 * n);
    c.q = (float*)(distill ? take(4 * n * K) : nullptr);
    c.teacher = (float4*)(distill ? take(16 * n) : nullptr);
    c.cls = (int32_t*)(distill ? nullptr : take(4 * np));
    c.pairs_in = (unsigned*)(distill ? take(4 * tiles * np) : nullptr);
    c.hc = (uint16_t*)take(2 * np * c.Dp);
    c.wc = (uint16_t*)(copy_w ? take(2 * (size_t)c.V * c.Dp) : nullptr);
    c.zt = (float*)take(4 * np * K);
    c.part = (float2*)take(8 * tiles * np);
    c.row = (VocabRow*)take(sizeof(VocabRow) * np);
    c.e = (uint16_t*)(c.vb > 0 ? take(2 * np * (size_t)c.vb) : nullptr);
    // one part and one piece: dh's sums are final when its product ends
    c.dhp = (float*)(c.splits > 1 || (c.splits == 1 && c.vb < c.V) ? take(4 * (size_t)c.splits * np * c.Dp) : nullptr);
    return at;
}

// The stream's workspace, held by `lock` from here on.
static int vocab_workspace(cudaStream_t st, VocabWorkspace** out, WorkspaceLock& lock) {
    WorkspaceKey key;
    const int rc = workspace_key(st, key);
    if (rc != GK_OK) return rc;
    VocabWorkspace* ws;
    {
        std::lock_guard<std::mutex> all(g_vocab_mu);
        ws = &g_vocab_ws[key];
    }
    lock = WorkspaceLock(ws->held);
    if (ws->sm_count == 0) GK_CUDA_TRY(cudaDeviceGetAttribute(&ws->sm_count, cudaDevAttrMultiProcessorCount, std::get<0>(key)));
    *out = ws;
    return GK_OK;
}

// At least `bytes` for a workspace that the caller holds.  What the last call reported goes along.
static int grow(VocabWorkspace& ws, size_t bytes, cudaStream_t st) {
    if (ws.bytes >= bytes) return GK_OK;
    const bool had = ws.base != nullptr;
    VocabCtl last = {};
    if (had) {
        GK_CUDA_TRY(cudaStreamSynchronize(st));   // work already enqueued may still use the old block
        GK_CUDA_TRY(cudaMemcpy(&last, ws.base, sizeof(last), cudaMemcpyDeviceToHost));
        GK_CUDA_TRY(cudaFree(ws.base));
        ws.base = nullptr;
        ws.bytes = 0;
    }
    void* p = nullptr;
    if (cudaMalloc(&p, bytes) != cudaSuccess) { cudaGetLastError(); return GK_ERR_NOMEM; }
    ws.base = p;
    ws.bytes = bytes;
    // (a stream that could be waited for is not being captured: the copy is staged before it returns)
    if (had) GK_CUDA_TRY(cudaMemcpyAsync(p, &last, sizeof(last), cudaMemcpyHostToDevice, st));
    else GK_CUDA_TRY(cudaMemsetAsync(p, 0, sizeof(last), st));
    return GK_OK;
}

static void size_call(VocabCall& c, bool want_dh, DwRows dw, int sm_count) {
    c.n_pad = round_up(c.n, kVocabRowPad);
    c.Dp = round_up(c.D, 64);
    c.vb = want_dh || dw != DwRows::none ? piece_columns(c.n_pad, c.V) : 0;
    c.splits = want_dh ? vocab_dh_splits(c.n, c.D, c.vb < c.V ? c.vb : c.V, dw, sm_count) : 0;
}

template <bool F16>
static int enqueue(const VocabCall& c, bool distill, int sms, cudaStream_t st) {
    const unsigned n = (unsigned)c.n, groups = (n + 31) / 32;
    const bool grad = c.dh || c.dw;
    if (distill) {
        k_vocab_teacher<<<(n + 7) / 8, 256, 0, st>>>(c);
        GK_CUDA_TRY(cudaGetLastError());
    }
    if (c.n > kRankRows) GK_CUDA_TRY(launch_next(k_vocab_rows, dim3(1), 1024, 0, st, c));
    const int64_t copies = c.wc ? (c.V * (c.Dp / 8) + 127) / 128 : 0;
    GK_CUDA_TRY(launch_next(c.n > kRankRows ? k_vocab_gather<F16, false> : k_vocab_gather<F16, true>,
                            dim3((unsigned)(c.n_pad + (copies < 16 * sms ? copies : 16 * sms))), 128, 0, st, c));
    note_launch(1 + (distill ? 1 : 0) + (c.n > kRankRows ? 1 : 0));
    const int64_t kept = grad ? (c.vb < c.V ? c.vb : c.V) : 0;
    int rc = GK_OK;
    if (kept > 0) rc = launch_vocab_logits(c, 0, kept, true, sms, st);
    if (rc == GK_OK && kept < c.V) rc = launch_vocab_logits(c, kept, c.V, false, sms, st);
    if (rc != GK_OK) return rc;
    const bool own = grad && (c.V + kVocabTile - 1) / kVocabTile <= kOwnTiles;
    if (!own) {
        GK_CUDA_TRY(launch_next(k_vocab_rows_done, dim3(groups), 1024, 0, st, c));
        note_launch();
    }
    if (!grad) return GK_OK;
    for (int64_t v0 = 0; v0 < c.V; v0 += c.vb) {
        const int64_t v1 = v0 + c.vb < c.V ? v0 + c.vb : c.V;
        if (v0 > 0) {
            rc = launch_vocab_again(c, v0, v1, sms, st);
            if (rc != GK_OK) return rc;
            GK_CUDA_TRY(launch_next(k_vocab_targets<F16>, dim3(n), 128, 0, st, c, v0, v1));
            note_launch();
        } else {
            const int cols = own ? kGradCols<true> : kGradCols<false>;
            const dim3 grid((unsigned)round_up(n, 64), (unsigned)((v1 + cols - 1) / cols));
            GK_CUDA_TRY(launch_next(own ? k_vocab_scale<F16, true> : k_vocab_scale<F16, false>, grid, 256, 0, st, c, v0, v1));
            note_launch();
        }
        rc = launch_vocab_grads(c, v0, v1, v0 == 0, sms, st);
        if (rc != GK_OK) return rc;
    }
    if (c.dhp) {
        GK_CUDA_TRY(launch_next(k_vocab_finish_dh<F16>, dim3(n, (unsigned)((c.D + 511) / 512)), 256, 0, st, c));
        note_launch();
    }
    return GK_OK;
}

static bool overlap(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + bn && y < x + an;
}
static size_t extent(int64_t rows, int64_t cols, int64_t ld) { return rows < 1 ? 0 : 2 * (size_t)((rows - 1) * ld + cols); }

// What both entry points check, in the order of the arguments.
static int check_head(const VocabCall& c, int32_t dtype) {
    if (c.n < 0 || c.D < 1 || c.V < 1) return GK_ERR_SIZE;
    if (c.n > (1 << 22) || c.D > (1 << 16) || c.V > (1 << 26)) return GK_ERR_LIMIT;
    if (dtype != GK_TYPE_BF16 && dtype != GK_TYPE_F16) return GK_ERR_TYPE;
    if (!c.w || (c.n > 0 && (!c.h || !c.loss || !c.lse))) return GK_ERR_NULL;
    if (c.ldh < c.D || c.ldw < c.D || (c.dh && c.lddh < c.D) || (c.dw && c.lddw < c.D)) return GK_ERR_STRIDE;
    if ((((uintptr_t)c.h | (uintptr_t)c.w | (uintptr_t)c.dh | (uintptr_t)c.dw) & 1) != 0) return GK_ERR_ALIGN;
    const size_t hb = extent(c.n, c.D, c.ldh), wb = extent(c.V, c.D, c.ldw);
    const size_t dhb = c.dh ? extent(c.n, c.D, c.lddh) : 0, dwb = c.dw ? extent(c.V, c.D, c.lddw) : 0;
    if (dhb && (overlap(c.dh, dhb, c.h, hb) || overlap(c.dh, dhb, c.w, wb))) return GK_ERR_ALIAS;
    if (dwb && (overlap(c.dw, dwb, c.h, hb) || overlap(c.dw, dwb, c.w, wb))) return GK_ERR_ALIAS;
    if (dhb && dwb && overlap(c.dh, dhb, c.dw, dwb)) return GK_ERR_ALIAS;
    return GK_OK;
}

// (no exception passes a C entry: the map's memory is the only source of one)
static int run_head(VocabCall& c, bool distill, cudaStream_t st) try {
    VocabWorkspace* ws = nullptr;
    WorkspaceLock held;
    int rc = vocab_workspace(st, &ws, held);
    if (rc != GK_OK) return rc;
    if (c.n == 0) {   // no rows: the weights' gradient is zero
        if (c.dw) GK_CUDA_TRY(cudaMemset2DAsync(c.dw, 2 * c.lddw, 0, 2 * c.D, (size_t)c.V, st));
        if (ws->base) GK_CUDA_TRY(cudaMemsetAsync(ws->base, 0, sizeof(VocabCtl), st));
        ws->called = true;
        return GK_OK;
    }
    // rows that start and end on 16-byte boundaries are copied to shared memory as they lie
    const bool w_vec = (((uintptr_t)c.w | (uintptr_t)(2 * c.ldw) | (uintptr_t)(2 * c.D)) & 15) == 0;
    const bool dw_vec = (((uintptr_t)c.dw | (uintptr_t)(2 * c.lddw) | (uintptr_t)(2 * c.D)) & 15) == 0;
    size_call(c, c.dh != nullptr, !c.dw ? DwRows::none : dw_vec ? DwRows::aligned : DwRows::unaligned, ws->sm_count);
    rc = grow(*ws, lay_out(c, distill, !w_vec, nullptr), st);
    if (rc != GK_OK) return rc;
    lay_out(c, distill, !w_vec, (char*)ws->base);
    ws->called = true;
    return c.f16 ? enqueue<true>(c, distill, ws->sm_count, st) : enqueue<false>(c, distill, ws->sm_count, st);
} catch (const std::bad_alloc&) {
    return GK_ERR_NOMEM;
}

}  // namespace gk

using namespace gk;

extern "C" int gk_vocab_loss(const void* h, int64_t ldh, const void* w, int64_t ldw, int32_t dtype, int64_t n, int64_t D,
                             int64_t V, const int64_t* target, int64_t ignore_index, const float* row_grad,
                             float* loss_out, float* lse_out, void* dh_out, int64_t lddh, void* dw_out, int64_t lddw,
                             gk_stream_t stream) {
    VocabCall c = {};
    c.n = n; c.D = D; c.V = V;
    c.h = h; c.ldh = ldh; c.w = w; c.ldw = ldw; c.dh = dh_out; c.lddh = lddh; c.dw = dw_out; c.lddw = lddw;
    c.target = target; c.ignore_index = ignore_index; c.row_grad = row_grad; c.loss = loss_out; c.lse = lse_out;
    const int rc = check_head(c, dtype);
    if (rc != GK_OK) return rc;
    if (n > 0 && !target) return GK_ERR_NULL;
    c.K = 1;
    c.f16 = dtype == GK_TYPE_F16;
    c.inv_T = 1.f;
    c.zscale = (float)kLog2e;
    return run_head(c, false, (cudaStream_t)stream);
}

extern "C" int gk_vocab_distill(const void* h, int64_t ldh, const void* w, int64_t ldw, int32_t dtype, int64_t n,
                                int64_t D, int64_t V, const int32_t* t_idx, const float* t_val, int32_t K,
                                const float* t_lse, float temperature, const float* row_grad, float* loss_out,
                                float* lse_out, void* dh_out, int64_t lddh, void* dw_out, int64_t lddw,
                                gk_stream_t stream) {
    VocabCall c = {};
    c.n = n; c.D = D; c.V = V;
    c.h = h; c.ldh = ldh; c.w = w; c.ldw = ldw; c.dh = dh_out; c.lddh = lddh; c.dw = dw_out; c.lddw = lddw;
    c.t_idx = t_idx; c.t_val = t_val; c.t_lse = t_lse; c.row_grad = row_grad; c.loss = loss_out; c.lse = lse_out;
    const int rc = check_head(c, dtype);
    if (rc != GK_OK) return rc;
    if (n > 0 && (!t_idx || !t_val)) return GK_ERR_NULL;
    if (K < 1 || K > kVocabMaxPairs) return GK_ERR_K;
    if (!temperature_ok(temperature)) return GK_ERR_TEMPERATURE;
    c.K = K;
    c.f16 = dtype == GK_TYPE_F16;
    c.inv_T = 1.f / temperature;
    c.zscale = (float)(kLog2e / (double)temperature);
    return run_head(c, true, (cudaStream_t)stream);
}

extern "C" int gk_vocab_set_budget(int64_t bytes) {
    if (bytes < 0) return GK_ERR_CAPACITY;
    g_vocab_budget.store(bytes);
    return GK_OK;
}

// What the largest call of up to n rows may ask for: a distillation with K pairs and both gradients (or no gradient),
// over rows of w on any boundary.  Fewer rows can need more: dh is split into more parts, and a piece of the
// vocabulary comes nearer to the budget.  Within 64 rows, a block of dw's sum, launch_time's tiles and blocks are the
// same and a part costs more with more rows, so the fewest rows have the most parts.
static size_t largest(VocabCall& c, int64_t n, int64_t D, int64_t V, int32_t K, int grad, int sms) {
    c.D = D; c.V = V; c.K = K;
    size_t most = 0;
    for (int64_t last = n; last > 0; last = (last - 1) / 64 * 64) {
        const int64_t few = (last - 1) / 64 * 64 + 1;
        for (DwRows dw : {DwRows::none, DwRows::aligned, DwRows::unaligned}) {     // dh is split by what it shares the SMs with
            c.n = few;
            size_call(c, grad != 0, grad ? dw : DwRows::none, sms);
            c.n = last;
            const size_t bytes = lay_out(c, true, D % 8 != 0, nullptr);
            most = bytes > most ? bytes : most;
            if (!grad) return most;      // grows with the rows
        }
    }
    return most;
}

static int head_sizes_ok(int64_t n, int64_t D, int64_t V, int32_t K) {
    if (n < 1 || D < 1 || V < 1) return GK_ERR_SIZE;
    if (n > (1 << 22) || D > (1 << 16) || V > (1 << 26)) return GK_ERR_LIMIT;
    return K < 1 || K > kVocabMaxPairs ? GK_ERR_K : GK_OK;
}

extern "C" int64_t gk_vocab_workspace_bytes(int64_t n, int64_t D, int64_t V, int32_t K, int grad) {
    if (head_sizes_ok(n, D, V, K) != GK_OK) return 0;
    VocabCall c = {};
    return (int64_t)largest(c, n, D, V, K, grad, 148);
}

extern "C" int gk_vocab_reserve(int64_t n, int64_t D, int64_t V, int32_t K, int grad, gk_stream_t stream) try {
    const int rc = head_sizes_ok(n, D, V, K);
    if (rc != GK_OK) return rc;
    VocabWorkspace* ws = nullptr;
    WorkspaceLock held;
    const int wrc = vocab_workspace((cudaStream_t)stream, &ws, held);
    if (wrc != GK_OK) return wrc;
    VocabCall c = {};
    return grow(*ws, largest(c, n, D, V, K, grad, ws->sm_count), (cudaStream_t)stream);
} catch (const std::bad_alloc&) {
    return GK_ERR_NOMEM;
}

extern "C" int gk_vocab_last_info(gk_stream_t stream, int64_t* host_out) {
    if (!host_out) return GK_ERR_NULL;
    WorkspaceKey key;
    const int rc = workspace_key((cudaStream_t)stream, key);
    if (rc != GK_OK) return rc;
    VocabWorkspace* ws = nullptr;
    {
        std::lock_guard<std::mutex> all(g_vocab_mu);
        auto it = g_vocab_ws.find(key);
        if (it != g_vocab_ws.end()) ws = &it->second;
    }
    if (!ws) return GK_ERR_NULL;
    GK_CUDA_TRY(cudaStreamSynchronize((cudaStream_t)stream));
    std::lock_guard<std::mutex> held(ws->held);
    if (!ws->called) return GK_ERR_NULL;
    VocabCtl ctl = {};
    if (ws->base)       // else no call had rows
        GK_CUDA_TRY(cudaMemcpy(&ctl, ws->base, sizeof(ctl), cudaMemcpyDeviceToHost));
    host_out[0] = ctl.status;
    host_out[1] = ctl.n_valid;
    return GK_OK;
}
