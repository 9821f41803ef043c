// The products of the vocabulary head (gk_vocab.cu) on the fifth-generation tensor cores.
//
// One persistent kernel, four uses of it.  A pair of SMs (a cluster of two CTAs) computes a
// 256 x 256 tile of the result with tcgen05.mma.cta_group::2: each CTA holds 128 rows of A, 128 of
// the 256 columns of B, and 128 x 256 fp32 sums in its tensor memory.  Operands arrive by TMA in
// blocks of 64 along the summed axis, six blocks in flight (32 KB each and CTA); the sums are
// double buffered (2 x 256 of the 512 columns of tensor memory), so that one tile is read out and
// finished by four warps while the next one is being summed.
//
//   use          A (M x K)            B (N x K)            what the readout does
//   kLogits      hc  rows x D         w   columns x D      maximum and sum of the tile's columns per row
//   kLogitsKeep  the same                                  and the logits, as 16-bit steps below the
//                                                          tile's maximum
//   kAgain       the same                                  logit gradients, the log-sum-exp being known
//   kDw          e^T columns x rows   hc^T D x rows        16-bit rows of dw
//   kDh          e   rows x columns   w^T  D x columns     fp32 partial sums of dh
//
// e, hc and w are stored once, by rows; where the summed axis is not the contiguous one the
// operand is read as it lies (MN-major descriptors) instead of being transposed in memory.
#include <cuda.h>

#include "gk_vocab.cuh"

namespace gk {

enum Product { kLogits, kLogitsKeep, kAgain, kDw, kDh };

constexpr int kTileM = 256, kTileN = 256, kBlockK = 64, kStages = 6;
constexpr int kOperandBytes = 128 * kBlockK * 2;            // one operand's share of a CTA in a block
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kProductSmem = kStages * kStageBytes + 1024;  // and the alignment of the first block
constexpr int kProductThreads = 256;
constexpr int kRasterRows = 8;   // row tiles that are walked together: 8 x 9 tiles at once share operands in L2
static_assert(kVocabTile == kTileN, "a tile of logits has one maximum and one sum a row");

// ---------------------------------------------------------------------------
// PTX
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded: gives up after two seconds, or 2^24 polls, whichever is first.
__device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity) {
    const unsigned long long t0 = global_timer_ns();
    for (int i = 0; i < (1 << 24); ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 63) == 63 && global_timer_ns() - t0 > 2000000000ull) return false;
    }
    return false;
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
#pragma unroll 1
    for (int i = 0; i < 16; ++i)
        if (mbar_try(bar, parity)) return true;
    return mbar_wait_slow(bar, parity);
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar_cluster) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar_cluster) : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives at the barrier of this offset in both CTAs once the products issued so far are done.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
        ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// 32 columns of this thread's lane.  All lanes of the warp take part, whatever rows they have.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr) : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// Shared-memory descriptors, 128-byte swizzle.  K-major: rows of 128 bytes (64 values of the summed
// axis), groups of 8 rows 1024 bytes apart; 16 values further along the summed axis are 32 bytes
// further.  MN-major: rows of 128 bytes hold 64 values along M or N for one value of the summed
// axis; the next 64 are a box (64 rows, 8192 bytes) away, the next 8 of the summed axis 1024
// bytes; 16 further along the summed axis are 2048 bytes.
template <bool MN>
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    const uint64_t lead = MN ? 8192 / 16 : 1, stride = 1024 / 16;
    return (uint64_t)((addr & 0x3ffff) >> 4) | lead << 16 | stride << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

struct ProductArgs {
    VocabCall c;
    int64_t v0, v1;
    int first;       // kDh: overwrite the partial sums
    int splits;      // kDh: parts of the summed axis
    int wide;        // kDw: rows of dw start on 16-byte boundaries
};

template <int P, bool F16, bool EDGE>
__device__ __forceinline__ void read_logits(const ProductArgs& p, uint32_t tmem, int64_t row, int n_valid, int64_t col0, int cols) {
    const VocabCall& c = p.c;
    float v[32];
    float m = -INFINITY;
#pragma unroll 1
    for (int ch = 0; ch < kTileN / 32; ++ch) {
        tmem_ld32(tmem + ch * 32, v);
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (!EDGE || ch * 32 + i < cols) m = fmaxf(m, v[i]);
    }
    const float ref = m == -INFINITY ? 0.f : m;   // all -inf: every term is exp(-inf)
    const float step = -c.zscale * kept_steps<F16>();
    float s[4] = {};
    uint4* to = (uint4*)(c.e + row * c.vb + (col0 - p.v0));
#pragma unroll 1
    for (int ch = 0; ch < kTileN / 32; ++ch) {
        tmem_ld32(tmem + ch * 32, v);
        unsigned code[16];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float d = v[i] - ref;
            const float e = exp2_fast(d * c.zscale);
            if (!EDGE || ch * 32 + i < cols) s[i & 3] += e;
            if constexpr (P == kLogitsKeep) {
                // 2^23 + x has x in its low bits; 65535 steps stand for themselves and more
                const unsigned x = __float_as_uint(fminf(fmaf(d, step, 8388608.f), 8388608.f + 65535.f));
                if (i & 1) code[i >> 1] = __byte_perm(code[i >> 1], x, 0x5410);
                else code[i >> 1] = x;
            }
        }
        if constexpr (P == kLogitsKeep) {
            if (row < n_valid) {
#pragma unroll
                for (int i = 0; i < 4; ++i) to[ch * 4 + i] = make_uint4(code[4 * i], code[4 * i + 1], code[4 * i + 2], code[4 * i + 3]);
            }
        }
    }
    if (row < n_valid) c.part[col0 / kVocabTile * c.n_pad + row] = make_float2(m * c.zscale, (s[0] + s[1]) + (s[2] + s[3]));
}

template <bool F16>
__device__ __forceinline__ void read_gradients(const ProductArgs& p, uint32_t tmem, int64_t row, int n_valid, int64_t col0) {
    const VocabCall& c = p.c;
    VocabRow vr = {};
    if (row < n_valid) vr = c.row[row];
    uint4* to = (uint4*)(c.e + row * c.vb + (col0 - p.v0));
#pragma unroll 1
    for (int ch = 0; ch < kTileN / 32; ++ch) {
        float v[32];
        tmem_ld32(tmem + ch * 32, v);
        unsigned o[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float a = vr.coef * exp2_fast(fmaf(v[2 * i], c.zscale, -vr.lse2));
            const float b = vr.coef * exp2_fast(fmaf(v[2 * i + 1], c.zscale, -vr.lse2));
            o[i] = row < n_valid ? pack16<F16>(a, b) : 0u;    // rows up to the padding are summed over by dw
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) to[ch * 4 + i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
    }
}

template <bool F16>
__device__ __forceinline__ void read_dw(const ProductArgs& p, uint32_t tmem, int64_t row, int64_t rows, int64_t col0, bool empty) {
    const VocabCall& c = p.c;
    const float inv = c.ctl->inv_scale;
    uint16_t* to = (uint16_t*)c.dw + (p.v0 + row) * c.lddw + col0;
#pragma unroll 1
    for (int ch = 0; ch < kTileN / 32; ++ch) {
        if (col0 + ch * 32 >= c.D) break;
        float v[32];
        tmem_ld32(tmem + ch * 32, v);
        if (row >= rows) continue;
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = empty ? 0.f : v[i] * inv;
        if (p.wide && col0 + ch * 32 + 32 <= c.D) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                ((uint4*)to)[ch * 4 + i] = make_uint4(pack16<F16>(v[8 * i], v[8 * i + 1]), pack16<F16>(v[8 * i + 2], v[8 * i + 3]),
                                                      pack16<F16>(v[8 * i + 4], v[8 * i + 5]), pack16<F16>(v[8 * i + 6], v[8 * i + 7]));
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (col0 + ch * 32 + i < c.D) to[ch * 32 + i] = to16<F16>(v[i]);
        }
    }
}

__device__ __forceinline__ void read_dh(const ProductArgs& p, uint32_t tmem, int64_t row, int n_valid, int64_t col0, int split, bool empty) {
    const VocabCall& c = p.c;
    float4* to = (float4*)(c.dhp + ((int64_t)split * c.n_pad + row) * c.Dp + col0);
#pragma unroll 1
    for (int ch = 0; ch < kTileN / 32; ++ch) {
        if (col0 + ch * 32 >= c.Dp) break;
        float v[32];
        tmem_ld32(tmem + ch * 32, v);
        if (row >= n_valid) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float4 x = empty ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            if (!p.first) {
                const float4 y = to[ch * 8 + i];
                x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
            }
            to[ch * 8 + i] = x;
        }
    }
}

// The tiles of a call in the order in which the clusters take them.
struct Tiles {
    int64_t tm, tn, total;
    int kb, splits;
    __device__ __forceinline__ void at(int64_t t, int64_t& m, int64_t& n, int& split) const {
        const int64_t per = tm * tn;
        split = (int)(t / per);
        t -= split * per;
        const int64_t band = t / (kRasterRows * tn), m0 = band * kRasterRows;
        const int64_t rows = tm - m0 < kRasterRows ? tm - m0 : kRasterRows;
        t -= band * kRasterRows * tn;
        m = m0 + t % rows;
        n = t / rows;
    }
    __device__ __forceinline__ void blocks(int split, int& k0, int& k1) const {
        k0 = (int)((int64_t)kb * split / splits);
        k1 = (int)((int64_t)kb * (split + 1) / splits);
    }
};

template <int P, bool F16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
k_vocab_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ ProductArgs p) {
    constexpr bool kMnA = P == kDw, kMnB = P == kDw || P == kDh;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bar_full[kStages], bar_empty[kStages], bar_sum[2], bar_free[2], bar_drain;
    __shared__ uint32_t tmem_slot;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t stage0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const VocabCall& c = p.c;
    const int n_valid = c.ctl->n_valid;

    Tiles tiles;
    {
        const int64_t nv = p.v1 - p.v0, rows = ((int64_t)n_valid + kTileM - 1) / kTileM;
        tiles.tm = P == kDw ? (nv + kTileM - 1) / kTileM : rows;
        tiles.tn = P == kDw || P == kDh ? (c.D + kTileN - 1) / kTileN : (nv + kTileN - 1) / kTileN;
        const int64_t K = P == kDw ? n_valid : P == kDh ? nv : c.D;
        tiles.kb = (int)((K + kBlockK - 1) / kBlockK);
        tiles.splits = P == kDh ? p.splits : 1;
        tiles.total = tiles.tm * tiles.tn * tiles.splits;
    }
    const int64_t cluster = blockIdx.x >> 1, clusters = gridDim.x >> 1;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&bar_full[s]), 1);
            mbar_init(smem_u32(&bar_empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&bar_sum[b]), 1);
            mbar_init(smem_u32(&bar_free[b]), 8);     // four warps of each CTA
        }
        mbar_init(smem_u32(&bar_drain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_slot;

    bool ok = true;
    if (warp == 0) {
        // producer: this CTA's 128 rows of A and of B; the leader's barrier counts both CTAs' bytes
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            for (int64_t t = cluster; t < tiles.total && ok; t += clusters) {
                int64_t m, n;
                int split, k0, k1;
                tiles.at(t, m, n, split);
                tiles.blocks(split, k0, k1);
                const int ma = (int)(m * kTileM + rank * 128), nb = (int)(n * kTileN + rank * 128);
                for (int k = k0; k < k1; ++k) {
                    if (!(ok = mbar_wait(smem_u32(&bar_empty[stage]), phase ^ 1))) break;
                    const uint32_t full = smem_u32(&bar_full[stage]);
                    if (rank == 0) mbar_expect(full, 2 * kStageBytes);
                    const uint32_t bar = in_cta(full, 0);
                    const uint32_t a = stage0 + stage * kStageBytes, b = a + kOperandBytes;
                    if constexpr (kMnA) {
                        tma_load(a, &map_a, ma, k * kBlockK, bar);
                        tma_load(a + 8192, &map_a, ma + 64, k * kBlockK, bar);
                    } else {
                        tma_load(a, &map_a, k * kBlockK, ma, bar);
                    }
                    const int vrow = (P == kDh ? (int)p.v0 : 0) + k * kBlockK;
                    if constexpr (kMnB) {
                        tma_load(b, &map_b, nb, vrow, bar);
                        tma_load(b + 8192, &map_b, nb + 64, vrow, bar);
                    } else {
                        tma_load(b, &map_b, k * kBlockK, (int)p.v0 + nb, bar);
                    }
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                }
            }
            if (!ok && rank == 0)   // the copies in flight land before the memory is given back
                for (int s = 0; s < kStages; ++s) mbar_wait(smem_u32(&bar_full[s]), s < stage ? phase : phase ^ 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            constexpr uint32_t idesc = 1u << 4 | (F16 ? 0u : 1u) << 7 | (F16 ? 0u : 1u) << 10 | (kMnA ? 1u : 0u) << 15 |
                                       (kMnB ? 1u : 0u) << 16 | (uint32_t)(kTileN / 8) << 17 | (uint32_t)(kTileM / 16) << 24;
            int stage = 0, buf = 0;
            uint32_t phase = 0, free_phase = 0;
            for (int64_t t = cluster; t < tiles.total && ok; t += clusters) {
                int64_t m, n;
                int split, k0, k1;
                tiles.at(t, m, n, split);
                tiles.blocks(split, k0, k1);
                if (!(ok = mbar_wait(smem_u32(&bar_free[buf]), free_phase ^ 1))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int k = k0; k < k1; ++k) {
                    if (!(ok = mbar_wait(smem_u32(&bar_full[stage]), phase))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t a = stage0 + stage * kStageBytes, b = a + kOperandBytes;
#pragma unroll
                    for (int j = 0; j < kBlockK / 16; ++j)
                        mma_pair(tmem + buf * kTileN, operand_desc<kMnA>(a + j * (kMnA ? 2048 : 32)),
                                 operand_desc<kMnB>(b + j * (kMnB ? 2048 : 32)), idesc, k > k0 || j > 0);
                    commit_pair(smem_u32(&bar_empty[stage]));
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                }
                if (!ok) break;
                commit_pair(smem_u32(&bar_sum[buf]));
                if (++buf == 2) { buf = 0; free_phase ^= 1; }
            }
            if (!ok) {   // products in flight end before the tensor memory is freed
                commit_pair(smem_u32(&bar_drain));
                mbar_wait(smem_u32(&bar_drain), 0);
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        const int quarter = warp & 3;    // the tensor memory lanes this warp can read
        int buf = 0;
        uint32_t phase = 0;
        for (int64_t t = cluster; t < tiles.total; t += clusters) {
            int64_t m, n;
            int split, k0, k1;
            tiles.at(t, m, n, split);
            tiles.blocks(split, k0, k1);
            ok = mbar_wait(smem_u32(&bar_sum[buf]), phase);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t from = tmem + buf * kTileN + ((uint32_t)(quarter * 32) << 16);
            const int64_t row = m * kTileM + rank * 128 + quarter * 32 + lane, col0 = n * kTileN;
            if constexpr (P == kLogits || P == kLogitsKeep) {
                const int64_t left = p.v1 - p.v0 - col0;
                if (left >= kTileN) read_logits<P, F16, false>(p, from, row, n_valid, p.v0 + col0, kTileN);
                else read_logits<P, F16, true>(p, from, row, n_valid, p.v0 + col0, (int)left);
            } else if constexpr (P == kAgain) {
                read_gradients<F16>(p, from, row, n_valid, p.v0 + col0);
            } else if constexpr (P == kDw) {
                read_dw<F16>(p, from, row, p.v1 - p.v0, col0, k0 == k1);
            } else {
                read_dh(p, from, row, n_valid, col0, split, k0 == k1);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(in_cta(smem_u32(&bar_free[buf]), 0));
            if (++buf == 2) { buf = 0; phase ^= 1; }
        }
    }
    if (!ok) atomicOr(&c.ctl->status, (unsigned)GK_DEV_TIMEOUT);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();
    if (warp == 2) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeFn encode_fn() {
    static EncodeFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return (EncodeFn) nullptr;
        }
        return (EncodeFn)p;
    }();
    return fn;
}

// Rows of `cols` 16-bit values, `pitch` values apart, in boxes of 64 values and `box_rows` rows.
// Every x a kernel starts a box at is a multiple of 64 values, so every copy starts on 16 bytes.
static int make_map(CUtensorMap* map, bool f16, const void* base, int64_t cols, int64_t rows, int64_t pitch, int box_rows) {
    EncodeFn fn = encode_fn();
    if (!fn) return cuda_fail(cudaErrorNotSupported);
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(2 * pitch)};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, steps[2] = {1, 1};
    const CUresult r = fn(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base),
                          dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? GK_OK : cuda_fail(cudaErrorInvalidValue);
}

template <int P, bool F16>
static int launch_product(const ProductArgs& p, int sm_count, cudaStream_t st) {
    const VocabCall& c = p.c;
    const void* w = c.wc ? (const void*)c.wc : c.w;
    const int64_t ldw = c.wc ? c.Dp : c.ldw, nv = p.v1 - p.v0;
    CUtensorMap a, b;
    int rc;
    if (P == kDw) {
        rc = make_map(&a, c.f16, c.e, nv, c.n_pad, c.vb, 64);
        if (rc == GK_OK) rc = make_map(&b, c.f16, c.hc, c.Dp, c.n_pad, c.Dp, 64);
    } else if (P == kDh) {
        rc = make_map(&a, c.f16, c.e, nv, c.n_pad, c.vb, 128);
        if (rc == GK_OK) rc = make_map(&b, c.f16, w, c.D, c.V, ldw, 64);
    } else {
        rc = make_map(&a, c.f16, c.hc, c.Dp, c.n_pad, c.Dp, 128);
        if (rc == GK_OK) rc = make_map(&b, c.f16, w, c.D, c.V, ldw, 128);
    }
    if (rc != GK_OK) return rc;
    const int64_t tm = ((P == kDw ? nv : c.n) + kTileM - 1) / kTileM;
    const int64_t tn = ((P == kDw || P == kDh ? c.D : nv) + kTileN - 1) / kTileN;
    const int64_t pairs = tm * tn * (P == kDh ? p.splits : 1);
    const int64_t most = sm_count / 2 > 0 ? sm_count / 2 : 1;
    GK_CUDA_TRY(cudaFuncSetAttribute(k_vocab_product<P, F16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem));
    k_vocab_product<P, F16><<<(unsigned)(2 * (pairs < most ? pairs : most)), kProductThreads, kProductSmem, st>>>(a, b, p);
    GK_CUDA_TRY(cudaGetLastError());
    note_launch();
    return GK_OK;
}

template <int P>
static int launch(const VocabCall& c, int64_t v0, int64_t v1, bool first, int sm_count, cudaStream_t st) {
    ProductArgs p;
    p.c = c;
    p.v0 = v0;
    p.v1 = v1;
    p.first = first;
    p.splits = c.splits > 0 ? c.splits : 1;
    p.wide = (((uintptr_t)c.dw | (uintptr_t)(2 * c.lddw)) & 15) == 0;
    return c.f16 ? launch_product<P, true>(p, sm_count, st) : launch_product<P, false>(p, sm_count, st);
}

int launch_vocab_logits(const VocabCall& c, int64_t v0, int64_t v1, bool keep, int sm_count, cudaStream_t st) {
    return keep ? launch<kLogitsKeep>(c, v0, v1, true, sm_count, st) : launch<kLogits>(c, v0, v1, true, sm_count, st);
}
int launch_vocab_again(const VocabCall& c, int64_t v0, int64_t v1, int sm_count, cudaStream_t st) {
    return launch<kAgain>(c, v0, v1, true, sm_count, st);
}
int launch_vocab_dw(const VocabCall& c, int64_t v0, int64_t v1, int sm_count, cudaStream_t st) {
    return launch<kDw>(c, v0, v1, true, sm_count, st);
}
int launch_vocab_dh(const VocabCall& c, int64_t v0, int64_t v1, bool first, int sm_count, cudaStream_t st) {
    return launch<kDh>(c, v0, v1, first, sm_count, st);
}

int vocab_dh_splits(int64_t n, int64_t D, int64_t vb, int sm_count) {
    (void)n; (void)D; (void)vb; (void)sm_count;
    return 1;
}

}  // namespace gk
