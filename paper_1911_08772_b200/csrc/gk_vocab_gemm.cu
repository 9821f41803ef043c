// The products of the vocabulary head (gk_vocab.cu) on the fifth-generation tensor cores.
//
// One persistent kernel and its uses.  A pair of SMs (a cluster of two CTAs) computes a tile of 256 rows of the
// result with tcgen05.mma.cta_group::2; each CTA holds 128 rows of A, half of the tile's rows of B, and the fp32 sums
// of its 128 rows in tensor memory.  Operands arrive by TMA in blocks of 64 along the summed axis, 192 KB of them in
// flight a CTA.  One warp sends for blocks, one issues products, eight read the sums out.  Bound by the tensor
// pipes, and those by the power limit: in 4096 x 2048 x 50000 the logits kept them 89 to 95 % busy and the gradients 95 %,
// at 1.4 to 1.5 GHz.
//
// Narrow tiles (256 columns, six blocks of 32 KB in flight): one half of the tensor memory is summed into while
// the other is read out.  Logits always are; they are summed in chunks (kChunk), which take turns on the halves.
// Wide tiles (512 columns, four blocks of 48 KB, three quarters of the bytes a product): gradients where
// launch_time expects them to be faster; 8192 x 4096 x 128000 took 20.2 ms a call with them, 23.0 with narrow
// ones on the same GPU (19.6 to 21.9 ms on others).  Their sums take all of the tensor memory, so the two halves of a tile are summed out of step at its
// ends: the first is ahead by up to four blocks at the end of a tile, so that it is read out while
// the second catches up, and again at the start of the next tile, while the second is read out.  (The logits
// of 4096 x 4096 x 32000 took 713 us in wide tiles and 749 in narrow ones, when they were not summed in chunks.)
//
// The readers copy 128 columns of 32 rows to registers and give the tensor memory back before they work on them.
//
//   use          A (M x K)            B (N x K)            what the readout does
//   kLogits      hc  rows x D         w   columns x D      maximum and sum of 128 columns per row
//   kLogitsKeep  the same                                  and the logits, as 16-bit steps below that
//                                                          maximum
//   kAgain       the same                                  logit gradients, the log-sum-exp being known
//   kGrads, dh   e   rows x columns   w^T  D x columns     16-bit rows of dh, or fp32 partial sums of them
//   kGrads, dw   e^T columns x rows   hc^T D x rows        16-bit rows of dw
//
// The two gradients are tiles of one launch, dh's long ones first, so that they fill the SMs together.
// e, hc and w are stored once, by rows; where the summed axis is not the contiguous one the
// operand is read as it lies (MN-major descriptors) instead of being transposed in memory.
// Results leave through shared memory, 32 rows x 128 bytes a warp, as TMA stores: a thread has a row of
// its own, and a store by all of them would be to 32 rows at once.
#include <cuda.h>

#include <atomic>

#include "gk_vocab.cuh"

namespace gk {

enum Product { kLogits, kLogitsKeep, kAgain, kGrads };

constexpr int kTileM = 256, kHalfN = 256, kTileN = 2 * kHalfN, kBlockK = 64;
constexpr int kOperandBytes = 128 * kBlockK * 2;            // a CTA's share of A, or of a half of B, in a block
constexpr int kBlockBytes = 12 * kOperandBytes;             // four blocks of a wide tile, six of a narrow one
constexpr int kMaxStages = 6;
// Logits are summed over 12 blocks (768 of D) at a time in tensor memory, and the chunks are added up in fp32
// registers: the tensor memory's sums are not rounded to nearest but lean one way, by more the longer they are.
// Losses and log-sum-exps of 8192 x 4096 x 128000 were off by up to 3.4e-6 of the largest in one piece, and are
// by 3e-7 to 6e-7, as a sum in fp32 is.  (dh and dw are rounded to 16 bits, which hides it.)
constexpr int kChunk = 12;
constexpr int kReaders = 8;                                 // warps that read the sums out
constexpr int kStagingBytes = 32 * 128;                     // of each of them
constexpr int kProductSmem = kBlockBytes + kReaders * kStagingBytes + 1024;   // and the alignment of the first block
constexpr int kProductThreads = 128 + 32 * kReaders;
constexpr int kRasterRows = 8;   // row tiles that are walked together: 8 x 9 tiles at once share operands in L2
static_assert(kVocabTile == 128, "a reading warp's columns have one maximum and one sum a row");

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
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000000) : "memory");
    return ok != 0;
}
// The same without waiting.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded: gives up after `limit` clocks, or 2^24 polls, whichever is first.
constexpr long long kWaitClocks = 1ll << 32;       // about two seconds
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, long long limit) {
    if (mbar_try(bar, parity)) return true;
    const long long t0 = clock64();
#pragma unroll 1
    for (int i = 0; i < (1 << 24); ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 63) == 63 && clock64() - t0 > limit) return false;
    }
    return false;
}
// The whole warp waits and the outcome is a vote: the loops run over values that the compiler knows to be the
// same in all lanes, and one elected lane only issues.  (Loops run by lane 0 alone could not keep the tensor pipe
// fed: 61 % busy, 4096 x 4096 x 32000.)
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, long long limit) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, limit));
}
__device__ __forceinline__ bool elected() {
    uint32_t p;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar_cluster) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar_cluster) : "memory");
}
// Descriptors as their lower words (address, leading distance); the upper words are constants.
__device__ __forceinline__ void mma_pair(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %5, 0;\n"
        "mov.b64 a, {%1, %3};\nmov.b64 b, {%2, %3};\n"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %4, p;\n}"
        ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// Arrives at the barrier of this offset in both CTAs once the products issued so far are done.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
        ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// 16 or 128 columns of this thread's lane.  All lanes of the warp take part, whatever rows they have.
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
          "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld128(uint32_t addr, float (&v)[128]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x128.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63, "
        "%64, %65, %66, %67, %68, %69, %70, %71, %72, %73, %74, %75, %76, %77, %78, %79, "
        "%80, %81, %82, %83, %84, %85, %86, %87, %88, %89, %90, %91, %92, %93, %94, %95, "
        "%96, %97, %98, %99, %100, %101, %102, %103, %104, %105, %106, %107, %108, %109, %110, %111, "
        "%112, %113, %114, %115, %116, %117, %118, %119, %120, %121, %122, %123, %124, %125, %126, %127}, [%128];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
          "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
          "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
          "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]),
          "=f"(v[32]), "=f"(v[33]), "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]),
          "=f"(v[40]), "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]),
          "=f"(v[48]), "=f"(v[49]), "=f"(v[50]), "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]),
          "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63]),
          "=f"(v[64]), "=f"(v[65]), "=f"(v[66]), "=f"(v[67]), "=f"(v[68]), "=f"(v[69]), "=f"(v[70]), "=f"(v[71]),
          "=f"(v[72]), "=f"(v[73]), "=f"(v[74]), "=f"(v[75]), "=f"(v[76]), "=f"(v[77]), "=f"(v[78]), "=f"(v[79]),
          "=f"(v[80]), "=f"(v[81]), "=f"(v[82]), "=f"(v[83]), "=f"(v[84]), "=f"(v[85]), "=f"(v[86]), "=f"(v[87]),
          "=f"(v[88]), "=f"(v[89]), "=f"(v[90]), "=f"(v[91]), "=f"(v[92]), "=f"(v[93]), "=f"(v[94]), "=f"(v[95]),
          "=f"(v[96]), "=f"(v[97]), "=f"(v[98]), "=f"(v[99]), "=f"(v[100]), "=f"(v[101]), "=f"(v[102]), "=f"(v[103]),
          "=f"(v[104]), "=f"(v[105]), "=f"(v[106]), "=f"(v[107]), "=f"(v[108]), "=f"(v[109]), "=f"(v[110]), "=f"(v[111]),
          "=f"(v[112]), "=f"(v[113]), "=f"(v[114]), "=f"(v[115]), "=f"(v[116]), "=f"(v[117]), "=f"(v[118]), "=f"(v[119]),
          "=f"(v[120]), "=f"(v[121]), "=f"(v[122]), "=f"(v[123]), "=f"(v[124]), "=f"(v[125]), "=f"(v[126]), "=f"(v[127])
        : "r"(addr) : "memory");
}
// A warp's 32 rows x 128 bytes in shared memory to global memory: 16-byte words are stored at
// (word ^ row mod 8), the 128-byte swizzle of the tensor map.
__device__ __forceinline__ void stage_word(uint32_t staging, int row, int word, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                 ::"r"(staging + row * 128 + ((word ^ (row & 7)) << 4)), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// the staging memory may be written again
__device__ __forceinline__ void stage_reuse(int lane) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
}
__device__ __forceinline__ void stage_store(uint32_t staging, int lane, const CUtensorMap* map, int x, int y) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];"
                     ::"l"(map), "r"(x), "r"(y), "r"(staging) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
__device__ __forceinline__ void stage_add(uint32_t staging, int lane, const CUtensorMap* map, int x, int y) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];"
                     ::"l"(map), "r"(x), "r"(y), "r"(staging) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}

// Shared-memory descriptors, 128-byte swizzle.  K-major: rows of 128 bytes (64 values of the summed
// axis), groups of 8 rows 1024 bytes apart; 16 values further along the summed axis are 32 bytes
// further.  MN-major: rows of 128 bytes hold 64 values along M or N for one value of the summed
// axis; the next 64 are a box (64 rows, 8192 bytes) away, the next 8 of the summed axis 1024
// bytes; 16 further along the summed axis are 2048 bytes.
template <bool MN>
__device__ __forceinline__ uint32_t operand_lo(uint32_t addr) {
    return (addr & 0x3ffff) >> 4 | (MN ? 8192u / 16 : 1u) << 16;
}
constexpr uint32_t kOperandHi = 1024 / 16 | 1u << 14 | 2u << 29;

struct ProductArgs {
    VocabCall c;
    int64_t v0, v1;
    int narrow;      // tiles of 256 columns instead of 512
    int first;       // dh: overwrite the partial sums
    long long wait_clocks;   // limit of every wait
    int extra_arrivals;      // test hook: arrivals the readers wait for that never come
    int splits;      // dh: parts of the summed axis
    int direct;      // dh: one part and one piece, 16-bit rows are stored at once
    int wide;        // dw: rows start and end on 16-byte boundaries
    int dh_unit, dw_unit;   // values in the boundary that rows start on: 1, 2, 4, 8
};

// What a reading warp finishes: 128 columns of 32 rows.
struct Patch {
    uint32_t tmem;       // its lanes and first column
    uint32_t staging;
    int lane;
    int64_t row0;        // of the warp; the thread's row is row0 + lane
    int64_t col0;        // of the 128
    int64_t cols;        // columns of the result from col0 on (may be more than 128, or none)
    int row;                 // kLogits, kLogitsKeep: the row's class, or the row's number with the caller
    unsigned pairs;          // its pairs in the 128 columns: the first's number + 2^16 how many
    int next;                // column of the first
};

// A row's class, or its teacher's pairs in ascending order, are met one patch of columns at a time: the logit at each is
// taken as it passes.  Taken from the same sums as the log-sum-exp, its error is that of the term it is in there, and
// goes out of the loss of a confident row (a dot product of its own left losses off by 1e-6 of the largest).
// Where a teacher's pairs are is in a table that k_vocab_teacher made (searching the row's pairs instead, six
// dependent loads by 32 rows apart, took 2048 x 2048 x 32000 with 64 pairs 746 us a call, the table 722).  What is
// found of them depends on one load after another, which are sent a chunk of sums apart and not waited for
// between: 728 us with all of them before the first sums, 716 so.
__device__ __forceinline__ void find_row(const VocabCall& c, Patch& w, int n_valid) {
    const int64_t row = w.row0 + w.lane;
    w.row = 0;
    w.pairs = 0;
    w.next = 0x7fffffff;
    if (row < n_valid) w.row = c.target ? c.cls[row] : c.row_of[row];
}
__device__ __forceinline__ void find_pairs(const VocabCall& c, Patch& w, int n_valid) {
    if (w.row0 + w.lane < n_valid && !c.target) w.pairs = c.pairs_in[w.col0 / kVocabTile * c.n_pad + w.row];
}
__device__ __forceinline__ void find_first(const VocabCall& c, Patch& w, int n_valid) {
    if (c.target) {
        if (w.row0 + w.lane < n_valid && w.row >= w.col0 && w.row < w.col0 + kVocabTile) {
            w.pairs = 1u << 16;
            w.next = w.row;
        }
    } else if (w.pairs >> 16) {
        w.next = c.t_idx[(int64_t)w.row * c.K + (w.pairs & 0xffff)];
    }
}
// `v`: the patch's columns; a register cannot be chosen at run time, so stretches of 32 columns with a pair in
// any of the warp's rows go through the staging memory.
__device__ __forceinline__ void take_pairs(const VocabCall& c, const Patch& w, const float (&v)[128]) {
    const int64_t row = w.row0 + w.lane;
    const int32_t* pairs = c.t_idx + (int64_t)w.row * c.K;       // used with more than one
    int j = (int)(w.pairs & 0xffff), next = w.next;
    const int pairs_end = j + (int)(w.pairs >> 16);
#pragma unroll
    for (int part = 0; part < 4; ++part) {
        const int from = (int)w.col0 + part * 32;
        const int end = from + (int)(w.cols - part * 32 < 32 ? w.cols - part * 32 : 32);
        if (__any_sync(0xffffffffu, next < end)) {
            stage_reuse(w.lane);
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                const float* x = v + part * 32 + g * 4;
                stage_word(w.staging, w.lane, g, __float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
            }
            while (next < end) {         // a row's own values: nothing to wait for
                const int col = next - from;
                float z;
                asm volatile("ld.shared.f32 %0, [%1];"
                             : "=f"(z) : "r"(w.staging + w.lane * 128 + (((col >> 2) ^ (w.lane & 7)) << 4) + (col & 3) * 4) : "memory");
                const int at = j++;
                next = j < pairs_end ? pairs[j] : 0x7fffffff;
                c.zt[row * c.K + at] = z;
            }
            __syncwarp();
        }
    }
}

// The readers work on 128 columns in registers: the tensor memory is free for the next tile's sums as soon as
// it has been copied (read out 16 columns at a time, a wide tile of 32 blocks took 24.2 us, 17.5 of them
// sums).  Columns past the result's end hold -inf in the uses that make logits.
template <int P, bool F16>
__device__ __forceinline__ void read_logits(const ProductArgs& p, const Patch& w, const CUtensorMap* out, int n_valid, float (&v)[128]) {
    const VocabCall& c = p.c;
    const int64_t row = w.row0 + w.lane;
    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < 128; ++i) top[i & 3] = fmaxf(top[i & 3], v[i]);
    const float m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    const float ref = m == -INFINITY ? 0.f : m;   // all -inf: every term is exp(-inf)
    float s[4] = {};
#pragma unroll
    for (int ch = 0; ch < 2; ++ch) {
        if constexpr (P == kLogitsKeep) stage_reuse(w.lane);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            unsigned code[4];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = (v[ch * 64 + g * 8 + i] - ref) * c.zscale;
                s[i & 3] += exp2_fast(d);
                if constexpr (P == kLogitsKeep) {
                    const unsigned x = kept_code<F16>(d);
                    if (i & 1) code[i >> 1] = __byte_perm(code[i >> 1], x, 0x5410);
                    else code[i >> 1] = x;
                }
            }
            if constexpr (P == kLogitsKeep) stage_word(w.staging, w.lane, g, code[0], code[1], code[2], code[3]);
        }
        if constexpr (P == kLogitsKeep)
            if (ch * 64 < w.cols) stage_store(w.staging, w.lane, out, (int)(w.col0 - p.v0) + ch * 64, (int)w.row0);
    }
    if (row < n_valid) c.part[w.col0 / kVocabTile * c.n_pad + row] = make_float2(m * c.zscale, (s[0] + s[1]) + (s[2] + s[3]));
}

template <bool F16>
__device__ __forceinline__ void read_gradients(const ProductArgs& p, const Patch& w, const CUtensorMap* out, int n_valid, float (&v)[128]) {
    const VocabCall& c = p.c;
    const int64_t row = w.row0 + w.lane;
    VocabRow vr = {};
    if (row < n_valid) vr = c.row[row];
#pragma unroll
    for (int ch = 0; ch < 2; ++ch) {
        if (ch * 64 >= w.cols) break;
        stage_reuse(w.lane);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            unsigned o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = vr.coef * exp2_fast(fmaf(v[ch * 64 + g * 8 + 2 * i], c.zscale, -vr.lse2));
                const float b = vr.coef * exp2_fast(fmaf(v[ch * 64 + g * 8 + 2 * i + 1], c.zscale, -vr.lse2));
                o[i] = row < n_valid ? pack16<F16>(a, b) : 0u;    // rows up to the padding are summed over by dw
            }
            stage_word(w.staging, w.lane, g, o[0], o[1], o[2], o[3]);
        }
        stage_store(w.staging, w.lane, out, (int)(w.col0 - p.v0) + ch * 64, (int)w.row0);
    }
}

// A warp's 32 rows x 64 16-bit columns from its staging memory to rows on boundaries of VEC values, VEC a lane:
// one row at a time by two values, two by four, four by eight; four steps' loads go before their stores.  The
// widest that the rows allow: with the 3000-byte rows of 700 x 1500 x 10000, both gradients took 62 us by two
// values and 50 by four.
// `to`: column 0 of the 64 in the result's row 0; `row`: the thread's own row there, -1: nowhere.
template <int VEC>
__device__ __forceinline__ void store_rows(uint32_t staging, int lane, uint16_t* to, int64_t ld, int row, int64_t cols) {
    constexpr int kLanes = 64 / VEC, kRows = 32 / kLanes, kSteps = 32 / kRows, kBatch = kSteps < 4 ? kSteps : 4;
    __syncwarp();
    const int col = lane % kLanes * VEC;
    const bool whole = col + VEC <= cols;
#pragma unroll 1
    for (int s0 = 0; s0 < kSteps; s0 += kBatch) {
        uint32_t x[kBatch][4];
        int at[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int r = (s0 + i) * kRows + lane / kLanes;
            at[i] = __shfl_sync(0xffffffffu, row, r);
            const uint32_t from = staging + r * 128 + (((col >> 3) ^ (r & 7)) << 4) + (col & 7) * 2;
            if constexpr (VEC == 2) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x[i][0]) : "r"(from) : "memory");
            else if constexpr (VEC == 4) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x[i][0]), "=r"(x[i][1]) : "r"(from) : "memory");
            else asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[i][0]), "=r"(x[i][1]), "=r"(x[i][2]), "=r"(x[i][3]) : "r"(from) : "memory");
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            uint16_t* p = to + at[i] * ld + col;
            if (at[i] < 0) continue;
            if (whole && (VEC > 2 || ((uintptr_t)p & 3) == 0)) {
                if constexpr (VEC == 2) *(uint32_t*)p = x[i][0];
                else if constexpr (VEC == 4) *(uint2*)p = make_uint2(x[i][0], x[i][1]);
                else *(uint4*)p = make_uint4(x[i][0], x[i][1], x[i][2], x[i][3]);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (col + e < cols) p[e] = (uint16_t)(x[i][e / 2] >> (e % 2 * 16));
            }
        }
    }
    __syncwarp();
}
// `unit`: the boundary in values that all rows start on.
__device__ __forceinline__ void store_rows(uint32_t staging, int lane, uint16_t* to, int64_t ld, int row, int64_t cols, int unit) {
    if (unit >= 8) store_rows<8>(staging, lane, to, ld, row, cols);
    else if (unit >= 4) store_rows<4>(staging, lane, to, ld, row, cols);
    else store_rows<2>(staging, lane, to, ld, row, cols);
}

template <bool F16>
__device__ __forceinline__ void stage16(const Patch& w, const float* v, float f, bool empty) {
    stage_reuse(w.lane);
#pragma unroll
    for (int g = 0; g < 8; ++g) {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = empty ? 0u : pack16<F16>(v[8 * g + 2 * i] * f, v[8 * g + 2 * i + 1] * f);
        stage_word(w.staging, w.lane, g, x[0], x[1], x[2], x[3]);
    }
}

template <bool F16>
__device__ __forceinline__ void read_dw(const ProductArgs& p, const Patch& w, const CUtensorMap* out, bool empty, float (&v)[128]) {
    const VocabCall& c = p.c;
    const float inv = c.ctl->inv_scale;
    const int64_t rows = p.v1 - p.v0 - w.row0;   // rows of the result from the warp's first on
    if (rows <= 0) return;
#pragma unroll
    for (int ch = 0; ch < 2; ++ch) {
        if (ch * 64 >= w.cols) break;
        stage16<F16>(w, v + ch * 64, inv, empty);
        if (p.wide) stage_store(w.staging, w.lane, out, (int)w.col0 + ch * 64, (int)w.row0);
        else store_rows(w.staging, w.lane, (uint16_t*)c.dw + (p.v0 + w.row0) * c.lddw + w.col0 + ch * 64, c.lddw, w.lane < rows ? w.lane : -1,
                        w.cols - ch * 64, p.dw_unit);
    }
}

template <bool F16>
__device__ __forceinline__ void read_dh(const ProductArgs& p, const Patch& w, const CUtensorMap* out, int n_valid, int split, float (&v)[128]) {
    const VocabCall& c = p.c;
    if (w.row0 >= n_valid) return;
    const int64_t row = w.row0 + w.lane;
    if (p.direct) {
        float f = 0.f;
        int to = -1;
        if (row < n_valid) {
            f = c.ctl->inv_scale;
            to = c.row_of[row];
        }
#pragma unroll
        for (int ch = 0; ch < 2; ++ch) {
            if (ch * 64 >= w.cols) break;
            stage16<F16>(w, v + ch * 64, f, false);
            store_rows(w.staging, w.lane, (uint16_t*)c.dh + w.col0 + ch * 64, c.lddh, to, w.cols - ch * 64, p.dh_unit);
        }
        return;
    }
    const int y = (int)(split * c.n_pad + w.row0);
#pragma unroll
    for (int part = 0; part < 4; ++part) {
        if (part / 2 * 64 >= w.cols) break;
        stage_reuse(w.lane);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            const float* x = v + part * 32 + g * 4;
            stage_word(w.staging, w.lane, g, __float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
        }
        const int x0 = (int)w.col0 + part * 32;
        // one tile adds to an element and launches follow one another: the order is fixed
        if (p.first) stage_store(w.staging, w.lane, out, x0, y);
        else stage_add(w.staging, w.lane, out, x0, y);
    }
}

// The tiles of a call in the order in which the clusters take them.  In 32 bits (the sums of 2^31 tiles'
// rows would take more memory than there is): 64-bit divisions cost a microsecond a tile.
struct Tiles {
    uint32_t tm, tn, total;
    int kb, splits;
    __device__ __forceinline__ void at(uint32_t t, int& m, int& n, int& split) const {
        const uint32_t per = tm * tn;
        uint32_t s = 0;
        if (splits > 1) {
            s = t / per;
            t -= s * per;
        }
        const uint32_t band = t / (kRasterRows * tn), m0 = band * kRasterRows;
        const uint32_t rows = tm - m0 < kRasterRows ? tm - m0 : kRasterRows;
        t -= m0 * tn;
        const uint32_t col = t / rows;
        m = (int)(m0 + t - col * rows);
        n = (int)col;
        split = (int)s;
    }
    __device__ __forceinline__ void blocks(int split, int& k0, int& k1) const {
        k0 = splits > 1 ? kb * split / splits : 0;
        k1 = splits > 1 ? kb * (split + 1) / splits : kb;
    }
};

__device__ __forceinline__ Tiles make_tiles(int64_t rows, int64_t cols, int64_t K, int width, int splits) {
    Tiles t;
    t.tm = (uint32_t)((rows + kTileM - 1) / kTileM);
    t.tn = (uint32_t)((cols + width - 1) / width);
    t.kb = (int)((K + kBlockK - 1) / kBlockK);
    t.splits = splits;
    t.total = t.tm * t.tn * splits;
    return t;
}

// A cluster's share of the tiles, in the order in which it takes them.  The first kind (dh's) is dealt
// out in turn, so that some clusters have one more than the others; the others then get as much of the
// second kind (dw's) as makes up for it, and the rest is dealt in turn again, beginning with them.
struct Deal {
    int n1, n2, clusters, heavy;      // heavy: clusters with one more of the first kind
    int extra;                        // tiles of the second kind that make up for it
    int index, at;                    // the cluster, its next tile of the present kind
    bool light;
    int kind;                             // 0: first, 1: extra, 2: rest
    __device__ __forceinline__ Deal(const Tiles& a, const Tiles& b, int cluster, int clusters_) {
        n1 = (int)a.total;
        n2 = (int)b.total;
        clusters = clusters_;
        heavy = n1 % clusters;
        light = cluster >= heavy;
        // a tile costs its blocks and about two more
        const int each = heavy ? (a.kb / a.splits + 2) / (b.kb + 2) : 0;
        extra = each * (clusters - heavy);
        if (extra > n2) extra = n2;
        at = cluster;
        kind = 0;
        index = cluster;
    }
    // The next tile: `dw`: of the second kind; false: none left.
    __device__ __forceinline__ bool next(uint32_t& t, bool& dw) {
        if (kind == 0) {
            if (at < n1) { t = (uint32_t)at; dw = false; at += clusters; return true; }
            kind = 1;
            at = light ? index - heavy : n2;
        }
        if (kind == 1) {
            if (at < extra) { t = (uint32_t)at; dw = true; at += clusters - heavy; return true; }
            kind = 2;
            at = extra + (light ? index - heavy : index + clusters - heavy);
        }
        if (at >= n2) return false;
        t = (uint32_t)at;
        dw = true;
        at += clusters;
        return true;
    }
};

// map_a2, map_b2, map_out2: dw's operands and result in kGrads.
template <int P, bool F16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
k_vocab_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_a2,
                const __grid_constant__ CUtensorMap map_b2, const __grid_constant__ CUtensorMap map_out2,
                const __grid_constant__ ProductArgs p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bar_full[kMaxStages], bar_empty[kMaxStages], bar_sum[2], bar_free[2], bar_drain;
    __shared__ uint32_t tmem_slot;
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = (int)__reduce_max_sync(0xffffffffu, (unsigned)tid >> 5);
    const uint32_t rank = cluster_rank();
    const uint32_t stage0 = (smem_u32(smem_raw) + 1023u) & ~1023u, staging0 = stage0 + kBlockBytes;
    const VocabCall& c = p.c;
    const bool narrow = P != kGrads || p.narrow;
    const int width = narrow ? kHalfN : kTileN;
    const int stages = narrow ? 6 : 4;
    const uint32_t stage_bytes = (narrow ? 2 : 3) * kOperandBytes;
    const int cluster = (int)(blockIdx.x >> 1), clusters = (int)(gridDim.x >> 1);

    if (tid == 32) {       // the descriptors are on their way while the rest is set up
        for (const CUtensorMap* m : {&map_a, &map_b, &map_out})
            asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
        if (P == kGrads)
            for (const CUtensorMap* m : {&map_a2, &map_b2, &map_out2})
                asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
    }
    if (tid == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            mbar_init(smem_u32(&bar_full[s]), 1);
            mbar_init(smem_u32(&bar_empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&bar_sum[b]), 1 + p.extra_arrivals);
            mbar_init(smem_u32(&bar_free[b]), 2 * kReaders);
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
    after_previous();

    const int n_valid = (int)__reduce_max_sync(0xffffffffu, (unsigned)c.ctl->n_valid);   // one value, known as such

    const int64_t nv = p.v1 - p.v0, n_cols = P == kGrads ? c.D : nv;      // columns of the result
    const Tiles tiles = P == kGrads ? make_tiles(c.dh ? n_valid : 0, c.D, nv, width, p.splits) : make_tiles(n_valid, nv, c.D, width, 1);
    const Tiles tiles2 = make_tiles(P == kGrads && c.dw ? nv : 0, c.D, n_valid, width, 1);

    bool ok = true;
    if (warp == 0) {
        // producer: this CTA's 128 rows of A and of each half of B; the leader's barrier counts both CTAs' bytes
        int stage = 0;
        uint32_t phase = 0;
        uint32_t t;
        bool dw;
        for (Deal deal(tiles, tiles2, cluster, clusters); ok && deal.next(t, dw);) {
            int m, n, split, k0, k1;
            if (P != kGrads) dw = false;
            (dw ? tiles2 : tiles).at(t, m, n, split);
            (dw ? tiles2 : tiles).blocks(split, k0, k1);
            const bool two = !narrow && n * kTileN + kHalfN < n_cols;
            const int ma = (int)(m * kTileM + rank * 128), nb = (int)(n * width + rank * 128);
            const uint32_t bytes = 2 * (two ? 3 : 2) * kOperandBytes;
            for (int k = k0; k < k1; ++k) {
                if (!(ok = warp_wait(smem_u32(&bar_empty[stage]), phase ^ 1, p.wait_clocks))) break;
                if (elected()) {
                    const uint32_t full = smem_u32(&bar_full[stage]);
                    if (rank == 0) mbar_expect(full, bytes);
                    const uint32_t bar = in_cta(full, 0);
                    const uint32_t a = stage0 + stage * stage_bytes, b = a + kOperandBytes;
                    if constexpr (P == kGrads) {
                        // B lies by the summed axis in both; A in dw
                        const CUtensorMap* mb = dw ? &map_b2 : &map_b;
                        const int y = (dw ? 0 : (int)p.v0) + k * kBlockK;
                        if (dw) {
                            tma_load(a, &map_a2, ma, y, bar);
                            tma_load(a + 8192, &map_a2, ma + 64, y, bar);
                        } else {
                            tma_load(a, &map_a, k * kBlockK, ma, bar);
                        }
                        tma_load(b, mb, nb, y, bar);
                        tma_load(b + 8192, mb, nb + 64, y, bar);
                        if (two) {
                            tma_load(b + kOperandBytes, mb, nb + kHalfN, y, bar);
                            tma_load(b + kOperandBytes + 8192, mb, nb + kHalfN + 64, y, bar);
                        }
                    } else {
                        tma_load(a, &map_a, k * kBlockK, ma, bar);
                        tma_load(b, &map_b, k * kBlockK, (int)p.v0 + nb, bar);
                    }
                }
                __syncwarp();
                if (++stage == stages) { stage = 0; phase ^= 1; }
            }
        }
        if (!ok && rank == 0)   // the copies in flight land before the memory is given back
            for (int s = 0; s < stages; ++s) mbar_wait(smem_u32(&bar_full[s]), s < stage ? phase : phase ^ 1, p.wait_clocks);
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr bool kMnB = P == kGrads;
            constexpr uint32_t kDesc = 1u << 4 | (F16 ? 0u : 1u) << 7 | (F16 ? 0u : 1u) << 10 | (kMnB ? 1u : 0u) << 16 |
                                       (uint32_t)(kHalfN / 8) << 17 | (uint32_t)(kTileM / 16) << 24;
            constexpr uint32_t step_b = (kMnB ? 2048 : 32) / 16;
            const uint32_t b0 = operand_lo<kMnB>(stage0 + kOperandBytes);
            uint32_t idesc = kDesc, step_a = 32 / 16, a0 = operand_lo<false>(stage0);
            // one block of one half, by the elected lane
            auto issue = [&](int stage, int half, bool fresh) {
                const uint32_t at = stage * (stage_bytes / 16);
                const uint32_t a = a0 + at, b = b0 + at + (narrow ? 0 : half * (kOperandBytes / 16));
                const uint32_t d = tmem + half * kHalfN;
                mma_pair(d, a, b, kOperandHi, idesc, !fresh);
#pragma unroll
                for (int j = 1; j < kBlockK / 16; ++j) mma_pair(d, a + j * step_a, b + j * step_b, kOperandHi, idesc, true);
            };
            int stage_a = 0, stage_b = 0;     // next block of the first half (of the only one), of the second half
            uint32_t phase = 0, free0 = 0, free1 = 0;
            int only = 0;                     // the half a narrow tile has
            uint32_t t;
            bool dw;
            for (Deal deal(tiles, tiles2, cluster, clusters); ok && deal.next(t, dw);) {
                int m, n, split, k0, k1;
                if (P != kGrads) dw = false;
                (dw ? tiles2 : tiles).at(t, m, n, split);
                (dw ? tiles2 : tiles).blocks(split, k0, k1);
                const int blocks = k1 - k0;
                const bool two = !narrow && n * kTileN + kHalfN < n_cols;
                if (dw) {
                    idesc = kDesc | 1u << 15;
                    step_a = 2048 / 16;
                    a0 = operand_lo<true>(stage0);
                }
                int a = 0, b = 0;             // blocks issued for each half
                int count = blocks;           // of a chunk
                auto first_half = [&](int half, bool release) {
                    ok = warp_wait(smem_u32(&bar_full[stage_a]), phase, p.wait_clocks);
                    if (!ok) return;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    if (elected()) {
                        issue(stage_a, half, a == 0);
                        if (release) commit_pair(smem_u32(&bar_empty[stage_a]));
                        if (a + 1 == count) commit_pair(smem_u32(&bar_sum[half]));
                    }
                    __syncwarp();
                    ++a;
                    if (++stage_a == stages) { stage_a = 0; phase ^= 1; }
                };
                auto second_half = [&]() {
                    if (elected()) {
                        issue(stage_b, 1, b == 0);
                        commit_pair(smem_u32(&bar_empty[stage_b]));
                        if (b + 1 == blocks) commit_pair(smem_u32(&bar_sum[1]));
                    }
                    __syncwarp();
                    ++b;
                    if (++stage_b == stages) stage_b = 0;
                };
                // the first half's sums, or a narrow tile's, have been read out
                auto wait_free = [&](int half) {
                    ok = warp_wait(smem_u32(&bar_free[half]), (half ? free1 : free0) ^ 1, p.wait_clocks);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    if (half) free1 ^= 1;
                    else free0 ^= 1;
                    if (ok && blocks == 0 && elected()) commit_pair(smem_u32(&bar_sum[half]));
                    __syncwarp();
                };
                if (!two) {
                    int left = blocks;
                    do {
                        wait_free(only);
                        count = P == kGrads || left < kChunk ? left : kChunk;
                        a = 0;
                        while (a < count && ok) first_half(only, true);
                        left -= count;
                        if (narrow) only ^= 1;
                    } while (ok && left > 0);
                    stage_b = stage_a;
                    continue;
                }
                wait_free(0);
                if (!ok) break;
                // ahead, as far as blocks are in flight, while the second half's sums are still being read out
                while (ok && a < blocks && a < stages && !__all_sync(0xffffffffu, mbar_test(smem_u32(&bar_free[1]), free1 ^ 1)))
                    first_half(0, false);
                if (ok) wait_free(1);
                if (!ok) break;
                while (b < a && a < blocks) second_half();
                while (ok && a < blocks - stages) {
                    first_half(0, false);
                    if (ok) second_half();
                }
                while (ok && a < blocks) first_half(0, false);      // ahead over the last blocks
                if (ok) while (b < blocks) second_half();
            }
            if (!ok) {   // products in flight end before the tensor memory is freed
                if (elected()) commit_pair(smem_u32(&bar_drain));
                __syncwarp();
                mbar_wait(smem_u32(&bar_drain), 0, p.wait_clocks);
            }
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, side = (warp - 4) >> 2;    // the tensor memory lanes this warp can read; its columns
        uint32_t phases = 0;    // a bit for each half
        int only = 0;           // the half a narrow tile has
        Patch w;
        w.lane = lane;
        w.staging = staging0 + (warp - 4) * kStagingBytes;
        uint32_t t;
        bool dw;
        for (Deal deal(tiles, tiles2, cluster, clusters); ok && deal.next(t, dw);) {
            int m, n, split, k0, k1;
            if (P != kGrads) dw = false;
            (dw ? tiles2 : tiles).at(t, m, n, split);
            (dw ? tiles2 : tiles).blocks(split, k0, k1);
            const bool two = !narrow && n * kTileN + kHalfN < n_cols;
            w.row0 = m * kTileM + (int)rank * 128 + quarter * 32;
            // rows that are used: those that count, and of logit gradients those that dw sums over
            const bool used_rows = P == kGrads || w.row0 < (P == kAgain ? round_up(n_valid, 64) : n_valid);
            const uint32_t lanes = tmem + side * 128 + ((uint32_t)(quarter * 32) << 16);
            float v[128];
            auto wait_sums = [&](int h) {
                ok = warp_wait(smem_u32(&bar_sum[h]), phases >> h & 1, p.wait_clocks);
                phases ^= 1u << h;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            };
            auto give_back = [&](int h) {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(in_cta(smem_u32(&bar_free[h]), 0));
            };
            if constexpr (P != kGrads) {
                const int64_t col = (int64_t)n * width + side * 128;
                w.cols = n_cols - col;
                w.col0 = p.v0 + col;
                const bool used = used_rows && w.cols > 0, pairs = P != kAgain && used && w.row0 < n_valid;
                if (pairs) find_row(c, w, n_valid);
                for (int done = 0; done < k1 - k0; done += kChunk) {
                    wait_sums(only);
                    if (!ok) break;
                    w.tmem = lanes + only * kHalfN;
                    if (used) {
                        __syncwarp();
                        if (done == 0) {
                            tmem_ld128(w.tmem, v);
                            if (pairs) find_pairs(c, w, n_valid);
                        } else {
                            if (pairs && done == kChunk) find_first(c, w, n_valid);
                            __syncwarp();       // lanes part there, and the copies below take the whole warp
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                float x[16];
                                tmem_ld16(w.tmem + i * 16, x);
#pragma unroll
                                for (int j = 0; j < 16; ++j) v[i * 16 + j] += x[j];
                            }
                        }
                    }
                    give_back(only);
                    only ^= 1;
                }
                if (!ok) break;
                if (pairs && k1 - k0 <= kChunk) find_first(c, w, n_valid);
                if (pairs) take_pairs(c, w, v);
                if (used) {
                    if (P != kAgain && w.cols < 128) {
#pragma unroll
                        for (int i = 0; i < 128; ++i) v[i] = i < w.cols ? v[i] : -INFINITY;
                    }
                    if constexpr (P == kLogits || P == kLogitsKeep) read_logits<P, F16>(p, w, &map_out, n_valid, v);
                    else read_gradients<F16>(p, w, &map_out, n_valid, v);
                }
            } else {
#pragma unroll 1
                for (int h = only; h < (two ? 2 : only + 1); ++h) {
                    w.col0 = (int64_t)n * width + (two ? h * kHalfN : 0) + side * 128;
                    w.cols = n_cols - w.col0;
                    wait_sums(h);
                    if (!ok) break;
                    __syncwarp();
                    tmem_ld128(lanes + h * kHalfN, v);
                    give_back(h);
                    if (w.cols > 0) {
                        if (dw) read_dw<F16>(p, w, &map_out2, k0 == k1, v);
                        else read_dh<F16>(p, w, &map_out, n_valid, split, v);
                    }
                }
                if (narrow) only ^= 1;
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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

// Rows of `cols` values, `pitch` values apart, in boxes of 128 bytes and `box_rows` rows.  Every x
// a kernel starts a box at is a multiple of 64 16-bit or 32 fp32 values, so every copy starts on 16 bytes.
enum Element { kBf16, kF16, kF32 };
static int make_map(CUtensorMap* map, Element type, const void* base, int64_t cols, int64_t rows, int64_t pitch, int box_rows) {
    EncodeFn fn = encode_fn();
    if (!fn) return cuda_fail(cudaErrorNotSupported);
    const int size = type == kF32 ? 4 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(size * pitch)};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / size), (cuuint32_t)box_rows}, steps[2] = {1, 1};
    const CUtensorMapDataType t = type == kF32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                : type == kF16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const CUresult r = fn(map, t, 2, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? GK_OK : cuda_fail(cudaErrorInvalidValue);
}

// An estimate of a launch's time in us, for choosing between tiles and parts: what the busiest pair of SMs does,
// and 4 us to fill and empty.  A tile takes its blocks of 64 or its readout, whichever is longer, and what of
// them does not overlap.  As measured: a block 0.60 us in a wide tile, 0.34 in a
// narrow one; a readout 6 and 3.4 us, by rows that do not start on 16 bytes 10 and 5.  Whole calls with wide and with
// narrow tiles for the gradients: 8192 x 4096 x 128000 20160 : 22950 us, 1024 x 1024 x 32000 216 : 215,
// 300 x 512 x 20000 75 : 63.  The first kind of tile (dh's, in `splits` parts) is dealt out before the second
// (dw's), which evens the shares out.
struct Share {
    int64_t rows, cols, kb;
    bool unaligned;
};
static double launch_time(const Share& first, int splits, const Share& second, bool narrow, int sm_count) {
    const int64_t width = narrow ? kHalfN : kTileN, most = sm_count / 2 > 0 ? sm_count / 2 : 1;
    const int64_t n1 = (first.rows + kTileM - 1) / kTileM * ((first.cols + width - 1) / width) * splits;
    const int64_t n2 = (second.rows + kTileM - 1) / kTileM * ((second.cols + width - 1) / width);
    auto tile = [&](int64_t kb, bool unaligned) {
        const double us = (double)kb * (narrow ? 0.34 : 0.60);
        const double read = unaligned ? (narrow ? 5.0 : 10.0) : narrow ? 3.4 : 6.0;
        return (us > read ? us : read) + (narrow ? 0.5 : 1.5);
    };
    const double t1 = tile((first.kb + splits - 1) / splits, first.unaligned), t2 = tile(second.kb, second.unaligned);
    const double rounds1 = (double)((n1 + most - 1) / most), all = ((double)n1 * t1 + (double)n2 * t2) / (double)most;
    const double longest = rounds1 * t1, even = n2 ? all + 0.5 * t2 : 0.0;
    return (longest > even ? longest : even) + 4.0;
}

template <int P, bool F16>
static int launch_product(ProductArgs p, int sm_count, cudaStream_t st) {
    const VocabCall& c = p.c;
    const void* w = c.wc ? (const void*)c.wc : c.w;
    const int64_t ldw = c.wc ? c.Dp : c.ldw, nv = p.v1 - p.v0;
    const Element type = F16 ? kF16 : kBf16;
    CUtensorMap a, b, out, a2, b2, out2;
    Share first, second = {0, 1, 1, false};
    int rc;
    if (P == kGrads) {
        rc = make_map(&a, type, c.e, nv, c.n_pad, c.vb, 128);
        if (rc == GK_OK) rc = make_map(&b, type, w, c.D, c.V, ldw, 64);
        out = a;     // not used by direct stores
        if (rc == GK_OK && c.dh && !p.direct) rc = make_map(&out, kF32, c.dhp, c.Dp, p.splits * c.n_pad, c.Dp, 32);
        if (rc == GK_OK) rc = make_map(&a2, type, c.e, nv, c.n_pad, c.vb, 64);
        if (rc == GK_OK) rc = make_map(&b2, type, c.hc, c.Dp, c.n_pad, c.Dp, 64);
        out2 = a2;   // rows on other boundaries are stored without a map
        if (rc == GK_OK && c.dw && p.wide) rc = make_map(&out2, type, (const uint16_t*)c.dw + p.v0 * c.lddw, c.D, nv, c.lddw, 32);
        first = {c.dh ? c.n : 0, c.D, (nv + kBlockK - 1) / kBlockK, false};
        second = {c.dw ? nv : 0, c.D, (c.n + kBlockK - 1) / kBlockK, !p.wide};
    } else {
        rc = make_map(&a, type, c.hc, c.Dp, c.n_pad, c.Dp, 128);
        if (rc == GK_OK) rc = make_map(&b, type, w, c.D, c.V, ldw, 128);
        out = a;     // kLogits keeps nothing
        if (rc == GK_OK && P != kLogits) rc = make_map(&out, type, c.e, nv, c.n_pad, c.vb, 32);
        a2 = b2 = out2 = a;
        first = {c.n, nv, (c.D + kBlockK - 1) / kBlockK, false};
    }
    if (rc != GK_OK) return rc;
    p.narrow = P != kGrads || launch_time(first, p.splits, second, true, sm_count) < launch_time(first, p.splits, second, false, sm_count);
    const int64_t width = p.narrow ? kHalfN : kTileN;
    const int64_t pairs = (first.rows + kTileM - 1) / kTileM * ((first.cols + width - 1) / width) * p.splits +
                          (second.rows + kTileM - 1) / kTileM * ((second.cols + width - 1) / width);
    const int64_t most = sm_count / 2 > 0 ? sm_count / 2 : 1;
    static std::atomic<unsigned long long> ready{0};      // devices on which the kernel may have its shared memory
    int dev = 0;
    GK_CUDA_TRY(cudaGetDevice(&dev));
    if (dev > 63 || !(ready.load() >> dev & 1)) {
        GK_CUDA_TRY(cudaFuncSetAttribute(k_vocab_product<P, F16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem));
        if (dev < 64) ready.fetch_or(1ull << dev);
    }
    GK_CUDA_TRY(launch_next(k_vocab_product<P, F16>, dim3((unsigned)(2 * (pairs < most ? pairs : most))), kProductThreads, kProductSmem, st,
                            a, b, out, a2, b2, out2, p));
    note_launch();
    return GK_OK;
}

template <int P>
static int launch(const VocabCall& c, int64_t v0, int64_t v1, bool first, int sm_count, cudaStream_t st) {
    ProductArgs p;
    p.c = c;
    p.v0 = v0;
    p.v1 = v1;
    p.narrow = 0;
    p.first = first;
    p.extra_arrivals = host_knob(kKnobExtraArrivals) > 0 ? 1 : 0;
    p.wait_clocks = p.extra_arrivals ? 1ll << 27 : kWaitClocks;
    // (a part without a block would have no sums: the last piece of the vocabulary can be shorter than the parts, which
    // the first, a full one, has four blocks for each of; parts that it does not reach keep the sums they have)
    const int64_t blocks = (v1 - v0 + kBlockK - 1) / kBlockK;
    p.splits = P == kGrads && c.splits > 0 ? (int)(c.splits < blocks ? c.splits : blocks) : 1;
    p.direct = c.dhp == nullptr;
    // (the copies' hardware cuts a row's end in steps of 16 bytes, so the rows' length counts too)
    p.wide = (((uintptr_t)c.dw | (uintptr_t)(2 * c.lddw) | (uintptr_t)(2 * c.D)) & 15) == 0;
    auto unit = [](const void* base, int64_t ld) {
        const uintptr_t x = (uintptr_t)base | (uintptr_t)(2 * ld);
        return (x & 15) == 0 ? 8 : (x & 7) == 0 ? 4 : (x & 3) == 0 ? 2 : 1;
    };
    p.dh_unit = unit(c.dh, c.lddh);
    p.dw_unit = unit(c.dw, c.lddw);
    return c.f16 ? launch_product<P, true>(p, sm_count, st) : launch_product<P, false>(p, sm_count, st);
}

int launch_vocab_logits(const VocabCall& c, int64_t v0, int64_t v1, bool keep, int sm_count, cudaStream_t st) {
    return keep ? launch<kLogitsKeep>(c, v0, v1, true, sm_count, st) : launch<kLogits>(c, v0, v1, true, sm_count, st);
}
int launch_vocab_again(const VocabCall& c, int64_t v0, int64_t v1, int sm_count, cudaStream_t st) {
    return launch<kAgain>(c, v0, v1, true, sm_count, st);
}
int launch_vocab_grads(const VocabCall& c, int64_t v0, int64_t v1, bool first, int sm_count, cudaStream_t st) {
    return launch<kGrads>(c, v0, v1, first, sm_count, st);
}

// Into how many parts the summed axis of dh is split.  dh has few tiles (rows / 256 x D / 512) and a
// long sum, so without parts most pairs of SMs would idle; parts cost a write and a read of fp32 sums,
// taken at 5 TB/s, and a launch that adds them.
int vocab_dh_splits(int64_t n, int64_t D, int64_t vb, DwRows dw, int sm_count) {
    const Share first = {n, D, (vb + kBlockK - 1) / kBlockK, false};
    const Share second = {dw == DwRows::none ? 0 : vb, D, (n + kBlockK - 1) / kBlockK, dw == DwRows::unaligned};
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 32 && (s == 1 || s * 4 <= first.kb); ++s) {
        const double wide = launch_time(first, s, second, false, sm_count), narrow = launch_time(first, s, second, true, sm_count);
        const double us = (wide < narrow ? wide : narrow) + (s > 1 ? 4.0 + (double)s * (double)n * (double)D * 8.0 / 5e6 : 0.0);
        if (s == 1 || us < least) { least = us; best = s; }
    }
    return best;
}

}  // namespace gk
