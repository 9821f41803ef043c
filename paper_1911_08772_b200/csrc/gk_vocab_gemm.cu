// The products of the vocabulary head (gk_vocab.cu), simplest form: one CTA a 64 x 64 tile of the
// result, operands read through their strides into shared memory, fp32 multiply-adds.
#include "gk_vocab.cuh"

namespace gk {

enum Product { kLogits, kLogitsKeep, kAgain, kDw, kDh };

template <int P, bool F16>
__global__ void __launch_bounds__(256) k_product(VocabCall c, int64_t v0, int64_t v1, bool first) {
    __shared__ float as[16][65], bs[16][65], tile[64][65];
    const int n_valid = c.ctl->n_valid;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const uint16_t* w = (const uint16_t*)(c.wc ? c.wc : c.w);
    const int64_t ldw = c.wc ? c.Dp : c.ldw;
    const int64_t m0 = (int64_t)blockIdx.x * 64, n0 = (int64_t)blockIdx.y * 64;
    // sizes and strides of A (M x K) and B (N x K)
    const int64_t nv = v1 - v0;
    const int64_t M = P == kDw ? nv : n_valid;
    const int64_t N = P == kDw || P == kDh ? c.D : nv;
    const int64_t Kd = P == kDw ? n_valid : P == kDh ? nv : c.D;
    const uint16_t* A = P == kDw || P == kDh ? c.e : c.hc;
    const int64_t ams = P == kDw ? 1 : P == kDh ? c.vb : c.Dp, aks = P == kDw ? c.vb : 1;
    const uint16_t* B = P == kDw ? c.hc : w + v0 * ldw;
    const int64_t bns = P == kDw || P == kDh ? 1 : ldw, bks = P == kDw ? c.Dp : P == kDh ? ldw : 1;
    if (m0 >= M) return;
    float acc[4][4] = {};
    for (int64_t k0 = 0; k0 < Kd; k0 += 16) {
        for (int i = tid; i < 64 * 16; i += 256) {
            const int r = i >> 4, k = i & 15;
            as[k][r] = m0 + r < M && k0 + k < Kd ? from16<F16>(A[(m0 + r) * ams + (k0 + k) * aks]) : 0.f;
            bs[k][r] = n0 + r < N && k0 + k < Kd ? from16<F16>(B[(n0 + r) * bns + (k0 + k) * bks]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(as[k][ty * 4 + i], bs[k][tx * 4 + j], acc[i][j]);
        __syncthreads();
    }
    if constexpr (P == kDw || P == kDh) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t r = m0 + ty * 4 + i, col = n0 + tx * 4 + j;
                if (r >= M || col >= N) continue;
                if constexpr (P == kDw) ((uint16_t*)c.dw)[(v0 + r) * c.lddw + col] = to16<F16>(acc[i][j] * c.ctl->inv_scale);
                else {
                    float* p = c.dhp + r * c.Dp + col;
                    *p = first ? acc[i][j] : *p + acc[i][j];
                }
            }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) tile[ty * 4 + i][tx * 4 + j] = acc[i][j] * c.zscale;
        __syncthreads();
        const int64_t row = m0 + tid;
        if (tid < 64 && row < M) {
            const int cols = (int)(N - n0 < 64 ? N - n0 : 64);
            if constexpr (P == kAgain) {
                const VocabRow vr = c.row[row];
                for (int j = 0; j < 64; ++j)
                    c.e[row * c.vb + n0 + j] = j < cols ? to16<F16>(vr.coef * exp2_fast(tile[tid][j] - vr.lse2)) : (uint16_t)0;
            } else {
                float m = -INFINITY, s = 0.f;
                for (int j = 0; j < cols; ++j) m = fmaxf(m, tile[tid][j]);
                const float ref = m == -INFINITY ? 0.f : m;
                for (int j = 0; j < 64; ++j) {
                    const float e = j < cols ? exp2_fast(tile[tid][j] - ref) : 0.f;
                    s += e;
                    if constexpr (P == kLogitsKeep) c.e[row * c.vb + n0 + j] = to16<F16>(e);
                }
                c.part[((v0 + n0) / kVocabTile) * c.n_pad + row] = make_float2(m, s);
            }
        }
    }
}

template <int P>
static int launch(const VocabCall& c, int64_t v0, int64_t v1, bool first, cudaStream_t st) {
    const int64_t M = P == kDw ? v1 - v0 : c.n, N = P == kDw || P == kDh ? c.D : v1 - v0;
    const dim3 grid((unsigned)((M + 63) / 64), (unsigned)((N + 63) / 64));
    if (c.f16) k_product<P, true><<<grid, 256, 0, st>>>(c, v0, v1, first);
    else k_product<P, false><<<grid, 256, 0, st>>>(c, v0, v1, first);
    GK_CUDA_TRY(cudaGetLastError());
    note_launch();
    return GK_OK;
}

int launch_vocab_logits(const VocabCall& c, int64_t v0, int64_t v1, bool keep, int, cudaStream_t st) {
    return keep ? launch<kLogitsKeep>(c, v0, v1, true, st) : launch<kLogits>(c, v0, v1, true, st);
}
int launch_vocab_again(const VocabCall& c, int64_t v0, int64_t v1, int, cudaStream_t st) { return launch<kAgain>(c, v0, v1, true, st); }
int launch_vocab_dw(const VocabCall& c, int64_t v0, int64_t v1, int, cudaStream_t st) { return launch<kDw>(c, v0, v1, true, st); }
int launch_vocab_dh(const VocabCall& c, int64_t v0, int64_t v1, bool first, int, cudaStream_t st) { return launch<kDh>(c, v0, v1, first, st); }
int vocab_dh_splits(int64_t, int64_t, int64_t, int) { return 1; }

}  // namespace gk
