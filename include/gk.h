/*
 * gk.h -- C ABI of the B200 error-compensated Gaussian_k gradient sparsifier
 *         and exact Top_k selection (arXiv 1911.08772).
 *
 * Conventions for every call
 *   - Pointers marked DEVICE are caller-owned global memory of the CUDA device
 *     that is current when the call is made; pointers marked HOST are ordinary
 *     host memory.  The library never frees or keeps caller pointers.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default
 *     stream).  All device work is enqueued on it and the call returns without
 *     synchronising, unless stated otherwise.
 *   - Vectors are fp32, indices int32, so 1 <= d <= 2^31 - 1.  Base pointers of
 *     g, eps and u must be 16-byte aligned.  Inputs must be finite.
 *   - The library owns a scratch workspace per (device, stream), created
 *     by the first call that needs it (cudaMalloc; use gk_reserve to do that
 *     ahead of time) and kept: small for the sparsifiers and gk_grad_*, up to gk_vocab_set_budget
 *     and more, in a block of its own, for the vocabulary head.  Two calls that overlap on the GPU must use different
 *     streams.  Calls of several host threads are safe on any streams: those
 *     on one stream are enqueued whole, one after the other in no promised
 *     order, and each thread's cudaStreamPerThread has a workspace of its own.
 *     (gk_sparsify_static's scratch is one for all: see there.)
 *   - A call that does not synchronise and has no workspace to allocate can be
 *     captured in a graph, which stays good until a call that needs more
 *     replaces the workspace of the stream that it was captured on.  All
 *     graphs captured on a stream share its workspace, on whatever streams
 *     they are replayed: their replays must not overlap.
 *   - Return value: GK_OK or a negative gk_status for errors detected on the
 *     host before anything is enqueued.  Conditions found on the device
 *     (truncated output, a bounded wait that ran out, a malformed segment
 *     table) are reported in gk_stats.status, never by a trap or a hang.
 */
#ifndef GK_H_
#define GK_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef void* gk_stream_t; /* a cudaStream_t */

typedef enum gk_status {
    GK_OK = 0,
    GK_ERR_NULL = -1,      /* a required pointer is NULL */
    GK_ERR_SIZE = -2,      /* d < 1 or d > 2^31 - 1, or S < 1 */
    GK_ERR_K = -3,         /* k < 1 or k > d; gk_vocab_logprob: k < 0, k > V or k > 128 */
    GK_ERR_ALIGN = -4,     /* g / eps / u not 16-byte aligned; gk_vocab_*, gk_grad_*: a pointer off its type's boundary */
    GK_ERR_ALIAS = -5,     /* g overlaps eps; gk_vocab_logprob_grad, gk_grad_clip: an output overlaps what it must not */
    GK_ERR_CUDA = -6,      /* a CUDA runtime call failed (see gk_last_cuda_error) */
    GK_ERR_NOMEM = -7,     /* workspace allocation failed */
    GK_ERR_CAPACITY = -8,  /* gk_set_capacity: cap < 0 */
    GK_ERR_LIMIT = -9,     /* size beyond a fixed built-in limit */
    GK_ERR_TYPE = -10,     /* gk_vocab_*, gk_grad_*: not one of the element types the call takes */
    GK_ERR_STRIDE = -11,   /* gk_vocab_*: a row stride shorter than the row */
    GK_ERR_TEMPERATURE = -12, /* gk_vocab_*: temperature or log2(e) over it not positive and finite */
    GK_ERR_NORM = -13      /* gk_grad_clip: max_norm not positive */
} gk_status;

/* Element types of the gk_vocab_* and gk_grad_* calls. */
typedef enum gk_type { GK_TYPE_F32 = 0, GK_TYPE_BF16 = 1, GK_TYPE_F16 = 2 } gk_type;

/* Values of gk_stats.status (bit flags, written by the device). */
#define GK_DEV_OK 0
#define GK_DEV_TRUNCATED 1    /* more survivors than the output capacity */
#define GK_DEV_TIMEOUT 2      /* a bounded look-back wait gave up; outputs invalid */
#define GK_DEV_BAD_SEGMENTS 4 /* seg_offsets not ascending from 0 to d, or seg_k out of range */
#define GK_DEV_BAD_SAMPLE 8   /* dgck_*: a sampled position outside [0, d) (it was clamped) */
#define GK_DEV_BAD_INDEX 16   /* gk_apply_*: a message index outside [0, d) (the entry was skipped) */

/*
 * What one Gaussian_k run decided (Algorithm 1 of the paper).  For the
 * segmented call there is one record per segment.
 */
typedef struct gk_stats {
    double mu;         /* mean of u */
    double sigma;      /* sample standard deviation of u (divisor d - 1) */
    double z;          /* Phi^-1(1 - k/d) */
    double thres0;     /* mu + sigma * z, the first threshold */
    double thr_final;  /* threshold of the mask that was returned */
    int64_t counts[4]; /* #{|u_i| > thres} seen in each executed round */
    int32_t rounds;    /* rounds executed, 0 when k >= d (everything selected) */
    int32_t status;    /* GK_DEV_* flags */
    int64_t nnz;       /* size of the returned mask (before any truncation) */
    int64_t emitted;   /* pairs actually written (= min(nnz, capacity)) */
} gk_stats;

/*
 * gk_sparsify -- one step of error-compensated sparsification, Eq. 2 of the
 * paper with Comp_k = Gaussian_k (Algorithm 1):
 *     u = g + eps;   (idx, val) = Gaussian_k(u);   eps <- u - Comp(u).
 * Gaussian_k takes mean and standard deviation of u, sets the first threshold
 * to the normal quantile at p = 1 - k/d, then for at most four rounds counts
 * #{|u_i| > thres} and halves the threshold when the count is below 2k/3,
 * multiplies it by 1.5 when above 4k/3, and stops otherwise.  The mask of the
 * last round evaluated is returned.
 *
 *   g        DEVICE in   d floats, the stochastic gradient; must not overlap eps
 *   eps      DEVICE i/o  d floats; in: residual eps_t, out: eps_{t+1}
 *                        (+0.0f at selected positions, u_i elsewhere)
 *   d, k     sizes, 1 <= k <= d
 *   idx_out  DEVICE out  capacity ints (see gk_set_capacity; default d):
 *                        positions with |u_i| > threshold, ascending
 *   val_out  DEVICE out  capacity floats: u at those positions
 *   nnz_out  DEVICE out  one int64: number of pairs written
 *   stream   the stream to enqueue on
 *
 * The number of survivors is data dependent and may be below or above k
 * (Appendix A.5 of the paper).  If it exceeds the capacity, only the first
 * `capacity` survivors in index order are written and only their eps slots are
 * cleared, so that Comp(u) + eps_{t+1} == u still holds; status gets
 * GK_DEV_TRUNCATED.
 */
int gk_sparsify(const float* g, float* eps, int64_t d, int64_t k, int32_t* idx_out,
                float* val_out, int64_t* nnz_out, gk_stream_t stream);

/*
 * gk_select -- Gaussian_k as an operator on a given vector (Algorithm 1 of the paper as
 * printed: input u, output the entries with |u_i| > threshold).  The same statistics,
 * first threshold, count-and-adjust rounds and returned mask as gk_sparsify, without the
 * accumulation before and the residual after: this is the form whose running time
 * Section 4.3 / Fig. 4 compares with Top_k and DGC_k (topk_exact and dgck_select here).
 *
 *   u        DEVICE in   d floats, not modified (16-byte aligned)
 *   d, k     sizes, 1 <= k <= d
 *   idx_out  DEVICE out  capacity ints (gk_set_capacity; default d), ascending positions
 *   val_out  DEVICE out  capacity floats: u at those positions
 *   nnz_out  DEVICE out  one int64: number of pairs written
 * Capacity rule, statistics record (gk_last_stats) and the choice of implementation
 * (gk_set_path) as for gk_sparsify.
 */
int gk_select(const float* u, int64_t d, int64_t k, int32_t* idx_out, float* val_out,
              int64_t* nnz_out, gk_stream_t stream);

/*
 * gk_sparsify_segmented -- the same step with Algorithm 1 run independently on
 * every contiguous segment [seg_offsets[s], seg_offsets[s+1]) with its own
 * mean, deviation, k_s and threshold (layer-wise selection).  The paper states
 * Algorithm 1 for the whole vector; applying it per layer is this library's
 * extension.  All S segments are processed by one batched launch per stage.
 *
 *   seg_offsets DEVICE in  S + 1 int64, seg_offsets[0] = 0 <= ... <= seg_offsets[S] = d;
 *                          boundaries need no alignment; empty segments allowed
 *   seg_k       DEVICE in  S int64, 1 <= seg_k[s] (values >= the segment length
 *                          select the whole segment)
 *   S           number of segments, 1 <= S <= 65536
 *   idx_out / val_out      as above; indices are global, segments appear in order,
 *                          so idx_out is ascending overall
 *   seg_nnz_out DEVICE out S int64: size of each segment's mask (may be NULL)
 *   nnz_out     DEVICE out one int64: total pairs written
 * A malformed table sets GK_DEV_BAD_SEGMENTS; nothing is then selected
 * (eps still receives u).
 */
int gk_sparsify_segmented(const float* g, float* eps, int64_t d, const int64_t* seg_offsets,
                          const int64_t* seg_k, int32_t S, int32_t* idx_out, float* val_out,
                          int64_t* seg_nnz_out, int64_t* nnz_out, gk_stream_t stream);

/*
 * topk_exact -- Top_k of Section 1 of the paper: the k entries of largest
 * absolute value with their indices, by radix select on the magnitude bits.
 * Entries of equal magnitude are taken in order of increasing index (+0 and
 * -0 tie).  Exactly k pairs are written, in ascending index order.
 *
 *   u        DEVICE in   d floats, not modified
 *   idx_out  DEVICE out  k ints;   val_out  DEVICE out  k floats
 */
int topk_exact(const float* u, int64_t d, int64_t k, int32_t* idx_out, float* val_out,
               gk_stream_t stream);

/*
 * topk_sparsify -- Eq. 2 of the paper with Comp_k = Top_k: u = g + eps, the exact
 * Top_k of u is written as k pairs, eps <- u - Top_k(u).  Arguments as for
 * gk_sparsify; exactly k pairs are written and *nnz_out = k.
 */
int topk_sparsify(const float* g, float* eps, int64_t d, int64_t k, int32_t* idx_out,
                  float* val_out, int64_t* nnz_out, gk_stream_t stream);

/*
 * dgck_select -- DGC_k, the hierarchical sampling selector the paper compares
 * Gaussian_k with (Section 3.3; Section 4.3 uses a 1 % sample).  The paper says
 * only that a small random sample estimates the threshold and that top-k
 * selection runs twice on subsets of the vector; the steps taken here:
 *   1. tau = the k_m-th largest of { |u[sample_idx[j]]| : j < m },
 *      k_m = ceil(k * m / d)                       (first top-k, on the sample);
 *   2. candidates = { i : |u_i| >= tau }, n of them;
 *   3. n > k: the k largest candidates, ties toward the lower index (second
 *      top-k, on the candidates); otherwise all n candidates.
 * min(n, k) pairs are written in ascending index order.
 *
 *   u          DEVICE in   d floats, not modified (16-byte aligned)
 *   sample_idx DEVICE in   m int32 positions in [0, d), repeats allowed: the random
 *                          draw is the caller's.  A position outside the range is
 *                          clamped and flagged GK_DEV_BAD_SAMPLE.
 *   m          sample size, 1 <= m <= 2^31 - 1
 *   idx_out    DEVICE out  k ints;   val_out  DEVICE out  k floats
 *   nnz_out    DEVICE out  one int64: min(n, k)
 * One cooperative kernel; vectors of more than 448 rows of 4096 elements per SM
 * (271 M elements on 148 SMs) and devices without cooperative launch return
 * GK_ERR_LIMIT.
 */
int dgck_select(const float* u, int64_t d, int64_t k, const int32_t* sample_idx, int64_t m,
                int32_t* idx_out, float* val_out, int64_t* nnz_out, gk_stream_t stream);

/*
 * dgck_sparsify -- Eq. 2 of the paper with Comp_k = DGC_k: u = g + eps (the sample
 * is taken from u), selection as in dgck_select, eps <- u - Comp(u).  g, eps as
 * for gk_sparsify; the other arguments as for dgck_select.
 */
int dgck_sparsify(const float* g, float* eps, int64_t d, int64_t k, const int32_t* sample_idx,
                  int64_t m, int32_t* idx_out, float* val_out, int64_t* nnz_out, gk_stream_t stream);

/* Synchronise `stream` and write what the last dgck_* call on it decided to HOST
 * host_out[0..3]: the fp32 bit pattern of tau, n, k_m, pairs written. */
int dgck_last_info(gk_stream_t stream, int64_t* host_out);

/*
 * gk_apply_sparse -- the model update of Eq. 2 from the P workers' messages:
 *     x <- x + alpha * sum_p Comp_k(u^p)          (alpha = -eta / P in the paper).
 * Message p is the ascending (index, value) list a sparsifier call wrote.  The
 * terms of a position are added in rank order p = 0, 1, ... in fp32 (one
 * addition per term), the sum is multiplied by alpha and added to x; positions
 * that occur in no message are not touched.  The paper does not fix the order
 * of the P terms; rank order makes the result independent of timing.
 *
 *   x          DEVICE i/o  d floats
 *   idx_lists  HOST   in   P pointers to DEVICE int32 lists, each strictly ascending;
 *   val_lists  HOST   in   P pointers to DEVICE float lists.  A list may live in
 *                          another GPU's memory that this device can address (peer
 *                          access): the kernel reads the lists with plain loads.
 *   nnz        DEVICE in   P int64: entries of each list (values above cap count as cap)
 *   P          number of messages, 1 <= P <= 64;  cap: upper bound of every nnz[p]
 * One kernel, no scratch vector, no atomics on x.  An index outside [0, d) is
 * skipped and flagged GK_DEV_BAD_INDEX in the status word gk_last_stats returns.
 *
 * gk_apply_gathered -- the same for messages in one buffer (as an all-gather
 * leaves them): list p starts at idx + p * cap and val + p * cap (DEVICE).
 */
int gk_apply_sparse(float* x, int64_t d, const int32_t* const* idx_lists, const float* const* val_lists,
                    const int64_t* nnz, int32_t P, int64_t cap, float alpha, gk_stream_t stream);
int gk_apply_gathered(float* x, int64_t d, const int32_t* idx, const float* val, const int64_t* nnz,
                      int32_t P, int64_t cap, float alpha, gk_stream_t stream);

/*
 * gk_sparsify_host -- gk_sparsify for HOST buffers (Eq. 2, Algorithm 1): copies g
 * and eps to library-owned device staging buffers, runs the step, copies
 * eps_{t+1}, the pairs and their count back, and synchronises before
 * returning.  All pointers are HOST memory (pinned memory makes the copies
 * faster); idx_out / val_out hold `capacity` entries (default d).
 */
int gk_sparsify_host(const float* g, float* eps, int64_t d, int64_t k, int32_t* idx_out,
                     float* val_out, int64_t* nnz_out, gk_stats* stats_out);

/*
 * gk_error_ratio -- the compression error ratio of Eq. 5 / Section 3.2 of the
 * paper, ||u - Comp(u)||^2 / ||u||^2, for a step that has just run (any of the
 * sparsifiers above): eps then holds u - Comp(u) with the selected slots at
 * zero, so ||u||^2 = ||eps||^2 + ||val||^2.  Hold it against 1 - k/d (Eq. 4)
 * and (1 - k/d)^2 (Theorem 1).
 *
 *   eps      DEVICE in   d floats: the residual the step left (16-byte aligned)
 *   val      DEVICE in   the selected values the step wrote
 *   nnz      DEVICE in   one int64: how many of them
 *   host_out HOST   out  3 doubles: the ratio, ||u - Comp(u)||^2, ||u||^2
 * One pass over eps in fp64, deterministic.  Enqueued on `stream`, which is then
 * synchronised.  A zero vector gives ratio 0.
 */
int gk_error_ratio(const float* eps, int64_t d, const float* val, const int64_t* nnz,
                   gk_stream_t stream, double* host_out);

/*
 * gk_histogram -- the histogram of u shown in the paper's gradient-distribution
 * figures (Section 3.1, Fig. 2; its running sum over d is the cumulative curve
 * of the appendix).  nbins equal bins starting at lo, bin width 1 / inv_w:
 *     t = (u_i - lo) * inv_w in fp32 (one subtraction, one multiplication);
 *     t < 0 counts as "below", t >= nbins (or NaN) as "above", else bin floor(t).
 *
 *   u          DEVICE in   d floats (16-byte aligned), not modified
 *   lo, inv_w  lower edge of the first bin; inv_w = nbins / (hi - lo) > 0, as a float
 *   nbins      1 <= nbins <= 8192
 *   counts_out DEVICE out  nbins + 2 int64: [0] below, [1 .. nbins] the bins,
 *                          [nbins + 1] above (zeroed by the call)
 * One pass over u, enqueued on `stream`; does not synchronise.
 */
int gk_histogram(const float* u, int64_t d, float lo, float inv_w, int32_t nbins, int64_t* counts_out,
                 gk_stream_t stream);

/*
 * gk_sparsify_static -- gk_sparsify for callers that must not allocate device
 * memory (the paper has no counterpart: this is a deployment variant of the
 * same step, not another method).  Think of a step that runs under a framework
 * allocator with a fixed budget, or of a service that bans cudaMalloc once it
 * is serving because that call stalls the whole device.  Same arguments, same
 * results and same capacity rule as gk_sparsify, but the call never reaches
 * cudaMalloc, cudaFree or any routine that allocates: its scratch is a fixed
 * 544 KB array inside the library image, present on every GPU that loads the
 * library for as long as the process lives.
 *
 * Limits: 1 <= k < d <= 2^31 - 1 (d beyond that returns GK_ERR_SIZE; k = d
 * returns GK_ERR_K: selecting everything is left to gk_sparsify); the device
 * must support cooperative launch, the launch must fit the array's 512
 * per-CTA slots, and the vector must not exceed 2^29 elements (the array has one
 * word per row of 4096 elements) nor 1024 rows per SM, else GK_ERR_LIMIT.
 *
 * The first call on a device looks up the array's device address
 * (cudaGetSymbolAddress) and keeps it; make that first call before any stream
 * capture begins.  All calls on a device share the one array, which keeps
 * whatever the previous call left in it; the call clears the words that have
 * to start at zero.  Two calls that overlap on the GPU (different streams)
 * would race on the array: keep them in order.  There is no statistics record
 * to read back for this call.
 */
int gk_sparsify_static(const float* g, float* eps, int64_t d, int64_t k, int32_t* idx_out,
                       float* val_out, int64_t* nnz_out, gk_stream_t stream);

/*
 * gk_set_params -- the two constants of Algorithm 1 that can be read in more than one way.
 *   unbiased_std  non-zero (default): "std" is the sample standard deviation, divisor d - 1
 *                 (the paper's operators are tensor-library calls whose default this is);
 *                 0: the population form, divisor d.
 *   max_rounds    rounds of the loop "for i = 0 -> 3": 4 by default (both bounds included),
 *                 1 .. 4 accepted; the mask of the last round run is returned.
 * Applies to gk_sparsify, gk_select, gk_sparsify_segmented, gk_sparsify_host and
 * gk_sparsify_static from the next call on.  Process-wide; the device-side values are set on
 * the current device.  Returns GK_ERR_SIZE for max_rounds outside 1 .. 4.
 */
int gk_set_params(int unbiased_std, int max_rounds);

/*
 * gk_vocab_loss -- softmax cross entropy at the vocabulary head of a language model, and its
 * gradient: the loss whose gradient the sparsifiers above compress (the paper's LSTM workload
 * has such a head; the paper does not treat it).  With z = h w^T, without keeping z,
 *     lse_n = log sum_v exp z_nv;   loss_n = lse_n - z_n,t(n);
 *     dz_nv = g_n (exp(z_nv - lse_n) - [v = t(n)]);   dh = dz w;   dw = dz^T h.
 * Products of 16-bit operands are summed in fp32 (logits in pieces of 768, the pieces in fp32 registers), lse
 * and loss are fp32.  The gradients go through 16 bits three times.  A logit of the vocabulary's first piece (see
 * below) is kept as a 16-bit distance from the largest of its 128 columns, which puts its probability off by at
 * most 6.8e-4 of itself (bf16) or 8.5e-5 (fp16; 2.5e-4 below 2^-8, and 2^-32 is the least); of later pieces it is
 * computed again in fp32.  dz is rounded to the operands' type, scaled so that the call's largest finite row
 * coefficient is a power of two (fp16: a row 2^-34 of it is lost).  dh and dw are rounded at the end.  Together, as
 * norms, at most 1.5 times the last rounding alone over many rows.  The same call gives the same bits; under
 * another gk_vocab_set_budget, or with one gradient instead of both, they can be others.
 *
 *   h          DEVICE in   n rows of D elements of `dtype`, row stride ldh >= D (in elements)
 *   w          DEVICE in   V rows of D elements, row stride ldw >= D.  Rows that start and end on
 *                          16-byte boundaries are read in place; otherwise the call copies w first.
 *   dtype      GK_TYPE_BF16 or GK_TYPE_F16, of h, w, dh and dw
 *   n, D, V    0 <= n <= 2^22, 1 <= D <= 2^16, 1 <= V <= 2^26
 *   target     DEVICE in   n int64 classes.  A row whose target is ignore_index, or outside
 *                          [0, V), is left out: loss 0, lse 0, a zero row in dh, no share in dw,
 *                          whatever h holds there (its infinities and NaN included), and no work.
 *   row_grad   DEVICE in   g: n floats, the gradient of each row's loss; NULL: 1 / rows that
 *                          count, the gradient of their mean
 *   loss_out, lse_out      DEVICE out  n floats each
 *   dh_out     DEVICE out  n rows of D, row stride lddh; NULL: not wanted
 *   dw_out     DEVICE out  V rows of D, row stride lddw; NULL: not wanted
 * With neither dh nor dw only the forward pass runs (scoring).  dh and dw must not overlap h, w or
 * each other.  Results do not depend on timing: no atomics on floating-point data.
 *
 * The workspace is the call's own, per (device, stream), grown on first use and kept until the process ends
 * (gk_vocab_reserve makes it ahead; a call that fits it allocates nothing).  For a capture in a graph reserve it on
 * the stream that is captured, which torch.cuda.graph makes anew unless it is given one.  The
 * largest part, with gradients, is one piece of the vocabulary as n rows of 16-bit values, bounded by
 * gk_vocab_set_budget; of the pieces after the first the product h w^T is taken twice.
 * Memory for 8 bytes a row and 128 columns (12 for gk_vocab_distill) is needed beside it.
 */
int gk_vocab_loss(const void* h, int64_t ldh, const void* w, int64_t ldw, int32_t dtype, int64_t n, int64_t D,
                  int64_t V, const int64_t* target, int64_t ignore_index, const float* row_grad, float* loss_out,
                  float* lse_out, void* dh_out, int64_t lddh, void* dw_out, int64_t lddw, gk_stream_t stream);

/*
 * gk_vocab_distill -- distillation from a teacher's top logits through the same head: each row
 * has K pairs (index, logit) of the teacher, as gk_vocab_topk writes them.  With temperature T,
 *     q_nj = exp(t_nj / T - L_n),  L_n = t_lse[n], or log sum_j exp(t_nj / T) where t_lse is NULL;
 *     lse_n = log sum_v exp(z_nv / T);
 *     loss_n = sum_j q_nj (log q_nj - z_n,i(n,j) / T + lse_n);
 *     dz_nv = (g_n / T) (exp(z_nv / T - lse_n) sum_j q_nj - sum_{j: i(n,j) = v} q_nj).
 *
 *   t_idx      DEVICE in   n x K int32 (contiguous), in any order; an index given twice counts
 *                          twice.  Rows in strictly ascending order, pairs left out last, as
 *                          gk_vocab_topk writes them, are faster: the logits at other rows' pairs
 *                          are dot products of their own (2048 x 2048 x 32000 with 64 pairs: 600
 *                          and 740 us).  Pairs with an index outside [0, V) or a logit of -inf are left
 *                          out (rows with fewer pairs are filled up with -1); a row without any
 *                          pair is left out as in gk_vocab_loss.
 *   t_val      DEVICE in   n x K floats, the teacher's logits (not divided by T)
 *   K          1 <= K <= 1024
 *   t_lse      DEVICE in   n floats, the teacher's log-sum-exp at T over its whole vocabulary
 *                          (gk_vocab_topk's lse_out): q is then the teacher's probability and
 *                          sums to at most 1.  NULL: q is normalised over the K pairs.
 *   temperature  T > 0, with a finite reciprocal
 * The other arguments as for gk_vocab_loss.
 */
int gk_vocab_distill(const void* h, int64_t ldh, const void* w, int64_t ldw, int32_t dtype, int64_t n, int64_t D,
                     int64_t V, const int32_t* t_idx, const float* t_val, int32_t K, const float* t_lse,
                     float temperature, const float* row_grad, float* loss_out, float* lse_out, void* dh_out,
                     int64_t lddh, void* dw_out, int64_t lddw, gk_stream_t stream);

/*
 * gk_vocab_topk -- the k largest logits of each row as a message for gk_vocab_distill, in the form
 * of topk_exact's: exactly k pairs a row in ascending index order, equal values taken in order of
 * increasing index (+0 and -0 tie, NaN counts as above +inf).  Values here are compared as
 * they are, not by magnitude.
 *
 *   logits     DEVICE in   n rows of V elements of `dtype` (GK_TYPE_F32, _BF16 or _F16), row stride ld >= V
 *   n, V, k    n >= 0, 1 <= V <= 2^31 - 1, 1 <= k <= min(V, 1024)
 *   temperature  T > 0 with a finite reciprocal, for lse_out only
 *   idx_out    DEVICE out  n x k int32;   val_out  DEVICE out  n x k floats
 *   lse_out    DEVICE out  n floats, log sum_v exp(logit / T); -inf for a row of nothing but
 *                          -inf.  NULL: not wanted
 */
int gk_vocab_topk(const void* logits, int64_t ld, int32_t dtype, int64_t n, int64_t V, int32_t k, float temperature,
                  int32_t* idx_out, float* val_out, float* lse_out, gk_stream_t stream);

/*
 * gk_vocab_logprob -- log probabilities of given tokens under rows of logits, with the rows' entropies and their most
 * probable tokens: what a policy or preference loss takes of its rollouts, and a server answers with.  With y = z / T,
 *     lse_n = log sum_v exp y_nv;   logp_nj = y_n,t(n,j) - lse_n;   p_nv = exp(y_nv - lse_n);
 *     entropy_n = -sum_v p_nv log p_nv;
 *     rank_n = #{v: z_nv > z_nt, or z_nv = z_nt and v < t},  t = t(n,0)   (0: the most probable).
 *
 *   logits     DEVICE in   n rows of V elements of `dtype` (any gk_type), row stride ld >= V
 *   n, V       n >= 0, 1 <= V <= 2^31 - 1
 *   token      DEVICE in   n x m int64 (contiguous), 0 <= m <= 128; NULL for m = 0.  A token outside [0, V) is left
 *                          out: logp 0.  A row that was given tokens, all of them left out, is left out itself:
 *                          zeros, rank -1, idx -1, whatever its logits hold
 *   temperature  T > 0 with a finite reciprocal
 *   k          alternatives, 0 <= k <= min(V, 128)
 *   logp_out   DEVICE out  n x m floats; NULL: not wanted (as the next three)
 *   rank_out   DEVICE out  n int32: the rank of the row's first token, in the order of idx_out; -1 where that is left
 *                          out or m = 0
 *   entropy_out, lse_out  DEVICE out  n floats each
 *   idx_out    DEVICE out  n x k int32: the k largest logits' places, the largest first, equal ones in order of
 *                          increasing index (+0 and -0 tie, NaN counts as above +inf)
 *   val_out    DEVICE out  n x k floats, their log probabilities.  Both, or k = 0
 * A row of nothing but -inf has lse -inf, entropy 0 and log probabilities -inf; +inf or NaN in a row that counts
 * gives what the formulas give with it: lse +inf, entropy NaN, log probabilities -inf (NaN at +inf); NaN everywhere.
 * One pass over the logits (two over rows whose exponents need it, at extreme temperatures or maxima); sums in fp32
 * relative to the row's maximum, of which powers below 2^-126 are nothing; no workspace; the same call gives the same
 * bits.
 *
 * gk_vocab_logprob_grad -- the gradient with respect to the logits of
 *     sum_nj a_nj logp_nj + sum_n b_n entropy_n + sum_n c_n lse_n:
 *     dz_nv = (1 / T) (sum_j a_nj ([v = t(n,j)] - p_nv) - b_n p_nv (log p_nv + entropy_n) + c_n p_nv).
 *
 *   logits, ld, dtype, n, V, token, m, temperature   as given to gk_vocab_logprob
 *   lse, entropy   DEVICE in   n floats each, what that call wrote; entropy may be NULL where entropy_grad is
 *   logp_grad  DEVICE in   a, n x m floats (those of tokens left out are not read); NULL: 0
 *   entropy_grad   DEVICE in   b, n floats; NULL: 0
 *   lse_grad   DEVICE in   c, n floats (a penalty on the log-sum-exp); NULL: 0
 *   dlogits    DEVICE out  n rows of V elements of `dtype`, row stride lddz >= V.  The logits themselves (same
 *                          pointer and stride: in place), or memory that shares nothing with them: before or behind
 *                          all of them, or, of the same stride, between their rows
 * A token given twice counts twice.  Rows left out get zeros, and so do rows whose lse is below -1e30: their masks, of
 * -inf or of fp32's or bf16's lowest value, leave nothing.  So do logits of -inf that are no token.  A row that counts
 * and whose lse is +inf or NaN gets NaN throughout.  log p is taken from lse and has its rounding, 2^-24 of |lse|.
 * Rounded once to `dtype`.  No workspace.
 */
int gk_vocab_logprob(const void* logits, int64_t ld, int32_t dtype, int64_t n, int64_t V, const int64_t* token, int32_t m,
                     float temperature, int32_t k, float* logp_out, int32_t* rank_out, float* entropy_out, float* lse_out,
                     int32_t* idx_out, float* val_out, gk_stream_t stream);
int gk_vocab_logprob_grad(const void* logits, int64_t ld, int32_t dtype, int64_t n, int64_t V, const int64_t* token,
                          int32_t m, float temperature, const float* lse, const float* entropy, const float* logp_grad,
                          const float* entropy_grad, const float* lse_grad, void* dlogits, int64_t lddz,
                          gk_stream_t stream);

/* Bytes that one piece of the vocabulary may take in the workspace of gk_vocab_loss and
 * gk_vocab_distill (default 2 GiB).  A piece has at least 256 columns.  Process-wide; returns
 * GK_ERR_CAPACITY if bytes < 0. */
int gk_vocab_set_budget(int64_t bytes);

/* Create (or grow) the workspace of (current device, stream) for gk_vocab_loss (K = 1) and
 * gk_vocab_distill calls of up to n rows and K pairs and of this D and V, at the present budget, with or
 * without gradients, with rows of w on 16-byte boundaries where D is a multiple of 8.  Synchronous.
 * gk_vocab_workspace_bytes: what that takes, on a B200. */
int gk_vocab_reserve(int64_t n, int64_t D, int64_t V, int32_t K, int grad, gk_stream_t stream);
int64_t gk_vocab_workspace_bytes(int64_t n, int64_t D, int64_t V, int32_t K, int grad);

/* Synchronise `stream` and write to HOST host_out[0..1] of the last gk_vocab_loss or
 * gk_vocab_distill call on it, one without rows included (0, 0): GK_DEV_* flags, rows that counted.
 * GK_ERR_NULL where there was no call. */
int gk_vocab_last_info(gk_stream_t stream, int64_t* host_out);

/*
 * gk_grad_norm -- the Euclidean norm over the gradients of many tensors together, and each tensor's own:
 *     norm = sqrt(sum_i sum_x g_i(x)^2);   norms_i = sqrt(sum_x g_i(x)^2).
 * What a training step looks at, and clips by, before its gradient is compressed (the paper does not treat it).
 *
 *   grads      HOST   in   T pointers to DEVICE tensors of sizes[i] contiguous elements, on an element's
 *                          boundary; NULL allowed for an empty one
 *   types      HOST   in   T gk_type: each tensor's own
 *   sizes      HOST   in   T int64, 0 <= sizes[i] <= 2^44
 *   T          0 <= T <= 65536; more than 1000 need gk_reserve(1, T) before a capture, fewer gk_reserve(1, 1)
 *   norm_out   DEVICE out  one float
 *   norms_out  DEVICE out  T floats; NULL: not wanted
 * The lists are read before the call returns (they travel as the kernel's argument); a captured call keeps them.
 * Any values: squares beyond fp32's range are taken in fp64, an infinity gives infinity, NaN gives NaN.  A tensor
 * given twice counts twice.  Sums of 32 squares (fp32) or 64 (16 bits) in fp32, the rest in fp64, in an order that the sizes, the
 * 16-byte boundaries within the tensors and the device decide: the same call gives the same bits.
 *
 * gk_grad_clip -- the gradients scaled so that their norm is at most max_norm, in place or into other tensors:
 *     out_i = c s g_i,   c = max_norm / norm where norm = |s| ||g|| is above max_norm and finite, else 1.
 * With outputs of fp32 one after the other in one buffer this is the step from a backward pass to the vector g
 * that gk_sparsify takes (local gradient clipping before compression).
 *
 *   grads, types, sizes, T   as above
 *   outs       HOST   in   T pointers to DEVICE tensors of the same sizes.  An output is its own input (same
 *                          pointer, same type: in place) or shares memory with no input and no other output
 *   out_types  HOST   in   T gk_type.  A product is taken in fp32 and rounded once to the output's type
 *   max_norm   > 0; infinity clips nothing
 *   scale      DEVICE in   s, one float, as the reciprocal of a loss scale; NULL: 1
 *   norm_in    DEVICE in   the norm, of the scaled gradients, where the caller knows it (over tensors that other
 *                          ranks hold, say); NULL: taken over these tensors
 *   norm_out   DEVICE out  one float, the norm before clipping; NULL: not wanted.  It shares memory with none of the
 *                          others, but may be norm_in, or scale where norm_in is NULL.  Scale and norm_in share
 *                          none with an output
 * A norm that is not finite as a float clips nothing (c = 1): the caller finds it in norm_out and drops the step.
 * A factor c s below 2^-126 has the absolute steps of fp32 there.  Where
 * nothing is clipped or scaled, tensors in place are not written.  One cooperative kernel (the device must support
 * that); should its bounded barrier run out, norm_out is NaN and no output is written.
 */
int gk_grad_norm(const void* const* grads, const int32_t* types, const int64_t* sizes, int32_t T, float* norm_out,
                 float* norms_out, gk_stream_t stream);
int gk_grad_clip(const void* const* grads, const int32_t* types, void* const* outs, const int32_t* out_types,
                 const int64_t* sizes, int32_t T, float max_norm, const float* scale, const float* norm_in,
                 float* norm_out, gk_stream_t stream);

/* Synchronise `stream` and write to HOST host_out[0..1] of the last gk_grad_clip call on it: GK_DEV_* flags,
 * whether it clipped.  GK_ERR_NULL where no call has made the stream's workspace. */
int gk_grad_last_info(gk_stream_t stream, int64_t* host_out);

/* Output capacity of idx_out / val_out for the sparsify calls, in pairs.
 * 0 (the default) means "d".  Process-wide; returns GK_ERR_CAPACITY if cap < 0. */
int gk_set_capacity(int64_t cap);

/*
 * Which implementation gk_sparsify, gk_select and gk_sparsify_host use.  Process-wide.
 *   0 (default)  vectors of up to 589,824 elements: one thread-block cluster of sixteen CTAs
 *                that holds u in shared memory and synchronises with cluster barriers;
 *                larger ones: one persistent cooperative kernel that keeps what fits of u in
 *                shared memory between the phases of Algorithm 1.  Falls back to path 1 where
 *                neither can be launched and for k = d.
 *   1            three kernels: accumulate + statistics, candidate counts,
 *                compaction by decoupled look-back.
 *   2            the persistent cooperative kernel at every size.
 * All give identical results.  Returns GK_ERR_SIZE for any other value.
 */
int gk_set_path(int path);

/* Create (or grow) the workspace of (current device, stream) for vectors of up
 * to d elements in up to S segments.  Synchronous; call outside timed regions
 * and before stream capture. */
int gk_reserve(int64_t d, int32_t S, gk_stream_t stream);

/* Bytes of scratch workspace a call with these sizes uses. */
int64_t gk_workspace_bytes(int64_t d, int32_t S);

/* Synchronise `stream` and copy the record of the last gk_sparsify (or the S
 * records of the last gk_sparsify_segmented) enqueued on it to HOST memory. */
int gk_last_stats(gk_stream_t stream, gk_stats* host_out);
int gk_last_segment_stats(gk_stream_t stream, int32_t S, gk_stats* host_out);

/*
 * Per-stage device timing (tracing aid, off by default; process-wide switch).
 * While enabled, every call records a CUDA event on its stream before its first
 * kernel and after each kernel.  gk_last_stage_ms synchronises the stream and
 * writes the durations in milliseconds of the stages of the last call enqueued on
 * it to HOST ms_out[0..*n_stages-1] (at most 8).  Single-kernel forms: the kernel,
 * then spans between timestamps the kernel takes itself (CTA 0 and the CTA that
 * leaves last).  gk_sparsify and gk_sparsify_segmented: accumulate incl. first
 * barrier and thresholds, counting loop, second barrier, replay of the rounds,
 * compaction, exit of the last CTA.  topk_exact and topk_sparsify: first pass,
 * barrier and first digit, second pass to second digit, third pass to third digit,
 * counts and fourth barrier, offsets and write-out, exit of the last CTA.
 * Multi-kernel forms, one value per kernel: accumulate, count, compact; for
 * Top_k three histogram passes and compact, with accumulate first in topk_sparsify.
 */
int gk_stage_timing(int enable);
int gk_last_stage_ms(gk_stream_t stream, float* ms_out, int* n_stages);

/*
 * Per-CTA trace of the last single-kernel gk_sparsify or gk_sparsify_segmented
 * call on `stream` (tracing aid).  Synchronises the stream and writes 8 uint64
 * per CTA to HOST host_out (room for 512 x 8), %globaltimer in ns.  gk_sparsify:
 * the CTA's start, before and after the first grid barrier, before and after the
 * second, before and after the third, its end.  gk_sparsify_segmented: start,
 * table read, end of the first phase, after the first barrier, thresholds formed,
 * end of the counting, after the second barrier, end.
 * *n_ctas receives the number of CTAs, 0 if the last call did not run such a kernel.
 */
int gk_last_cta_trace(gk_stream_t stream, uint64_t* host_out, int* n_ctas);

/*
 * gk_debug_set -- test hooks (the paper has no counterpart).  They exist so that tests can
 * reach the give-up branch of every bounded wait without hanging anything, and both sides of
 * the library's run-time decisions.  Process-wide; the device-side values are set on the
 * current device.  Defaults are restored by setting the default value again.
 *   key 0  polls of a grid barrier before a CTA gives up and sets GK_DEV_TIMEOUT (default 2^24)
 *   key 1  polls of a predecessor's status word in the look-back compaction (default 2^22)
 *   key 2  arrivals the barriers of the fused gk_sparsify kernel wait for beyond the grid
 *          size (default 0).  With 1 no barrier can complete: every CTA's wait runs out,
 *          the call ends with GK_DEV_TIMEOUT in gk_stats.status and invalid outputs.  Also in the
 *          products of gk_vocab_loss and gk_vocab_distill, whose readers then wait for sums that never
 *          arrive (a sixteenth of a second instead of two): GK_DEV_TIMEOUT in gk_vocab_last_info.
 *   key 3  a tile of the look-back compaction that keeps its status word to itself, so
 *          that its successors' waits run out (default -1: none)
 *   key 4  counting against predicted thresholds in the fused gk_sparsify / gk_select
 *          kernel: -1 automatic (large vectors), 0 never, 1 whenever the vector has 128
 *          elements or more
 *   key 5  the second phase of that kernel counting only the candidates it expects the rounds
 *          to reach: -1 automatic, 0 never, 1 always and with thres0 alone (any further
 *          round then asks for a candidate left out, and the count is taken again in full)
 * Returns GK_ERR_SIZE for an unknown key or a value outside [-1, 2^31 - 1].
 */
int gk_debug_set(int key, int64_t value);

/*
 * How the last single-kernel gk_sparsify / gk_select call on `stream` took its counts
 * (tracing aid).  Synchronises the stream and writes 6 int64 to HOST host_out: CTAs that
 * formed a prediction of the thresholds from the sample; CTAs whose predicted bands held the
 * exact thresholds (their counts come from the first phase plus the cells it left over);
 * 1 if the rounds needed a candidate the short way leaves out, so that a full count followed;
 * (row, warp) cells of 128 elements left to the second phase by CTAs with a prediction; CTAs
 * of the launch (0 if the call did not run that kernel); CTAs that counted, in the second
 * phase, only the candidates they expected the rounds to reach.
 */
int gk_last_path_info(gk_stream_t stream, int64_t* host_out);

/* Number of kernels the library has launched so far in this process. */
int64_t gk_launch_count(void);

/* Text for a gk_status; the CUDA error string of the last GK_ERR_CUDA. */
const char* gk_strerror(int code);
const char* gk_last_cuda_error(void);

/* Library version, major * 1000 + minor. */
int gk_version(void);

#ifdef __cplusplus
}
#endif
#endif /* GK_H_ */
