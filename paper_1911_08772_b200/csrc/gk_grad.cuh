// The gradients of many tensors (gk_grad_norm, gk_grad_clip): their part of the workspace, and the
// 16-byte words of the library's element types.  Internal; the public interface is include/gk.h.
#pragma once

#include "gk_common.cuh"
#include "gk_vocab.cuh"

namespace gk {

constexpr int kGradMaxCtas = 1024;

// At the start of a workspace's gradient block.  Zero when the workspace is made; the counters are back at
// zero when a call ends.
struct GradCtl {
    unsigned arrived, left;     // the barrier of gk_grad_clip
    unsigned done;              // CTAs of gk_grad_norm that have finished
    int status;                 // GK_DEV_* flags of the last gk_grad_clip
    int clipped;                // its norm was above the limit
};
size_t grad_scratch_bytes(int32_t S);

#ifdef __CUDACC__

template <int TYPE>
__device__ __forceinline__ void unpack16B(const uint4& x, float (&f)[TYPE == GK_TYPE_F32 ? 4 : 8]) {
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

#endif  // __CUDACC__

}  // namespace gk
