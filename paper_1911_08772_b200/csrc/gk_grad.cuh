// The gradients of many tensors (gk_grad_norm, gk_grad_clip): their part of the workspace.  Internal;
// the public interface is include/gk.h.
#pragma once

#include "gk_common.cuh"

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

}  // namespace gk
