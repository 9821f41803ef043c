// Elements of the library's types in 16-byte words, keys in the order of their values, and pairs of fp32
// operations: what the kernels over rows of logits and over gradients share.  Internal; the public interface is
// include/gk.h.
#pragma once

#include "gk_vocab.cuh"

namespace gk {

#ifdef __CUDACC__

// Unsigned key in the order of the values; -0 ties with +0, NaN is above +inf.
__device__ __forceinline__ unsigned order_key(float v) {
    if (v != v) return 0xffffffffu;
    const unsigned b = __float_as_uint(v == 0.f ? 0.f : v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);   // 0xffffffff: a NaN
}

template <int TYPE>
__device__ __forceinline__ float load_logit(const char* row, int64_t i) {
    if constexpr (TYPE == GK_TYPE_F32) return __ldg((const float*)row + i);
    else return from16<TYPE == GK_TYPE_F16>(__ldg((const uint16_t*)row + i));
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <int TYPE>
__device__ __forceinline__ void unpack(const uint4& x, float (&f)[TYPE == GK_TYPE_F32 ? 4 : 8]) {
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
