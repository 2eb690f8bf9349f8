// Rows of logits as the kernels over them load them: 16 bytes to a lane.  Rows start at any element, so the loads are unaligned ones.
#pragma once
#include "common.h"

namespace rn50 {

constexpr int kMaxRows = 1 << 22;  // a launch has fewer than 2^32 threads

template <class T> struct RowVec { static constexpr int N = 16 / (int)sizeof(T); };  // elements of a load
template <class T> __device__ inline uint4 row_load16(const T *p)
{
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
template <class T> __device__ inline void row_store16(T *p, uint4 v) { __builtin_memcpy(p, &v, 16); }

__device__ inline float row_ld(const float *p, long i) { return p[i]; }
__device__ inline float row_ld(const bf16_t *p, long i) { return __uint_as_float((uint32_t)p[i] << 16); }
__device__ inline void row_st(float *p, long i, float v) { p[i] = v; }
__device__ inline void row_st(bf16_t *p, long i, float v) { p[i] = (bf16_t)bf16_rne(v); }

}  // namespace rn50
