// What the operators behind the feature maps share: storage types, vectors of them, sums over a wave.
#pragma once

#include "mdcnn_internal.h"

namespace mdcnn {

// VEC neighbouring channels as they lie in memory, and as floats.  A 16-byte vector where channels, strides and pointers allow
// it, one channel otherwise.
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
    T v[VEC];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(_Float16 x) { return (float)x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return (float)x; }

template <typename T, int VEC>
__device__ __forceinline__ void unpack(const Pack<T, VEC>& p, float (&f)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = to_f32(p.v[i]);
}
template <typename T, int VEC>
__device__ __forceinline__ Pack<T, VEC> pack(const float (&f)[VEC]) {
    Pack<T, VEC> p;
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.v[i] = (T)f[i];
    return p;
}

// Sum over `width` (a power of two, up to 64) neighbouring lanes, in all of them.
__device__ __forceinline__ float sum_lanes(float v, int width) {
    for (int m = 1; m < width; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace mdcnn
