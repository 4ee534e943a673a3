// Rotary positions: pairs of channels turned by position times frequency.
//
// The angle of a pair is position x step modulo 2^64, in 2^64ths of a turn: integer arithmetic that is exact at any position, where
// a product of floats has lost 0.06 rad at position 10^6.  Its upper 32 bits are brought to an eighth of a turn and the sine and
// cosine summed as Taylor series (next terms below 2e-9 and 2e-10 there), once per token and pair; the heads that share them are
// gone through by the same thread.  What bounds it is the memory, every value read and written once; with few tokens, the launch.
// 32768 tokens of 40 bf16 heads of 128 channels (671 MB read and written) 130 us, 5.2 TB/s; 13824 tokens of 16 fp32 heads of 32 by three positions
// (57 MB) 14 us, 4.0 TB/s, part of that the time until all blocks have begun; 48 tokens 3.7 us.
#include "ops_device.h"
#include "ops_internal.h"

namespace mdcnn {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void sin_cos_turn(int phase, float& s, float& c) {
    const int quarter = (int)((unsigned)phase + 0x20000000u) >> 30;                      // to the nearest quarter turn
    const float x = (float)(int)((unsigned)phase - ((unsigned)quarter << 30)) * 1.46291807926716e-09f;   // 2 pi / 2^32
    const float x2 = x * x;
    const float sn = x + x * x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880))));
    const float cs = 1.f + x2 * (-0.5f + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 + x2 * (-1.f / 3628800)))));
    const float a = quarter & 1 ? cs : sn, b = quarter & 1 ? sn : cs;
    s = quarter & 2 ? -a : a;
    c = (quarter + 1) & 2 ? -b : b;
}

// Sine and cosine of N pairs from pair `first` of token t, times the magnitude.
template <int N>
__device__ __forceinline__ void turns_of(const RotaryJob& j, long long t, int first, float (&s)[N], float (&c)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int p = first + i, axis = (p >= j.per ? 1 : 0) + (p >= 2 * j.per ? 1 : 0) + (p >= 3 * j.per ? 1 : 0);
        const long long pos = j.pos[t * j.axes + axis];
        sin_cos_turn((int)(((unsigned long long)pos * j.steps[p]) >> 32), s[i], c[i]);
        s[i] *= j.inverse ? -j.magnitude : j.magnitude;
        c[i] *= j.magnitude;
    }
}

// A thread: one token, one unit of its heads - turned vectors first (one of VEC/2 interleaved pairs, or the two that hold VEC pairs of
// halves), then copied ones - and j.group heads.
template <typename T, int VEC, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void k_rotary(RotaryJob j) {
    const int u = threadIdx.x % j.units;
    const long long t = (long long)blockIdx.x * j.tokens_per_block + threadIdx.x / j.units;
    if (threadIdx.x >= j.units * j.tokens_per_block || t >= j.tokens) return;
    constexpr int PAIRS = INTERLEAVED ? (VEC > 1 ? VEC / 2 : 1) : VEC;
    const int h0 = blockIdx.y * j.group, h1 = min(h0 + j.group, j.maps[0].heads + j.maps[1].heads);
    if (u < j.turned_units) {
        float s[PAIRS], c[PAIRS];
        turns_of(j, t, u * PAIRS, s, c);
#pragma unroll 4
        for (int h = h0; h < h1; ++h) {
            const int second = h >= j.maps[0].heads;
            const RotaryMap& m = j.maps[second];
            const int hh = second ? h - j.maps[0].heads : h;
            const T* x = (const T*)m.x + t * m.x_token + hh * m.x_head;
            T* y = (T*)m.y + t * m.y_token + hh * m.y_head;
            if constexpr (INTERLEAVED && VEC > 1) {
                float f[VEC];
                unpack(*(const Pack<T, VEC>*)(x + u * VEC), f);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    const float a = f[2 * i], b = f[2 * i + 1];
                    f[2 * i] = a * c[i] - b * s[i];
                    f[2 * i + 1] = a * s[i] + b * c[i];
                }
                *(Pack<T, VEC>*)(y + u * VEC) = pack<T, VEC>(f);
            } else {
                const int at = INTERLEAVED ? 2 * u : u * VEC, over = INTERLEAVED ? 1 : j.turned / 2;
                float a[VEC], b[VEC];
                unpack(*(const Pack<T, VEC>*)(x + at), a);
                unpack(*(const Pack<T, VEC>*)(x + at + over), b);
                float p[VEC], q[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    p[i] = a[i] * c[i] - b[i] * s[i];
                    q[i] = a[i] * s[i] + b[i] * c[i];
                }
                *(Pack<T, VEC>*)(y + at) = pack<T, VEC>(p);
                *(Pack<T, VEC>*)(y + at + over) = pack<T, VEC>(q);
            }
        }
    } else {
        const int at = j.turned + (u - j.turned_units) * VEC;
#pragma unroll 4
        for (int h = h0; h < h1; ++h) {
            const int second = h >= j.maps[0].heads;
            const RotaryMap& m = j.maps[second];
            const int hh = second ? h - j.maps[0].heads : h;
            *(Pack<T, VEC>*)((T*)m.y + t * m.y_token + hh * m.y_head + at) = *(const Pack<T, VEC>*)((const T*)m.x + t * m.x_token + hh * m.x_head + at);
        }
    }
}

template <typename T, int VEC>
hipError_t launch(const RotaryJob& j, bool interleaved, hipStream_t st) {
    const dim3 grid((unsigned)((j.tokens + j.tokens_per_block - 1) / j.tokens_per_block), (unsigned)((j.maps[0].heads + j.maps[1].heads + j.group - 1) / j.group));
    if (interleaved) k_rotary<T, VEC, true><<<grid, kThreads, 0, st>>>(j);
    else k_rotary<T, VEC, false><<<grid, kThreads, 0, st>>>(j);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryJob& j, int dtype, int vec, bool interleaved, hipStream_t st) {
    if (dtype == MDCNN_F32) return vec == 4 ? launch<float, 4>(j, interleaved, st) : launch<float, 1>(j, interleaved, st);
    if (dtype == MDCNN_F16) return vec == 8 ? launch<_Float16, 8>(j, interleaved, st) : vec == 4 ? launch<_Float16, 4>(j, interleaved, st) : launch<_Float16, 1>(j, interleaved, st);
    return vec == 8 ? launch<__bf16, 8>(j, interleaved, st) : vec == 4 ? launch<__bf16, 4>(j, interleaved, st) : launch<__bf16, 1>(j, interleaved, st);
}

}  // namespace mdcnn
