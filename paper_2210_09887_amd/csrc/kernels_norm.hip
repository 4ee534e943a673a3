// Group norm with an activation, channels last, and its gradients.
//
//   z = (x - mean) rstd,  y = act(gamma z + beta);     t = gamma act'(u) dy,  dx = rstd (t - mean(t) - z mean(t z))
//
// Both directions need sums over an image and group before a single output can be made, so a map is gone over twice; what
// bounds it is the memory.  Channels last, a thread owns one 16-byte vector of channels and walks down the pixels: neighbouring
// lanes read neighbouring channels, and everything that depends on the channel alone stays in registers.
//  - Maps that the registers of a block hold (held_*): one launch, one read.
//  - Larger ones: a launch that leaves the sums of chunks of pixels, one that joins them and goes over the map again, with the
//    same blocks for the same pixels (the second read then comes from the caches as far as they reach).  Beyond 64 chunks an image,
//    whose joining would be most of a block's work, they are joined by a launch of their own.
// Variances are sums of squares about a value of the channel itself, then about the means of ever larger sets: a mean that is large
// beside the deviation costs no digits.  No atomics: sums are taken in one order.
// 16 bf16 maps of 128 x 128 x 256 (134 MB): sums 26 us (5.1 TB/s), second pass with silu 56 (4.8), sums of the gradients 62 (4.3), dx 75 (5.4); one fp16
// map of 12 x 9 x 256 8 us, a launch and two trips to memory.
#include <type_traits>

#include "ops_device.h"
#include "ops_internal.h"

namespace mdcnn {

namespace {

constexpr int kThreads = 256;
constexpr int kJoinHere = 64;                  // chunks of an image that every block joins for itself

__device__ __forceinline__ long long at_pixel(const mdcnn_strides& s, int p, int W, int flat) {
    return flat ? (long long)p * s.x : (long long)(p / W) * s.y + (long long)(p % W) * s.x;
}

// s = 1 / (1 + exp(-u)) and 1 - s.  Maps of fp32: from the exponential of -|u|, so that neither is a difference; of 16 bits: the exponent a rounded
// product and 1 - s a difference, which take |u| 2^-24 of a value, far less than its own rounding.
struct Sigmoid {
    float s, rest;
};
template <typename T>
__device__ __forceinline__ Sigmoid sigmoid_of(float u) {
    if constexpr (sizeof(T) == 4) {
        const float e = expf(-fabsf(u)), big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
        return u < 0.f ? Sigmoid{small, big} : Sigmoid{big, small};
    } else {
        const float s = __builtin_amdgcn_rcpf(1.f + exp2_fast(-1.44269504f * u));
        return {s, 1.f - s};
    }
}
template <int ACT, typename T>
__device__ __forceinline__ float act_of(float u) {
    if (ACT == MDCNN_ACT_SILU) return u * sigmoid_of<T>(u).s;
    if (ACT == MDCNN_ACT_RELU) return u < 0.f ? 0.f : u;
    return u;
}
// act'(u).  silu: s + u s (1 - s); nothing of it overflows.
template <int ACT, typename T>
__device__ __forceinline__ float slope_of(float u) {
    if (ACT == MDCNN_ACT_SILU) {
        const Sigmoid g = sigmoid_of<T>(u);
        return __builtin_fmaf(u * g.s, g.rest, g.s);
    }
    if (ACT == MDCNN_ACT_RELU) return u > 0.f ? 1.f : u == u ? 0.f : u;
    return 1.f;
}

// f with the activation as a constant: one decision to a loop instead of one to a value.
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    if (act == MDCNN_ACT_SILU) f(std::integral_constant<int, MDCNN_ACT_SILU>());
    else if (act == MDCNN_ACT_RELU) f(std::integral_constant<int, MDCNN_ACT_RELU>());
    else f(std::integral_constant<int, MDCNN_ACT_NONE>());
}

// Block of a chunked launch: image, chunk, slice of channels and the thread's place in it.
struct Place {
    int n, chunk, c0, nc, lane, row, r0, r1;
};
__device__ __forceinline__ Place place_of(const NormJob& j, unsigned blk) {
    Place p;
    const int slice = blk % j.slices;
    blk /= j.slices;
    p.chunk = blk % j.chunks;
    p.n = blk / j.chunks;
    p.c0 = slice * j.slice;
    p.nc = min(j.slice, j.C - p.c0);
    p.lane = threadIdx.x % j.lanes;
    p.row = threadIdx.x / j.lanes;
    p.r0 = p.chunk * j.rows;
    p.r1 = min(j.P, p.r0 + j.rows);
    return p;
}

__device__ __forceinline__ int pow2_over(int n) { return n >= 64 ? 64 : n <= 1 ? 1 : 1 << (32 - __clz(n - 1)); }

// Lanes to a group: as many as the block has for all its groups, no more than there are elements.
__device__ __forceinline__ int lanes_for(int groups, int elements) {
    int w = pow2_over(elements);
    while (w > 1 && w * groups > (int)blockDim.x) w >>= 1;
    return w;
}

// Per group of the slice, from what the rows of threads left in s[row][c] - mean and squares about it of a channel's pixels row, row + row_lanes .. - the
// same over all its channels and pixels: out(group, mean, squares).
template <typename F>
__device__ __forceinline__ void join_groups(const float2* s, int nc, int cpg, int row_lanes, int pixels, F&& out) {
    __syncthreads();
    const int groups = nc / cpg, rows = min(row_lanes, pixels), w = lanes_for(groups, rows * cpg), lane = threadIdx.x % w;
    const int whole = (pixels + row_lanes - 1) / row_lanes, more = pixels % row_lanes, dr = w / cpg, dc = w % cpg;
    const float inv = 1.f / ((float)pixels * (float)cpg);
    for (int g = threadIdx.x / w; g < groups; g += blockDim.x / w) {
        auto each = [&](auto&& f) {
#pragma unroll 4
            for (int r = lane / cpg, c = lane % cpg; r < rows;) {
                f(s[r * nc + g * cpg + c], (float)(!more || r < more ? whole : whole - 1));
                r += dr;
                c += dc;
                if (c >= cpg) { c -= cpg; ++r; }
            }
        };
        float m = 0.f, sq = 0.f;
        each([&](float2 v, float k) { m = __builtin_fmaf(v.x, k, m); });
        m = sum_lanes(m, w) * inv;
        each([&](float2 v, float k) { sq += __builtin_fmaf((v.x - m) * (v.x - m), k, v.y); });
        sq = sum_lanes(sq, w);
        if (lane == 0) out(g, m, sq);
    }
}
// Sums of the rows of threads per channel: in s[0][c].
__device__ __forceinline__ void add_rows(float2* s, int nc, int row_lanes) {
    __syncthreads();
    if (row_lanes < 2) return;
    // sets of threads over the channels each take every sets-th row, then the first takes the sets
    const int sets = max(1, min(row_lanes, (int)blockDim.x / nc));
    const int set = threadIdx.x / nc;
    if (set < sets)
        for (int c = threadIdx.x - set * nc; c < nc; c += sets > 1 ? nc : blockDim.x) {
            float a = 0.f, b = 0.f;
#pragma unroll 4
            for (int r = set; r < row_lanes; r += sets) { const float2 v = s[r * nc + c]; a += v.x; b += v.y; }
            s[set * nc + c] = make_float2(a, b);           // (a row that only this thread reads)
        }
    __syncthreads();
    if (sets > 1) {
        if (set == 0) {
            float a = 0.f, b = 0.f;
            for (int r = 0; r < sets; ++r) { const float2 v = s[r * nc + threadIdx.x]; a += v.x; b += v.y; }
            s[threadIdx.x] = make_float2(a, b);
        }
        __syncthreads();
    }
}
template <typename F>
__device__ __forceinline__ void add_channels(const float2* s, int nc, int cpg, F&& out) {
    const int groups = nc / cpg, w = lanes_for(groups, cpg), lane = threadIdx.x % w;
    for (int g = threadIdx.x / w; g < groups; g += blockDim.x / w) {
        float a = 0.f, b = 0.f;
#pragma unroll 4
        for (int c = lane; c < cpg; c += w) { const float2 v = s[g * cpg + c]; a += v.x; b += v.y; }
        a = sum_lanes(a, w);
        b = sum_lanes(b, w);
        if (lane == 0) out(g, a, b);
    }
}
// Chunks of image n and group g joined by w lanes.
__device__ __forceinline__ float2 join_chunks(const NormJob& j, int n, int g, int lane, int w) {
    const float2* p = (const float2*)j.part + ((size_t)n * j.chunks) * j.groups + g;
    const float whole = (float)j.rows, last = (float)(j.P - (j.chunks - 1) * j.rows), inv = 1.f / (float)j.P;
    float m = 0.f, sq = 0.f;
#pragma unroll 4
    for (int k = lane; k < j.chunks; k += w) m += p[(size_t)k * j.groups].x * ((k == j.chunks - 1 ? last : whole) * inv);
    m = sum_lanes(m, w);
#pragma unroll 4
    for (int k = lane; k < j.chunks; k += w) {
        const float2 v = p[(size_t)k * j.groups];
        sq += v.y + (k == j.chunks - 1 ? last : whole) * (float)j.cpg * (v.x - m) * (v.x - m);
    }
    sq = sum_lanes(sq, w);
    return make_float2(m, 1.f / sqrtf(sq * j.inv_count + j.eps));
}
__device__ __forceinline__ float2 add_chunks(const NormJob& j, int n, int g, int lane, int w) {
    const float2* p = (const float2*)j.part + ((size_t)n * j.chunks) * j.groups + g;
    float a = 0.f, b = 0.f;
#pragma unroll 4
    for (int k = lane; k < j.chunks; k += w) { const float2 v = p[(size_t)k * j.groups]; a += v.x; b += v.y; }
    return make_float2(sum_lanes(a, w) * j.inv_count, sum_lanes(b, w) * j.inv_count);
}

// Groups of the channels c .. c + VEC - 1, counted from `first`, one division for all.
template <int VEC, typename F>
__device__ __forceinline__ void each_group(const NormJob& j, int c, int first, F&& f) {
    int g = c / j.cpg, in = c - g * j.cpg;
    g -= first;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        f(i, g);
        if (++in == j.cpg) { in = 0; ++g; }
    }
}

// What of a vector of channels does not change from pixel to pixel: y = act((x - mean) scale + beta), scale = gamma rstd.
template <int VEC>
struct Channels {
    float mean[VEC], scale[VEC], beta[VEC];
    __device__ __forceinline__ void load_affine(const NormJob& j, int c) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            scale[i] = j.gamma ? j.gamma[c + i] : 1.f;
            beta[i] = j.beta ? j.beta[c + i] : 0.f;
        }
    }
    __device__ __forceinline__ void load_stats(const NormJob& j, int c, const float* mean_of, const float* rstd_of, int first_group) {
        each_group<VEC>(j, c, first_group, [&](int i, int g) { mean[i] = mean_of[g]; scale[i] *= rstd_of[g]; });
    }
    template <int ACT, typename T>
    __device__ __forceinline__ Pack<T, VEC> apply(const Pack<T, VEC>& x) const {
        float f[VEC];
        unpack(x, f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = act_of<ACT, T>(__builtin_fmaf(f[i] - mean[i], scale[i], beta[i]));
        return pack<T, VEC>(f);
    }
};
// The same for gradients, with du = act'(u) dy and d = x - mean:
//   dx = scale du - rstd m1 - rstd^2 m2' d,   m2' = mean(gamma du d)
template <int VEC>
struct GradChannels {
    float mean[VEC], scale[VEC], beta[VEC];
    __device__ __forceinline__ void load(const NormJob& j, int n, int c) {
        each_group<VEC>(j, c, 0, [&](int i, int g) {
            const size_t at = (size_t)n * j.groups + g;
            mean[i] = j.mean[at];
            scale[i] = j.rstd[at] * (j.gamma ? j.gamma[c + i] : 1.f);
            beta[i] = j.beta ? j.beta[c + i] : 0.f;
        });
    }
    template <int ACT, typename T>
    __device__ __forceinline__ void of(const Pack<T, VEC>& x, const Pack<T, VEC>& dy, float (&du)[VEC], float (&d)[VEC]) const {
        unpack(x, d);
        unpack(dy, du);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            d[i] -= mean[i];
            if (ACT != MDCNN_ACT_NONE) du[i] *= slope_of<ACT, T>(__builtin_fmaf(d[i], scale[i], beta[i]));
        }
    }
};
// The two terms that a group's sums take from its gradients.
template <int VEC>
struct GradTerms {
    float one[VEC], two[VEC];
    __device__ __forceinline__ void load(const NormJob& j, int n, int c, const float2* sums, int first_group) {
        each_group<VEC>(j, c, first_group, [&](int i, int g) {
            const float r = j.rstd[(size_t)n * j.groups + first_group + g];
            const float2 v = sums[g];
            one[i] = r * v.x;
            two[i] = r * v.y;
        });
    }
    template <typename T>
    __device__ __forceinline__ Pack<T, VEC> gradient(const GradChannels<VEC>& ch, const float (&du)[VEC], const float (&d)[VEC]) const {
        float f[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = __builtin_fmaf(du[i], ch.scale[i], -__builtin_fmaf(d[i], two[i], one[i]));
        return pack<T, VEC>(f);
    }
};

// ---- forward ----------------------------------------------------------------------------------------------------------
template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void k_norm_stats(NormJob j) {
    extern __shared__ float2 s[];
    const Place p = place_of(j, blockIdx.x);
    const T* x = (const T*)j.x + (long long)p.n * j.xs.n + p.c0;
    if (p.row < j.row_lanes)
        for (int c = p.lane * VEC; c < p.nc; c += j.lanes * VEC) {
            float pivot[VEC], s1[VEC], s2[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) pivot[i] = s1[i] = s2[i] = 0.f;
            const int first = p.r0 + p.row;
            if (first < p.r1) unpack(*(const Pack<T, VEC>*)(x + at_pixel(j.xs, first, j.W, j.flat) + c), pivot);
#pragma unroll 4
            for (int r = first + j.row_lanes; r < p.r1; r += j.row_lanes) {
                float f[VEC];
                unpack(*(const Pack<T, VEC>*)(x + at_pixel(j.xs, r, j.W, j.flat) + c), f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float d = f[i] - pivot[i];
                    s1[i] += d;
                    s2[i] = __builtin_fmaf(d, d, s2[i]);
                }
            }
            const int k = first < p.r1 ? (p.r1 - first + j.row_lanes - 1) / j.row_lanes : 1;
            const float inv = 1.f / (float)k;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = s1[i] * inv, sq = s2[i] - s1[i] * d;
                s[p.row * p.nc + c + i] = make_float2(pivot[i] + d, sq < 0.f ? 0.f : sq);
            }
        }
    float2* out = (float2*)j.part + ((size_t)p.n * j.chunks + p.chunk) * j.groups + p.c0 / j.cpg;
    join_groups(s, p.nc, j.cpg, j.row_lanes, p.r1 - p.r0, [&](int g, float m, float sq) { out[g] = make_float2(m, sq); });
}

__global__ __launch_bounds__(kThreads) void k_norm_join(NormJob j) {
    const long long i = (long long)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    if (i >= (long long)j.N * j.groups) return;
    const int n = (int)(i / j.groups), g = (int)(i % j.groups), lane = threadIdx.x & 63;
    const float2 v = join_chunks(j, n, g, lane, 64);
    if (lane == 0) { j.mean[i] = v.x; j.rstd[i] = v.y; }
}

template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void k_norm_apply(NormJob j) {
    extern __shared__ float2 s[];
    float* mean = (float*)s;
    float* rstd = mean + j.slice / j.cpg;
    const Place p = place_of(j, gridDim.x - 1 - blockIdx.x);              // what was read last comes first: the caches hold that
    const int g0 = p.c0 / j.cpg;
    if (j.chunks <= kJoinHere) {
        const int w = lanes_for(p.nc / j.cpg, j.chunks), lane = threadIdx.x % w;
        for (int g = threadIdx.x / w; g * j.cpg < p.nc; g += kThreads / w) {
            const float2 v = join_chunks(j, p.n, g0 + g, lane, w);
            if (lane == 0) {
                mean[g] = v.x;
                rstd[g] = v.y;
                if (p.chunk == 0) { j.mean[(size_t)p.n * j.groups + g0 + g] = v.x; j.rstd[(size_t)p.n * j.groups + g0 + g] = v.y; }
            }
        }
    } else {
        for (int g = threadIdx.x; g * j.cpg < p.nc; g += kThreads) {
            mean[g] = j.mean[(size_t)p.n * j.groups + g0 + g];
            rstd[g] = j.rstd[(size_t)p.n * j.groups + g0 + g];
        }
    }
    __syncthreads();
    if (p.row >= j.row_lanes) return;
    const T* x = (const T*)j.x + (long long)p.n * j.xs.n;
    T* y = (T*)j.y + (long long)p.n * j.ys.n;
    for (int c = p.c0 + p.lane * VEC; c < p.c0 + p.nc; c += j.lanes * VEC) {
        Channels<VEC> ch;
        ch.load_affine(j, c);
        ch.load_stats(j, c, mean, rstd, g0);
        with_act(j.act, [&](auto act) {
#pragma unroll 4
            for (int r = p.r0 + p.row; r < p.r1; r += j.row_lanes)
                *(Pack<T, VEC>*)(y + at_pixel(j.ys, r, j.W, j.flat) + c) = ch.template apply<act()>(*(const Pack<T, VEC>*)(x + at_pixel(j.xs, r, j.W, j.flat) + c));
        });
    }
}

// The map of a block in its registers: HELD vectors a thread.
template <typename T, int VEC, int HELD>
__global__ __launch_bounds__(VEC == 8 ? 512 : 1024) void k_norm_held(NormJob j) {
    extern __shared__ float2 s[];
    const Place p = place_of(j, blockIdx.x);
    const T* x = (const T*)j.x + (long long)p.n * j.xs.n;
    const int c = p.c0 + p.lane * VEC;
    const bool on = p.row < j.row_lanes && p.lane * VEC < p.nc;
    Pack<T, VEC> v[HELD];
    const int k = on && p.row < j.P ? (j.P - p.row + j.row_lanes - 1) / j.row_lanes : 0;
#pragma unroll
    for (int q = 0; q < HELD; ++q)
        if (q < k) v[q] = *(const Pack<T, VEC>*)(x + at_pixel(j.xs, p.row + q * j.row_lanes, j.W, j.flat) + c);
    Channels<VEC> ch;
    if (on) {
        ch.load_affine(j, c);
        float m[VEC], sq[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) m[i] = sq[i] = 0.f;
#pragma unroll
        for (int q = 0; q < HELD; ++q)
            if (q < k) {
                float f[VEC];
                unpack(v[q], f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) m[i] += f[i];
            }
        const float inv = 1.f / (float)max(k, 1);
#pragma unroll
        for (int i = 0; i < VEC; ++i) m[i] *= inv;
#pragma unroll
        for (int q = 0; q < HELD; ++q)
            if (q < k) {
                float f[VEC];
                unpack(v[q], f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sq[i] = __builtin_fmaf(f[i] - m[i], f[i] - m[i], sq[i]);
            }
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[p.row * p.nc + p.lane * VEC + i] = make_float2(m[i], sq[i]);
    }
    const int g0 = p.c0 / j.cpg;
    // behind the channels: mean and rstd of the groups
    float* mean = (float*)(s + (size_t)j.row_lanes * p.nc);
    float* rstd = mean + p.nc / j.cpg;
    join_groups(s, p.nc, j.cpg, j.row_lanes, j.P, [&](int g, float m, float sq) {
        const float r = 1.f / sqrtf(sq * j.inv_count + j.eps);
        mean[g] = m;
        rstd[g] = r;
        j.mean[(size_t)p.n * j.groups + g0 + g] = m;
        j.rstd[(size_t)p.n * j.groups + g0 + g] = r;
    });
    __syncthreads();
    if (!on) return;
    T* y = (T*)j.y + (long long)p.n * j.ys.n;
    ch.load_stats(j, c, mean, rstd, g0);
    with_act(j.act, [&](auto act) {
#pragma unroll
        for (int q = 0; q < HELD; ++q)
            if (q < k) *(Pack<T, VEC>*)(y + at_pixel(j.ys, p.row + q * j.row_lanes, j.W, j.flat) + c) = ch.template apply<act()>(v[q]);
    });
}

// ---- gradients --------------------------------------------------------------------------------------------------------
template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void k_norm_grad_sums(NormJob j) {
    extern __shared__ float2 s[];
    const Place p = place_of(j, blockIdx.x);
    const T* x = (const T*)j.x + (long long)p.n * j.xs.n;
    const T* dy = (const T*)j.dy + (long long)p.n * j.ds.n;
    if (p.row < j.row_lanes)
        for (int c = p.c0 + p.lane * VEC; c < p.c0 + p.nc; c += j.lanes * VEC) {
            GradChannels<VEC> ch;
            ch.load(j, p.n, c);
            float s1[VEC], s2[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) s1[i] = s2[i] = 0.f;
            with_act(j.act, [&](auto act) {
#pragma unroll 4
                for (int r = p.r0 + p.row; r < p.r1; r += j.row_lanes) {
                    float du[VEC], d[VEC];
                    ch.template of<act()>(*(const Pack<T, VEC>*)(x + at_pixel(j.xs, r, j.W, j.flat) + c), *(const Pack<T, VEC>*)(dy + at_pixel(j.ds, r, j.W, j.flat) + c), du, d);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        s1[i] += du[i];
                        s2[i] = __builtin_fmaf(du[i], d[i], s2[i]);
                    }
                }
            });
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[p.row * p.nc + c - p.c0 + i] = make_float2(s1[i], s2[i]);
        }
    add_rows(s, p.nc, j.row_lanes);
    float2* cpart = (float2*)j.cpart + ((size_t)p.n * j.chunks + p.chunk) * j.C + p.c0;
    for (int c = threadIdx.x; c < p.nc; c += kThreads) {
        const float r = j.rstd[(size_t)p.n * j.groups + (p.c0 + c) / j.cpg];
        const float2 v = make_float2(s[c].x, s[c].y * r);  // of du and of du z
        cpart[c] = v;
        const float gamma = j.gamma ? j.gamma[p.c0 + c] : 1.f;
        s[c] = make_float2(v.x * gamma, v.y * gamma * r);
    }
    __syncthreads();
    float2* out = (float2*)j.part + ((size_t)p.n * j.chunks + p.chunk) * j.groups + p.c0 / j.cpg;
    add_channels(s, p.nc, j.cpg, [&](int g, float a, float b) { out[g] = make_float2(a, b); });
}

__global__ __launch_bounds__(kThreads) void k_norm_grad_join(NormJob j) {
    const long long i = (long long)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    if (i >= (long long)j.N * j.groups) return;
    const int n = (int)(i / j.groups), g = (int)(i % j.groups), lane = threadIdx.x & 63;
    const float2 v = add_chunks(j, n, g, lane, 64);
    if (lane == 0) ((float2*)j.joined)[i] = v;
}

// dgamma, dbeta of 16 channels: the sums that the chunks of all images left, 16 rows of threads.
constexpr int kColumn = 16;
__device__ __forceinline__ void channel_gradients(const NormJob& j, int blk, float2* s) {
    const int c = blk * kColumn + threadIdx.x % kColumn, row = threadIdx.x / kColumn;
    const long long rows = (long long)j.N * j.chunks;
    float a = 0.f, b = 0.f;
    if (c < j.C) {
#pragma unroll 8
        for (long long r = row; r < rows; r += kThreads / kColumn) {
            const float2 v = ((const float2*)j.cpart)[r * j.C + c];
            a += v.x;
            b += v.y;
        }
    }
    s[threadIdx.x] = make_float2(a, b);
    __syncthreads();
    if (row == 0 && c < j.C) {
        for (int r = 1; r < kThreads / kColumn; ++r) { a += s[r * kColumn + threadIdx.x].x; b += s[r * kColumn + threadIdx.x].y; }
        j.dbeta[c] = a;
        j.dgamma[c] = b;
    }
}
__global__ __launch_bounds__(kThreads) void k_norm_grad_channels(NormJob j) {
    __shared__ float2 s[kThreads];
    channel_gradients(j, blockIdx.x, s);
}

template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void k_norm_grad_apply(NormJob j) {
    extern __shared__ float2 s[];
    const unsigned columns = (j.C + kColumn - 1) / kColumn;
    if (blockIdx.x < columns) {
        channel_gradients(j, blockIdx.x, s);
        return;
    }
    const Place p = place_of(j, gridDim.x - 1 - blockIdx.x);              // what was read last comes first: the caches hold that
    const int g0 = p.c0 / j.cpg;
    if (j.chunks <= kJoinHere) {
        const int w = lanes_for(p.nc / j.cpg, j.chunks), lane = threadIdx.x % w;
        for (int g = threadIdx.x / w; g * j.cpg < p.nc; g += kThreads / w) {
            const float2 v = add_chunks(j, p.n, g0 + g, lane, w);
            if (lane == 0) s[g] = v;
        }
    } else {
        for (int g = threadIdx.x; g * j.cpg < p.nc; g += kThreads) s[g] = ((const float2*)j.joined)[(size_t)p.n * j.groups + g0 + g];
    }
    __syncthreads();
    if (p.row >= j.row_lanes) return;
    const T* x = (const T*)j.x + (long long)p.n * j.xs.n;
    const T* dy = (const T*)j.dy + (long long)p.n * j.ds.n;
    T* dx = (T*)j.y + (long long)p.n * j.ys.n;
    for (int c = p.c0 + p.lane * VEC; c < p.c0 + p.nc; c += j.lanes * VEC) {
        GradChannels<VEC> ch;
        ch.load(j, p.n, c);
        GradTerms<VEC> terms;
        terms.load(j, p.n, c, s, g0);
        with_act(j.act, [&](auto act) {
#pragma unroll 2
            for (int r = p.r0 + p.row; r < p.r1; r += j.row_lanes) {
                float du[VEC], d[VEC];
                ch.template of<act()>(*(const Pack<T, VEC>*)(x + at_pixel(j.xs, r, j.W, j.flat) + c), *(const Pack<T, VEC>*)(dy + at_pixel(j.ds, r, j.W, j.flat) + c), du, d);
                *(Pack<T, VEC>*)(dx + at_pixel(j.ys, r, j.W, j.flat) + c) = terms.template gradient<T>(ch, du, d);
            }
        });
    }
}

template <typename T, int VEC, int HELD>
__global__ __launch_bounds__(VEC == 8 ? 512 : 1024) void k_norm_grad_held(NormJob j) {
    extern __shared__ float2 s[];
    const Place p = place_of(j, blockIdx.x);
    const T* x = (const T*)j.x + (long long)p.n * j.xs.n;
    const T* dy = (const T*)j.dy + (long long)p.n * j.ds.n;
    const int c = p.c0 + p.lane * VEC;
    const bool on = p.row < j.row_lanes && p.lane * VEC < p.nc;
    Pack<T, VEC> v[HELD], w[HELD];
    GradChannels<VEC> ch;
    const int k = on && p.row < j.P ? (j.P - p.row + j.row_lanes - 1) / j.row_lanes : 0;
#pragma unroll
    for (int q = 0; q < HELD; ++q)
        if (q < k) {
            v[q] = *(const Pack<T, VEC>*)(x + at_pixel(j.xs, p.row + q * j.row_lanes, j.W, j.flat) + c);
            w[q] = *(const Pack<T, VEC>*)(dy + at_pixel(j.ds, p.row + q * j.row_lanes, j.W, j.flat) + c);
        }
    if (on) {
        ch.load(j, p.n, c);
        float s1[VEC], s2[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) s1[i] = s2[i] = 0.f;
        with_act(j.act, [&](auto act) {
#pragma unroll
            for (int q = 0; q < HELD; ++q)
                if (q < k) {
                    float du[VEC], d[VEC];
                    ch.template of<act()>(v[q], w[q], du, d);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        s1[i] += du[i];
                        s2[i] = __builtin_fmaf(du[i], d[i], s2[i]);
                    }
                }
        });
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[p.row * p.nc + p.lane * VEC + i] = make_float2(s1[i], s2[i]);
    }
    add_rows(s, p.nc, j.row_lanes);
    for (int q = threadIdx.x; q < p.nc; q += blockDim.x) {
        const float r = j.rstd[(size_t)p.n * j.groups + (p.c0 + q) / j.cpg];
        const float2 t = make_float2(s[q].x, s[q].y * r);
        if (j.N == 1) {                                    // this block's sums are the gradients
            j.dbeta[p.c0 + q] = t.x;
            j.dgamma[p.c0 + q] = t.y;
        } else {
            ((float2*)j.cpart)[(size_t)p.n * j.C + p.c0 + q] = t;
        }
        const float gamma = j.gamma ? j.gamma[p.c0 + q] : 1.f;
        s[q] = make_float2(t.x * gamma, t.y * gamma * r);
    }
    __syncthreads();
    float2* sums = s + (size_t)j.row_lanes * p.nc;
    add_channels(s, p.nc, j.cpg, [&](int g, float a, float b) { sums[g] = make_float2(a * j.inv_count, b * j.inv_count); });
    __syncthreads();
    if (!on) return;
    T* dx = (T*)j.y + (long long)p.n * j.ys.n;
    GradTerms<VEC> terms;
    terms.load(j, p.n, c, sums, p.c0 / j.cpg);
    with_act(j.act, [&](auto act) {
#pragma unroll
        for (int q = 0; q < HELD; ++q)
            if (q < k) {
                float du[VEC], d[VEC];
                ch.template of<act()>(v[q], w[q], du, d);
                *(Pack<T, VEC>*)(dx + at_pixel(j.ys, p.row + q * j.row_lanes, j.W, j.flat) + c) = terms.template gradient<T>(ch, du, d);
            }
    });
}

// LDS: a float2 per row of threads and channel, behind them two floats per group.
size_t lds_of(const NormJob& j) { return ((size_t)j.row_lanes * j.slice + j.slice / j.cpg) * sizeof(float2); }

template <typename T, int VEC>
hipError_t forward(const NormJob& j, int held, hipStream_t st) {
    const unsigned blocks = (unsigned)((long long)j.N * j.chunks * j.slices);
    if (held) {
        const unsigned threads = (unsigned)(j.lanes * j.row_lanes + 63) / 64 * 64;
        switch (held) {
            case 1: k_norm_held<T, VEC, 1><<<blocks, threads, lds_of(j), st>>>(j); break;
            case 2: k_norm_held<T, VEC, 2><<<blocks, threads, lds_of(j), st>>>(j); break;
            case 4: k_norm_held<T, VEC, 4><<<blocks, threads, lds_of(j), st>>>(j); break;
            default: k_norm_held<T, VEC, 8><<<blocks, threads, lds_of(j), st>>>(j); break;
        }
        return hipGetLastError();
    }
    k_norm_stats<T, VEC><<<blocks, kThreads, (size_t)j.row_lanes * j.slice * sizeof(float2), st>>>(j);
    if (j.chunks > kJoinHere) k_norm_join<<<(unsigned)(((long long)j.N * j.groups + 3) / 4), kThreads, 0, st>>>(j);
    k_norm_apply<T, VEC><<<blocks, kThreads, (size_t)(j.slice / j.cpg) * 8, st>>>(j);
    return hipGetLastError();
}

template <typename T, int VEC>
hipError_t gradients(const NormJob& j, int held, hipStream_t st) {
    const unsigned blocks = (unsigned)((long long)j.N * j.chunks * j.slices), columns = (unsigned)(j.C + kColumn - 1) / kColumn;
    if (held && j.N) {
        const unsigned threads = (unsigned)(j.lanes * j.row_lanes + 63) / 64 * 64;
        switch (held) {
            case 1: k_norm_grad_held<T, VEC, 1><<<blocks, threads, lds_of(j), st>>>(j); break;
            case 2: k_norm_grad_held<T, VEC, 2><<<blocks, threads, lds_of(j), st>>>(j); break;
            default: k_norm_grad_held<T, VEC, 4><<<blocks, threads, lds_of(j), st>>>(j); break;
        }
        if (j.N == 1) return hipGetLastError();
    }
    if (held || !j.N) {
        k_norm_grad_channels<<<columns, kThreads, 0, st>>>(j);
        return hipGetLastError();
    }
    k_norm_grad_sums<T, VEC><<<blocks, kThreads, (size_t)j.row_lanes * j.slice * sizeof(float2), st>>>(j);
    if (j.chunks > kJoinHere) k_norm_grad_join<<<(unsigned)(((long long)j.N * j.groups + 3) / 4), kThreads, 0, st>>>(j);
    const size_t lds = (size_t)max(j.slice / j.cpg, kThreads) * sizeof(float2);
    k_norm_grad_apply<T, VEC><<<blocks + columns, kThreads, lds, st>>>(j);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormJob& j, int dtype, int vec, int held, hipStream_t st) {
    if (dtype == MDCNN_F32) return vec > 1 ? forward<float, 4>(j, held, st) : forward<float, 1>(j, held, st);
    if (dtype == MDCNN_F16) return vec > 1 ? forward<_Float16, 8>(j, held, st) : forward<_Float16, 1>(j, held, st);
    return vec > 1 ? forward<__bf16, 8>(j, held, st) : forward<__bf16, 1>(j, held, st);
}
hipError_t launch_norm_grad(const NormJob& j, int dtype, int vec, int held, hipStream_t st) {
    if (dtype == MDCNN_F32) return vec > 1 ? gradients<float, 4>(j, held, st) : gradients<float, 1>(j, held, st);
    if (dtype == MDCNN_F16) return vec > 1 ? gradients<_Float16, 8>(j, held, st) : gradients<_Float16, 1>(j, held, st);
    return vec > 1 ? gradients<__bf16, 8>(j, held, st) : gradients<__bf16, 1>(j, held, st);
}

}  // namespace mdcnn
