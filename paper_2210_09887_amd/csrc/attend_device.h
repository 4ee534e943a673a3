// What the attention kernels share: which tokens a row sees, codes as matrix operands, queries as such.
//
// Rows.  The queries of a sequence that read one head of the cache - n queries of g heads each - are n g rows: row r is query
// r / g, head r % g of the group.  Every kernel computes S' = K Q' (tokens by rows) and O' = V' P', so that a lane holds tokens of
// one row: maxima and sums over tokens stay in the lane but for two or one steps, and P' leaves the first product in the registers in which
// the second takes it.  Which token a row of an instruction is is free as long as both products agree: lanes get runs of
// neighbouring tokens, which is how the values lie in a page.
//
// Codes become halves without a conversion: a byte c + 128 in the low byte of 0x6400 is the half 1152 + c, minus 1152 is c,
// exactly.  The scale of a page's keys is multiplied into the logits.  That of its values goes into the exponent,
//   w = 2^(x + log2 vs - T + kRoom),  T the row's largest x + log2 vs when it was last moved,
// so that w is a half next to what counts most in this row, whatever the sizes of scales and values: sum w code / sum (w / vs) is the result,
// 2^(T - kRoom) sum (w / vs) the sum of the exponentials.  Weights near 2^kRoom at the top leave the halves' range to those below: one has all its bits
// down to 2^-24 of the largest, and a step of 2^-34 of it from there (a first token 14 above 4096 others: with the largest at 1 the others' part of the result
// was off by 1 %).  T is moved by pages that have values: those that are all zeros (vs below 2^-100) or not
// numbers count in the second sum only, with the scale of the page before.  (Scales of one sequence and head may lie 2^100 apart.)
#pragma once

#include "ops_device.h"
#include "ops_internal.h"

namespace mdcnn {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Eight codes as halves.
__device__ __forceinline__ half8 halves_of(unsigned a, unsigned b) {
    union { unsigned u[4]; half2v h[4]; half8 v; } r;
    a ^= 0x80808080u;
    b ^= 0x80808080u;
    r.u[0] = __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u);
    r.u[1] = __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u);
    r.u[2] = __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u);
    r.u[3] = __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u);
    const half2v off = {(_Float16)1152, (_Float16)1152};
#pragma unroll
    for (int i = 0; i < 4; ++i) r.h[i] -= off;
    return r.v;
}

// Sequence of a block and what its rows see.
struct Rows {
    int len, n, rows;            // tokens in the cache, queries, rows (queries x group)
    long long q0;                // first query of the sequence in the maps
    __device__ __forceinline__ bool load(const AttendJob& j, int seq) {
        const int s0 = j.starts[seq];
        n = min(min(j.starts[seq + 1], j.tokens) - s0, j.max_new);
        if (s0 < 0 || n <= 0) return false;
        len = max(0, min(j.lengths[seq], j.max_len));
        q0 = s0;
        rows = n * j.group;
        return true;
    }
    // positions that query i sees: lo <= position < hi
    __device__ __forceinline__ int hi(const AttendJob& j, int i) const { return j.causal ? max(0, len - n + i + 1) : len; }
    // (a window of any size: nothing negative less nothing negative)
    __device__ __forceinline__ int lo(const AttendJob& j, int i) const { return j.window ? max(0, hi(j, i) - j.window) : 0; }
};

// Pages of the rows r0 .. r1 - 1 of a sequence, of which split z has the run [first, last).
struct Run {
    int first, last, splits;
    __device__ __forceinline__ Run(const AttendJob& j, const Rows& s, int r0, int r1, int z) {
        const int lo = s.lo(j, r0 / j.group), hi = s.hi(j, (r1 - 1) / j.group);
        const int p0 = lo / MDCNN_PAGE_TOKENS, p1 = min(hi / MDCNN_PAGE_TOKENS + (hi % MDCNN_PAGE_TOKENS > 0), j.max_pages);
        splits = max(0, (p1 - p0 + j.run - 1) / j.run);
        first = p0 + z * j.run;
        last = min(p1, first + j.run);
    }
};

// Where weights lie: the largest that T knows at 2^kRoom.  32 of them in a lane (a page of the tiles) add up to 2^15 then, below kMuch.
constexpr float kRoom = 10.f, kUnroom = 1.f / 1024;
// Weights of fp32 calls as two halves: the second one holds 2^11 times what the first leaves, or it would end where the first does, and is multiplied with codes by 2^-11
// (exact: they are whole numbers up to 127).
constexpr float kSecond = 2048.f;
constexpr _Float16 kSecondBack = (_Float16)(1.f / 2048);

// The scale of a page's values in the exponent: log2 vs as a whole number and a part below one, 24 bits of it, so that a weight is as exact as its
// logit whatever the size of the values.  What is left of that is in the weights of both sums: the inverse is the scale's own.
struct ValueScale {
    float scale = 1.f;                                     // the page's, or the last one that could be used
    bool none = false, bad = false;                        // weights do not count in the sum of values; not a number
    __device__ __forceinline__ void next(float vs) {
        bad = vs != vs;
        none = vs < 7.8886090522101181e-31f;               // 2^-100; any scale does then: that of the page before
        if (!none && !bad) scale = vs;
        asm volatile("" : "+v"(scale));                  // scalar registers are short in tiles of 256 channels
    }
    __device__ __forceinline__ float whole() const { return (float)((int)(__float_as_uint(scale) >> 23) - 127); }
    __device__ __forceinline__ float part() const { return __builtin_amdgcn_logf(__uint_as_float((__float_as_uint(scale) & 0x7fffffu) | 0x3f800000u)); }
    __device__ __forceinline__ float inverse() const {
        const float r = __builtin_amdgcn_rcpf(scale);
        return __builtin_fmaf(__builtin_fmaf(-scale, r, 1.f), r, r);
    }
    __device__ __forceinline__ float log() const { return whole() + part(); }
    // of the weights of a row: the exponent of a logit of zero
    __device__ __forceinline__ float base(float top) const { return whole() + kRoom - (top == -INFINITY ? 0.f : top) + part(); }
};

// In place of a row's factor (which is not negative): its query is not finite.  It goes through as zeros, so that hidden tokens stay hidden, and its sum
// becomes NaN at the end if it has seen any token.
constexpr float kSpoiled = -1.f;

// Factor of the products of a row with a page's keys.  Never zero: a hidden token's minus infinity stays that.
__device__ __forceinline__ float factor_of(float logit, float ks) {
    const float by = logit * ks;
    return by < 1e-30f ? 1e-30f : by;
}
// T of a row is moved - and what has been summed faded - only where the weights of a lane add up to more than this (they have to be
// halves, of which the largest is 65504; where no values follow, what the sum takes of them has to stay below 2^110): weights are made
// before anyone looks for a maximum, and on nearly all pages no one does.
constexpr float kMuch = 65504.f;
__device__ __forceinline__ float much(const ValueScale& val) { return val.none || val.bad ? fminf(val.scale * 0x1p120f, 0x1p127f) : kMuch; }

// T of a row after a page whose largest x + log2 vs is `most` (minus infinity: the row sees none of it), and what the sums fade by.  The first page with
// values sets it, whatever pages without values left (their sum is kept: no further down than that stays finite).
struct NextTop {
    float top, fade, fade_out;
    __device__ __forceinline__ NextTop(float was, float most, bool moves, bool values, float& valued) {
        const bool sets = values && valued == 0.f && most > -INFINITY;
        top = !moves ? was : sets ? fmaxf(most, was - 100.f) : fmaxf(was, most);
        fade = was == -INFINITY ? 1.f : exp2_fast(was - top);              // (nothing summed so far: nothing to fade)
        fade_out = valued == 0.f ? 0.f : fade;                            // (nothing but zeros so far)
        valued = sets ? 1.f : valued;
    }
};

// Whether it holds in one of the lanes n and n + 32 (n, n + 16, n + 32, n + 48) that share a row.
__device__ __forceinline__ bool row_of_two(bool here, int n) {
    const unsigned long long b = __ballot(here);
    return ((b | b >> 32) >> n & 1) != 0;
}
__device__ __forceinline__ bool row_of_four(bool here, int n) {
    unsigned long long b = __ballot(here);
    b |= b >> 32;
    return ((b | b >> 16) >> n & 1) != 0;
}

// The larger one of the two lanes 32 (16) apart, in both.
__device__ __forceinline__ float max_over_32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_over_16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// Page numbers of a run, asked for in ascending order: 64 of them in a register of the wave.  (A scalar load for each would be waited for
// together with whatever LDS reads are on their way.)
struct PageIds {
    const int* table;
    int ids, begin, last, pages, lane;
    __device__ __forceinline__ PageIds(const AttendJob& j, int seq, const Run& run, int first, int lane_) : table(j.table + (long long)seq * j.max_pages), last(run.last), pages(j.pages), lane(lane_) { fetch(first); }
    __device__ __forceinline__ void fetch(int p) {
        begin = p;
        ids = p + lane < last ? table[p + lane] : -1;
        ids = ids >= 0 && ids < pages ? ids : -1;
    }
    // -1: no page
    __device__ __forceinline__ int at(int p) {
        if (p >= last) return -1;
        if (p - begin >= 64) fetch(p);
        return __builtin_amdgcn_readlane(ids, p - begin);
    }
};

// The power of two that brings the largest magnitude of a row to 2^13 .. 2^14 (1 for none, or one that is not finite).
__device__ __forceinline__ int exponent_of(float top) {
    const int e = (int)(__float_as_uint(top) >> 23);
    return top > 0.f && e < 255 ? e - 127 - 13 : 0;
}
__device__ __forceinline__ float scaled(float x, int e) { return ldexpf(x, e); }

// Eight channels of a query from c on (dim is a multiple of eight), zeros beyond.
template <typename T>
__device__ __forceinline__ void eight_of(const T* q, int c, int dim, bool whole, float (&f)[8]) {
    if (c >= dim) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 0.f;
    } else if (whole) {                                    // on 16 bytes
        constexpr int N = 16 / sizeof(T);
#pragma unroll
        for (int k = 0; k < 8 / N; ++k) {
            float g[N];
            unpack(*(const Pack<T, N>*)(q + c + N * k), g);
#pragma unroll
            for (int i = 0; i < N; ++i) f[N * k + i] = g[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = to_f32(q[c + i]);
    }
}

// Which of 16 tokens from `pos` on have a nonzero byte, as bits.
__device__ __forceinline__ unsigned mask_bits(const uint8_t* row, int pos, int end, bool whole) {
    unsigned bits = 0;
    if (whole && pos + 16 <= end) {
        const uint4v w = *(const uint4v*)(row + pos);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) bits |= (w[i] >> (8 * e) & 0xff ? 1u : 0u) << (4 * i + e);
    } else {
        for (int i = 0; i < 16; ++i)
            if (pos + i < end && row[pos + i]) bits |= 1u << i;
    }
    return bits;
}

// What::go<storage type, pitch>(j, st)
template <typename What, typename T>
hipError_t for_pitch(const AttendJob& j, hipStream_t st) {
    switch (j.pitch) {
        case 32: return What::template go<T, 32>(j, st);
        case 64: return What::template go<T, 64>(j, st);
        case 96: return What::template go<T, 96>(j, st);
        case 128: return What::template go<T, 128>(j, st);
        case 192: return What::template go<T, 192>(j, st);
        default: return What::template go<T, 256>(j, st);
    }
}
template <typename What>
hipError_t for_type_and_pitch(const AttendJob& j, int dtype, hipStream_t st) {
    if (dtype == MDCNN_F32) return for_pitch<What, float>(j, st);
    if (dtype == MDCNN_F16) return for_pitch<What, _Float16>(j, st);
    return for_pitch<What, __bf16>(j, st);
}

}  // namespace mdcnn
