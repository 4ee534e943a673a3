// Keys and values into and out of pages of 8-bit codes.
//
// A page holds 64 tokens: keys [head][token][pitch], values [head][pitch][token], so that the attention's matrix instructions find both with the
// channels (keys) or the tokens (values) they sum over side by side.  One scale for each page and head: max |x| / 127 over its tokens, so
// that a code is off by half a scale at most.  Codes of a page that grows are rounded again; growing by a quarter at least keeps what
// that adds below half of 1 + 0.8 + 0.64 .. = 5, 2.5 codes, however often a page grows.  Scale and quotient are IEEE
// divisions: a code is what the formula says, not a neighbour.
// A block has one page and head of the keys or of the values; the memory bounds it, with one new token the chain table - scale -
// values - code.
#include "ops_device.h"
#include "ops_internal.h"

namespace mdcnn {

namespace {

constexpr int kThreads = 256;
constexpr int kPage = MDCNN_PAGE_TOKENS;

// Block of a page: sequence, the page's place in its table row, head, keys or values.
struct PageOf {
    int seq, slot, head, is_v;
    int row, first, count;       // first row, its position and number of tokens that the call has for the sequence
    long long page;              // -1: none
    __device__ __forceinline__ bool find(const CacheJob& j) {
        head = blockIdx.y % j.heads;
        is_v = blockIdx.y / j.heads;
        seq = blockIdx.x / j.slots;
        const int s0 = j.starts[seq];
        first = j.first[seq];
        row = s0;
        count = min(min(j.starts[seq + 1], j.tokens) - s0, j.max_new);
        slot = first / kPage + blockIdx.x % j.slots;
        if (s0 < 0 || count <= 0 || first < 0 || slot * (long long)kPage >= (long long)first + count) return false;
        page = -1;
        if (slot < j.max_pages) {
            const int p = j.table[(long long)seq * j.max_pages + slot];
            if (p >= 0 && p < j.pages) page = p;
        }
        return true;
    }
};

// Largest magnitude as bits (a NaN is above infinity), over the block.
__device__ __forceinline__ unsigned block_max(unsigned v, unsigned* s) {
    for (int m = 1; m < 64; m <<= 1) v = max(v, (unsigned)__shfl_xor((int)v, m, 64));
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = max(max(s[0], s[1]), max(s[2], s[3]));
    __syncthreads();
    return v;
}

__device__ __forceinline__ int code_of(float x, float scale) {
    if (!(scale > 0.f)) return 0;                                            // all zeros, or not finite
    return (int)fminf(fmaxf(rintf(x / scale), -127.f), 127.f);
}

// Channels VEC beside one another; the tokens' values pass through LDS as floats, so that they are read once.
template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void k_cache_store(CacheJob j) {
    extern __shared__ float vals[];                                          // [tokens][dim + 1]
    __shared__ unsigned s_max[4];
    PageOf p;
    if (!p.find(j) || p.page < 0) return;
    const CacheMap& m = p.is_v ? j.v : j.k;
    const int base = p.slot * kPage;                                         // position of the page's first token
    const int t0 = max(p.first - base, 0), t1 = min(p.count - (base - p.first), kPage);   // its tokens that are new
    const long long row0 = (long long)p.row + (base - p.first);
    const T* x = (const T*)m.x + p.head * m.x_head;
    const int vecs = j.dim / VEC, n = (t1 - t0) * vecs, pitch = j.dim + 1;
    unsigned top = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int t = i / vecs, c = (i % vecs) * VEC;
        float f[VEC];
        unpack(*(const Pack<T, VEC>*)(x + (row0 + t0 + t) * m.x_token + c), f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            vals[t * pitch + c + e] = f[e];
            top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
        }
    }
    top = block_max(top, s_max);
    float* scale_at = (p.is_v ? j.v_scale : j.k_scale) + p.page * j.heads + p.head;
    const float need = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(top) / 127.f;
    float scale = need, ratio = 1.f;
    if (t0 > 0) {                                                            // the page holds t0 tokens already
        const float old = *scale_at;
        if (need <= old) {
            scale = old;
        } else {
            scale = old != old || need != need ? __uint_as_float(0x7fc00000u) : fmaxf(need, 1.25f * old);
            ratio = scale > 0.f ? old / scale : 0.f;
        }
    }
    __syncthreads();                                                         // everyone has read the old scale
    if (threadIdx.x == 0) *scale_at = scale;
    int8_t* codes = (p.is_v ? j.v_codes : j.k_codes) + (p.page * j.heads + p.head) * (long long)(kPage * j.pitch);
    if (p.is_v) {
        // four tokens of a channel to a word of codes
        for (int i = threadIdx.x; i < j.dim * (kPage / 4); i += kThreads) {
            const int c = i / (kPage / 4), t = (i % (kPage / 4)) * 4;
            if (t >= t1 || (t + 3 < t0 && ratio == 1.f)) continue;
            unsigned* at = (unsigned*)(codes + c * kPage + t);
            unsigned word = t < t0 || t + 3 >= t1 ? *at : 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int tt = t + e;
                if (tt >= t1) continue;
                int q = (int8_t)(word >> (8 * e));
                if (tt >= t0) q = code_of(vals[(tt - t0) * pitch + c], scale);
                else if (ratio != 1.f) q = (int)rintf((float)q * ratio);
                word = (word & ~(0xffu << (8 * e))) | (unsigned)(q & 0xff) << (8 * e);
            }
            *at = word;
        }
    } else {
        const int words = j.dim / 4;
        for (int i = threadIdx.x + (ratio == 1.f ? t0 * words : 0); i < t1 * words; i += kThreads) {
            const int t = i / words, c = (i % words) * 4;
            unsigned* at = (unsigned*)(codes + t * j.pitch + c);
            unsigned word = t < t0 ? *at : 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                int q = (int8_t)(word >> (8 * e));
                if (t >= t0) q = code_of(vals[(t - t0) * pitch + c + e], scale);
                else q = (int)rintf((float)q * ratio);
                word = (word & ~(0xffu << (8 * e))) | (unsigned)(q & 0xff) << (8 * e);
            }
            *at = word;
        }
    }
}

// Values of a page and head back, through LDS where the tokens lie side by side.
template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void k_cache_read(CacheJob j) {
    extern __shared__ unsigned words[];                                      // [dim][kPage / 4 + 1]
    PageOf p;
    if (!p.find(j)) return;
    const CacheMap& m = p.is_v ? j.v : j.k;
    const int base = p.slot * kPage;
    const int t0 = max(p.first - base, 0), t1 = min(p.count - (base - p.first), kPage);
    const long long row0 = (long long)p.row + (base - p.first);
    T* y = (T*)m.y + p.head * m.y_head;
    const long long at = p.page < 0 ? 0 : p.page * j.heads + p.head;
    const float scale = p.page < 0 ? 0.f : (p.is_v ? j.v_scale : j.k_scale)[at];
    const int8_t* codes = (p.is_v ? j.v_codes : j.k_codes) + at * (kPage * j.pitch);
    constexpr int kRow = kPage / 4 + 1;
    if (p.is_v && p.page >= 0) {
        for (int i = threadIdx.x; i < j.dim * (kPage / 4); i += kThreads) {
            const int c = i / (kPage / 4), w = i % (kPage / 4);
            words[c * kRow + w] = *(const unsigned*)(codes + c * kPage + w * 4);
        }
        __syncthreads();
    }
    const int vecs = j.dim / VEC;
    for (int i = threadIdx.x; i < (t1 - t0) * vecs; i += kThreads) {
        const int t = t0 + i / vecs, c = (i % vecs) * VEC;
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            int q = 0;
            if (p.page >= 0) q = p.is_v ? (int8_t)(words[(c + e) * kRow + t / 4] >> (8 * (t & 3))) : codes[t * j.pitch + c + e];
            f[e] = p.page >= 0 ? (float)q * scale : 0.f;
        }
        *(Pack<T, VEC>*)(y + (row0 + t) * m.y_token + c) = pack<T, VEC>(f);
    }
}

template <typename T, int VEC>
hipError_t launch(const CacheJob& j, bool store, hipStream_t st) {
    const dim3 grid((unsigned)(j.n_seq * j.slots), (unsigned)(2 * j.heads));
    if (store) k_cache_store<T, VEC><<<grid, kThreads, (size_t)min(kPage, j.max_new) * (j.dim + 1) * 4, st>>>(j);
    else k_cache_read<T, VEC><<<grid, kThreads, (size_t)j.dim * (kPage / 4 + 1) * 4, st>>>(j);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache(const CacheJob& j, int dtype, int vec, bool store, hipStream_t st) {
    if (dtype == MDCNN_F32) return vec == 4 ? launch<float, 4>(j, store, st) : launch<float, 1>(j, store, st);
    if (dtype == MDCNN_F16) return vec == 8 ? launch<_Float16, 8>(j, store, st) : launch<_Float16, 1>(j, store, st);
    return vec == 8 ? launch<__bf16, 8>(j, store, st) : launch<__bf16, 1>(j, store, st);
}

}  // namespace mdcnn
