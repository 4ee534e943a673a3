// Keys and values into and out of pages of 8-bit codes.
//
// A page holds 64 tokens: keys [head][token][pitch], values [head][pitch][token], so that the attention's matrix instructions find both with the
// channels (keys) or the tokens (values) they sum over side by side.  One scale for each page and head: max |x| / 127 over its tokens, so
// that a code is off by half a scale at most.  Codes of a page that grows are rounded again; growing by a quarter at least keeps what
// that adds below half of 1 + 0.8 + 0.64 .. = 5, 2.5 codes, however often a page grows.  Scale and quotient are IEEE
// divisions: a code is what the formula says, not a neighbour.
// A block has one page and head of the keys or of the values; the memory bounds it, with one new token the chain table - scale -
// values - code.  Prompts of 9327 tokens, 8 fp16 heads of 128 channels (57 MB each way): stored in 20 us (2.9 TB/s), read back in 15 (3.8); 1300 blocks
// with a maximum over the page between what they read and what they write, 2600 are few for 256 compute units.  One bf16 token to each of 48
// sequences 8 us, the pages they are in read back 8.
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

// Codes of four values, a byte each: the quotients rounded to nearest even.  A product with the reciprocal is off by 2^-15 at most: only where that
// could decide between two codes are the divisions made.
__device__ __forceinline__ unsigned codes_of(const float (&x)[4], float scale, float inverse) {
    if (!(scale > 0.f)) return 0;                                            // all zeros, or not finite
    float q[4], near = inverse < 3e38f ? 0.f : 1.f;                          // (a scale below 2^-128 has no finite reciprocal)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y = x[i] * inverse;
        q[i] = rintf(y);
        near = fmaxf(near, fabsf(y - q[i]));
    }
    if (!(near < 0.4999f))
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = rintf(x[i] / scale);
    unsigned word = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) word |= ((unsigned)(int)fminf(fmaxf(q[i], -127.f), 127.f) & 0xffu) << (8 * i);
    return word;
}
// Old codes of a page whose scale has grown.
__device__ __forceinline__ unsigned smaller(unsigned word, float ratio) {
    unsigned r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= ((unsigned)(int)rintf((float)(int8_t)(word >> (8 * i)) * ratio) & 0xffu) << (8 * i);
    return r;
}

// A thread has VEC channels of four tokens (of four more every pass) in registers from the one read to the codes.  Values are turned in LDS, so that
// they leave as 16 tokens of a channel.
template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void k_cache_store(CacheJob j) {
    constexpr int kPasses = 16 / VEC < 1 ? 1 : 16 / VEC;                     // 256 channels
    extern __shared__ __align__(16) unsigned turned[];                       // values: [dim][kPage / 4 + 4], in words of four tokens
    constexpr int kRow = kPage / 4 + 4;
    __shared__ unsigned s_max[4];
    PageOf p;
    if (!p.find(j) || p.page < 0) return;
    const CacheMap& m = p.is_v ? j.v : j.k;
    const int base = p.slot * kPage;                                         // position of the page's first token
    const int t0 = max(p.first - base, 0), t1 = min(p.count - (base - p.first), kPage);   // its tokens that are new
    const T* x = (const T*)m.x + p.head * m.x_head + ((long long)p.row + (base - p.first)) * m.x_token;
    const int vecs = j.dim / VEC, sets = kThreads / vecs, set = threadIdx.x / vecs, c = (threadIdx.x - set * vecs) * VEC;
    Pack<T, VEC> v[kPasses][4];
    unsigned top = 0;
#pragma unroll
    for (int q = 0; q < kPasses; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * (set + q * sets) + i;
            if (set < sets && t >= t0 && t < t1) v[q][i] = *(const Pack<T, VEC>*)(x + t * m.x_token + c);
        }
#pragma unroll
    for (int q = 0; q < kPasses; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * (set + q * sets) + i;
            if (set < sets && t >= t0 && t < t1) {
                float f[VEC];
                unpack(v[q][i], f);
#pragma unroll
                for (int e = 0; e < VEC; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
            }
        }
    float* scale_at = (p.is_v ? j.v_scale : j.k_scale) + p.page * j.heads + p.head;
    const float old = t0 > 0 ? *scale_at : 0.f;
    top = block_max(top, s_max);                                             // (behind it, everyone has read the old scale)
    const float need = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(top) / 127.f;
    float scale = need, ratio = 1.f;
    if (t0 > 0) {                                                            // the page holds t0 tokens already
        if (need <= old) {
            scale = old;
        } else {
            scale = old != old || need != need ? __uint_as_float(0x7fc00000u) : fmaxf(need, 1.25f * old);
            ratio = scale > 0.f ? old / scale : 0.f;
        }
    }
    if (threadIdx.x == 0) *scale_at = scale;
    const float inverse = 1.f / scale;
    int8_t* codes = (p.is_v ? j.v_codes : j.k_codes) + (p.page * j.heads + p.head) * (long long)(kPage * j.pitch);
    if (!p.is_v) {
        if (ratio != 1.f)
            for (int i = threadIdx.x; i < t0 * (j.dim / 4); i += kThreads) {
                unsigned* at = (unsigned*)(codes + i / (j.dim / 4) * j.pitch + i % (j.dim / 4) * 4);
                *at = smaller(*at, ratio);
            }
#pragma unroll
        for (int q = 0; q < kPasses; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 4 * (set + q * sets) + i;
                if (set < sets && t >= t0 && t < t1) {
                    float f[VEC];
                    unpack(v[q][i], f);
                    int8_t* at = codes + t * j.pitch + c;
                    if constexpr (VEC >= 4) {
                        Pack<unsigned, VEC / 4> w;
#pragma unroll
                        for (int k = 0; k < VEC / 4; ++k) {
                            const float g[4] = {f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]};
                            w.v[k] = codes_of(g, scale, inverse);
                        }
                        *(Pack<unsigned, VEC / 4>*)at = w;
                    } else {
                        const float g[4] = {f[0], 0.f, 0.f, 0.f};
                        *at = (int8_t)codes_of(g, scale, inverse);
                    }
                }
            }
        return;
    }
    if (set < sets)
#pragma unroll
        for (int q = 0; q < kPasses; ++q) {
            const int t = 4 * (set + q * sets);
            if (t < kPage && t + 4 > t0 && t < t1) {
                float f[4][VEC];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (t + i >= t0 && t + i < t1) {
                        unpack(v[q][i], f[i]);
                    } else {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) f[i][e] = 0.f;
                    }
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float g[4] = {f[0][e], f[1][e], f[2][e], f[3][e]};
                    turned[(c + e) * kRow + t / 4] = codes_of(g, scale, inverse);
                }
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < j.dim * (kPage / 16); i += kThreads) {
        const int ch = i / (kPage / 16), t = i % (kPage / 16) * 16;
        if (t >= t1 || (t + 16 <= t0 && ratio == 1.f)) continue;
        Pack<unsigned, 4>* at = (Pack<unsigned, 4>*)(codes + ch * kPage + t);
        Pack<unsigned, 4> w = *(const Pack<unsigned, 4>*)(turned + ch * kRow + t / 4);
        if (t < t0 || t + 16 > t1) {                                         // codes that stay
            const Pack<unsigned, 4> was = *at;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int a = t + 4 * k;                                     // bytes a .. a + 3, of which t0 <= byte < t1 are new
                unsigned fresh = 0xffffffffu;
                if (a < t0) fresh = a + 4 <= t0 ? 0u : fresh << (8 * (t0 - a));
                if (a + 4 > t1) fresh &= a >= t1 ? 0u : 0xffffffffu >> (8 * (a + 4 - t1));
                const unsigned kept = ratio != 1.f && a < t0 ? smaller(was.v[k], ratio) : was.v[k];
                w.v[k] = (w.v[k] & fresh) | (kept & ~fresh);
            }
        }
        *at = w;
    }
}

// Values of a page and head back: a thread has eight channels of four tokens.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_cache_read(CacheJob j) {
    extern __shared__ __align__(16) unsigned turned[];                       // values: [dim][kPage / 4 + 4]
    constexpr int kRow = kPage / 4 + 4;
    PageOf p;
    if (!p.find(j)) return;
    const CacheMap& m = p.is_v ? j.v : j.k;
    const int base = p.slot * kPage;
    const int t0 = max(p.first - base, 0), t1 = min(p.count - (base - p.first), kPage);
    T* y = (T*)m.y + p.head * m.y_head + ((long long)p.row + (base - p.first)) * m.y_token;
    const bool there = p.page >= 0;
    const long long at = there ? p.page * j.heads + p.head : 0;
    const float scale = there ? (p.is_v ? j.v_scale : j.k_scale)[at] : 0.f;
    const int8_t* codes = (p.is_v ? j.v_codes : j.k_codes) + at * (kPage * j.pitch);
    if (p.is_v && there) {
        for (int i = threadIdx.x; i < j.dim * (kPage / 16); i += kThreads)
            *(Pack<unsigned, 4>*)(turned + i / (kPage / 16) * kRow + i % (kPage / 16) * 4) = *(const Pack<unsigned, 4>*)(codes + i * 16);
        __syncthreads();
    }
    const int vecs = j.dim / 8, sets = kThreads / vecs, set = threadIdx.x / vecs, c = (threadIdx.x - set * vecs) * 8;
    if (set >= sets) return;
    for (int t = 4 * set; t < t1; t += 4 * sets) {
        if (t + 4 <= t0) continue;
        unsigned w[8];                                                       // values: word e has channel c + e of the four tokens; keys: words 2 i, 2 i + 1 token i
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = there ? p.is_v ? turned[(c + e) * kRow + t / 4] : *(const unsigned*)(codes + (t + e / 2) * j.pitch + c + e % 2 * 4) : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (t + i < t0 || t + i >= t1) continue;
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int q = p.is_v ? (int8_t)(w[e] >> (8 * i)) : (int8_t)(w[2 * i + e / 4] >> (8 * (e % 4)));
                f[e] = there ? (float)q * scale : 0.f;
            }
            T* to = y + (t + i) * m.y_token + c;
            if constexpr (WHOLE) {
                constexpr int N = 16 / sizeof(T);
#pragma unroll
                for (int k = 0; k < 8 / N; ++k) {
                    float g[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) g[e] = f[N * k + e];
                    *(Pack<T, N>*)(to + N * k) = pack<T, N>(g);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) to[e] = (T)f[e];
            }
        }
    }
}

template <typename T, int VEC>
hipError_t launch(const CacheJob& j, bool store, hipStream_t st) {
    const dim3 grid((unsigned)(j.n_seq * j.slots), (unsigned)(2 * j.heads));
    const size_t lds = (size_t)j.dim * (kPage / 4 + 4) * 4;
    if (store) k_cache_store<T, VEC><<<grid, kThreads, lds, st>>>(j);
    else k_cache_read<T, (VEC > 1)><<<grid, kThreads, lds, st>>>(j);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache(const CacheJob& j, int dtype, int vec, bool store, hipStream_t st) {
    if (dtype == MDCNN_F32) return vec == 4 ? launch<float, 4>(j, store, st) : launch<float, 1>(j, store, st);
    if (dtype == MDCNN_F16) return vec == 8 ? launch<_Float16, 8>(j, store, st) : launch<_Float16, 1>(j, store, st);
    return vec == 8 ? launch<__bf16, 8>(j, store, st) : launch<__bf16, 1>(j, store, st);
}

}  // namespace mdcnn
