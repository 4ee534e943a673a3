// Attention over a cache of 8-bit pages, tiles of 128 rows: prompts and the pixels of frames.
//
// A block has 128 rows of one sequence and head, four waves 32 each.  A page's codes are made halves once, on their way to LDS (the next
// page's are loaded while this one is worked on), and read by the four waves.  Per page and wave: 64 x 32 products of the keys with the
// queries (v_mfma_f32_32x32x16_f16, the queries stay in registers), the weights, as many products with the values; the weights need not leave
// the registers they come to be in (attend_device.h).
// What bounds it is the issue of vector instructions beside the matrix ones (an exponential, a product and sum, a sum and half a conversion for each weight, ten
// to make eight codes halves): 56 and 39 % of the busy time with 128 channels.  4 x 4096 queries of 32 bf16 heads of 128 channels over 8 and 8192 tokens
// 2.35 ms, 935 TFLOP/s (64 channels 1.36 ms, 805; 32 channels, 16 x 2048 queries of 8 heads, 0.52 ms, 530).
// Weights of 16-bit calls are one half: it takes up to 2^-12 of each, and fp16 results of 32 channels are off by 2.3e-4 of their norm instead of 2.1e-4, bf16 ones by 1.7e-3 with either.
// As two halves 2 x 1728 pixels over 13824 tokens of 8 heads of 32 would take 191 us instead of 149, three prompts of 128 channels 909 instead of 680.
// Rows of LDS are 16-byte chunks that are permuted by their row (chunk ^ row), so that neither the reads of 16 rows side by side nor the
// writes meet in a bank.
#include "attend_device.h"

namespace mdcnn {

namespace {

constexpr int kThreads = 256;
constexpr int kPage = MDCNN_PAGE_TOKENS;

// LDS of a page: keys [64 rows][pitch of a power of two] and values [DP rows][64], as halves, and what the mask adds to a token.
template <int DP>
struct Stage {
    static constexpr int kRow = DP <= 32 ? 32 : DP <= 64 ? 64 : DP <= 128 ? 128 : 256;     // halves of a row of keys
    static constexpr int kKeys = kPage * kRow, kValues = DP * kPage;
    static constexpr int kBytes = (kKeys + kValues) * 2 + kPage * 4 + 16;               // .. and the two scales
    // rows of the first product: MFMA row m of tile a is row 32 a + m, token 32 (m / 4 % 2) + 16 a + 4 (m / 8) + m % 4
    __device__ static __forceinline__ int row_of(int t) { return 32 * (t >> 4 & 1) + 8 * (t >> 2 & 3) + 4 * (t >> 5) + (t & 3); }
    __device__ static __forceinline__ int key_at(int row, int chunk) {
        constexpr int kChunks = kRow / 8, kShift = kChunks == 4 ? 2 : kChunks == 8 ? 1 : 0;
        return row * kRow + ((chunk ^ (row >> kShift & (kChunks < 16 ? kChunks - 1 : 15))) << 3);
    }
    __device__ static __forceinline__ int value_at(int d, int chunk) { return kKeys + d * kPage + ((chunk ^ (d >> 1 & 7)) << 3); }
};

// Matrix instructions in turn with reads of LDS that are AHEAD of them, N of each.
template <int N, int AHEAD>
__device__ __forceinline__ void ahead_of() {
    constexpr int kFirst = AHEAD < N ? AHEAD : N;
    __builtin_amdgcn_sched_group_barrier(0x100, kFirst, 0);
#pragma unroll
    for (int i = 0; i < N - kFirst; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, kFirst, 0);
}

// LDS is waited for, loads from memory are not.
__device__ __forceinline__ void page_over() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// More waves to a SIMD help: one wave issues a vector instruction every five
// cycles, two or three together one every three.  (64 channels of 16 bits: two waves 1468 us for 4 x 4096 queries of 32 heads over 8192 tokens, three 1360.)
template <typename T, int DP, bool MASK>
__global__ __launch_bounds__(kThreads, attend_tile_blocks(sizeof(T), DP)) void k_attend_tiles(AttendJob j) {
    constexpr bool kTwo = sizeof(T) == 4;
    constexpr int NS = DP / 16, ND = DP / 32, NL = DP / 32;               // steps of channels, tiles of channels, 16-byte loads of a thread
    constexpr int kHeld = DP > 192 ? 9 : NS;                              // steps of the queries in registers; the others lie in LDS behind the two stages
    constexpr bool kAhead = DP <= 192;                                    // the next page's codes wait in registers while this one is worked on
    constexpr bool kAnew = DP > 128 || (DP == 64 && MASK);                // places in LDS are worked out anew for each page: registers are short
    using S = Stage<DP>;
    extern __shared__ __align__(16) unsigned char lds[];
    unsigned b = blockIdx.x;
    const int head = b % j.heads;                          // (tiles of a head on one XCD where there are eight heads)
    b /= j.heads;
    const int seq = b % j.n_seq;
    b /= j.n_seq;
    const int tile = j.tiles - 1 - b % j.tiles, split = b / j.tiles;       // the last tiles see most: they begin first
    Rows s;
    if (!s.load(j, seq)) return;
    const int r0 = tile * kAttendTile, r1 = min(r0 + kAttendTile, s.rows);
    if (r0 >= s.rows) return;
    const Run run(j, s, r0, r1, split);
    if (split > 0 && run.first >= run.last) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;

    const int row = r0 + 32 * wave + n, query = row / j.group;
    const bool live = row < s.rows;
    half8 qh[kHeld], ql[kTwo ? NS : 1];
    half8* beyond = (half8*)(lds + 2 * S::kBytes) + threadIdx.x;
    int e;
    bool spoiled;
    {
        const T* q = (const T*)j.q + (s.q0 + (live ? query : 0)) * j.q_token + (long long)(head * j.group + (live ? row % j.group : 0)) * j.q_head;
        float top = 0.f, zero = 0.f;
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            float f[8];
            eight_of(q, 16 * st + 8 * half, live ? j.dim : 0, j.q_whole, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                top = fmaxf(top, fabsf(f[i]));
                zero = __builtin_fmaf(f[i], 0.f, zero);
            }
        }
        spoiled = row_of_two(zero != zero, n);
        top = max_over_32(top);
        e = exponent_of(top);
        const float sign = j.scale < 0.f ? -1.f : 1.f;
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            float f[8];
            eight_of(q, 16 * st + 8 * half, live ? j.dim : 0, j.q_whole, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[i] = spoiled ? 0.f : scaled(f[i], -e) * sign;
                if constexpr (kTwo) ql[st][i] = (_Float16)(f[i] - (float)(_Float16)f[i]);
            }
            half8 h;
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = (_Float16)f[i];
            if (st < kHeld) qh[st < kHeld ? st : 0] = h;
            else beyond[(st - kHeld) * kThreads] = h;
        }
    }
    const float logit = spoiled ? kSpoiled : scaled(fabsf(j.scale) * kLog2E, e);
    const int hi = live ? s.hi(j, query) : 0, lo = live ? s.lo(j, query) : 0;
    // of the wave's rows: what every one sees, what any one sees
    const int w0 = min(r0 + 32 * wave, s.rows - 1) / j.group, w1 = min(r0 + 32 * wave + 31, s.rows - 1) / j.group;
    const bool any_row = r0 + 32 * wave < s.rows;
    const int all_hi = s.hi(j, w0), all_lo = s.lo(j, w1), any_hi = any_row ? s.hi(j, w1) : 0, any_lo = s.lo(j, w0);
    const uint8_t* mask = MASK ? j.mask + seq * j.mask_row : nullptr;

    float top = -INFINITY, sum = 0.f;                      // T and sum of this lane's row
    float valued = 0.f;                                    // 1: the row has seen values (a mask would take two scalar registers, which are short)
    ValueScale val;
    float16v out[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) out[d][i] = 0.f;

    PageIds page(j, seq, run, run.first, lane);
    // a thread's loads: 16 codes of a key or of a channel's values each, consecutive ones side by side
    constexpr int kKeyLoads = kPage * DP / 16;
    uint4v codes[NL];
    unsigned char seen_byte = 1;
    float scale = 0.f;
    auto load = [&](int id, int p) {
        const long long at = ((long long)max(id, 0) * j.heads + head) * (kPage * DP);
#pragma unroll
        for (int q = 0; q < NL; ++q) {
            const int i = threadIdx.x + kThreads * q;
            codes[q] = *(const uint4v*)((i < kKeyLoads ? j.k_codes : j.v_codes - kPage * DP) + at + 16 * i);
        }
        if (threadIdx.x < 2) scale = (threadIdx.x ? j.v_scale : j.k_scale)[(long long)max(id, 0) * j.heads + head];
        if (MASK && threadIdx.x < kPage) seen_byte = p * kPage + (int)threadIdx.x < s.len ? mask[p * kPage + threadIdx.x] : 0;
    };
    auto stage = [&](_Float16* to) {
        int thread = threadIdx.x;
        if (kAnew) asm volatile("" : "+v"(thread));
#pragma unroll
        for (int q = 0; q < NL; ++q) {
            const int i = thread + kThreads * q;
            int a, c;
            if (i < kKeyLoads) {
                const int r = S::row_of(i / (DP / 16)), chunk = i % (DP / 16) * 2;
                a = S::key_at(r, chunk);
                c = S::key_at(r, chunk + 1);
            } else {
                const int k = i - kKeyLoads, d = k / (kPage / 16), chunk = k % (kPage / 16) * 2;
                a = S::value_at(d, chunk);
                c = S::value_at(d, chunk + 1);
            }
            *(half8*)(to + a) = halves_of(codes[q][0], codes[q][1]);
            *(half8*)(to + c) = halves_of(codes[q][2], codes[q][3]);
        }
        float* beside = (float*)(to + S::kKeys + S::kValues);
        if (threadIdx.x < 2) beside[kPage + threadIdx.x] = scale;
        if (MASK && threadIdx.x < kPage) beside[threadIdx.x] = seen_byte ? 0.f : -INFINITY;
    };
    int id = page.at(run.first), next = page.at(run.first + 1);
    _Float16* now = (_Float16*)lds;
    _Float16* then = (_Float16*)(lds + S::kBytes);
    if (run.first < run.last) {
        load(id, run.first);
        stage(now);
    }
    __syncthreads();
    for (int p = run.first; p < run.last; ++p) {
        const int after = page.at(p + 2);
        if (kAhead && p + 1 < run.last) load(next, p + 1);
        const int pos = p * kPage;
        if (id >= 0 && pos < any_hi && pos + kPage > any_lo) {
            const float* beside = (const float*)(now + S::kKeys + S::kValues);
            const float ks = uniform(beside[kPage]), vs = uniform(beside[kPage + 1]);
            int place = n;
            if (kAnew) asm volatile("" : "+v"(place));
            float16v x[2];
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                if constexpr (MASK) {
                    const float4v* add = (const float4v*)(beside + 32 * half + 16 * a);
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[a][i] = add[i / 4][i % 4];
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[a][i] = 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 2 * NS; ++i) {             // the two sums in turn, so that neither waits for itself; where registers are short one by one
                const int st = DP <= 128 ? i / 2 : i % NS, a = DP <= 128 ? i % 2 : i / NS;
                const half8 k = *(const half8*)(now + S::key_at(32 * a + place, 2 * st + half));
                x[a] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, st < kHeld ? qh[st < kHeld ? st : 0] : beyond[(st - kHeld) * kThreads], x[a], 0, 0, 0);
                if constexpr (kTwo) x[a] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, ql[st], x[a], 0, 0, 0);
            }
            // x[a][i] is token 32 half + 16 a + i
            if (pos < all_lo || pos + kPage > all_hi) {
                const int from = lo - pos - 32 * half, to = hi - pos - 32 * half;
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (16 * a + i < from || 16 * a + i >= to) x[a][i] = -INFINITY;
            }
            const float by = factor_of(logit, ks);
            val.next(vs);
            bool bad = false;                              // the row sees tokens whose scale is not a number
            if (__builtin_expect(ks != ks || val.bad, 0)) {
#pragma unroll
                for (int t = 0; t < 32; ++t) bad = bad || x[t / 16][t % 16] != -INFINITY;
                bad = row_of_two(bad, n);
            }
            if (ks == ks) {
                // weights, at first as if T stayed
                float add;
                half8 ph[4], pl[kTwo ? 4 : 1];
                auto weigh = [&]() {
                    const float base = val.base(top);
                    float part[4];
#pragma unroll
                    for (int t = 0; t < 32; ++t) {
                        const float w = exp2_fast(__builtin_fmaf(x[t / 16][t % 16], by, base));
                        part[t % 4] = t < 4 ? w : part[t % 4] + w;
                        ph[t / 8][t % 8] = (_Float16)w;
                        if constexpr (kTwo) pl[t / 8][t % 8] = (_Float16)((w - (float)ph[t / 8][t % 8]) * kSecond);
                        if (t % 8 == 7) __builtin_amdgcn_sched_barrier(0);           // eight at a time: registers are short
                    }
                    add = (part[0] + part[1]) + (part[2] + part[3]);
                };
                weigh();
                const bool values = !val.none && !val.bad;
                bool moves = add > much(val) || (live && valued == 0.f);
                if (__builtin_expect(__any(moves), 0)) {
                    moves = row_of_two(moves, n);
                    float m[4] = {x[0][0], x[0][1], x[0][2], x[0][3]};
#pragma unroll
                    for (int t = 4; t < 32; ++t) m[t % 4] = fmaxf(m[t % 4], x[t / 16][t % 16]);
                    const float most = max_over_32(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]))) * by + val.log();
                    const NextTop to(top, most, moves, values, valued);
                    top = to.top;
                    sum *= to.fade;
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) out[d][i] *= to.fade_out;
                    weigh();
                }
                sum += add * kUnroom * val.inverse();
                auto add_values = [&]() __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < 4 * ND; ++i) {
                        const int st = DP <= 128 ? i / ND : i % 4, d = DP <= 128 ? i % ND : i / 4;
                        const half8 v = *(const half8*)(now + S::value_at(32 * d + place, 4 * half + st));
                        out[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, ph[st], out[d], 0, 0, 0);
                        if constexpr (kTwo) out[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v * kSecondBack, pl[st], out[d], 0, 0, 0);
                    }
                };
                auto spoil = [&]() __attribute__((always_inline)) {
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) out[d][i] = bad ? vs : out[d][i];
                };
                if constexpr (DP <= 128) {
                    // Nothing is added: by weights of zero, so that the sums are moved into no other registers (64 moves a page with 128 channels).
                    if (__builtin_expect(!values, 0)) {
#pragma unroll
                        for (int t = 0; t < 32; ++t) {
                            ph[t / 8][t % 8] = 0;
                            if constexpr (kTwo) pl[t / 8][t % 8] = 0;
                        }
                        if (val.bad) spoil();
                    }
                    add_values();
                    if constexpr (!kTwo) ahead_of<4 * ND, 6>();
                } else if (__builtin_expect(val.bad, 0)) {
                    spoil();
                } else if (!val.none) {
                    add_values();
                }
            } else {
                sum = bad ? ks : sum;
            }
        }
        if (!kAhead && p + 1 < run.last) load(next, p + 1);
        if (p + 1 < run.last) stage(then);
        page_over();
        _Float16* swap = now;
        now = then;
        then = swap;
        id = next;
        next = after;
    }
    if (!live) return;
    if (logit == kSpoiled && top > -INFINITY) sum = NAN;
    sum += __shfl_xor(sum, 32, 64);
    const bool whole = run.splits <= 1;
    const long long slot = ((((long long)seq * j.heads + head) * j.tiles + tile) * j.splits + split) * kAttendTile + 32 * wave + n;
    const float inv = whole ? (top == -INFINITY && sum == 0.f ? 0.f : 1.f / sum) : 1.f;
    T* y = (T*)j.y + (s.q0 + query) * j.y_token + (long long)(head * j.group + row % j.group) * j.y_head;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = 32 * d + 8 * q + 4 * half;       // four channels beside one another
            if (!whole) {
                *(float4v*)(j.part_out + slot * DP + c) = float4v{out[d][4 * q], out[d][4 * q + 1], out[d][4 * q + 2], out[d][4 * q + 3]} * kUnroom;
            } else if (c < j.dim) {
#pragma unroll
                for (int i = 0; i < 4; ++i) y[c + i] = (T)(out[d][4 * q + i] * kUnroom * inv);
            }
        }
    if (half == 0) {
        if (!whole) j.part_top[slot] = float2{top, sum};
        else if (j.lse) j.lse[(s.q0 + query) * (j.heads * j.group) + head * j.group + row % j.group] = kLn2 * (top + __log2f(sum));
    }
}

struct Tiles {
    template <typename T, int DP>
    static hipError_t go(const AttendJob& j, hipStream_t st) {
        if constexpr (sizeof(T) == 4 && DP > 192) return hipErrorInvalidValue;           // (no registers for them: attend_tiles_fit)
        else return j.mask ? tiles<T, DP, true>(j, st) : tiles<T, DP, false>(j, st);
    }
    template <typename T, int DP, bool MASK>
    static hipError_t tiles(const AttendJob& j, hipStream_t st) {
        constexpr int kLds = 2 * Stage<DP>::kBytes + (DP > 192 ? (DP / 16 - 9) * kThreads * 16 : 0);
        const auto kern = k_attend_tiles<T, DP, MASK>;
        if (kLds > 64 * 1024) {
            const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
            if (err != hipSuccess) return err;
        }
        kern<<<(unsigned)((long long)j.splits * j.tiles * j.n_seq * j.heads), kThreads, kLds, st>>>(j);
        return hipGetLastError();
    }
};

}  // namespace

bool attend_tiles_fit(int dtype, int pitch) { return dtype != MDCNN_F32 || pitch <= 192; }
hipError_t launch_attend_tiles(const AttendJob& j, int dtype, hipStream_t st) { return for_type_and_pitch<Tiles>(j, dtype, st); }

}  // namespace mdcnn
