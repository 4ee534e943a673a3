// Attention over a cache of 8-bit pages, rows by sixteen: single tokens, a few queries, anything (the tiles of prompts and frames:
// kernels_attend_tiles.hip).
//
// With few rows the cache's bytes bound it: each is read once, 16 bytes a lane, straight into the registers of the wave that multiplies
// them; the next page's keys are on their way while the softmax and the values of this one are worked on, and the other way
// round.  A wave has pages of its own (every fourth of its block's run) with a maximum and a sum of its own; the four are joined
// in LDS.  Runs of pages are split over blocks where rows alone would not fill the GPU, and joined by a second launch.
// One bf16 token of 32 heads over 8 for each of 48 sequences of 1 to 16384 tokens (193 MB) 51-54 us, 3.6 TB/s (the longest sequences end last), and 5 to join;
// two sequences of 150001 tokens, 2 heads (154 MB) 28 us, 5.4 TB/s, and 6 to join; 700 tokens of fp32 9 us.
#include "attend_device.h"

namespace mdcnn {

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kPage = MDCNN_PAGE_TOKENS;

// Place of a block.  Heads and sequences lie side by side and splits last: neighbouring blocks go to different XCDs, and only the first
// splits of short sequences have work.  (Splits side by side, 32 of them: all first ones on one XCD, 194 us for 48 sequences instead of 62.)
struct AttendBlock {
    int split, tile, head, seq;
    __device__ __forceinline__ AttendBlock(const AttendJob& j, unsigned b) {
        head = b % j.heads;
        b /= j.heads;
        seq = b % j.n_seq;
        b /= j.n_seq;
        tile = b % j.tiles;
        split = b / j.tiles;
    }
};

// TWO: weights as two halves, 22 bits, else one, 11 bits.  fp32 calls always; 16-bit ones where sixteen rows are all there are, whose results are then those of weights in 32
// bits rounded once.  One half / two, 16 bf16 sequences of 8192 tokens, 8 heads: 1 row of 64 channels 30.2 / 31.5 us, of 128 47.5 / 48.0, of 256 109 / 111;
// 64 rows 63.5 / 77.6, 118 / 123, 294 / 319, more than the bits are worth: one half takes up to 2^-12 of a weight, fp16 results are off by 2.3e-4 of their norm
// instead of 2.1e-4, bf16 ones by 1.7e-3 with either.  The second half of 16-bit calls is what the first leaves, 2^-35 of the largest weight at its finest; in fp32
// calls 2^11 times that (attend_device.h).
template <typename T, int DP, bool TWO>
__global__ __launch_bounds__(kThreads, DP <= 128 ? 2 : 1) void k_attend_rows(AttendJob j) {
    constexpr bool kTwo = sizeof(T) == 4;                  // fp32 queries as sums of two halves
    constexpr int NS = DP / 32, NV = DP / 16;              // steps of 32 channels, tiles of 16
    constexpr int U = DP / 64;                             // pairs of steps that a 16-byte load serves
    __shared__ float s_top[kWaves][16], s_sum[kWaves][16];
    __shared__ __align__(16) float s_out[kWaves][16][DP + 4];
    const AttendBlock blk(j, blockIdx.x);
    const int head = blk.head, seq = blk.seq;
    Rows s;
    if (!s.load(j, seq)) return;
    const int r0 = blk.tile * 16, r1 = min(r0 + 16, s.rows);
    if (r0 >= s.rows) return;
    const Run run(j, s, r0, r1, blk.split);
    if (blk.split > 0 && run.first >= run.last) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, quad = lane >> 4;

    // Queries of this lane's row, channels in the order in which the keys are loaded.
    const int row = r0 + n, query = row / j.group;
    const bool live = row < s.rows;
    const T* q = (const T*)j.q + (s.q0 + (live ? query : 0)) * j.q_token + (long long)(head * j.group + (live ? row % j.group : 0)) * j.q_head;
    half8 qh[NS], ql[kTwo ? NS : 1];
    int e;
    bool spoiled;
    {
        float f[NS][8], top = 0.f, zero = 0.f;
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            eight_of(q, st < 2 * U ? 64 * (st / 2) + 16 * quad + 8 * (st & 1) : 64 * U + 8 * quad, live ? j.dim : 0, j.q_whole, f[st]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                top = fmaxf(top, fabsf(f[st][i]));
                zero = __builtin_fmaf(f[st][i], 0.f, zero);
            }
        }
        spoiled = row_of_four(zero != zero, n);
        top = max_over_32(max_over_16(top));
        e = exponent_of(top);
        const float sign = j.scale < 0.f ? -1.f : 1.f;
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = spoiled ? 0.f : scaled(f[st][i], -e) * sign;
                qh[st][i] = (_Float16)x;
                if constexpr (kTwo) ql[st][i] = (_Float16)(x - (float)qh[st][i]);
            }
    }
    const float logit = spoiled ? kSpoiled : scaled(fabsf(j.scale) * kLog2E, e);         // (the queries have its sign)
    const int hi = live ? s.hi(j, query) : 0, lo = live ? s.lo(j, query) : 0;
    const int all_hi = s.hi(j, r0 / j.group), all_lo = s.lo(j, (r1 - 1) / j.group);      // seen by every row
    const uint8_t* mask = j.mask ? j.mask + seq * j.mask_row : nullptr;

    float top = -INFINITY, sum = 0.f;                      // T and sum of this lane's row
    float valued = 0.f;                                    // 1: the row has seen values (a mask would take two scalar registers, which are short)
    ValueScale val;
    float4v out[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) out[v] = float4v{0.f, 0.f, 0.f, 0.f};

    PageIds page(j, seq, run, run.first, lane);
    const int per_head = kPage * DP;
    uint4v kr[4][U ? U : 1];
    uint2v kx[4];
    uint4v vr[NV];
    // Scales come by vector loads ahead of the keys, whose return they do not wait for.
    int beside;
    asm("v_mov_b32 %0, 0" : "=v"(beside));
    float ks = 0.f, vs = 0.f;
    auto load_scales = [&](int id) {
        const long long at = (long long)max(id, 0) * j.heads + head + beside;
        ks = j.k_scale[at];
        vs = j.v_scale[at];
    };
    // (no page: what the first one holds, which is then not looked at; there is one wherever there is a run)
    auto load_keys = [&](int id) {
        const int8_t* k = j.k_codes + ((long long)max(id, 0) * j.heads + head) * per_head;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int8_t* r = k + (16 * (n >> 2) + 4 * t + (n & 3)) * DP;
#pragma unroll
            for (int u = 0; u < U; ++u) kr[t][u] = *(const uint4v*)(r + 64 * u + 16 * quad);
            if constexpr (DP % 64 != 0) kx[t] = *(const uint2v*)(r + 64 * U + 8 * quad);
        }
    };
    auto load_values = [&](int id) {
        const int8_t* v = j.v_codes + ((long long)max(id, 0) * j.heads + head) * per_head;
#pragma unroll
        for (int t = 0; t < NV; ++t) vr[t] = *(const uint4v*)(v + (16 * t + n) * kPage + 16 * quad);
    };
    int p = run.first + wave, id = page.at(p), next = page.at(p + kWaves);
    if (p < run.last) {
        load_scales(id);
        load_keys(id);
        load_values(id);
    }
    for (; p < run.last; p += kWaves) {
        const int after = page.at(p + 2 * kWaves);
        if (id < 0) {                                      // no page: its tokens do not exist
            id = next;
            next = after;
            load_scales(id);
            load_keys(id);
            load_values(id);
            continue;
        }
        float4v acc[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            acc[t] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                const half8 k = st < 2 * U ? (st & 1 ? halves_of(kr[t][st / 2][2], kr[t][st / 2][3]) : halves_of(kr[t][st / 2][0], kr[t][st / 2][1])) : halves_of(kx[t][0], kx[t][1]);
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, qh[st], acc[t], 0, 0, 0);
                if constexpr (kTwo) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, ql[st], acc[t], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);             // or all codes are made halves first, in as many registers
        }
        const float by = factor_of(logit, uniform(ks)), vs_now = uniform(vs);
        load_scales(next);
        load_keys(next);
        val.next(vs_now);
        float x[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) x[t] = acc[t / 4][t % 4];
        unsigned seen = 0xffffu;
        const int pos = p * kPage + 16 * quad;
        if (p * kPage < all_lo || (p + 1) * kPage > all_hi || mask) {
            if (mask) seen = mask_bits(mask, pos, s.len, j.mask_whole);
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                if (pos + t < lo || pos + t >= hi) seen &= ~(1u << t);
                x[t] = seen >> t & 1 ? x[t] : -INFINITY;
            }
        }
        if (by == by) {
            // weights, at first as if T stayed
            float add;
            half8 ph[2], pl[TWO ? 2 : 1];
            auto weigh = [&]() {
                const float base = val.base(top);
                float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    const float w = exp2_fast(__builtin_fmaf(x[t], by, base));
                    part[t % 4] += w;
                    ph[t / 8][t % 8] = (_Float16)w;
                    if constexpr (TWO) pl[t / 8][t % 8] = (_Float16)((w - (float)ph[t / 8][t % 8]) * (kTwo ? kSecond : 1.f));
                }
                add = (part[0] + part[1]) + (part[2] + part[3]);
            };
            weigh();
            const bool values = !val.none && !val.bad;
            bool moves = add > much(val) || (live && valued == 0.f);
            if (__any(moves)) {
                moves = row_of_four(moves, n);
                float m[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                for (int t = 4; t < 16; ++t) m[t % 4] = fmaxf(m[t % 4], x[t]);
                const float most = max_over_32(max_over_16(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])))) * by + val.log();
                const NextTop to(top, most, moves, values, valued);
                top = to.top;
                sum *= to.fade;
#pragma unroll
                for (int v = 0; v < NV; ++v) out[v] *= to.fade_out;
                weigh();
            }
            sum += add * kUnroom * val.inverse();
            if (val.bad) {
                const bool bad = row_of_four(seen != 0, n);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < 4; ++i) out[v][i] = bad ? vs_now : out[v][i];
            } else if (!val.none) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const half8 a = halves_of(vr[v][0], vr[v][1]), b = halves_of(vr[v][2], vr[v][3]);
                    out[v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, ph[0], out[v], 0, 0, 0);
                    out[v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b, ph[1], out[v], 0, 0, 0);
                    if constexpr (TWO) {
                        out[v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kTwo ? a * kSecondBack : a, pl[0], out[v], 0, 0, 0);
                        out[v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kTwo ? b * kSecondBack : b, pl[1], out[v], 0, 0, 0);
                    }
                    if (v % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {                                           // the row sees tokens whose scale is not a number
            sum = row_of_four(seen != 0, n) ? by : sum;
        }
        id = next;
        next = after;
        load_values(id);
    }
    if (logit == kSpoiled && top > -INFINITY) sum = NAN;
    // join the four waves
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (quad == 0) { s_top[wave][n] = top; s_sum[wave][n] = sum; }
#pragma unroll
    for (int v = 0; v < NV; ++v) *(float4v*)&s_out[wave][n][16 * v + 4 * quad] = out[v];
    __syncthreads();
    const int m = threadIdx.x / 16, c0 = threadIdx.x % 16;
    if (r0 + m >= s.rows) return;
    float peak = s_top[0][m], total = 0.f, weight[kWaves];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) peak = fmaxf(peak, s_top[w][m]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        weight[w] = exp2_fast(s_top[w][m] - (peak == -INFINITY ? 0.f : peak));
        total += weight[w] * s_sum[w][m];
    }
    const bool whole = run.splits <= 1;
    const int r = r0 + m;
    const long long slot = (((long long)seq * j.heads + head) * j.tiles + blk.tile) * j.splits + blk.split;
    T* y = (T*)j.y + (s.q0 + r / j.group) * j.y_token + (long long)(head * j.group + r % j.group) * j.y_head;
    const float inv = peak == -INFINITY && total == 0.f ? 0.f : 1.f / total;
    for (int c = c0; c < DP; c += 16) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x += weight[w] * s_out[w][m][c];
        x *= kUnroom;
        if (!whole) j.part_out[(slot * 16 + m) * DP + c] = x;
        else if (c < j.dim) y[c] = (T)(x * inv);
    }
    if (c0 == 0) {
        if (!whole) j.part_top[slot * 16 + m] = float2{peak, total};
        else if (j.lse) j.lse[(s.q0 + r / j.group) * (j.heads * j.group) + head * j.group + r % j.group] = kLn2 * (peak + __log2f(total));
    }
}

// Joins the splits of rows.  A thread has four channels of a row and every j.sets-th split; a block as many rows as it has threads for.
template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void k_attend_join(AttendJob j) {
    constexpr int kLanes = DP / 4;
    __shared__ float4v s_part[kThreads];
    __shared__ float2 s_top[kThreads];
    const int per_block = kThreads / (kLanes * j.sets), blocks = (j.max_new * j.group + per_block - 1) / per_block;
    const int c = threadIdx.x % kLanes, set = threadIdx.x / kLanes % j.sets, slot_row = threadIdx.x / (kLanes * j.sets);
    const int r = blockIdx.x % blocks * per_block + slot_row, head = blockIdx.x / blocks % j.heads, seq = blockIdx.x / blocks / j.heads;
    Rows s;
    const bool any = s.load(j, seq);
    const int tile = r / j.tile_rows, m = r % j.tile_rows;
    bool on = any && slot_row < per_block && r < s.rows;
    int splits = 0;
    if (on) splits = Run(j, s, tile * j.tile_rows, min((tile + 1) * j.tile_rows, s.rows), 0).splits;
    on = on && splits > 1;                                 // (a single one has written the row itself)
    const long long slot = (((long long)seq * j.heads + head) * j.tiles + tile) * j.splits;
    float top = -INFINITY, total = 0.f;
    float4v x = float4v{0.f, 0.f, 0.f, 0.f};
    auto take = [&](float2 t, float4v y) {
        const float next = fmaxf(top, t.x), base = next == -INFINITY ? 0.f : next, fade = exp2_fast(top - base), w = exp2_fast(t.x - base);
        top = next;
        total = total * fade + t.y * w;
        x = x * fade + y * w;
    };
    if (on) {
#pragma unroll 4
        for (int z = set; z < splits; z += j.sets) {
            const long long at = (slot + z) * j.tile_rows + m;
            take(j.part_top[at], *(const float4v*)(j.part_out + at * DP + 4 * c));
        }
    }
    if (j.sets > 1) {
        s_part[threadIdx.x] = x;
        s_top[threadIdx.x] = float2{top, total};
        __syncthreads();
        on = on && set == 0;
        if (on)
            for (int k = 1; k < j.sets; ++k) take(s_top[threadIdx.x + k * kLanes], s_part[threadIdx.x + k * kLanes]);
    }
    if (!on) return;
    const float inv = top == -INFINITY && total == 0.f ? 0.f : 1.f / total;
    T* y = (T*)j.y + (s.q0 + r / j.group) * j.y_token + (long long)(head * j.group + r % j.group) * j.y_head;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * c + i < j.dim) y[4 * c + i] = (T)(x[i] * inv);
    if (c == 0 && j.lse) j.lse[(s.q0 + r / j.group) * (j.heads * j.group) + head * j.group + r % j.group] = kLn2 * (top + __log2f(total));
}

template <typename T, int DP>
hipError_t launch_join(AttendJob j, hipStream_t st) {
    if (j.splits < 2) return hipSuccess;
    // up to eight splits to a thread, as far as a block has threads
    j.sets = 1;
    while (j.sets * 8 < j.splits && 2 * j.sets * (DP / 4) <= kThreads) j.sets *= 2;
    const long long per_block = kThreads / (DP / 4 * j.sets), rows = (long long)j.max_new * j.group;
    k_attend_join<T, DP><<<(unsigned)((rows + per_block - 1) / per_block * j.n_seq * j.heads), kThreads, 0, st>>>(j);
    return hipGetLastError();
}
template <typename T, int DP>
hipError_t launch(const AttendJob& j, hipStream_t st) {
    const unsigned blocks = (unsigned)((long long)j.splits * j.tiles * j.n_seq * j.heads);
    if (sizeof(T) == 4 || j.tiles == 1) k_attend_rows<T, DP, true><<<blocks, kThreads, 0, st>>>(j);
    else k_attend_rows<T, DP, sizeof(T) == 4><<<blocks, kThreads, 0, st>>>(j);
    return hipGetLastError();
}
struct Rows16 {
    template <typename T, int DP>
    static hipError_t go(const AttendJob& j, hipStream_t st) { return launch<T, DP>(j, st); }
};
struct Join {
    template <typename T, int DP>
    static hipError_t go(const AttendJob& j, hipStream_t st) { return launch_join<T, DP>(j, st); }
};

}  // namespace

hipError_t launch_attend_rows(const AttendJob& j, int dtype, hipStream_t st) { return for_type_and_pitch<Rows16>(j, dtype, st); }
hipError_t launch_attend_join(const AttendJob& j, int dtype, hipStream_t st) { return for_type_and_pitch<Join>(j, dtype, st); }

}  // namespace mdcnn
