// Jobs of the operators behind the feature maps, as the host fills them in and the kernels read them.
#pragma once

#include "mdcnn_internal.h"

namespace mdcnn {

// Sets the text of mdcnn_last_error (mdcnn_api.hip).
mdcnn_status fail_with(mdcnn_status st, const char* text);

inline size_t storage_bytes(int dtype) { return dtype == MDCNN_F32 ? 4 : 2; }

// Group norm -----------------------------------------------------------------------------------------------------------
struct NormJob {
    const void* x;
    const void* dy;              // gradients only
    void* y;                     // forward: the output; gradients: dx
    const float* gamma;          // nullptr: ones
    const float* beta;           // nullptr: zeros
    float* mean;                 // [N][groups], written forward, read for gradients
    float* rstd;
    float* dgamma;               // gradients only
    float* dbeta;
    float* part;                 // [N][chunks][groups][2]: mean and sum of squares about it; gradients: the two sums
    float* joined;               // [N][groups][2] gradients, where the chunks are joined by a launch of their own
    float* cpart;                // [N * chunks][C][2] gradients: sums of every channel
    mdcnn_strides xs, ys, ds;    // of x; of y (or dx); of dy
    int N, W, P, C, groups, cpg; // P = H * W pixels of an image
    int flat;                    // the rows of all maps follow one another: pixel p lies at p * stride.x
    int slice, slices;           // channels of a block: whole groups
    int lanes, row_lanes;        // threads beside one another over a slice's vectors, rows of threads
    int rows, chunks;            // pixels of a block, blocks of an image
    int act;
    float eps, inv_count;        // 1 / (P * cpg)
};
// vec: channels to a vector (1, or 16 bytes of them).  held: 16-byte vectors (or single channels) a thread keeps in registers, 0: in chunks.
hipError_t launch_norm(const NormJob& j, int dtype, int vec, int held, hipStream_t st);
hipError_t launch_norm_grad(const NormJob& j, int dtype, int vec, int held, hipStream_t st);

// Rotary positions -------------------------------------------------------------------------------------------------------
struct RotaryMap {
    const void* x;
    void* y;
    int heads;
    long long x_token, x_head, y_token, y_head;
};
struct RotaryJob {
    RotaryMap maps[2];           // of the second, 0 heads if there is none
    const int* pos;              // [tokens][axes]
    const unsigned long long* steps;
    long long tokens;
    int axes, per;               // per: pairs to an axis
    int turned;
    int turned_units, units;     // vectors of a head that a thread each turns; these and those that are copied
    int tokens_per_block, group; // group: heads a thread goes through
    int inverse;
    float magnitude;
};
hipError_t launch_rotary(const RotaryJob& j, int dtype, int vec, bool interleaved, hipStream_t st);

// The cache --------------------------------------------------------------------------------------------------------------
struct CacheMap {
    const void* x;
    void* y;
    long long x_token, x_head, y_token, y_head;
};
struct CacheJob {
    int8_t* k_codes;
    int8_t* v_codes;
    float* k_scale;
    float* v_scale;
    const int* table;
    const int* starts;           // [n_seq + 1]
    const int* first;            // [n_seq] position of a sequence's first token of the call
    CacheMap k, v;
    int pages, heads, dim, pitch, n_seq, max_pages, max_new, tokens;
    int slots;                   // pages that a sequence's tokens may lie in
};
hipError_t launch_cache(const CacheJob& j, int dtype, int vec, bool store, hipStream_t st);

// Attention over the cache -----------------------------------------------------------------------------------------------
struct AttendJob {
    const void* q;
    void* y;
    float* lse;
    const int8_t* k_codes;
    const int8_t* v_codes;
    const float* k_scale;
    const float* v_scale;
    const int* table;
    const int* starts;
    const int* lengths;
    const uint8_t* mask;
    float2* part_top;            // [seq][head][tile][split][tile_rows]: T and sum of a row
    float* part_out;             // [..][16][pitch]
    long long q_token, q_head, y_token, y_head, mask_row;
    int pages, heads, group, dim, pitch, n_seq, max_pages;   // group: query heads to a head of the cache
    int tokens, max_new, max_len, causal, window;
    int mask_whole, q_whole;     // rows of the mask, heads of the queries begin on 16 bytes
    int tile_rows;               // rows of a block
    int tiles, splits, run;      // tiles of rows and splits of a sequence and head (bounds), pages to a split
    int sets;                    // of a row's splits when they are joined
    float scale;
};
hipError_t launch_attend_rows(const AttendJob& j, int dtype, hipStream_t st);
bool attend_tiles_fit(int dtype, int pitch);             // whether launch_attend_tiles takes them
hipError_t launch_attend_tiles(const AttendJob& j, int dtype, hipStream_t st);
hipError_t launch_attend_join(const AttendJob& j, int dtype, hipStream_t st);     // nothing if there is one split
constexpr int kAttendRows = 16, kAttendTile = 128;       // rows of a block of the two
// Blocks of 128 rows on a compute unit (waves on a SIMD), as queries, sums, products and weights leave room for them in the registers.
constexpr int attend_tile_blocks(int value_bytes, int pitch) { return value_bytes == 2 ? (pitch <= 64 ? 3 : pitch <= 128 ? 2 : 1) : pitch == 32 ? 3 : pitch <= 96 ? 2 : 1; }

}  // namespace mdcnn
