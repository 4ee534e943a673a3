// Host side of the operators behind the feature maps: argument checks, launch shapes.  Allocates nothing and never waits.
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <cmath>
#include <numeric>

#include "ops_internal.h"

using namespace mdcnn;

namespace {

mdcnn_status fail(mdcnn_status st, const char* fmt, ...) {
    char text[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof(text), fmt, ap);
    va_end(ap);
    return fail_with(st, text);
}

bool known_dtype(int dtype) { return dtype == MDCNN_F32 || dtype == MDCNN_F16 || dtype == MDCNN_BF16; }
bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
mdcnn_status launched(hipError_t err, const char* what) {
    return err == hipSuccess ? MDCNN_OK : fail(MDCNN_ERR_HIP, "%s launch: %s", what, hipGetErrorString(err));
}

// ---- group norm ---------------------------------------------------------------------------------------------------------
constexpr int kNormThreads = 256;              // of the chunked launches (kernels_norm.hip)

mdcnn_status check_strides(const mdcnn_group_norm_desc& d, const mdcnn_strides& s, const char* what, bool written) {
    const long long top = 1ll << 46;
    if (s.n < 0 || s.y < 0 || s.x < 0 || s.n > top || s.y > top || s.x > top) return fail(MDCNN_ERR_SHAPE, "group_norm: strides of %s out of range", what);
    if (written) {
        const long long row = (d.W > 1 ? (d.W - 1) * s.x : 0) + d.C, map = (d.H > 1 ? (d.H - 1) * s.y : 0) + row;
        if ((d.W > 1 && s.x < d.C) || (d.H > 1 && s.y < row) || (d.N > 1 && s.n < map))
            return fail(MDCNN_ERR_SHAPE, "group_norm: pixels of %s overlap", what);
    }
    return MDCNN_OK;
}

mdcnn_status check_norm(const mdcnn_group_norm_desc* d, bool backward) {
    if (!d) return fail(MDCNN_ERR_NULL, "group_norm: descriptor is NULL");
    if (!known_dtype(d->dtype)) return fail(MDCNN_ERR_DTYPE, "group_norm: unknown dtype %d", d->dtype);
    if (d->N < 0 || d->H < 1 || d->W < 1 || d->C < 1 || d->groups < 1) return fail(MDCNN_ERR_SHAPE, "group_norm: sizes must be positive");
    if (d->C > 4096 || (long long)d->H * d->W > (1 << 24) || d->N > (1 << 24)) return fail(MDCNN_ERR_SIZE, "group_norm: C <= 4096, H W <= 2^24, N <= 2^24");
    if (d->C % d->groups) return fail(MDCNN_ERR_SHAPE, "group_norm: %d channels in %d groups", d->C, d->groups);
    if (d->act < MDCNN_ACT_NONE || d->act > MDCNN_ACT_SILU) return fail(MDCNN_ERR_SHAPE, "group_norm: unknown activation %d", d->act);
    if (!(d->eps >= 0.f) || d->eps > 1e30f) return fail(MDCNN_ERR_SHAPE, "group_norm: eps out of range");
    if (!aligned(d->gamma_dev, 4) || !aligned(d->beta_dev, 4)) return fail(MDCNN_ERR_ALIGN, "group_norm: misaligned gamma or beta");
    mdcnn_status st = check_strides(*d, d->xs, "x", false);
    if (!st) st = check_strides(*d, d->ys, backward ? "dx" : "y", true);
    if (!st && backward) st = check_strides(*d, d->ds, "dy", false);
    return st;
}

// Whether every pixel of a map begins on a vector of vec channels.
bool vectors_fit(const mdcnn_group_norm_desc& d, const mdcnn_strides& s, int vec) {
    return (d.N == 1 || s.n % vec == 0) && (d.H == 1 || s.y % vec == 0) && (d.W == 1 || s.x % vec == 0);
}

// Launch shape with vectors of vec channels; returns the vectors held per thread, 0: in chunks.
int plan_norm(const mdcnn_group_norm_desc& d, bool backward, int vec, NormJob& j) {
    j.N = d.N; j.C = d.C; j.groups = d.groups; j.cpg = d.C / d.groups; j.W = d.W; j.P = d.H * d.W;
    j.act = d.act; j.eps = d.eps; j.inv_count = 1.f / ((float)j.P * (float)j.cpg);
    j.gamma = d.gamma_dev; j.beta = d.beta_dev;
    const int unit = std::lcm(j.cpg, vec);         // a slice holds whole groups and whole vectors
    const int esize = (int)storage_bytes(d.dtype), images = std::max(d.N, 1);
    // Held in registers: slices of 64 bytes of channels (a memory segment) at least, threads so that the LDS takes 32 KiB.  Held / in chunks, forward and
    // backward: 12 x 9 x 256 16 / 28 us, 24 x 18 x 128 19 / 30, 16 maps of 16 x 16 x 512 25 / 33, of 32 x 32 x 256 (forward only) 14 / 18.
    {
        const int most = std::min(1024, 4096 / vec), deep = backward ? 4 : 8;
        int slice = unit * std::max(1, (64 / esize + unit - 1) / unit);
        slice = std::min(slice, j.C);
        const int lanes = slice / vec;
        if (lanes <= most) {
            const int row_lanes = std::min(j.P, most / lanes), held = (j.P + row_lanes - 1) / row_lanes;
            if (held <= deep) {
                j.slice = slice; j.slices = (j.C + slice - 1) / slice;
                j.lanes = lanes; j.row_lanes = row_lanes;
                j.rows = j.P; j.chunks = 1;
                return held <= 1 ? 1 : held <= 2 ? 2 : held <= 4 ? 4 : 8;
            }
        }
    }
    // In chunks: up to 128 vectors beside one another, so that few of 256 threads are left over; 32 vectors to a thread, fewer
    // (down to 4) where that leaves less than four blocks to a compute unit.  (Forward and backward of 16 bf16 maps of 128 x 128 x 256: 16 vectors 234 us,
    // 32 223, 64 238.)
    j.slice = std::min(j.C, unit * std::max(1, 128 * vec / unit));
    j.slices = (j.C + j.slice - 1) / j.slice;
    j.lanes = std::min(j.slice / vec, kNormThreads);
    j.row_lanes = kNormThreads / j.lanes;
    const long long per_row = (long long)images * j.slices;
    long long deep = 32;
    while (deep > 4 && per_row * ((j.P + deep * j.row_lanes - 1) / (deep * j.row_lanes)) < 1024) deep /= 2;
    j.rows = (int)std::min<long long>(j.P, deep * j.row_lanes);
    j.chunks = (j.P + j.rows - 1) / j.rows;
    return 0;
}

struct NormWork { size_t part, joined, cpart, total; };
NormWork norm_work(const NormJob& j, bool backward, int held) {
    NormWork w{};
    const size_t blocks = (size_t)j.N * j.chunks;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t o = at; at += up256(n); return o; };
    w.part = take(held ? 0 : blocks * j.groups * 8);
    w.joined = take(backward && !held ? (size_t)j.N * j.groups * 8 : 0);
    w.cpart = take(backward && !(held && j.N == 1) ? blocks * j.C * 8 : 0);
    w.total = at;
    return w;
}

size_t norm_bytes(const mdcnn_group_norm_desc& d, bool backward) {
    size_t most = 0;
    for (int vec : {1, (int)(16 / storage_bytes(d.dtype))}) {              // (what the pointers allow is not known yet)
        if (d.C % vec) continue;
        NormJob j{};
        const int held = plan_norm(d, backward, vec, j);
        most = std::max(most, norm_work(j, backward, held).total);
    }
    return most;
}

mdcnn_status run_norm(const mdcnn_group_norm_desc& d, bool backward, const void* x, const void* dy, void* y, float* mean, float* rstd, float* dgamma, float* dbeta,
                      void* work, size_t work_bytes, void* stream) {
    const size_t e = storage_bytes(d.dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(dy, e) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4) || !aligned(work, 16))
        return fail(MDCNN_ERR_ALIGN, "group_norm: misaligned pointer");
    int vec = (int)(16 / e);
    if (d.C % vec || !aligned(x, 16) || !aligned(y, 16) || !aligned(dy, 16) || !vectors_fit(d, d.xs, vec) || !vectors_fit(d, d.ys, vec) ||
        (backward && !vectors_fit(d, d.ds, vec)))
        vec = 1;
    NormJob j{};
    const int held = plan_norm(d, backward, vec, j);
    const NormWork w = norm_work(j, backward, held);
    const size_t need = norm_bytes(d, backward);
    if (work_bytes < need) return fail(MDCNN_ERR_SIZE, "group_norm: workspace of %zu bytes, %zu needed", work_bytes, need);
    if (need && !work) return fail(MDCNN_ERR_NULL, "group_norm: workspace is NULL");
    if ((long long)j.N * j.chunks * j.slices > 0x7fff0000ll) return fail(MDCNN_ERR_SIZE, "group_norm: too large");
    j.x = x; j.dy = dy; j.y = y; j.mean = mean; j.rstd = rstd; j.dgamma = dgamma; j.dbeta = dbeta;
    j.part = (float*)((char*)work + w.part); j.joined = (float*)((char*)work + w.joined); j.cpart = (float*)((char*)work + w.cpart);
    j.xs = d.xs; j.ys = d.ys; j.ds = d.ds;
    j.flat = 1;
    for (mdcnn_strides* s : {&j.xs, &j.ys, &j.ds}) {
        if (d.W == 1) s->x = s->y;                                         // one column: pixels are rows
        else if (d.H > 1 && s->y != d.W * s->x && (backward || s != &j.ds)) j.flat = 0;
    }
    if (backward) return launched(launch_norm_grad(j, d.dtype, vec, held, (hipStream_t)stream), "group_norm_backward");
    if (!j.N) return MDCNN_OK;
    return launched(launch_norm(j, d.dtype, vec, held, (hipStream_t)stream), "group_norm");
}

// ---- rotary positions -----------------------------------------------------------------------------------------------------
mdcnn_status check_heads(const mdcnn_heads& m, const char* call, const char* what, int dim, long long tokens, size_t e, bool reads, bool writes) {
    const long long top = 1ll << 46;
    if (m.heads < 1 || m.heads > 65535) return fail(MDCNN_ERR_SHAPE, "%s: heads of %s out of range", call, what);
    if ((reads && !m.x_dev) || (writes && !m.y_dev)) return fail(MDCNN_ERR_NULL, "%s: %s is NULL", call, what);
    if ((reads && !aligned(m.x_dev, e)) || (writes && !aligned(m.y_dev, e))) return fail(MDCNN_ERR_ALIGN, "%s: %s is misaligned", call, what);
    if (reads && (m.x_token < 0 || m.x_head < 0 || m.x_token > top || m.x_head > top)) return fail(MDCNN_ERR_SHAPE, "%s: strides of %s out of range", call, what);
    if (writes) {
        // heads within tokens or tokens within heads: either way none may reach into the next; where there is one of them its stride counts for nothing
        const bool several = m.heads > 1, more = tokens > 1;
        if (m.y_token > top || m.y_head > top) return fail(MDCNN_ERR_SHAPE, "%s: strides of %s out of range", call, what);
        if ((more && m.y_token < dim) || (several && m.y_head < dim)) return fail(MDCNN_ERR_SHAPE, "%s: heads of %s overlap", call, what);
        if (several && more && m.y_token >= m.y_head && m.y_token < (m.heads - 1) * m.y_head + dim) return fail(MDCNN_ERR_SHAPE, "%s: tokens of %s overlap", call, what);
        if (several && more && m.y_token < m.y_head && m.y_head < (tokens - 1) * m.y_token + dim) return fail(MDCNN_ERR_SHAPE, "%s: heads of %s overlap", call, what);
    }
    return MDCNN_OK;
}

// ---- the cache ------------------------------------------------------------------------------------------------------------
mdcnn_status check_cache(const mdcnn_cache_desc* c, const char* call) {
    if (!c) return fail(MDCNN_ERR_NULL, "%s: cache is NULL", call);
    if (!mdcnn_cache_pitch(c->dim)) return fail(MDCNN_ERR_SHAPE, "%s: %d channels to a head (8 to 256, a multiple of 8)", call, c->dim);
    if (c->heads < 1 || c->heads > 32767) return fail(MDCNN_ERR_SHAPE, "%s: %d heads", call, c->heads);
    if (c->pages < 0 || c->n_seq < 0 || c->max_pages < 0 || c->max_pages > (1 << 24)) return fail(MDCNN_ERR_SIZE, "%s: pages, sequences or table out of range", call);
    // (an empty tensor has no memory: a table without entries, a pool without pages)
    const bool table = c->n_seq && c->max_pages, pool = table && c->pages;
    if ((table && !c->table_dev) || (pool && (!c->k_dev || !c->v_dev || !c->k_scale_dev || !c->v_scale_dev))) return fail(MDCNN_ERR_NULL, "%s: NULL pointer in the cache", call);
    if (!aligned(c->k_dev, 16) || !aligned(c->v_dev, 16) || !aligned(c->k_scale_dev, 4) || !aligned(c->v_scale_dev, 4) || !aligned(c->table_dev, 4))
        return fail(MDCNN_ERR_ALIGN, "%s: misaligned pointer in the cache", call);
    return MDCNN_OK;
}

mdcnn_status run_cache(const mdcnn_cache_desc* c, const mdcnn_heads* k, const mdcnn_heads* v, int tokens, const int* starts, const int* first, int max_new, int dtype, bool store, void* stream) {
    const char* call = store ? "cache_store" : "cache_read";
    mdcnn_status st = check_cache(c, call);
    if (st) return st;
    if (!known_dtype(dtype)) return fail(MDCNN_ERR_DTYPE, "%s: unknown dtype %d", call, dtype);
    if (!k || !v) return fail(MDCNN_ERR_NULL, "%s: NULL map", call);
    if (max_new < 0 || tokens < 0) return fail(MDCNN_ERR_SHAPE, "%s: max_new %d, %d tokens", call, max_new, tokens);
    max_new = std::min(max_new, tokens);
    if (!c->n_seq || !max_new) return MDCNN_OK;
    if (!starts || !first) return fail(MDCNN_ERR_NULL, "%s: starts or positions are NULL", call);
    if (!aligned(starts, 4) || !aligned(first, 4)) return fail(MDCNN_ERR_ALIGN, "%s: starts or positions are misaligned", call);
    const size_t e = storage_bytes(dtype);
    CacheJob j{};
    int vec = (int)(16 / e);
    for (const mdcnn_heads* m : {k, v}) {
        const char* what = m == k ? "the keys" : "the values";
        if (m->heads != c->heads) return fail(MDCNN_ERR_SHAPE, "%s: %d heads in %s, %d in the cache", call, m->heads, what, c->heads);
        st = check_heads(*m, call, what, c->dim, tokens, e, store, !store);
        if (st) return st;
        const void* at = store ? m->x_dev : m->y_dev;
        const long long token = store ? m->x_token : m->y_token, head = store ? m->x_head : m->y_head;
        if (!aligned(at, 16) || (tokens > 1 && token % vec) || (m->heads > 1 && head % vec)) vec = 1;
        (m == k ? j.k : j.v) = CacheMap{m->x_dev, m->y_dev, m->x_token, m->x_head, m->y_token, m->y_head};
    }
    j.k_codes = c->k_dev; j.v_codes = c->v_dev; j.k_scale = c->k_scale_dev; j.v_scale = c->v_scale_dev;
    j.table = c->table_dev; j.starts = starts; j.first = first;
    j.pages = c->pages; j.heads = c->heads; j.dim = c->dim; j.pitch = mdcnn_cache_pitch(c->dim);
    j.n_seq = c->n_seq; j.max_pages = c->max_pages; j.max_new = max_new; j.tokens = tokens;
    j.slots = (int)(((long long)max_new + MDCNN_PAGE_TOKENS - 2) / MDCNN_PAGE_TOKENS) + 1;      // the first page may be begun
    if ((long long)j.n_seq * j.slots > 0x7fffffffll) return fail(MDCNN_ERR_SIZE, "%s: %d sequences of up to %d tokens", call, j.n_seq, max_new);
    return launched(launch_cache(j, dtype, vec, store, (hipStream_t)stream), call);
}

// ---- attention ------------------------------------------------------------------------------------------------------------
mdcnn_status check_attend(const mdcnn_cache_desc* c, const mdcnn_attend_desc* a, int q_heads) {
    const mdcnn_status st = check_cache(c, "cache_attend");
    if (st) return st;
    if (!a) return fail(MDCNN_ERR_NULL, "cache_attend: description is NULL");
    if (q_heads < 1 || q_heads % c->heads || q_heads > 65535) return fail(MDCNN_ERR_SHAPE, "cache_attend: %d query heads over %d", q_heads, c->heads);
    if (a->tokens < 0 || a->max_new < 0 || a->max_len < 0) return fail(MDCNN_ERR_SHAPE, "cache_attend: negative sizes");
    if ((a->causal & ~1) || a->window < 0 || (a->window && !a->causal)) return fail(MDCNN_ERR_SHAPE, "cache_attend: causal is 0 or 1, a window needs it");
    if (!std::isfinite(a->scale)) return fail(MDCNN_ERR_SHAPE, "cache_attend: scale is not finite");
    if (c->n_seq && (!a->starts_dev || !a->lengths_dev)) return fail(MDCNN_ERR_NULL, "cache_attend: starts or lengths are NULL");
    if (!aligned(a->starts_dev, 4) || !aligned(a->lengths_dev, 4)) return fail(MDCNN_ERR_ALIGN, "cache_attend: starts or lengths are misaligned");
    if (a->mask_dev && a->mask_row < a->max_len) return fail(MDCNN_ERR_SIZE, "cache_attend: mask rows of %lld bytes, %d tokens", a->mask_row, a->max_len);
    return MDCNN_OK;
}

// Rows to a block and pages to a split.  Up to 16 rows go by sixteen, whose blocks read the cache's bytes and little else, more than 64 by 128, whose codes are read once and made halves
// once; 17 to 64 by sixteen - two to four blocks that each read and decode - but for heads of 64 to 128 channels of 16 bits as soon as those are more than the 1024 blocks that
// fill the GPU twice (of 32 channels a tile's own work is the longer, of 192 and more or of fp32 there is one tile to a compute unit).  By sixteen / by 128, us, 8 bf16 heads:
//   128 channels: 16 x 8192 tokens, 16 rows 50 / 72, 48 rows 102 / 85, 64 rows 118 / 87, 128 rows 225 / 114; 64 x 8192, 32 rows 383 / 224, 64 rows 830 / 284; 2 x 30000, 48 rows 50 / 52;
//   1 x 2000, 48 rows 18 / 26.  64 channels: 16 x 8192, 32 rows 37 / 42, 64 rows 60 / 54; 64 x 1024, 64 rows 43 / 35.  32 channels: 64 x 8192, 48 rows 123 / 160.
//   256 channels: 16 x 8192, 48 rows 246 / 331.  fp32, 128 channels: 16 x 8192, 64 rows 140 / 181.
// Runs of 12 to 32 pages by sixteen rows: shorter ones are mostly what a block does once (its queries, its sums: two sequences of 150001 tokens, 2 heads,
// 63 us with 4 pages, 46 with 8, 36 with 24), longer ones leave the last blocks of ragged sequences alone on the GPU; in between just under the 512 blocks that
// the GPU holds.  By 128 rows as many runs as the GPU holds blocks, but none shorter than 8 pages: a run leaves its sums in 32 bits, and one that begins when others
// end leaves the GPU half empty (against about 2048 blocks: prompt of 2000 tokens, 32 heads of 128 channels over 8, 81 and 134 us; 1000 rows over 8192 tokens, 8
// heads of 128 channels, 76 and 100).
mdcnn_status plan_attend(const mdcnn_cache_desc& c, const mdcnn_attend_desc& a, int q_heads, int dtype, AttendJob& j, size_t* bytes) {
    j.pages = c.pages; j.heads = c.heads; j.group = q_heads / c.heads; j.dim = c.dim; j.pitch = mdcnn_cache_pitch(c.dim);
    j.n_seq = c.n_seq; j.max_pages = c.pages ? c.max_pages : 0;
    j.tokens = a.tokens; j.max_new = std::min(a.max_new, a.tokens); j.max_len = a.max_len;
    j.causal = a.causal; j.window = a.window; j.scale = a.scale;
    const long long rows = (long long)j.max_new * j.group;
    if (rows > 0x7fffff00ll || rows * c.n_seq * c.heads > 0x7fffffffll) return fail(MDCNN_ERR_SIZE, "cache_attend: too many rows");
    long long most = std::min<long long>((a.max_len + (long long)MDCNN_PAGE_TOKENS - 1) / MDCNN_PAGE_TOKENS, c.max_pages);
    if (a.window) most = std::min<long long>(most, (a.window + (long long)j.max_new + 2 * MDCNN_PAGE_TOKENS - 2) / MDCNN_PAGE_TOKENS);
    most = std::max(most, 1ll);
    long long columns, live;
    auto cut = [&](int tile_rows) {
        j.tile_rows = tile_rows;
        j.tiles = (int)((rows + tile_rows - 1) / tile_rows);
        columns = (long long)j.tiles * c.n_seq * c.heads;
        live = std::min(columns, ((long long)j.tokens * j.group / tile_rows + c.n_seq) * c.heads);        // (no more of them have rows)
        if (tile_rows == kAttendRows) {
            const long long run = std::min(32ll, std::max(12ll, (most * live + 479) / 480));
            j.splits = live >= 2048 ? 1 : (int)((most + run - 1) / run);
        } else {
            j.splits = (int)std::max(1ll, std::min((most + 7) / 8, 256ll * attend_tile_blocks((int)storage_bytes(dtype), j.pitch) / std::max(1ll, live)));
        }
    };
    cut(kAttendRows);
    const bool lean = storage_bytes(dtype) == 2 && j.pitch >= 64 && j.pitch <= 128;
    if (attend_tiles_fit(dtype, j.pitch) && (rows > 64 || (rows > 16 && lean && live * j.splits > 1024))) cut(kAttendTile);
    j.run = j.splits == 1 ? 1 << 30 : (int)((most + j.splits - 1) / j.splits);          // all alike
    if (columns * j.splits > 0x7fffffffll) return fail(MDCNN_ERR_SIZE, "cache_attend: too large");
    *bytes = j.splits > 1 ? (size_t)columns * j.splits * j.tile_rows * (8 + 4 * (size_t)j.pitch) + 256 : 0;
    return MDCNN_OK;
}

}  // namespace

extern "C" {

mdcnn_status mdcnn_group_norm_bytes(const mdcnn_group_norm_desc* d, int backward, size_t* bytes) {
    const mdcnn_status st = check_norm(d, backward != 0);
    if (st) return st;
    if (!bytes) return fail(MDCNN_ERR_NULL, "group_norm_bytes: bytes is NULL");
    *bytes = norm_bytes(*d, backward != 0);
    return MDCNN_OK;
}

mdcnn_status mdcnn_group_norm(const mdcnn_group_norm_desc* d, const void* x_dev, void* y_dev, float* mean_dev, float* rstd_dev, void* work_dev, size_t work_bytes,
                              void* stream) {
    const mdcnn_status st = check_norm(d, false);
    if (st) return st;
    if (d->N && (!x_dev || !y_dev || !mean_dev || !rstd_dev)) return fail(MDCNN_ERR_NULL, "group_norm: NULL argument");
    return run_norm(*d, false, x_dev, nullptr, y_dev, mean_dev, rstd_dev, nullptr, nullptr, work_dev, work_bytes, stream);
}

mdcnn_status mdcnn_group_norm_backward(const mdcnn_group_norm_desc* d, const void* x_dev, const void* dy_dev, const float* mean_dev, const float* rstd_dev, void* dx_dev,
                                       float* dgamma_dev, float* dbeta_dev, void* work_dev, size_t work_bytes, void* stream) {
    const mdcnn_status st = check_norm(d, true);
    if (st) return st;
    if (!dgamma_dev || !dbeta_dev || (d->N && (!x_dev || !dy_dev || !mean_dev || !rstd_dev || !dx_dev))) return fail(MDCNN_ERR_NULL, "group_norm_backward: NULL argument");
    return run_norm(*d, true, x_dev, dy_dev, dx_dev, const_cast<float*>(mean_dev), const_cast<float*>(rstd_dev), dgamma_dev, dbeta_dev, work_dev, work_bytes, stream);
}

mdcnn_status mdcnn_rotary_table(const mdcnn_rotary_desc* d, uint64_t* steps) {
    if (!d || !steps) return fail(MDCNN_ERR_NULL, "rotary_table: NULL argument");
    if (d->axes < 1 || d->axes > 4 || d->turned < 2 || d->turned > 4096 || d->turned % (2 * d->axes)) return fail(MDCNN_ERR_SHAPE, "rotary_table: %d channels on %d axes", d->turned, d->axes);
    if (!(d->base > 1.0) || !std::isfinite(d->base)) return fail(MDCNN_ERR_SHAPE, "rotary_table: base must be above 1");
    if (d->scaling < MDCNN_ROTARY_PLAIN || d->scaling > MDCNN_ROTARY_PARTS) return fail(MDCNN_ERR_SHAPE, "rotary_table: unknown scaling %d", d->scaling);
    if (d->scaling != MDCNN_ROTARY_PLAIN && (!(d->factor >= 1.0) || !std::isfinite(d->factor))) return fail(MDCNN_ERR_SHAPE, "rotary_table: factor must be 1 or more");
    if (d->scaling == MDCNN_ROTARY_PARTS && (!(d->original > 0.0) || !(d->slow >= 0.0) || !(d->fast > d->slow) || !std::isfinite(d->original) || !std::isfinite(d->fast)))
        return fail(MDCNN_ERR_SHAPE, "rotary_table: original > 0 and 0 <= slow < fast are needed");
    const int n = d->turned / 2 / d->axes;
    const double two_pi = 6.283185307179586476925;
    double base = d->base;
    if (d->scaling == MDCNN_ROTARY_BASE && n > 1) base *= std::pow(d->factor, (double)n / (n - 1));
    for (int i = 0; i < d->turned / 2; ++i) {
        double f = std::pow(base, -(double)(i % n) / n);
        if (d->scaling == MDCNN_ROTARY_LINEAR) f /= d->factor;
        if (d->scaling == MDCNN_ROTARY_PARTS) {
            const double keep = std::min(1.0, std::max(0.0, (d->original * f / two_pi - d->slow) / (d->fast - d->slow)));
            f = f * keep + f / d->factor * (1.0 - keep);
        }
        steps[i] = (uint64_t)std::rint(std::ldexp(f / two_pi, 64));
    }
    return MDCNN_OK;
}

mdcnn_status mdcnn_rotary(const mdcnn_heads* maps, int n_maps, int tokens, int dim, int dtype, const int* pos_dev, int axes, const uint64_t* steps_dev, int turned, int interleaved,
                          int inverse, float magnitude, void* stream) {
    if (!maps) return fail(MDCNN_ERR_NULL, "rotary: maps is NULL");
    if (!known_dtype(dtype)) return fail(MDCNN_ERR_DTYPE, "rotary: unknown dtype %d", dtype);
    if (n_maps < 1 || n_maps > 2) return fail(MDCNN_ERR_SHAPE, "rotary: one or two maps");
    if (tokens < 0) return fail(MDCNN_ERR_SHAPE, "rotary: %d tokens", tokens);
    if (dim < 2 || dim > 256) return fail(MDCNN_ERR_SIZE, "rotary: 2 to 256 channels to a head");
    if (axes < 1 || axes > 4 || turned < 2 || turned > dim || turned % (2 * axes)) return fail(MDCNN_ERR_SHAPE, "rotary: %d of %d channels on %d axes", turned, dim, axes);
    if ((interleaved | inverse) & ~1) return fail(MDCNN_ERR_SHAPE, "rotary: interleaved and inverse are 0 or 1");
    if (!std::isfinite(magnitude)) return fail(MDCNN_ERR_SHAPE, "rotary: magnitude is not finite");
    const size_t e = storage_bytes(dtype);
    RotaryJob j{};
    for (int i = 0; i < n_maps; ++i) {
        mdcnn_status st = tokens ? check_heads(maps[i], "rotary", i ? "the second map" : "the first map", dim, tokens, e, true, true) : MDCNN_OK;
        if (st) return st;
        j.maps[i] = RotaryMap{maps[i].x_dev, maps[i].y_dev, maps[i].heads, maps[i].x_token, maps[i].x_head, maps[i].y_token, maps[i].y_head};
    }
    if (!tokens) return MDCNN_OK;
    if (!pos_dev || !steps_dev) return fail(MDCNN_ERR_NULL, "rotary: positions or steps are NULL");
    if (!aligned(pos_dev, 4) || !aligned(steps_dev, 8)) return fail(MDCNN_ERR_ALIGN, "rotary: positions or steps are misaligned");
    // The widest vectors that the turned and the copied channels consist of and every head begins on.
    int vec = 1;
    for (int v : {(int)(16 / e), 4}) {
        const size_t bytes = v * e;
        bool ok = (interleaved ? turned : turned / 2) % v == 0 && (dim - turned) % v == 0;
        for (int i = 0; i < n_maps; ++i) {
            const RotaryMap& m = j.maps[i];
            ok = ok && aligned(m.x, bytes) && aligned(m.y, bytes) && (tokens == 1 || (m.x_token % v == 0 && m.y_token % v == 0)) && (m.heads == 1 || (m.x_head % v == 0 && m.y_head % v == 0));
        }
        if (ok) { vec = v; break; }
    }
    bool in_place = true;
    for (int i = 0; i < n_maps; ++i) in_place = in_place && j.maps[i].x == j.maps[i].y && j.maps[i].x_token == j.maps[i].y_token && j.maps[i].x_head == j.maps[i].y_head;
    j.pos = pos_dev; j.steps = (const unsigned long long*)steps_dev;
    j.tokens = tokens; j.axes = axes; j.per = turned / 2 / axes; j.turned = turned;
    j.turned_units = interleaved ? (vec > 1 ? turned / vec : turned / 2) : turned / 2 / vec;
    j.units = j.turned_units + (in_place ? 0 : (dim - turned) / vec);
    j.tokens_per_block = 256 / j.units;
    j.inverse = inverse; j.magnitude = magnitude;
    // A thread goes through up to 16 heads with the same sines; fewer where that leaves less than eight blocks to a compute unit.  (40 bf16 heads of 128
    // channels: 32768 tokens 130 us, one head to a thread 147; 48 tokens 3.6 us, 16 heads to a thread 9.1.)
    const int heads = j.maps[0].heads + j.maps[1].heads;
    const long long blocks = ((long long)tokens + j.tokens_per_block - 1) / j.tokens_per_block;
    j.group = std::min(heads, 16);
    while (j.group > 1 && blocks * ((heads + j.group - 1) / j.group) < 2048) j.group = (j.group + 1) / 2;      // (the second extent of the grid is 8192 at most)
    return launched(launch_rotary(j, dtype, vec, interleaved != 0, (hipStream_t)stream), "rotary");
}

int mdcnn_cache_pitch(int dim) {
    if (dim < 8 || dim > 256 || dim % 8) return 0;
    for (int p : {32, 64, 96, 128, 192})
        if (p >= dim) return p;
    return 256;
}

mdcnn_status mdcnn_cache_store(const mdcnn_cache_desc* c, const mdcnn_heads* k, const mdcnn_heads* v, int tokens, const int* starts_dev, const int* held_dev, int max_new, int dtype, void* stream) {
    return run_cache(c, k, v, tokens, starts_dev, held_dev, max_new, dtype, true, stream);
}

mdcnn_status mdcnn_cache_read(const mdcnn_cache_desc* c, const mdcnn_heads* k, const mdcnn_heads* v, int tokens, const int* starts_dev, const int* first_dev, int max_new, int dtype, void* stream) {
    return run_cache(c, k, v, tokens, starts_dev, first_dev, max_new, dtype, false, stream);
}

mdcnn_status mdcnn_cache_attend_bytes(const mdcnn_cache_desc* c, const mdcnn_attend_desc* a, int q_heads, int dtype, size_t* bytes) {
    mdcnn_status st = check_attend(c, a, q_heads);
    if (st) return st;
    if (!known_dtype(dtype)) return fail(MDCNN_ERR_DTYPE, "cache_attend_bytes: unknown dtype %d", dtype);
    if (!bytes) return fail(MDCNN_ERR_NULL, "cache_attend_bytes: bytes is NULL");
    AttendJob j{};
    return plan_attend(*c, *a, q_heads, dtype, j, bytes);
}

mdcnn_status mdcnn_cache_attend(const mdcnn_cache_desc* c, const mdcnn_attend_desc* a, const mdcnn_heads* q, int dtype, float* lse_dev, void* work_dev, size_t work_bytes, void* stream) {
    if (!q) return fail(MDCNN_ERR_NULL, "cache_attend: queries are NULL");
    mdcnn_status st = check_attend(c, a, q->heads);
    if (st) return st;
    if (!known_dtype(dtype)) return fail(MDCNN_ERR_DTYPE, "cache_attend: unknown dtype %d", dtype);
    AttendJob j{};
    size_t need = 0;
    st = plan_attend(*c, *a, q->heads, dtype, j, &need);
    if (st) return st;
    if (!c->n_seq || !a->tokens || !a->max_new) return MDCNN_OK;
    st = check_heads(*q, "cache_attend", "the queries", c->dim, a->tokens, storage_bytes(dtype), true, true);
    if (st) return st;
    if (!aligned(lse_dev, 4) || !aligned(work_dev, 16)) return fail(MDCNN_ERR_ALIGN, "cache_attend: misaligned pointer");
    if (work_bytes < need) return fail(MDCNN_ERR_SIZE, "cache_attend: workspace of %zu bytes, %zu needed", work_bytes, need);
    if (need && !work_dev) return fail(MDCNN_ERR_NULL, "cache_attend: workspace is NULL");
    j.q = q->x_dev; j.y = q->y_dev; j.lse = lse_dev;
    j.q_token = q->x_token; j.q_head = q->x_head; j.y_token = q->y_token; j.y_head = q->y_head;
    j.k_codes = c->k_dev; j.v_codes = c->v_dev; j.k_scale = c->k_scale_dev; j.v_scale = c->v_scale_dev; j.table = c->table_dev;
    j.starts = a->starts_dev; j.lengths = a->lengths_dev; j.mask = a->mask_dev; j.mask_row = a->mask_row;
    j.mask_whole = aligned(a->mask_dev, 16) && (c->n_seq == 1 || a->mask_row % 16 == 0);
    const long long per = 16 / (long long)storage_bytes(dtype);
    j.q_whole = aligned(q->x_dev, 16) && (a->tokens == 1 || q->x_token % per == 0) && (q->heads == 1 || q->x_head % per == 0);
    j.part_out = (float*)work_dev;
    j.part_top = (float2*)((char*)work_dev + (size_t)j.n_seq * j.heads * j.tiles * j.splits * j.tile_rows * j.pitch * 4);
    const auto first = j.tile_rows == kAttendRows ? launch_attend_rows : launch_attend_tiles;
    hipError_t err = first(j, dtype, (hipStream_t)stream);
    if (err == hipSuccess) err = launch_attend_join(j, dtype, (hipStream_t)stream);
    return launched(err, "cache_attend");
}

}  // extern "C"
