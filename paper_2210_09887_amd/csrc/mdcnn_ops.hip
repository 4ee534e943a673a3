// Host side of the operators behind the feature maps: argument checks, launch shapes.  Allocates nothing and never waits.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
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
    // Held in registers: slices of 64 bytes of channels (a memory segment) at least, threads so that the LDS takes 32 KiB.
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
    // In chunks: up to 128 vectors beside one another, so that few of 256 threads are left over; 16 vectors to a thread, fewer
    // (down to 4) where that leaves less than four blocks to a compute unit.
    j.slice = std::min(j.C, unit * std::max(1, 128 * vec / unit));
    j.slices = (j.C + j.slice - 1) / j.slice;
    j.lanes = std::min(j.slice / vec, kNormThreads);
    j.row_lanes = kNormThreads / j.lanes;
    const long long per_row = (long long)images * j.slices;
    long long deep = 16;
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

}  // extern "C"
