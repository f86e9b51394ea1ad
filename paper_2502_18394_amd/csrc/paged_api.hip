// C ABI of the paged attention layers: argument checks and launches.  Every entry point validates on the host, enqueues on the caller's stream and
// returns; nothing is allocated.
#include <climits>
#include <cmath>
#include <cstdint>

#include "internal.h"
#include "norm.h"
#include "paged.h"

namespace spectre {
namespace {

constexpr int kLongest = SPECTRE_KV_MAX_TABLE * 256;   // tokens that a sequence can have

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

int check_dtype(spectre_dtype io, const char *who) {
    return io == SPECTRE_F32 || io == SPECTRE_BF16 ? SPECTRE_OK : fail(SPECTRE_EINVAL, "%s: unknown dtype %d", who, (int)io);
}

int check_sizes(const spectre_kv *kv, const char *who) {
    if (!kv) return fail(SPECTRE_EINVAL, "%s: null pool", who);
    if (kv->layers < 1 || kv->pages < 1 || kv->Hkv < 1 || kv->seqs < 1 || kv->max_pages < 1) return fail(SPECTRE_EINVAL, "%s: a size of the pool is below 1", who);
    if (kv->dtype != SPECTRE_E4M3) {
        const int rc = check_dtype(kv->dtype, who);
        if (rc) return rc;
    }
    if (kv->d != 64 && kv->d != 128) return fail(SPECTRE_EUNSUPPORTED, "%s: d = %d (64 and 128 are supported)", who, kv->d);
    if (kv->page < 16 || kv->page > 256 || (kv->page & (kv->page - 1))) return fail(SPECTRE_EUNSUPPORTED, "%s: %d tokens a page (16, 32, 64, 128, 256 are supported)", who, kv->page);
    if (kv->seqs > SPECTRE_KV_MAX_SEQS || kv->max_pages > SPECTRE_KV_MAX_TABLE || kv->pages > (1 << 28) || kv->Hkv > 4096 || kv->layers > 65536)
        return fail(SPECTRE_EUNSUPPORTED, "%s: pool of %d pages, %d sequences of %d pages, %d heads", who, kv->pages, kv->seqs, kv->max_pages, kv->Hkv);
    return SPECTRE_OK;
}

int check_pool(const spectre_kv *kv, const char *who) {
    const int rc = check_sizes(kv, who);
    if (rc) return rc;
    if (!kv->k || !kv->v || !kv->book) return fail(SPECTRE_EINVAL, "%s: null array in the pool", who);
    if (!aligned(kv->k, 16) || !aligned(kv->v, 16) || !aligned(kv->book, 4)) return fail(SPECTRE_EINVAL, "%s: pool array not aligned", who);
    if (kv->dtype == SPECTRE_E4M3 && (!kv->scales || !aligned(kv->scales, 8))) return fail(SPECTRE_EINVAL, "%s: scales of the pool null or not aligned", who);
    return SPECTRE_OK;
}

int check_ws(const void *ws, size_t have, size_t need, const char *who) {
    if (!ws || have < need) return fail(SPECTRE_EWORKSPACE, "%s: workspace %zu < %zu bytes", who, ws ? have : (size_t)0, need);
    if (!aligned(ws, 16)) return fail(SPECTRE_EINVAL, "%s: workspace not 16-byte aligned", who);
    return SPECTRE_OK;
}

// Type of the rows that calls on a pool take.
spectre_dtype rows_of(const spectre_kv *kv) { return kv->dtype == SPECTRE_E4M3 ? SPECTRE_BF16 : kv->dtype; }

struct Span {
    const void *at;
    long long stride;                // elements a token
    int heads;
    const char *name;
};
int size_of(spectre_dtype io) { return io == SPECTRE_BF16 ? 2 : 4; }

int check_rows(const Span &x, int d, spectre_dtype io, const char *who) {
    if (!x.at) return fail(SPECTRE_EINVAL, "%s: null %s", who, x.name);
    if (!aligned(x.at, 16)) return fail(SPECTRE_EINVAL, "%s: %s not 16-byte aligned", who, x.name);
    if (x.stride < (long long)x.heads * d) return fail(SPECTRE_EINVAL, "%s: stride of %s below its heads' channels", who, x.name);
    if (x.stride * size_of(io) % 16 || x.stride > LLONG_MAX / 64) return fail(SPECTRE_EINVAL, "%s: stride of %s not a multiple of 16 bytes", who, x.name);
    return SPECTRE_OK;
}
// Outputs are dense; an input may hold other rows between its own, so only ranges that interleave with them count as overlap.
bool overlap(const Span &in, const void *out, int out_heads, int T, int d, spectre_dtype io) {
    const uintptr_t size = size_of(io), a = reinterpret_cast<uintptr_t>(in.at), b = reinterpret_cast<uintptr_t>(out);
    const uintptr_t a_end = a + ((uintptr_t)(T - 1) * in.stride + (uintptr_t)in.heads * d) * size, b_end = b + (uintptr_t)T * out_heads * d * size;
    return a < b_end && b < a_end;
}

int check_heads(const spectre_heads *P, const int *positions, int T, int H, int Hkv, spectre_dtype io, const char *who) {
    if (!P) return fail(SPECTRE_EINVAL, "%s: null parameters", who);
    int rc = check_dtype(io, who);
    if (rc) return rc;
    if (T < 0 || H < 1 || Hkv < 1) return fail(SPECTRE_EINVAL, "%s: T below 0, or H or Hkv below 1", who);
    if (H > 65536 || Hkv > 65536) return fail(SPECTRE_EUNSUPPORTED, "%s: %d and %d heads", who, H, Hkv);
    if (P->d != 64 && P->d != 128) return fail(SPECTRE_EUNSUPPORTED, "%s: d = %d (64 and 128 are supported)", who, P->d);
    if (P->rot < 0 || P->rot > P->d || P->rot % 16) return fail(SPECTRE_EUNSUPPORTED, "%s: %d rotated channels (multiples of 16 up to d are supported)", who, P->rot);
    if (P->rot && !P->inv_freq) return fail(SPECTRE_EINVAL, "%s: null inv_freq", who);
    if (!P->wq != !P->wk) return fail(SPECTRE_EINVAL, "%s: one of wq and wk is null", who);
    if (P->wq && !(P->eps >= 0.f && std::isfinite(P->eps))) return fail(SPECTRE_EINVAL, "%s: eps", who);
    if (P->interleaved != 0 && P->interleaved != 1) return fail(SPECTRE_EINVAL, "%s: interleaved is neither 0 nor 1", who);
    if (P->axes < 0) return fail(SPECTRE_EINVAL, "%s: axes below 0", who);
    if (P->axes > SPECTRE_HEADS_MAX_AXES) return fail(SPECTRE_EUNSUPPORTED, "%s: %d axes (up to %d are supported)", who, P->axes, SPECTRE_HEADS_MAX_AXES);
    if (P->axes > 1 && P->rot && !P->axis) return fail(SPECTRE_EINVAL, "%s: null axis", who);
    if (P->axes > 1 && P->rot && !positions && T > 0) return fail(SPECTRE_EINVAL, "%s: null positions, which several axes need", who);
    if (!aligned(positions, 4) || !aligned(P->axis, 4)) return fail(SPECTRE_EINVAL, "%s: positions or axis not aligned", who);
    return SPECTRE_OK;
}

int check_layer(const spectre_kv *kv, int layer, const char *who) {
    return layer >= 0 && layer < kv->layers ? SPECTRE_OK : fail(SPECTRE_EINVAL, "%s: layer %d of %d", who, layer, kv->layers);
}

int check_batch(const spectre_kv *kv, const int *start, int B, int T, int H, const char *who) {
    if (!start) return fail(SPECTRE_EINVAL, "%s: null start", who);
    if (B < (T > 0) || T < 0 || H < 1) return fail(SPECTRE_EINVAL, "%s: T below 0, or B or H below 1", who);
    if (B > kv->seqs) return fail(SPECTRE_EINVAL, "%s: %d sequences, the table has %d", who, B, kv->seqs);
    if (H % kv->Hkv) return fail(SPECTRE_EINVAL, "%s: %d heads do not divide among %d key heads", who, H, kv->Hkv);
    if (H > 65536) return fail(SPECTRE_EUNSUPPORTED, "%s: %d heads", who, H);
    return SPECTRE_OK;
}

int done(hipError_t e, const char *who) { return e == hipSuccess ? SPECTRE_OK : fail_hip(e, who); }

int check_attend(const spectre_kv *kv, int B, int T, int H, int max_new, int max_len, int window, const char *who) {
    if (B < (T > 0) || T < 0 || H < 1 || H % kv->Hkv) return fail(SPECTRE_EINVAL, "%s: B, T or H", who);
    if (max_new < 1 || max_len < 1 || window < 0) return fail(SPECTRE_EINVAL, "%s: max_new or max_len below 1, or window below 0", who);
    const long long rows = (long long)max_new * (H / kv->Hkv), tiles = (rows + 127) / 128;
    if (rows > INT_MAX || tiles * B * kv->Hkv > (1 << 24) || (long long)B * kv->Hkv > (1 << 22) || (long long)T * H > INT_MAX)
        return fail(SPECTRE_EUNSUPPORTED, "%s: %d sequences of %d new tokens, %d heads", who, B, max_new, H);
    return SPECTRE_OK;
}

int check_norm(const float *w, int T, int D, float eps, spectre_dtype io, const char *who) {
    const int rc = check_dtype(io, who);
    if (rc) return rc;
    if (T < 0 || D < 1) return fail(SPECTRE_EINVAL, "%s: T below 0, or D below 1", who);
    if ((long long)D * size_of(io) % 16 || (long long)D * size_of(io) > kNormMostBytes)
        return fail(SPECTRE_EUNSUPPORTED, "%s: rows of %d channels (multiples of 16 bytes up to %d are supported)", who, D, kNormMostBytes);
    if (!(eps >= 0.f && std::isfinite(eps))) return fail(SPECTRE_EINVAL, "%s: eps", who);
    if (w && !aligned(w, 16)) return fail(SPECTRE_EINVAL, "%s: w not 16-byte aligned", who);
    return SPECTRE_OK;
}

// `bytes` of an output against the rows of an input, or another output's bytes.
bool meets(const void *out, size_t bytes, const void *at, size_t span) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(out), b = reinterpret_cast<uintptr_t>(at);
    return a < b + span && b < a + bytes;
}
size_t span_of(const Span &x, int T, int D, spectre_dtype io) { return ((size_t)(T - 1) * x.stride + D) * size_of(io); }

int check_plan(const AttendPlan &p, int B, int H, int max_new, const char *who) {
    return p.fits ? SPECTRE_OK : fail(SPECTRE_EUNSUPPORTED, "%s: %d sequences of %d new tokens, %d heads: more workgroups than a launch has", who, B, max_new, H);
}

}  // namespace
}  // namespace spectre

using namespace spectre;

#pragma GCC visibility push(default)
extern "C" {

size_t spectre_kv_bytes(const spectre_kv *kv, int which) {
    if (check_sizes(kv, "kv_bytes")) return 0;
    const size_t rows = (size_t)kv->layers * kv->pages * kv->Hkv * kv->page * kv->d * kv_size_of(kv->dtype);
    if (which == SPECTRE_KV_K || which == SPECTRE_KV_V) return rows;
    if (which == SPECTRE_KV_BOOK) return ((size_t)kKvStatusWords + kv->seqs + kv->pages + (size_t)kv->seqs * kv->max_pages) * sizeof(int);
    if (which == SPECTRE_KV_SCALES && kv->dtype == SPECTRE_E4M3) return (size_t)kv->layers * kv->pages * kv->Hkv * (kv->page / kKvBlock) * 2 * sizeof(float);
    fail(SPECTRE_EINVAL, "kv_bytes: unknown array %d", which);
    return 0;
}

int spectre_kv_prepare(void) {
    hipError_t (*const loaders[])() = {load_kernels_heads, load_kernels_pages, load_kernels_attend, load_kernels_append8, load_kernels_norm};
    for (auto load : loaders) {
        const hipError_t e = load();
        if (e != hipSuccess) return fail_hip(e, "kv_prepare: loading kernels");
    }
    return SPECTRE_OK;
}

int spectre_kv_init(const spectre_kv *kv, void *stream) {
    const int rc = check_pool(kv, "kv_init");
    if (rc) return rc;
    return done(launch_kv_init(kv_view(kv, 0), static_cast<hipStream_t>(stream)), "kv_init");
}

size_t spectre_kv_workspace_bytes(const spectre_kv *kv, int n) {
    if (check_sizes(kv, "kv_workspace") || n < 0) return 0;
    // eight words, then page lists: every page (reserve), two a child (fork), three a page (compact)
    const size_t words = 3 * (size_t)kv->pages > 2 * (size_t)n ? 3 * (size_t)kv->pages : 2 * (size_t)n;
    return align256((words + 8) * sizeof(int));
}

int spectre_kv_reserve(const spectre_kv *kv, const int *seqs, const int *add, int n, void *ws, size_t ws_bytes, void *stream) {
    int rc = check_pool(kv, "kv_reserve");
    if (rc) return rc;
    if (n < 0 || (n && (!seqs || !add))) return fail(SPECTRE_EINVAL, "kv_reserve: null list or negative count");
    if (n == 0) return SPECTRE_OK;
    rc = check_ws(ws, ws_bytes, spectre_kv_workspace_bytes(kv, n), "kv_reserve");
    if (rc) return rc;
    return done(launch_kv_reserve(kv_view(kv, 0), seqs, add, n, static_cast<int *>(ws), static_cast<hipStream_t>(stream)), "kv_reserve");
}

int spectre_kv_fork(const spectre_kv *kv, const int *src, const int *dst, int n, void *ws, size_t ws_bytes, void *stream) {
    int rc = check_pool(kv, "kv_fork");
    if (rc) return rc;
    if (n < 0 || (n && (!src || !dst))) return fail(SPECTRE_EINVAL, "kv_fork: null list or negative count");
    if (n > kv->seqs) return fail(SPECTRE_EINVAL, "kv_fork: %d children, the table has %d rows", n, kv->seqs);
    if (n == 0) return SPECTRE_OK;
    rc = check_ws(ws, ws_bytes, spectre_kv_workspace_bytes(kv, n), "kv_fork");
    if (rc) return rc;
    return done(launch_kv_fork(kv_view(kv, 0), kv->layers, kv->d, (int)kv->dtype, src, dst, n, static_cast<int *>(ws), static_cast<hipStream_t>(stream)), "kv_fork");
}

int spectre_kv_free(const spectre_kv *kv, const int *seqs, int n, void *stream) {
    const int rc = check_pool(kv, "kv_free");
    if (rc) return rc;
    if (n < 0 || (n && !seqs)) return fail(SPECTRE_EINVAL, "kv_free: null list or negative count");
    if (n == 0) return SPECTRE_OK;
    return done(launch_kv_free(kv_view(kv, 0), seqs, n, static_cast<hipStream_t>(stream)), "kv_free");
}

int spectre_kv_compact(const spectre_kv *kv, void *ws, size_t ws_bytes, void *stream) {
    int rc = check_pool(kv, "kv_compact");
    if (rc) return rc;
    rc = check_ws(ws, ws_bytes, spectre_kv_workspace_bytes(kv, 0), "kv_compact");
    if (rc) return rc;
    return done(launch_kv_compact(kv_view(kv, 0), kv->layers, static_cast<int *>(ws), static_cast<hipStream_t>(stream)), "kv_compact");
}

int spectre_kv_copy(const spectre_kv *kv, const int *src, const int *dst, int n, void *stream) {
    const int rc = check_pool(kv, "kv_copy");
    if (rc) return rc;
    if (n < 0 || (n && (!src || !dst))) return fail(SPECTRE_EINVAL, "kv_copy: null list or negative count");
    if (n == 0) return SPECTRE_OK;
    return done(launch_kv_copy(kv_view(kv, 0), kv->layers, src, dst, n, static_cast<hipStream_t>(stream)), "kv_copy");
}

int spectre_heads_forward(const spectre_heads *P, const void *q, long long q_stride, const void *k, long long k_stride, const int *positions, int T, int H, int Hkv,
                          spectre_dtype io, void *q_out, void *k_out, void *stream) {
    const char *who = "heads_forward";
    int rc = check_heads(P, positions, T, H, Hkv, io, who);
    if (rc || T == 0) return rc;
    const Span in[2] = {{q, q_stride, H, "q"}, {k, k_stride, Hkv, "k"}};
    for (const Span &x : in)
        if ((rc = check_rows(x, P->d, io, who))) return rc;
    const Span out[2] = {{q_out, (long long)H * P->d, H, "q_out"}, {k_out, (long long)Hkv * P->d, Hkv, "k_out"}};
    for (const Span &y : out) {
        if ((rc = check_rows(y, P->d, io, who))) return rc;
        for (const Span &x : in)
            if (overlap(x, y.at, y.heads, T, P->d, io)) return fail(SPECTRE_EINVAL, "%s: %s overlaps %s", who, y.name, x.name);
    }
    if (overlap(out[0], k_out, Hkv, T, P->d, io)) return fail(SPECTRE_EINVAL, "%s: outputs overlap", who);
    const HeadRows x = {q, k, nullptr, q_stride, k_stride, 0, T, H, Hkv};
    return done(launch_heads_forward(*P, (int)io, x, positions, q_out, k_out, static_cast<hipStream_t>(stream)), who);
}

size_t spectre_heads_backward_workspace_bytes(int T, int d) {
    if (T < 0 || (d != 64 && d != 128)) return 0;
    return align256((size_t)heads_backward_blocks(T) * 2 * d * sizeof(double));
}

int spectre_heads_backward(const spectre_heads *P, const void *dq, long long dq_stride, const void *dk, long long dk_stride, const void *q, long long q_stride, const void *k,
                           long long k_stride, const int *positions, int T, int H, int Hkv, spectre_dtype io, void *gq, void *gk, float *gwq, float *gwk, void *ws,
                           size_t ws_bytes, void *stream) {
    const char *who = "heads_backward";
    int rc = check_heads(P, positions, T, H, Hkv, io, who);
    if (rc) return rc;
    if (P->wq && (!gwq || !gwk)) return fail(SPECTRE_EINVAL, "%s: null gwq or gwk", who);
    if (T == 0) return P->wq ? done(launch_heads_backward(*P, (int)io, HeadRows{}, HeadRows{}, nullptr, nullptr, nullptr, gwq, gwk, nullptr, static_cast<hipStream_t>(stream)), who) : SPECTRE_OK;
    const Span in[4] = {{dq, dq_stride, H, "dq"}, {dk, dk_stride, Hkv, "dk"}, {q, q_stride, H, "q"}, {k, k_stride, Hkv, "k"}};
    for (const Span &x : in)
        if ((rc = check_rows(x, P->d, io, who))) return rc;
    const Span out[2] = {{gq, (long long)H * P->d, H, "gq"}, {gk, (long long)Hkv * P->d, Hkv, "gk"}};
    for (const Span &y : out) {
        if ((rc = check_rows(y, P->d, io, who))) return rc;
        for (const Span &x : in)
            if (overlap(x, y.at, y.heads, T, P->d, io)) return fail(SPECTRE_EINVAL, "%s: %s overlaps %s", who, y.name, x.name);
    }
    if (overlap(out[0], gk, Hkv, T, P->d, io)) return fail(SPECTRE_EINVAL, "%s: outputs overlap", who);
    if (P->wq) {
        rc = check_ws(ws, ws_bytes, spectre_heads_backward_workspace_bytes(T, P->d), who);
        if (rc) return rc;
    }
    const HeadRows x = {q, k, nullptr, q_stride, k_stride, 0, T, H, Hkv}, y = {dq, dk, nullptr, dq_stride, dk_stride, 0, T, H, Hkv};
    return done(launch_heads_backward(*P, (int)io, x, y, positions, gq, gk, gwq, gwk, static_cast<double *>(ws), static_cast<hipStream_t>(stream)), who);
}

int spectre_kv_append(const spectre_kv *kv, int layer, const spectre_heads *P, const void *q, long long q_stride, const void *k, long long k_stride, const void *v,
                      long long v_stride, const int *start, const int *seqs, int B, int T, int H, void *q_out, void *stream) {
    return spectre_kv_append_at(kv, layer, P, q, q_stride, k, k_stride, v, v_stride, nullptr, start, seqs, B, T, H, q_out, stream);
}

int spectre_kv_append_at(const spectre_kv *kv, int layer, const spectre_heads *P, const void *q, long long q_stride, const void *k, long long k_stride, const void *v,
                         long long v_stride, const int *positions, const int *start, const int *seqs, int B, int T, int H, void *q_out, void *stream) {
    const char *who = "kv_append";
    int rc = check_pool(kv, who);
    if (rc) return rc;
    if ((rc = check_layer(kv, layer, who))) return rc;
    const spectre_dtype io = rows_of(kv);
    if ((rc = check_heads(P, positions, T, H, kv->Hkv, io, who))) return rc;
    if (P->d != kv->d) return fail(SPECTRE_EINVAL, "%s: d = %d, the pool has %d", who, P->d, kv->d);
    if ((rc = check_batch(kv, start, B, T, H, who))) return rc;
    if (T == 0) return SPECTRE_OK;
    const Span in[3] = {{q, q_stride, H, "q"}, {k, k_stride, kv->Hkv, "k"}, {v, v_stride, kv->Hkv, "v"}};
    for (const Span &x : in)
        if ((rc = check_rows(x, kv->d, io, who))) return rc;
    if ((rc = check_rows({q_out, (long long)H * kv->d, H, "q_out"}, kv->d, io, who))) return rc;
    for (const Span &x : in)
        if (overlap(x, q_out, H, T, kv->d, io)) return fail(SPECTRE_EINVAL, "%s: q_out overlaps %s", who, x.name);
    const HeadRows x = {q, k, v, q_stride, k_stride, v_stride, T, H, kv->Hkv};
    if (kv->dtype == SPECTRE_E4M3) return done(launch_heads_append8(*P, x, kv_view(kv, layer), positions, start, seqs, B, q_out, static_cast<hipStream_t>(stream)), who);
    return done(launch_heads_append(*P, (int)io, x, kv_view(kv, layer), positions, start, seqs, B, q_out, static_cast<hipStream_t>(stream)), who);
}

size_t spectre_kv_attend_workspace_bytes(const spectre_kv *kv, int B, int T, int H, int max_new, int max_len, int window) {
    if (check_sizes(kv, "kv_attend") || check_attend(kv, B, T, H, max_new, max_len, window, "kv_attend")) return 0;
    if (window >= kLongest) window = 0;
    const AttendPlan p = attend_plan(kv->d, (int)kv->dtype, B, T, H, kv->Hkv, max_new, max_len, window);
    if (check_plan(p, B, H, max_new, "kv_attend")) return 0;
    return align256(p.partial_bytes + 1);
}

int spectre_kv_attend(const spectre_kv *kv, int layer, const void *q, long long q_stride, const int *start, const int *seqs, int B, int T, int H, int max_new, int max_len,
                      float scale, int window, void *out, float *lse, void *ws, size_t ws_bytes, void *stream) {
    const char *who = "kv_attend";
    int rc = check_pool(kv, who);
    if (rc) return rc;
    if ((rc = check_layer(kv, layer, who))) return rc;
    if ((rc = check_batch(kv, start, B, T, H, who))) return rc;
    if ((rc = check_attend(kv, B, T, H, max_new, max_len, window, who))) return rc;
    // statistics are kept in powers of two: scale and its inverse have to leave them their range
    if (!(scale >= 1e-30f && scale <= 1e30f)) return fail(SPECTRE_EINVAL, "%s: scale is not between 1e-30 and 1e30", who);
    if (window >= kLongest) window = 0;                 // sees everything there can be
    if (T == 0) return SPECTRE_OK;
    const Span x = {q, q_stride, H, "q"};
    const spectre_dtype io = rows_of(kv);
    if ((rc = check_rows(x, kv->d, io, who))) return rc;
    if ((rc = check_rows({out, (long long)H * kv->d, H, "out"}, kv->d, io, who))) return rc;
    if (overlap(x, out, H, T, kv->d, io)) return fail(SPECTRE_EINVAL, "%s: out overlaps q", who);
    const AttendPlan p = attend_plan(kv->d, (int)kv->dtype, B, T, H, kv->Hkv, max_new, max_len, window);
    if ((rc = check_plan(p, B, H, max_new, who))) return rc;
    if (p.partial_bytes && (rc = check_ws(ws, ws_bytes, align256(p.partial_bytes + 1), who))) return rc;
    const AttendArgs a = {q, q_stride, start, seqs, B, T, H, window, scale, out, lse};
    return done(launch_attend(kv_view(kv, layer), kv->layers, kv->d, (int)io, a, p, ws, static_cast<hipStream_t>(stream)), who);
}

int spectre_norm_forward(const void *x, long long x_stride, const void *delta, long long delta_stride, const float *w, int T, int D, float eps, spectre_dtype io, void *sum,
                         void *y, spectre_dtype y_type, float *scales, void *stream) {
    const char *who = "norm_forward";
    int rc = check_norm(w, T, D, eps, io, who);
    if (rc) return rc;
    if (y_type != io && y_type != SPECTRE_E4M3) return fail(SPECTRE_EINVAL, "%s: y is neither of the rows' type nor of 8 bits", who);
    const bool coded = y_type == SPECTRE_E4M3;
    if (coded && D % kNormGroup) return fail(SPECTRE_EUNSUPPORTED, "%s: %d channels in 8 bits (multiples of %d are supported)", who, D, kNormGroup);
    if (T == 0) return SPECTRE_OK;
    if (coded != (scales != nullptr)) return fail(SPECTRE_EINVAL, "%s: scales with y of the rows' type, or none with y of 8 bits", who);
    if (!delta != !sum) return fail(SPECTRE_EINVAL, "%s: one of delta and sum is null", who);
    const Span in[2] = {{x, x_stride, 1, "x"}, {delta, delta_stride, 1, "delta"}};
    const size_t rows = (size_t)T * D;
    const struct { const void *at; size_t bytes; const char *name; } out[3] = {
        {y, rows * (coded ? 1 : size_of(io)), "y"}, {sum, rows * size_of(io), "sum"}, {scales, rows / kNormGroup * sizeof(float), "scales"}};
    if (!y || !aligned(y, 16) || !aligned(sum, 16) || !aligned(scales, 4)) return fail(SPECTRE_EINVAL, "%s: an output is null or not aligned", who);
    for (int i = 0; i < (delta ? 2 : 1); ++i) {
        if ((rc = check_rows(in[i], D, io, who))) return rc;
        for (const auto &o : out)
            if (o.at && meets(o.at, o.bytes, in[i].at, span_of(in[i], T, D, io))) return fail(SPECTRE_EINVAL, "%s: %s overlaps %s", who, o.name, in[i].name);
    }
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < i; ++j)
            if (out[i].at && out[j].at && meets(out[i].at, out[i].bytes, out[j].at, out[j].bytes)) return fail(SPECTRE_EINVAL, "%s: outputs overlap", who);
    const NormRows n = {x, delta, x_stride, delta_stride, w, eps, T, D};
    return done(launch_norm(n, (int)io, sum, y, scales, static_cast<hipStream_t>(stream)), who);
}

size_t spectre_norm_backward_workspace_bytes(int T, int D, spectre_dtype io) {
    if (check_norm(nullptr, T, D, 0.f, io, "norm_backward")) return 0;
    const int blocks = norm_backward_blocks(T, D * size_of(io) / 16, true);
    return blocks > 1 ? align256((size_t)blocks * D * sizeof(float)) : 0;
}

int spectre_norm_backward(const void *dy, long long dy_stride, const void *sum, long long sum_stride, const void *dsum, long long dsum_stride, const float *w, int T, int D,
                          float eps, spectre_dtype io, void *gx, float *gw, void *ws, size_t ws_bytes, void *stream) {
    const char *who = "norm_backward";
    int rc = check_norm(w, T, D, eps, io, who);
    if (rc) return rc;
    if (!aligned(gw, 16)) return fail(SPECTRE_EINVAL, "%s: gw not 16-byte aligned", who);
    const NormRows n = {sum, nullptr, sum_stride, 0, w, eps, T, D};
    const NormGrads g = {dy, dsum, dy_stride, dsum_stride};
    if (T == 0) return gw ? done(launch_norm_backward(n, g, (int)io, gx, gw, nullptr, static_cast<hipStream_t>(stream)), who) : SPECTRE_OK;
    const Span in[3] = {{dy, dy_stride, 1, "dy"}, {sum, sum_stride, 1, "sum"}, {dsum, dsum_stride, 1, "dsum"}};
    if (!gx || !aligned(gx, 16)) return fail(SPECTRE_EINVAL, "%s: gx is null or not aligned", who);
    const size_t bytes = (size_t)T * D * size_of(io);
    for (int i = 0; i < (dsum ? 3 : 2); ++i) {
        if ((rc = check_rows(in[i], D, io, who))) return rc;
        if (meets(gx, bytes, in[i].at, span_of(in[i], T, D, io)) || (gw && meets(gw, D * sizeof(float), in[i].at, span_of(in[i], T, D, io))))
            return fail(SPECTRE_EINVAL, "%s: an output overlaps %s", who, in[i].name);
    }
    if (gw && meets(gx, bytes, gw, D * sizeof(float))) return fail(SPECTRE_EINVAL, "%s: outputs overlap", who);
    const size_t need = gw ? spectre_norm_backward_workspace_bytes(T, D, io) : 0;
    if (need && (rc = check_ws(ws, ws_bytes, need, who))) return rc;
    return done(launch_norm_backward(n, g, (int)io, gx, gw, static_cast<float *>(ws), static_cast<hipStream_t>(stream)), who);
}

}  // extern "C"
#pragma GCC visibility pop
