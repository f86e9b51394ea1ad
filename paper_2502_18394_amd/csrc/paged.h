// Keys and values in pages: layout, views of the bookkeeping, launchers of the kernels that work on them.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/spectre.h"

namespace spectre {

constexpr int kKvStatusWords = 8;
constexpr int kKvBlock = SPECTRE_KV_BLOCK, kKvBlockLog = 4;
static_assert(kKvBlock == 1 << kKvBlockLog && kKvBlock == 16, "a block of tokens is a 16-byte group of values");
inline int kv_size_of(int dtype) { return dtype == SPECTRE_BF16 ? 2 : dtype == SPECTRE_E4M3 ? 1 : 4; }

// One pool as the kernels see it.  A page of one key/value head is page * d elements of K, [d / E][page][E], and as many of V,
// [page / E][d][E], E = 16 bytes of elements: the 16-byte groups that a lane of a matrix instruction holds as its operand (adjacent channels of
// a key for Q K^T, adjacent keys of a channel for P V), so tiles go from memory to the matrix cores in wide loads without a transposition.
struct KvView {
    void *k, *v;                     // of one layer
    float *scales;                   // the same, pages of 8 bits: [page][head][block of kKvBlock tokens][keys, values]
    int *status, *lens, *refs, *table;
    int P, S, M, Hkv, page_log;      // pages, sequences, table row, key/value heads, log2(tokens a page)
    long long layer_bytes;           // of K, and of V
    long long layer_scales;          // 0: pages of another type
};

inline KvView kv_view(const spectre_kv *kv, int layer) {
    KvView w;
    w.layer_bytes = (long long)kv->pages * kv->Hkv * kv->page * kv->d * kv_size_of(kv->dtype);
    w.layer_scales = kv->dtype == SPECTRE_E4M3 ? (long long)kv->pages * kv->Hkv * (kv->page / kKvBlock) * 2 : 0;
    w.scales = w.layer_scales ? kv->scales + layer * w.layer_scales : nullptr;
    w.k = (char *)kv->k + (long long)layer * w.layer_bytes;
    w.v = (char *)kv->v + (long long)layer * w.layer_bytes;
    w.status = kv->book;
    w.lens = kv->book + kKvStatusWords;
    w.refs = w.lens + kv->seqs;
    w.table = w.refs + kv->pages;
    w.P = kv->pages; w.S = kv->seqs; w.M = kv->max_pages; w.Hkv = kv->Hkv;
    w.page_log = 0;
    while ((1 << w.page_log) < kv->page) ++w.page_log;
    return w;
}

hipError_t load_kernels_heads();
hipError_t load_kernels_pages();
hipError_t load_kernels_attend();
hipError_t load_kernels_append8();

// heads.hip
struct HeadRows {                    // token t, head h, channel c at base + (t * stride + h * d + c)
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    int T, H, Hkv;
};
hipError_t launch_heads_forward(const spectre_heads &P, int io, const HeadRows &x, const int *positions, void *q_out, void *k_out, hipStream_t st);
hipError_t launch_heads_append(const spectre_heads &P, int io, const HeadRows &x, const KvView &kv, const int *positions, const int *start, const int *seqs, int B, void *q_out,
                               hipStream_t st);
hipError_t launch_heads_append8(const spectre_heads &P, const HeadRows &x, const KvView &kv, const int *positions, const int *start, const int *seqs, int B, void *q_out,
                                hipStream_t st);   // append8.hip
int heads_backward_blocks(int T);
hipError_t launch_heads_backward(const spectre_heads &P, int io, const HeadRows &x, const HeadRows &dy, const int *positions, void *gq, void *gk, float *gwq, float *gwk,
                                 double *partial, hipStream_t st);

// pages.hip
hipError_t launch_kv_init(const KvView &kv, hipStream_t st);
hipError_t launch_kv_reserve(const KvView &kv, const int *seqs, const int *add, int n, int *ws, hipStream_t st);
hipError_t launch_kv_fork(const KvView &kv, int layers, int d, int io, const int *src, const int *dst, int n, int *ws, hipStream_t st);
hipError_t launch_kv_free(const KvView &kv, const int *seqs, int n, hipStream_t st);
hipError_t launch_kv_compact(const KvView &kv, int layers, int *ws, hipStream_t st);
hipError_t launch_kv_copy(const KvView &kv, int layers, const int *src, const int *dst, int n, hipStream_t st);

// attend.hip
struct AttendPlan {
    bool fits;                       // a launch can have that many workgroups
    int few, tile;                   // whether each kernel is launched
    int few_rows;                    // rows (new tokens x heads of a key head) that the kernel of few rows takes, 0 if it is not launched
    int few_splits, tile_splits, tiles, tile_waves, part_keys;
    bool packed;                     // rows have as many places for partial results as parts, not all the same number
    int few_tokens;                  // of a sequence, that have places of their own for few rows (0: all tokens of the batch)
    long long few_places, tile_places;
    size_t partial_bytes;            // of all rows' split results
};
struct AttendArgs {
    const void *q;
    long long q_stride;
    const int *start, *seqs;
    int B, T, H, window;
    float scale;
    void *out;
    float *lse;
};
AttendPlan attend_plan(int d, int dtype, int B, int T, int H, int Hkv, int max_new, int max_len, int window);
hipError_t launch_attend(const KvView &kv, int layers, int d, int io, const AttendArgs &a, const AttendPlan &p, void *ws, hipStream_t st);

}  // namespace spectre
