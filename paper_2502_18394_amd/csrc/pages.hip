// Pages of a cache: given to sequences, shared by forks, copied, freed, and the pool made dense again.
//
// The bookkeeping lives on the device (lengths, users of each page, page numbers), so a captured decode loop can take pages without the host.  A page nobody
// uses is free; pages are taken lowest number first, in the order of the call's list, so results do not depend on what ran when.  Each call checks
// everything it is given before it changes anything: one that cannot be done as a whole sets bits of the status and changes nothing.
// Bookkeeping is one workgroup's work (a scan over the page users, latency of a launch); the page data moves in a second launch over the whole
// card, bound by memory: 200 pages of 4 layers (210 MB read and written) 41 us, 5.1 TB/s, a large copy's rate; 537 MB of pages moved by a compaction 94 us, 5.7 TB/s.
// The bookkeeping takes 3.5 (free) to 7.5 us (reserve).
#include "common.h"
#include "paged.h"

namespace spectre {
namespace {

constexpr int kScan = 1024;                        // threads of a bookkeeping workgroup
constexpr int kSeqWords = SPECTRE_KV_MAX_SEQS / 32;
constexpr int kWsHead = 8;                         // words in front of a workspace's lists: [0] = done, [1] = how many

// Sum over the threads before this one; *total = over all.
__device__ __forceinline__ int scan_before(int x, int *total, int *waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = x;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int y = __shfl_up(s, m, 64);
        if (lane >= m) s += y;
    }
    __syncthreads();                               // `waves` of the scan before has been read
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kScan / 64; ++w) {
        const int y = waves[w];
        if (w < wave) before += y;
        all += y;
    }
    *total = all;
    return before + s - x;
}

// Marks sequence s; true if it was marked before.
__device__ __forceinline__ bool mark(uint32_t *bits, int s) {
    const uint32_t bit = 1u << (s & 31);
    return (atomicOr(&bits[s >> 5], bit) & bit) != 0;
}

// The first `want` free pages into `list`, in order; how many there were.  Each thread looks at four pages a step.
__device__ int list_free(const KvView &kv, int want, int *list, int *waves) {
    int found = 0;
    for (int base = 0; base < kv.P && found < want; base += 4 * kScan) {
        const int p0 = base + 4 * threadIdx.x;
        int free[4], n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            free[i] = p0 + i < kv.P && kv.refs[p0 + i] <= 0;
            n += free[i];
        }
        int total;
        int at = found + scan_before(n, &total, waves);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (free[i]) {
                if (at < want) list[at] = p0 + i;
                ++at;
            }
        found += total;
    }
    return found;
}

__global__ __launch_bounds__(256) void k_kv_init(KvView kv) {
    const long long n = (long long)kKvStatusWords + kv.S + kv.P + (long long)kv.S * kv.M, table = kKvStatusWords + kv.S + kv.P;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) kv.status[i] = i < table ? 0 : -1;
}

// ws: [0] done, [2 ..] page lists.  Sequences grow by add[i] tokens.
__global__ __launch_bounds__(kScan) void k_kv_reserve(KvView kv, const int *seqs, const int *add, int n, int *ws) {
    __shared__ uint32_t seen[kSeqWords];
    __shared__ int waves[kScan / 64];
    __shared__ int bad;
    const int page = 1 << kv.page_log;
    for (int i = threadIdx.x; i < (kv.S + 31) / 32; i += kScan) seen[i] = 0;
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    int need = 0;
    for (int base = 0; base < n; base += kScan) {
        const int i = base + threadIdx.x;
        int mine = 0;
        if (i < n) {
            const int s = seqs[i], more = add[i];
            if ((unsigned)s >= (unsigned)kv.S || more < 0) atomicOr(&bad, SPECTRE_KV_BAD_ARGUMENT);
            else if (mark(seen, s)) atomicOr(&bad, SPECTRE_KV_BAD_ARGUMENT);
            else {
                const long long had = kv.lens[s], has = had + more;
                if (had < 0) atomicOr(&bad, SPECTRE_KV_BAD_ARGUMENT);
                else if (((has + page - 1) >> kv.page_log) > kv.M) atomicOr(&bad, SPECTRE_KV_TOO_LONG);
                else mine = (int)(((has + page - 1) >> kv.page_log) - ((had + page - 1) >> kv.page_log));
            }
        }
        int total;
        scan_before(mine, &total, waves);
        need += total;
        if (need > kv.P) break;                    // more than there are, whatever follows
    }
    __syncthreads();
    if (bad == 0 && need > kv.P && threadIdx.x == 0) bad = SPECTRE_KV_NO_PAGES;
    __syncthreads();
    int *list = ws + kWsHead;
    if (bad == 0 && list_free(kv, need, list, waves) < need && threadIdx.x == 0) bad = SPECTRE_KV_NO_PAGES;
    __syncthreads();
    if (bad) {
        if (threadIdx.x == 0) atomicOr(&kv.status[0], bad);
        return;
    }
    int first = 0;
    for (int base = 0; base < n; base += kScan) {
        const int i = base + threadIdx.x;
        int had = 0, mine = 0, s = 0;
        if (i < n) {
            s = seqs[i];
            had = (kv.lens[s] + page - 1) >> kv.page_log;
            mine = ((kv.lens[s] + add[i] + page - 1) >> kv.page_log) - had;
        }
        int total;
        const int at = first + scan_before(mine, &total, waves);
        if (i < n) {
            kv.lens[s] += add[i];
            for (int j = 0; j < mine; ++j) {
                const int p = list[at + j];
                kv.table[(long long)s * kv.M + had + j] = p;
                kv.refs[p] = 1;
            }
        }
        first += total;
    }
}

// Whether the last page of sequence s, of `len` tokens, has to be copied for a child: it is not full, and in the pool (one that is absent is absent in the child, too).
__device__ __forceinline__ bool copies_last(const KvView &kv, int s, int len) {
    if ((len & ((1 << kv.page_log) - 1)) == 0) return false;
    return (unsigned)kv.table[(long long)s * kv.M + (len >> kv.page_log)] < (unsigned)kv.P;
}

// Which parents' last pages have to be copied, and the pages that take them: ws [0] done, list[i] = page of child i or -1.
__global__ __launch_bounds__(kScan) void k_kv_fork_plan(KvView kv, const int *src, const int *dst, int n, int *ws) {
    __shared__ uint32_t from[kSeqWords], to[kSeqWords];
    __shared__ int waves[kScan / 64];
    __shared__ int bad;
    for (int i = threadIdx.x; i < (kv.S + 31) / 32; i += kScan) from[i] = to[i] = 0;
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    int need = 0;
    for (int base = 0; base < n; base += kScan) {
        const int i = base + threadIdx.x;
        int mine = 0;
        if (i < n) {
            const int a = src[i], b = dst[i];
            if ((unsigned)a >= (unsigned)kv.S || (unsigned)b >= (unsigned)kv.S) atomicOr(&bad, SPECTRE_KV_BAD_ARGUMENT);
            else {
                mark(from, a);
                if (mark(to, b)) atomicOr(&bad, SPECTRE_KV_BAD_ARGUMENT);
                if (kv.lens[b] != 0) atomicOr(&bad, SPECTRE_KV_NOT_EMPTY);
                const int len = kv.lens[a];
                if (len < 0 || len > (long long)kv.M << kv.page_log) atomicOr(&bad, SPECTRE_KV_BAD_ARGUMENT);
                else mine = copies_last(kv, a, len);
            }
        }
        int total;
        scan_before(mine, &total, waves);
        need += total;
    }
    __syncthreads();
    for (int w = threadIdx.x; w < (kv.S + 31) / 32; w += kScan)
        if (from[w] & to[w]) atomicOr(&bad, SPECTRE_KV_BAD_ARGUMENT);       // a sequence that is read and written
    int *child = ws + kWsHead, *list = child + n;
    __syncthreads();
    if (bad == 0 && need > n) need = n;
    if (bad == 0 && list_free(kv, need, list, waves) < need && threadIdx.x == 0) bad = SPECTRE_KV_NO_PAGES;
    __syncthreads();
    if (threadIdx.x == 0) ws[0] = bad == 0;
    if (bad) {
        if (threadIdx.x == 0) atomicOr(&kv.status[0], bad);
        return;
    }
    if (threadIdx.x == 0) kv.status[1] = need;
    int first = 0;
    for (int base = 0; base < n; base += kScan) {
        const int i = base + threadIdx.x;
        const int mine = i < n && copies_last(kv, src[i], kv.lens[src[i]]);
        int total;
        const int at = first + scan_before(mine, &total, waves);
        if (i < n) child[i] = mine ? list[at] : -1;
        first += total;
    }
}

// Child i's row of the table, and the tokens of its last page: block x = child, y = slices of the layers' K and V.  Parents' rows and lengths are only
// read (no child is a parent), users are counted with integer atomics, whose order changes nothing.
__global__ __launch_bounds__(256) void k_kv_fork(KvView kv, int layers, int d, int E, const int *src, const int *dst, int n, const int *ws) {
    if (!ws[0]) return;
    const int i = blockIdx.x, a = src[i], b = dst[i], len = kv.lens[a], page = 1 << kv.page_log;
    const int full = len >> kv.page_log, rest = len & (page - 1), fresh = ws[kWsHead + i];
    if (blockIdx.y == 0) {
        for (int j = threadIdx.x; j < kv.M; j += 256) {
            int p = -1;
            if (j < full || (j == full && rest && fresh < 0)) {
                p = kv.table[(long long)a * kv.M + j];
                if ((unsigned)p < (unsigned)kv.P) atomicAdd(&kv.refs[p], 1);
            } else if (j == full && rest) {
                p = fresh;
                kv.refs[p] = 1;
            }
            kv.table[(long long)b * kv.M + j] = p;
        }
        if (threadIdx.x == 0) kv.lens[b] = len;
    }
    if (!rest || fresh < 0) return;
    const int old = kv.table[(long long)a * kv.M + full];
    // The 16-byte groups that hold the tokens: K rows of `some` groups of a page's `page`, V rows one after the other.
    const int some = (rest + E - 1) / E * E, lanes = d / E;
    const long long block = (long long)kv.Hkv * lanes << kv.page_log;          // groups of one page
    const long long rows = (long long)layers * 2 * kv.Hkv;                     // (layer, K or V, head)
    const int part = some * lanes;                                             // groups a row
    for (long long u = blockIdx.y; u < rows; u += gridDim.y) {
        const int h = (int)(u % kv.Hkv), which = (int)(u / kv.Hkv) & 1, layer = (int)(u / (2 * kv.Hkv));
        uint4 *base = reinterpret_cast<uint4 *>((which ? (char *)kv.v : (char *)kv.k) + layer * kv.layer_bytes);
        const long long at = (long long)h * lanes << kv.page_log;
        const uint4 *x = base + old * block + at;
        uint4 *y = base + fresh * block + at;
        for (int g = threadIdx.x; g < part; g += 256) {
            const int o = which ? g : ((g / some) << kv.page_log) + g % some;
            y[o] = x[o];
        }
    }
}

// One workgroup a sequence; the one that takes the length away frees the pages, so a sequence listed twice is freed once.
__global__ __launch_bounds__(256) void k_kv_free(KvView kv, const int *seqs, int n) {
    __shared__ int len;
    const int s = seqs[blockIdx.x];
    if ((unsigned)s >= (unsigned)kv.S) {
        if (threadIdx.x == 0) atomicOr(&kv.status[0], SPECTRE_KV_BAD_ARGUMENT);
        return;
    }
    if (threadIdx.x == 0) len = atomicExch(&kv.lens[s], 0);
    __syncthreads();
    const int pages = min((max(len, 0) + (1 << kv.page_log) - 1) >> kv.page_log, kv.M);
    for (int j = threadIdx.x; j < pages; j += 256) {
        const int p = kv.table[(long long)s * kv.M + j];
        if ((unsigned)p < (unsigned)kv.P) atomicSub(&kv.refs[p], 1);
        kv.table[(long long)s * kv.M + j] = -1;
    }
}

// The i-th page in use at or above the number of pages in use goes to the i-th free page below it.  ws: [1] moves, to[P] (new numbers of
// pages that move), moved[P], hole[P].
__global__ __launch_bounds__(kScan) void k_kv_compact_plan(KvView kv, int *ws) {
    __shared__ int waves[kScan / 64];
    int *to = ws + kWsHead, *moved = to + kv.P, *hole = moved + kv.P;
    int live = 0;
    for (int base = 0; base < kv.P; base += 4 * kScan) {
        int n = 0, total;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = base + 4 * (int)threadIdx.x + i;
            n += p < kv.P && kv.refs[p] > 0;
        }
        scan_before(n, &total, waves);
        live += total;
    }
    int moves = 0, holes = 0;
    for (int base = 0; base < kv.P; base += 4 * kScan) {
        int used[4], n = 0, total;                 // below `live` a free page counts, above it one in use
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = base + 4 * (int)threadIdx.x + i;
            used[i] = p < kv.P && kv.refs[p] > 0;
            if (p < kv.P) n += p < live ? (used[i] ? 0 : 1) : (used[i] ? 1 << 16 : 0);
        }
        const int before = scan_before(n, &total, waves);        // at most 4096 of each: both counts in one word
        int h = holes + (before & 0xffff), m = moves + (before >> 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = base + 4 * (int)threadIdx.x + i;
            if (p >= kv.P) continue;
            if (p < live && !used[i]) hole[h++] = p;
            if (p >= live && used[i]) moved[m++] = p;
            if (p >= live && !used[i]) to[p] = p;
        }
        holes += total & 0xffff;
        moves += total >> 16;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < moves; i += kScan) {
        const int a = moved[i], b = hole[i];
        to[a] = b;
        kv.refs[b] = kv.refs[a];
        kv.refs[a] = 0;
    }
    if (threadIdx.x == 0) {
        ws[1] = moves;
        ws[2] = live;
        kv.status[1] = moves;
        kv.status[2] = live;
    }
}

// Copies whole pages of every layer's K and V: units of kUnit groups, dealt to workgroups in turn; with four 16-byte loads a thread on their way.
constexpr int kUnit = 4 * 256;
__device__ __forceinline__ void copy_pages(const KvView &kv, int layers, long long groups, const int *src, const int *dst, int n, int first, int stride) {
    const int units = (int)((groups + kUnit - 1) / kUnit);
    const long long all = (long long)n * layers * 2 * units;
    for (long long u = first; u < all; u += stride) {
        const int unit = (int)(u % units);
        const long long x = u / units;
        const int which = (int)(x & 1), layer = (int)((x >> 1) % layers), i = (int)((x >> 1) / layers);
        const int a = src[i], b = dst[i];
        if ((unsigned)a >= (unsigned)kv.P || (unsigned)b >= (unsigned)kv.P) {
            if (threadIdx.x == 0 && unit == 0) atomicOr(&kv.status[0], SPECTRE_KV_BAD_ARGUMENT);
            continue;
        }
        float4 *base = reinterpret_cast<float4 *>((which ? (char *)kv.v : (char *)kv.k) + layer * kv.layer_bytes);
        const float4 *p = base + a * groups;
        float4 *q = base + b * groups;
        float4 r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long g = (long long)unit * kUnit + j * 256 + threadIdx.x;
            if (g < groups) r[j] = stream_load(p + g);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long g = (long long)unit * kUnit + j * 256 + threadIdx.x;
            if (g < groups) stream_store(q + g, r[j]);
        }
    }
}

__global__ __launch_bounds__(256) void k_kv_copy(KvView kv, int layers, long long groups, const int *src, const int *dst, int n) {
    copy_pages(kv, layers, groups, src, dst, n, blockIdx.x, gridDim.x);
}

// Page data and page numbers after k_kv_compact_plan: sources are at or above the pages in use, destinations below, so no page is both.
__global__ __launch_bounds__(256) void k_kv_compact(KvView kv, int layers, long long groups, const int *ws) {
    const int moves = ws[1], live = ws[2];
    if (!moves) return;
    const int *to = ws + kWsHead;
    const long long n = (long long)kv.S * kv.M;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int p = kv.table[i];
        if (p >= live && p < kv.P) kv.table[i] = to[p];
    }
    copy_pages(kv, layers, groups, to + kv.P, to + 2 * kv.P, moves, blockIdx.x, gridDim.x);
}

long long page_groups(const KvView &kv) { return kv.layer_bytes / 16 / kv.P; }

}  // namespace

hipError_t load_kernels_pages() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, reinterpret_cast<const void *>(k_kv_init));
}

hipError_t launch_kv_init(const KvView &kv, hipStream_t st) {
    k_kv_init<<<256, 256, 0, st>>>(kv);
    return hipGetLastError();
}

hipError_t launch_kv_reserve(const KvView &kv, const int *seqs, const int *add, int n, int *ws, hipStream_t st) {
    k_kv_reserve<<<1, kScan, 0, st>>>(kv, seqs, add, n, ws);
    return hipGetLastError();
}

hipError_t launch_kv_fork(const KvView &kv, int layers, int d, int io, const int *src, const int *dst, int n, int *ws, hipStream_t st) {
    k_kv_fork_plan<<<1, kScan, 0, st>>>(kv, src, dst, n, ws);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int rows = layers * 2 * kv.Hkv, most = (2048 + n - 1) / n;
    k_kv_fork<<<dim3(n, rows < most ? rows : most), 256, 0, st>>>(kv, layers, d, io == SPECTRE_BF16 ? 8 : 4, src, dst, n, ws);
    return hipGetLastError();
}

hipError_t launch_kv_free(const KvView &kv, const int *seqs, int n, hipStream_t st) {
    k_kv_free<<<n, 256, 0, st>>>(kv, seqs, n);
    return hipGetLastError();
}

hipError_t launch_kv_compact(const KvView &kv, int layers, int *ws, hipStream_t st) {
    k_kv_compact_plan<<<1, kScan, 0, st>>>(kv, ws);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_kv_compact<<<2048, 256, 0, st>>>(kv, layers, page_groups(kv), ws);
    return hipGetLastError();
}

hipError_t launch_kv_copy(const KvView &kv, int layers, const int *src, const int *dst, int n, hipStream_t st) {
    const long long units = (long long)n * layers * 2 * ((page_groups(kv) + kUnit - 1) / kUnit);
    k_kv_copy<<<(int)(units < 2048 ? units : 2048), 256, 0, st>>>(kv, layers, page_groups(kv), src, dst, n);
    return hipGetLastError();
}

}  // namespace spectre
