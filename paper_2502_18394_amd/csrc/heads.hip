// Norms of query and key heads with the rotation by their position, in one pass: training forms (forward, backward) and the serving form
// that writes keys and values into their pages.
//
// Per row x of d channels: r = (mean x^2 + eps)^-1/2, y = w r x, and each pair (a, b) of y turned by the angle pos * f_i:
// (a cos - b sin, b cos + a sin).  Backward with g = the output's gradient turned back: g_w = sum g r x over rows, h = g w,
// g_x = r (h - r x mean(h r x)).  Rows are read and written once; memory bounds the long calls, the launch the short ones.  32768 tokens of 32 + 8 bf16 heads, d = 64:
// forward 68 to 75 us by the machine (336 MB, 4.5 to 4.9 TB/s), backward 98 to 108 (503 MB, 4.7 to 5.1 TB/s, the sums of the weights' gradients in it), the two in turn 160 to 166,
// against 5.2 TB/s of a large copy; 8192 tokens into pages 22 us (4.6 TB/s); one token 5.
#include <math.h>

#include "common.h"
#include "paged.h"

namespace spectre {
namespace {

constexpr int kThreads = 256, kTokens = 8;      // tokens a workgroup: one 16-byte group of V pages, two in fp32
constexpr int kMostHalf = 64;                   // pairs of a row of 128 channels

struct Bf16Group {
    static constexpr int E = 8;
    typedef uint16_t elem_t;
    __device__ static __forceinline__ void unpack(uint4 g, float (&x)[8]) {
        const uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = IoBf16::pack(make_float2(x[2 * i], x[2 * i + 1]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
struct F32Group {
    static constexpr int E = 4;
    typedef uint32_t elem_t;
    __device__ static __forceinline__ void unpack(uint4 g, float (&x)[4]) {
        x[0] = __uint_as_float(g.x); x[1] = __uint_as_float(g.y); x[2] = __uint_as_float(g.z); x[3] = __uint_as_float(g.w);
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

struct HeadParams {
    const double *freq;
    const float *wq, *wk;
    float eps;
    int half;                       // pairs a row, 0: no rotation
    int interleaved;
};

// cos and sin of the angles of a workgroup's tokens, one pair a thread.  The turns pos * f / 2 pi are formed and reduced in 64 bits: a position of
// 131072 leaves 32 bits with an angle that is wrong in the third digit.
__device__ __forceinline__ void fill_turns(const HeadParams &P, const int *pos, int count, float2 (*turns)[kMostHalf]) {
    for (int i = threadIdx.x; i < count * P.half; i += kThreads) {
        const int t = i / P.half, f = i - t * P.half;
        double rev = (double)pos[t] * P.freq[f] * 0.15915494309189533577;
        rev -= rint(rev);
        float s, c;
        sincospif((float)(2.0 * rev), &s, &c);
        turns[t][f] = make_float2(c, s);
    }
}

// What a lane needs of its E channels, the same for every row it visits: its pairs' cos and sin (sin negated in the first half of split pairs)
// and the lane that holds the partners.
template <typename IO, int D>
struct Lane {
    static constexpr int E = IO::E, kLanes = D / E;
    int lane, partner;              // within a row; the partner's lane in the wave
    bool turned;
    float c[E], s[E];

    __device__ __forceinline__ void set(const HeadParams &P, const float2 *turns, float sign) {
        lane = threadIdx.x % kLanes;
        const int groups = 2 * P.half / E;             // lanes of a row that hold rotated channels
        turned = lane < groups;
        int at = lane;
        if (!P.interleaved && turned) at = lane < groups / 2 ? lane + groups / 2 : lane - groups / 2;
        partner = (threadIdx.x & 63) - lane + at;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            c[e] = 1.f; s[e] = 0.f;
            if (turned) {
                const int ch = lane * E + e;
                const int f = P.interleaved ? ch >> 1 : (ch < P.half ? ch : ch - P.half);
                const float2 t = turns[f];
                const bool first = P.interleaved ? !(ch & 1) : ch < P.half;
                c[e] = t.x;
                s[e] = first ? -sign * t.y : sign * t.y;
            }
        }
    }
    // y of this lane's channels, z of their partners'.  Channels that are not turned (whole lanes of them) pass through: a zero times an infinite neighbour is NaN.
    __device__ __forceinline__ void turn(const HeadParams &P, const float (&y)[E], const float (&z)[E], float (&o)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float t = y[e] * c[e] + (P.interleaved ? y[e ^ 1] : z[e]) * s[e];
            o[e] = turned ? t : y[e];
        }
    }
};

// Sum over the 8, 16 or 32 lanes of a row, in all of them: moves inside the vector unit, not through LDS.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float row_sum(float x) {
    static_assert(LANES == 8 || LANES == 16 || LANES == 32, "lanes of a row");
    x += dpp<0xB1>(x);                              // lane ^ 1
    x += dpp<0x4E>(x);                              // lane ^ 2
    x += dpp<0x141>(x);                             // the other four of eight
    if constexpr (LANES >= 16) x += dpp<0x140>(x);  // the other eight of sixteen
    if constexpr (LANES == 32) {
        typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
        const u32x2_t y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    return x;
}

// Rows of gradients and of training's outputs: through plain stores while the L2s hold them together for whoever comes next, streaming beyond that, which
// leaves the memory-side cache to what is read again (32768 tokens of 40 bf16 heads, forward and backward: 163 instead of 181 us; 8000 fp32 tokens 91 instead of 93).
__device__ __forceinline__ void put(uint4 *p, uint4 v, bool stream) {
    const float4 w = __builtin_bit_cast(float4, v);
    if (stream) stream_store(reinterpret_cast<float4 *>(p), w);
    else *reinterpret_cast<float4 *>(p) = w;
}

__device__ __forceinline__ uint4 shuffle(uint4 g, int lane) {
    return make_uint4(__shfl((int)g.x, lane, 64), __shfl((int)g.y, lane, 64), __shfl((int)g.z, lane, 64), __shfl((int)g.w, lane, 64));
}

// One row's norm and rotation.
template <typename IO, int D>
__device__ __forceinline__ uint4 head_row(const HeadParams &P, const Lane<IO, D> &L, const float *w, uint4 raw) {
    constexpr int E = IO::E;
    float x[E], z[E], o[E];
    IO::unpack(raw, x);
    const uint4 other = (P.half && !P.interleaved) ? shuffle(raw, L.partner) : raw;
    IO::unpack(other, z);
    if (w) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) sq += x[e] * x[e];
        const float r = rsqrtf(row_sum<D / E>(sq) * (1.f / D) + P.eps);
        const int base = L.lane * E, mate = (L.lane + (L.partner - (int)(threadIdx.x & 63))) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] = x[e] * r * w[base + e];
            z[e] = z[e] * r * w[mate + e];
        }
    }
    if (P.half) L.turn(P, x, z, o);
    else
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = x[e];
    return IO::pack(o);
}

// Place of a workgroup's tokens.  Training: kTokens tokens from kTokens * block on.  Serving: the tokens of one sequence that fall into one
// kTokens-aligned run of cache indexes, so that runs inside a chunk fill whole groups of the V pages.  Sequence b's runs are numbered from
// start[b] / kTokens + 2 b on: n tokens touch at most n / kTokens + 2 runs, so no two sequences' numbers meet.
struct Run {
    int first, count;               // tokens
    int index;                      // cache index of the first one
    int seq;                        // its row of the table
};

// Bits of the status that a reserve which could not be done leaves.  Its sequences have not grown, so what would be taken for the new tokens' places holds their last ones:
// nothing is written while a bit stands.
constexpr int kNotReserved = SPECTRE_KV_NO_PAGES | SPECTRE_KV_TOO_LONG | SPECTRE_KV_BAD_ARGUMENT;

__device__ __forceinline__ bool find_run(const KvView &kv, const int *start, const int *seqs, int B, int T, int block, Run *r) {
    const int status = kv.status[0];
    int lo = 0, hi = B;             // the last b with start[b] / kTokens + 2 b <= block: 64 asked at once (19 fp32 sequences of up to 700 tokens 18.6 us, by halves 19.0)
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, mid = lo + step * (int)(threadIdx.x & 63);
        const bool behind = mid == lo || (mid < hi && start[mid] / kTokens + 2 * mid <= block);
        lo += step * (__popcll(__ballot(behind)) - 1);
        hi = min(hi, lo + step);
    }
    const int from = start[lo], to = min(start[lo + 1], T), n = to - from;
    const int row = seqs ? seqs[lo] : lo;
    if ((status & kNotReserved) || from < 0 || n <= 0 || (unsigned)row >= (unsigned)kv.S) return false;
    const int had = kv.lens[row] - n;          // tokens before the new ones
    if (had < 0) return false;
    const int run = block - (from / kTokens + 2 * lo);
    const int a = max((had / kTokens + run) * kTokens, had), b = min((had / kTokens + run + 1) * kTokens, had + n);
    if (run < 0 || a >= b) return false;
    r->first = from + (a - had);
    r->count = b - a;
    r->index = a;
    r->seq = row;
    return true;
}

template <typename IO, int D, bool SERVE>
__global__ __launch_bounds__(kThreads) void k_heads(HeadParams P, HeadRows X, const int *positions, uint4 *q_out, uint4 *k_out, KvView kv, const int *start, const int *seqs,
                                                    int B, bool stream) {
    constexpr int E = IO::E, LANES = D / E, ROWS = kThreads / LANES;
    __shared__ float2 turns[kTokens][kMostHalf];
    __shared__ int pos[kTokens];
    __shared__ float weights[2][D];
    Run run{(int)blockIdx.x * kTokens, min(kTokens, X.T - (int)blockIdx.x * kTokens), 0, 0};
    if (SERVE && !find_run(kv, start, seqs, B, X.T, blockIdx.x, &run)) return;
    if (threadIdx.x < run.count) pos[threadIdx.x] = SERVE ? run.index + threadIdx.x : (positions ? positions[run.first + threadIdx.x] : run.first + (int)threadIdx.x);
    for (int i = threadIdx.x; i < D; i += kThreads) {
        weights[0][i] = P.wq ? P.wq[i] : 1.f;
        weights[1][i] = P.wk ? P.wk[i] : 1.f;
    }
    int page = 0, slot = 0;
    if (SERVE) {                                   // kTokens divides a page: one page a workgroup
        const int p = run.index >> kv.page_log;
        page = p < kv.M ? kv.table[(long long)run.seq * kv.M + p] : -1;
        slot = run.index & ((1 << kv.page_log) - 1);
    }
    __syncthreads();
    fill_turns(P, pos, run.count, turns);
    __syncthreads();

    // A page with several users holds another sequence's tokens, too: a reserve would have given the new ones a page of their own.  (Looked at where keys are written.)
    const bool in_pool = SERVE && (unsigned)page < (unsigned)kv.P;
    const int users = in_pool ? kv.refs[page] : 0;

    // rows in the order (head, token), tokens padded to a power of two, so that a thread stays with one token and one group of channels
    int tl = 0;
    while ((1 << tl) < run.count) ++tl;
    const int token = (threadIdx.x / LANES) & ((1 << tl) - 1);
    const bool there = token < run.count;
    Lane<IO, D> L;
    L.set(P, turns[there ? token : 0], 1.f);
    const long long t = run.first + token;
    const int heads = X.H + X.Hkv, step = ROWS >> tl;          // ROWS >= kTokens
    const uint4 *q = reinterpret_cast<const uint4 *>(X.q), *k = reinterpret_cast<const uint4 *>(X.k);
    const int first = (threadIdx.x / LANES) >> tl;
    constexpr int AHEAD = 4;                                   // rows on their way at once (the first of them before the angles are formed: 3 to 7 % slower)
    for (int h0 = first + (int)blockIdx.y * AHEAD * step; h0 - first < heads; h0 += AHEAD * step * (int)gridDim.y) {
        uint4 raw[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int h = h0 + i * step;
            raw[i] = make_uint4(0, 0, 0, 0);
            if (there && h < heads) raw[i] = h < X.H ? q[(t * X.q_stride + h * D) / E + L.lane] : k[(t * X.k_stride + (h - X.H) * D) / E + L.lane];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int h = h0 + i * step;
            const bool key = h >= X.H;
            const uint4 o = head_row<IO, D>(P, L, P.wq ? weights[key] : nullptr, raw[i]);
            if (!there || h >= heads) continue;
            if (!key) put(&q_out[(t * X.H + h) * LANES + L.lane], o, stream);
            else if (!SERVE) put(&k_out[(t * X.Hkv + h - X.H) * LANES + L.lane], o, stream);
            else if (in_pool && users <= 1) {
                const long long block = ((long long)page * X.Hkv + h - X.H) * LANES + L.lane;
                reinterpret_cast<uint4 *>(kv.k)[(block << kv.page_log) + slot + token] = o;
            }
        }
    }
    if (!in_pool) return;
    if (users > 1) {
        if (threadIdx.x == 0) atomicOr(&kv.status[0], SPECTRE_KV_SHARED);
        return;
    }
    // values: a lane holds one channel of every token of the run and writes whole groups where the run has them
    typedef typename IO::elem_t elem_t;
    const elem_t *v = reinterpret_cast<const elem_t *>(X.v);
    for (int i = threadIdx.x + kThreads * blockIdx.y; i < X.Hkv * D; i += kThreads * gridDim.y) {
        const int h = i / D, c = i % D;
        elem_t x[kTokens];
        const int off = slot & (kTokens - 1);      // runs of more than one token in front of an aligned index start inside a group
#pragma unroll
        for (int j = 0; j < kTokens; ++j) x[j] = (j >= off && j - off < run.count) ? v[(run.first + j - off) * X.v_stride + i] : 0;
        elem_t *to = reinterpret_cast<elem_t *>(kv.v) + ((((long long)page * X.Hkv + h) << kv.page_log) * D);
#pragma unroll
        for (int g = 0; g < kTokens / E; ++g) {
            elem_t *at = to + ((long long)((slot - off) / E + g) * D + c) * E;
            const int a = max(off - g * E, 0), b = min(off + run.count - g * E, E);
            if (a == 0 && b == E) {
                uint32_t w[4];
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if constexpr (E == 8) w[m] = (uint32_t)x[g * E + 2 * m] | ((uint32_t)x[g * E + 2 * m + 1] << 16);
                    else w[m] = x[g * E + m];
                }
                *reinterpret_cast<uint4 *>(at) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e >= a && e < b) at[e] = x[g * E + e];
            }
        }
    }
}

// Backward.  Weight gradients: a thread sums fewer than 2 kChain rows in fp32 (40 with 40 heads of 64 bf16 channels); these sums, the lanes' and the
// workgroups' are added in fp64, all in a fixed order, so results do not change from run to run.  LONG: threads have more rows than that and add up in between, which
// costs registers (8000 fp32 tokens of 20 heads, d = 128, forward and backward: 92.2 us with LONG, 89.9 without).
constexpr int kRunsEach = 4, kChain = 64;

template <typename IO, int D, bool LONG>
__global__ __launch_bounds__(kThreads) void k_heads_backward(HeadParams P, HeadRows X, HeadRows Y, const int *positions, uint4 *gq, uint4 *gk, double *partial, bool stream) {
    constexpr int E = IO::E, LANES = D / E, ROWS = kThreads / LANES;
    __shared__ float2 turns[kTokens][kMostHalf];
    __shared__ int pos[kTokens];
    __shared__ float weights[2][D];
    __shared__ double sums[kThreads / 64][2][D];
    for (int i = threadIdx.x; i < D; i += kThreads) {
        weights[0][i] = P.wq ? P.wq[i] : 1.f;
        weights[1][i] = P.wk ? P.wk[i] : 1.f;
    }
    float part[2][E];
#pragma unroll
    for (int e = 0; e < E; ++e) part[0][e] = part[1][e] = 0.f;
    if constexpr (LONG)
        for (int i = threadIdx.x & 63; i < 2 * D; i += 64) (&sums[threadIdx.x >> 6][0][0])[i] = 0.0;   // a wave's own
    const uint4 *xq = reinterpret_cast<const uint4 *>(X.q), *xk = reinterpret_cast<const uint4 *>(X.k);
    const uint4 *yq = reinterpret_cast<const uint4 *>(Y.q), *yk = reinterpret_cast<const uint4 *>(Y.k);
    const int heads = X.H + X.Hkv, token = (threadIdx.x / LANES) & (kTokens - 1), lane = threadIdx.x % LANES;
    constexpr int step = ROWS / kTokens;
    const int first = (threadIdx.x / LANES) / kTokens;
    int held = 0;                                   // rows in `part`
    // the lanes of a wave that hold the same channels; the waves come last
    auto add_up = [&]() {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                double s = part[n][e];
                part[n][e] = 0.f;
#pragma unroll
                for (int m = LANES; m < 64; m <<= 1) s += __shfl_xor(s, m, 64);
                double &sum = sums[threadIdx.x >> 6][n][lane * E + e];
                if ((threadIdx.x & 63) < LANES) sum = LONG ? sum + s : s;
            }
    };
    for (int t0 = blockIdx.x * kTokens; t0 < X.T; t0 += gridDim.x * kTokens) {
        const int count = min(kTokens, X.T - t0);
        const bool there = token < count;
        const long long t = t0 + token;
        uint4 rx, ry, nx, ny;                       // this row, and the next one on its way; two at a time cost registers, and with them waves: 122 instead of 108 us
        auto request = [&](int h, uint4 &x, uint4 &y) {
            x = y = make_uint4(0, 0, 0, 0);
            if (there && h < heads) {
                x = h < X.H ? xq[(t * X.q_stride + h * D) / E + lane] : xk[(t * X.k_stride + (h - X.H) * D) / E + lane];
                y = h < X.H ? yq[(t * Y.q_stride + h * D) / E + lane] : yk[(t * Y.k_stride + (h - X.H) * D) / E + lane];
            }
        };
        request(first, rx, ry);                     // on their way while the angles are formed
        __syncthreads();                            // the run before has read `turns`
        if (threadIdx.x < count) pos[threadIdx.x] = positions ? positions[t0 + threadIdx.x] : t0 + (int)threadIdx.x;
        __syncthreads();
        fill_turns(P, pos, count, turns);
        __syncthreads();
        Lane<IO, D> L;
        L.set(P, turns[there ? token : 0], -1.f);
        for (int h0 = 0; h0 == 0 || (LONG && h0 < heads); h0 += kChain * step) {
            const int end = LONG ? min(heads, h0 + kChain * step) : heads;
            for (int h = first + h0; h - first < end; h += step) {
                request(h + step, nx, ny);
                const bool key = h >= X.H;
                float y[E], z[E], g[E], x[E];
                IO::unpack(ry, y);
                if (P.half) {
                    const uint4 other = P.interleaved ? ry : shuffle(ry, L.partner);
                    IO::unpack(other, z);
                    L.turn(P, y, z, g);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) g[e] = y[e];
                }
                if (P.wq) {
                    IO::unpack(rx, x);
                    const float *w = weights[key] + lane * E;
                    float sq = 0.f, dot = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        sq += x[e] * x[e];
                        dot += g[e] * w[e] * x[e];
                    }
                    // a row that only pads adds nothing: without an epsilon its root would be infinite, and its sums NaN
                    const float rms = rsqrtf(row_sum<LANES>(sq) * (1.f / D) + P.eps), r = there && h < heads ? rms : 0.f;
                    const float m = row_sum<LANES>(dot) * r * (1.f / D);          // mean(h r x)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float xh = x[e] * r, gx = g[e] * xh;
                        if (key) part[1][e] += gx;
                        else part[0][e] += gx;
                        g[e] = r * (g[e] * w[e] - xh * m);
                    }
                }
                if (there && !key) put(&gq[(t * X.H + h) * LANES + lane], IO::pack(g), stream);
                else if (there && h < heads) put(&gk[(t * X.Hkv + h - X.H) * LANES + lane], IO::pack(g), stream);
                rx = nx;
                ry = ny;
            }
            if constexpr (LONG) {
                held += (end - h0 + step - 1) / step;
                if (P.wq && held >= kChain) {
                    add_up();
                    held = 0;
                }
            }
        }
    }
    if (!P.wq) return;
    add_up();
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) s += (&sums[w][0][0])[i];
        partial[(long long)blockIdx.x * 2 * D + i] = s;
    }
}

// Eight channels a workgroup, 32 threads each.
template <int D>
__global__ __launch_bounds__(256) void k_heads_weights(const double *partial, int blocks, float *gwq, float *gwk) {
    __shared__ double sums[32][8];
    const int c = threadIdx.x & 7, part = threadIdx.x >> 3, i = blockIdx.x * 8 + c;
    double s = 0.0;
#pragma unroll 8
    for (int b = part; b < blocks; b += 32) s += partial[(long long)b * 2 * D + i];
    sums[part][c] = s;
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int p = 1; p < 32; ++p) s += sums[p][c];
    if (i < D) gwq[i] = (float)s;
    else gwk[i - D] = (float)s;
}

// A run's heads are divided among workgroups while there are few of those: 3700 fp32 tokens of 16 heads, d = 128, 19.6 instead of 23.4 us.
int head_parts(int blocks) {
    const int parts = 2048 / (blocks > 0 ? blocks : 1);
    return parts < 1 ? 1 : parts > 4 ? 4 : parts;
}

bool streams(const HeadRows &x, int d, int io) { return (size_t)x.T * (x.H + x.Hkv) * d * (io == SPECTRE_BF16 ? 2 : 4) > kL2Bytes; }

HeadParams params(const spectre_heads &P) {
    HeadParams p;
    p.freq = P.inv_freq; p.wq = P.wq; p.wk = P.wk; p.eps = P.eps; p.half = P.rot / 2; p.interleaved = P.interleaved;
    return p;
}

}  // namespace

hipError_t load_kernels_heads() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, reinterpret_cast<const void *>(k_heads_weights<64>));
}

#define SPECTRE_HEADS_DISPATCH(CALL)                                  \
    if (io == SPECTRE_BF16 && P.d == 64) { CALL(Bf16Group, 64); }     \
    else if (io == SPECTRE_BF16) { CALL(Bf16Group, 128); }            \
    else if (P.d == 64) { CALL(F32Group, 64); }                       \
    else { CALL(F32Group, 128); }

hipError_t launch_heads_forward(const spectre_heads &P, int io, const HeadRows &x, const int *positions, void *q_out, void *k_out, hipStream_t st) {
    const int blocks = (x.T + kTokens - 1) / kTokens;
#define CALL(IO, D) k_heads<IO, D, false><<<dim3(blocks, head_parts(blocks)), kThreads, 0, st>>>(params(P), x, positions, (uint4 *)q_out, (uint4 *)k_out, KvView{}, nullptr, nullptr, 0, streams(x, P.d, io))
    SPECTRE_HEADS_DISPATCH(CALL)
#undef CALL
    return hipGetLastError();
}

hipError_t launch_heads_append(const spectre_heads &P, int io, const HeadRows &x, const KvView &kv, const int *start, const int *seqs, int B, void *q_out, hipStream_t st) {
    const int blocks = x.T / kTokens + 2 * B;
#define CALL(IO, D) k_heads<IO, D, true><<<dim3(blocks, head_parts(blocks)), kThreads, 0, st>>>(params(P), x, nullptr, (uint4 *)q_out, nullptr, kv, start, seqs, B, false)
    SPECTRE_HEADS_DISPATCH(CALL)
#undef CALL
    return hipGetLastError();
}

// One run a workgroup up to four workgroups a compute unit, then up to kRunsEach.
int heads_backward_blocks(int T) {
    const int runs = (T + kTokens - 1) / kTokens, most = (runs + kRunsEach - 1) / kRunsEach;
    return runs < 1024 ? runs : most > 1024 ? most : 1024;
}

hipError_t launch_heads_backward(const spectre_heads &P, int io, const HeadRows &x, const HeadRows &dy, const int *positions, void *gq, void *gk, float *gwq, float *gwk,
                                 double *partial, hipStream_t st) {
    const int blocks = heads_backward_blocks(x.T), lanes = P.d / (io == SPECTRE_BF16 ? 8 : 4), step = kThreads / lanes / kTokens;
    const long long runs = blocks ? ((x.T + kTokens - 1) / kTokens + blocks - 1) / blocks : 0;             // of a workgroup
    const bool many = P.wq && runs * ((x.H + x.Hkv + step - 1) / step) >= 2 * kChain;
#define CALL(IO, D)                                                                                                              \
    if (blocks && many) k_heads_backward<IO, D, true><<<blocks, kThreads, 0, st>>>(params(P), x, dy, positions, (uint4 *)gq, (uint4 *)gk, partial, streams(x, P.d, io)); \
    else if (blocks) k_heads_backward<IO, D, false><<<blocks, kThreads, 0, st>>>(params(P), x, dy, positions, (uint4 *)gq, (uint4 *)gk, partial, streams(x, P.d, io)); \
    if (P.wq) k_heads_weights<D><<<2 * D / 8, 256, 0, st>>>(partial, blocks, gwq, gwk)
    SPECTRE_HEADS_DISPATCH(CALL)
#undef CALL
    return hipGetLastError();
}

}  // namespace spectre
