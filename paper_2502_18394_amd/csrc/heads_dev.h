// What the kernels that norm and rotate heads share: rows in 16-byte groups, angles, the norm of a row, places of new tokens.
#pragma once
#include <math.h>

#include "common.h"
#include "paged.h"

namespace spectre {

constexpr int kThreads = 256;
constexpr int kMostHalf = 64;                   // pairs of a row of 128 channels
constexpr int kMostAxes = SPECTRE_HEADS_MAX_AXES;

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
    int axes;                       // positions of a token
    const int *axis;                // of each pair, null: one axis
};
inline HeadParams head_params(const spectre_heads &P) {
    HeadParams p;
    p.freq = P.inv_freq; p.wq = P.wq; p.wk = P.wk; p.eps = P.eps; p.half = P.rot / 2; p.interleaved = P.interleaved;
    p.axes = P.axes > 1 ? P.axes : 1;
    p.axis = P.axes > 1 ? P.axis : nullptr;
    return p;
}

// Positions of a workgroup's `count` tokens from `first` on: given, [axes][T], or (null) from `from` on one after the other.  Kernels have AXES where there may be several
// axes, as forms of their own: with one axis it would cost registers (backward, and with them waves) and 4 % of the time of 19 sequences' turns into pages.
template <bool AXES, int TOKENS>
__device__ __forceinline__ void fill_positions(const HeadParams &P, const int *positions, int T, int first, int from, int count, int (*pos)[TOKENS]) {
    if constexpr (AXES) {
        for (int i = threadIdx.x; i < TOKENS * P.axes; i += kThreads) {
            const int a = i / TOKENS, t = i % TOKENS;
            if (t < count) pos[a][t] = positions[(long long)a * T + first + t];
        }
    } else if (threadIdx.x < count) {
        pos[0][threadIdx.x] = positions ? positions[first + threadIdx.x] : from + (int)threadIdx.x;
    }
}
template <bool AXES>
constexpr int kAxesOf = AXES ? kMostAxes : 1;

// cos and sin of the angles of a workgroup's tokens, one pair a thread.  The turns pos * f / 2 pi are formed and reduced in 64 bits: a position of
// 131072 leaves 32 bits with an angle that is wrong in the third digit.
// EARLY: what a thread's first angle needs is asked for before the positions are there, and serves all its angles where a row's pairs divide the threads (24000
// tokens of three axes, forward and backward: 123.4 instead of 126.2 us; 19 sequences' turns 17.8 instead of 18.1).  Not in the backward pass, where it costs registers.
struct FirstTurn {
    double freq;
    int axis;
};
template <bool AXES>
__device__ __forceinline__ FirstTurn first_turn(const HeadParams &P) {
    FirstTurn t{0.0, 0};
    if (P.half) {
        const int f = threadIdx.x % P.half;
        t.freq = P.freq[f];
        if (AXES && P.axis) t.axis = P.axis[f];
    }
    return t;
}
template <bool AXES, bool EARLY, int TOKENS>
__device__ __forceinline__ void fill_turns(const HeadParams &P, FirstTurn first, const int (*pos)[TOKENS], int count, float2 (*turns)[kMostHalf]) {
    for (int i = threadIdx.x; i < count * P.half; i += kThreads) {
        const int t = i / P.half, f = i - t * P.half;
        if (!EARLY || kThreads % P.half) {
            first.freq = P.freq[f];
            if (AXES && P.axis) first.axis = P.axis[f];
        }
        const int a = AXES ? (int)min((unsigned)first.axis, (unsigned)P.axes - 1u) : 0;
        double rev = (double)pos[a][t] * first.freq * 0.15915494309189533577;
        rev -= rint(rev);
        float s, c;
        sincospif((float)(2.0 * rev), &s, &c);
        turns[t][f] = make_float2(c, s);
    }
}

// How rows are turned.  Whole rows have forms of their own, in which nothing is chosen element by element and adjacent pairs do without their partners' lane; the vector
// unit works four fifths of these kernels' time.  6126 tokens of adjacent pairs into pages, d = 128: 15.6 us, in the one form for all 20.9; 24000 of halves, forward and backward, 120 and 124.
enum { kAnyTurn, kHalves, kPairs };
inline int turn_of(const spectre_heads &P) { return P.rot != P.d ? kAnyTurn : P.interleaved ? kPairs : kHalves; }

// a c + b s with one rounding of b s, whatever form it is compiled in: all give the same bits.
__device__ __forceinline__ float turned_sum(float a, float c, float b, float s) {
#pragma clang fp contract(off)
    const float product = b * s;
    return fmaf(a, c, product);
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
    template <int TURN>
    __device__ __forceinline__ void turn(const HeadParams &P, const float (&y)[E], const float (&z)[E], float (&o)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float other = TURN == kPairs ? y[e ^ 1] : TURN == kHalves ? z[e] : P.interleaved ? y[e ^ 1] : z[e];
            const float t = turned_sum(y[e], c[e], other, s[e]);
            o[e] = TURN != kAnyTurn || turned ? t : y[e];
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

// One row's norm and rotation: this lane's channels.
template <typename IO, int D, int TURN>
__device__ __forceinline__ void head_channels(const HeadParams &P, const Lane<IO, D> &L, const float *w, uint4 raw, float (&o)[IO::E]) {
    constexpr int E = IO::E;
    float x[E], z[E];
    IO::unpack(raw, x);
    constexpr bool MATE = TURN != kPairs;             // a partner's channels are looked at
    if constexpr (MATE) {
        const uint4 other = TURN == kHalves || (P.half && !P.interleaved) ? shuffle(raw, L.partner) : raw;
        IO::unpack(other, z);
    }
    if (w) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) sq += x[e] * x[e];
        const float r = rsqrtf(row_sum<D / E>(sq) * (1.f / D) + P.eps);
        const int base = L.lane * E, mate = (L.lane + (L.partner - (int)(threadIdx.x & 63))) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] = x[e] * r * w[base + e];
            if (MATE) z[e] = z[e] * r * w[mate + e];
        }
    }
    if (TURN != kAnyTurn || P.half) L.template turn<TURN>(P, x, z, o);
    else
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = x[e];
}
template <typename IO, int D, int TURN>
__device__ __forceinline__ uint4 head_row(const HeadParams &P, const Lane<IO, D> &L, const float *w, uint4 raw) {
    float o[IO::E];
    head_channels<IO, D, TURN>(P, L, w, raw, o);
    return IO::pack(o);
}

// Place of a workgroup's tokens.  Training: TOKENS tokens from TOKENS * block on.  Serving: the tokens of one sequence that fall into one
// TOKENS-aligned run of cache indexes, so that runs inside a chunk fill whole groups of the V pages.  Sequence b's runs are numbered from
// start[b] / TOKENS + 2 b on: n tokens touch at most n / TOKENS + 2 runs, so no two sequences' numbers meet.
struct Run {
    int first, count;               // tokens
    int index;                      // cache index of the first one
    int seq;                        // its row of the table
};

// Bits of the status that a reserve which could not be done leaves.  Its sequences have not grown, so what would be taken for the new tokens' places holds their last ones:
// nothing is written while a bit stands.
constexpr int kNotReserved = SPECTRE_KV_NO_PAGES | SPECTRE_KV_TOO_LONG | SPECTRE_KV_BAD_ARGUMENT;

template <int TOKENS>
__device__ __forceinline__ bool find_run(const KvView &kv, const int *start, const int *seqs, int B, int T, int block, Run *r) {
    const int status = kv.status[0];
    int lo = 0, hi = B;             // the last b with start[b] / TOKENS + 2 b <= block: 64 asked at once (19 fp32 sequences of up to 700 tokens 18.6 us, by halves 19.0)
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, mid = lo + step * (int)(threadIdx.x & 63);
        const bool behind = mid == lo || (mid < hi && start[mid] / TOKENS + 2 * mid <= block);
        lo += step * (__popcll(__ballot(behind)) - 1);
        hi = min(hi, lo + step);
    }
    const int from = start[lo], to = min(start[lo + 1], T), n = to - from;
    const int row = seqs ? seqs[lo] : lo;
    if ((status & kNotReserved) || from < 0 || n <= 0 || (unsigned)row >= (unsigned)kv.S) return false;
    const int had = kv.lens[row] - n;          // tokens before the new ones
    if (had < 0) return false;
    const int run = block - (from / TOKENS + 2 * lo);
    const int a = max((had / TOKENS + run) * TOKENS, had), b = min((had / TOKENS + run + 1) * TOKENS, had + n);
    if (run < 0 || a >= b) return false;
    r->first = from + (a - had);
    r->count = b - a;
    r->index = a;
    r->seq = row;
    return true;
}

}  // namespace spectre
