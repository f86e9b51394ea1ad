// Norms of query and key heads with the rotation by their position, in one pass: training forms (forward, backward) and the serving form
// that writes keys and values into their pages.
//
// Per row x of d channels: r = (mean x^2 + eps)^-1/2, y = w r x, and each pair (a, b) of y turned by the angle pos * f_i:
// (a cos - b sin, b cos + a sin).  Backward with g = the output's gradient turned back: g_w = sum g r x over rows, h = g w,
// g_x = r (h - r x mean(h r x)).  Rows are read and written once; memory bounds the long calls, the launch the short ones.  32768 tokens of 32 + 8 bf16 heads, d = 64:
// forward 68 to 75 us by the machine (336 MB, 4.5 to 4.9 TB/s), backward 98 to 108 (503 MB, 4.7 to 5.1 TB/s, the sums of the weights' gradients in it), the two in turn 158 to 166,
// against 5.2 TB/s of a large copy; 8192 tokens into pages 22 us (4.6 TB/s); one token 5.  24000 tokens of three axes, forward and backward 120 us (614 MB, 5.1 TB/s); 6126 of 16 + 4
// heads, d = 128, three axes, adjacent pairs, into pages 15.6 us (75 MB, 4.8 TB/s).
#include "heads_dev.h"

namespace spectre {
namespace {

constexpr int kTokens = 8;                      // a workgroup: one 16-byte group of V pages, two in fp32

template <typename IO, int D, bool SERVE, bool AXES, int TURN>
__global__ __launch_bounds__(kThreads) void k_heads(HeadParams P, HeadRows X, const int *positions, uint4 *q_out, uint4 *k_out, KvView kv, const int *start, const int *seqs,
                                                    int B, bool stream) {
    constexpr int E = IO::E, LANES = D / E, ROWS = kThreads / LANES;
    __shared__ float2 turns[kTokens][kMostHalf];
    __shared__ int pos[kAxesOf<AXES>][kTokens];
    __shared__ float weights[2][D];
    Run run{(int)blockIdx.x * kTokens, min(kTokens, X.T - (int)blockIdx.x * kTokens), 0, 0};
    if (SERVE && !find_run<kTokens>(kv, start, seqs, B, X.T, blockIdx.x, &run)) return;
    const FirstTurn first_angle = first_turn<AXES>(P);
    fill_positions<AXES, kTokens>(P, SERVE && !AXES ? nullptr : positions, X.T, run.first, SERVE ? run.index : run.first, run.count, pos);
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
    fill_turns<AXES, true>(P, first_angle, pos, run.count, turns);
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
            const uint4 o = head_row<IO, D, TURN>(P, L, P.wq ? weights[key] : nullptr, raw[i]);
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

template <typename IO, int D, bool LONG, bool AXES, int TURN>
__global__ __launch_bounds__(kThreads) void k_heads_backward(HeadParams P, HeadRows X, HeadRows Y, const int *positions, uint4 *gq, uint4 *gk, double *partial, bool stream) {
    constexpr int E = IO::E, LANES = D / E, ROWS = kThreads / LANES;
    __shared__ float2 turns[kTokens][kMostHalf];
    __shared__ int pos[kAxesOf<AXES>][kTokens];
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
        fill_positions<AXES, kTokens>(P, positions, X.T, t0, t0, count, pos);
        __syncthreads();
        fill_turns<AXES, false>(P, FirstTurn{}, pos, count, turns);
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
                if (TURN != kAnyTurn || P.half) {
                    if constexpr (TURN != kPairs) {
                        const uint4 other = TURN == kAnyTurn && P.interleaved ? ry : shuffle(ry, L.partner);
                        IO::unpack(other, z);
                    }
                    L.template turn<TURN>(P, y, z, g);
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

}  // namespace

hipError_t load_kernels_heads() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, reinterpret_cast<const void *>(k_heads_weights<64>));
}

#define BY_TURN(LAUNCH, KERNEL, ...)                                                   \
    (turn_of(P) == kHalves  ? LAUNCH(KERNEL<__VA_ARGS__, kHalves>)                     \
     : turn_of(P) == kPairs ? LAUNCH(KERNEL<__VA_ARGS__, kPairs>)                      \
                            : LAUNCH(KERNEL<__VA_ARGS__, kAnyTurn>))
#define SPECTRE_HEADS_DISPATCH(CALL)                                  \
    if (io == SPECTRE_BF16 && P.d == 64) { CALL(Bf16Group, 64); }     \
    else if (io == SPECTRE_BF16) { CALL(Bf16Group, 128); }            \
    else if (P.d == 64) { CALL(F32Group, 64); }                       \
    else { CALL(F32Group, 128); }

hipError_t launch_heads_forward(const spectre_heads &P, int io, const HeadRows &x, const int *positions, void *q_out, void *k_out, hipStream_t st) {
    const int blocks = (x.T + kTokens - 1) / kTokens;
    auto launch = [&](auto kernel) {
        kernel<<<dim3(blocks, head_parts(blocks)), kThreads, 0, st>>>(head_params(P), x, positions, (uint4 *)q_out, (uint4 *)k_out, KvView{}, nullptr, nullptr, 0, streams(x, P.d, io));
    };
#define CALL(IO, D)                                                  \
    if (P.axes > 1 && positions) BY_TURN(launch, k_heads, IO, D, false, true); \
    else BY_TURN(launch, k_heads, IO, D, false, false)
    SPECTRE_HEADS_DISPATCH(CALL)
#undef CALL
    return hipGetLastError();
}

hipError_t launch_heads_append(const spectre_heads &P, int io, const HeadRows &x, const KvView &kv, const int *positions, const int *start, const int *seqs, int B, void *q_out,
                               hipStream_t st) {
    const int blocks = x.T / kTokens + 2 * B;
    auto launch = [&](auto kernel) {
        kernel<<<dim3(blocks, head_parts(blocks)), kThreads, 0, st>>>(head_params(P), x, positions, (uint4 *)q_out, nullptr, kv, start, seqs, B, false);
    };
#define CALL(IO, D)                                                  \
    if (positions) BY_TURN(launch, k_heads, IO, D, true, true);      \
    else BY_TURN(launch, k_heads, IO, D, true, false)
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
    auto launch = [&](auto kernel) {
        if (blocks) kernel<<<blocks, kThreads, 0, st>>>(head_params(P), x, dy, positions, (uint4 *)gq, (uint4 *)gk, partial, streams(x, P.d, io));
    };
#define CALL(IO, D)                                                              \
    if (P.axes > 1 && positions && many) BY_TURN(launch, k_heads_backward, IO, D, true, true);  \
    else if (P.axes > 1 && positions) BY_TURN(launch, k_heads_backward, IO, D, false, true);    \
    else if (many) BY_TURN(launch, k_heads_backward, IO, D, true, false);        \
    else BY_TURN(launch, k_heads_backward, IO, D, false, false);                 \
    if (P.wq) k_heads_weights<D><<<2 * D / 8, 256, 0, st>>>(partial, blocks, gwq, gwk)
    SPECTRE_HEADS_DISPATCH(CALL)
#undef CALL
    return hipGetLastError();
}

}  // namespace spectre
