// A residual's addition and the root-mean-square norm of the sum, in one pass: s = x + delta, y = w s (mean s^2 + eps)^-1/2, y in the rows' type or in 8 bits with a
// scale for each 128 channels.  Backward, with g = dL/dy and e = dL/ds from the residual's path: u = s r, h = g w, dL/dx = dL/ddelta = r (h - u mean(h u)) + e,
// dL/dw = sum over rows of g u.
//
// s is rounded to the rows' type where it is stored, and the norm is of what is stored: the backward pass, which reads it, finds the same numbers.
//
// Memory bounds the long calls, the launch the short ones.  16384 rows of 2048 bf16 channels: forward 49 to 51 us (268 MB, 5.4 TB/s), backward 50 to 52 (268 MB) and 5 for the weights'
// gradient; 12001 rows of 4096 in 8 bits 57 us (346 MB, 6.0 TB/s); one row 2.  Rows of more than 1024 groups of 16 bytes (two a thread) hold their weights and the sums of
// the weights' gradient beside each other, 45 registers more than there are: 2048 rows of 16384 bf16 channels, backward, 120 us with that gradient, 51 without; rows of 8192 56.
#include <math.h>

#include <algorithm>

#include "e4m3.h"
#include "heads_dev.h"
#include "norm.h"

namespace spectre {
namespace {

__device__ __forceinline__ float wave_sum(float x) {
    x = row_sum<16>(x);
    typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
    const u32x2_t a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const u32x2_t b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }     // NaN if one is
template <int LANES>
__device__ __forceinline__ float row_largest(float x) {
    x = larger(x, dpp<0xB1>(x));
    x = larger(x, dpp<0x4E>(x));
    x = larger(x, dpp<0x141>(x));
    x = larger(x, dpp<0x140>(x));
    if constexpr (LANES == 32) {
        typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
        const u32x2_t a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = larger(__uint_as_float(a[0]), __uint_as_float(a[1]));
    }
    return x;
}

// A row's threads are a wave, of which a workgroup has four, or the workgroup.
template <int LANES>
constexpr int kGroupThreads = LANES > 256 ? LANES : 256;

// Sums over the LANES threads of a row, in all of them; `sums` of the workgroup's waves, turn: 0 and 1 from row to row, so that one barrier does.
template <int LANES, int N>
__device__ __forceinline__ void sum_row(float (&x)[N], float (*sums)[kGroupThreads<LANES> / 64][N], int turn) {
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = wave_sum(x[n]);
    if constexpr (LANES > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) sums[turn][wave][n] = x[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            x[n] = sums[turn][0][n];
#pragma unroll
            for (int w = 1; w < LANES / 64; ++w) x[n] += sums[turn][w][n];
        }
    }
}

template <typename IO>
__device__ __forceinline__ void load_weights(const float *w, long long at, bool there, float (&y)[IO::E]) {
#pragma unroll
    for (int e = 0; e < IO::E; e += 4) {
        const float4 f = w && there ? *reinterpret_cast<const float4 *>(w + at + e) : make_float4(1.f, 1.f, 1.f, 1.f);
        y[e] = f.x; y[e + 1] = f.y; y[e + 2] = f.z; y[e + 3] = f.w;
    }
}

// LANES threads have a row (a wave, or the workgroup), CHUNKS groups of 16 bytes each; a workgroup goes through rows a grid apart, the next row on its way.
template <typename IO, int LANES, int CHUNKS, bool CODED>
__global__ __launch_bounds__((kGroupThreads<LANES>)) void k_norm(NormRows N, uint4 *sum, void *out, float *scales, bool stream) {
    constexpr int E = IO::E, ROWS = kGroupThreads<LANES> / LANES, GROUP = kNormGroup / E;
    __shared__ float sums[2][kGroupThreads<LANES> / 64][1];
    const int lane = threadIdx.x % LANES, groups = N.D / E;
    const float inv_d = 1.f / (float)N.D;
    float w[CHUNKS][E];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) load_weights<IO>(N.w, (long long)(lane + LANES * c) * E, lane + LANES * c < groups, w[c]);
    const uint4 *x = reinterpret_cast<const uint4 *>(N.x), *delta = reinterpret_cast<const uint4 *>(N.delta);
    uint4 xr[CHUNKS], dr[CHUNKS];
    auto request = [&](long long row) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int g = lane + LANES * c;
            xr[c] = dr[c] = make_uint4(0, 0, 0, 0);
            if (row < N.T && g < groups) {
                xr[c] = x[row * (N.x_stride / E) + g];
                if (delta) dr[c] = delta[row * (N.delta_stride / E) + g];
            }
        }
    };
    const long long step = (long long)gridDim.x * ROWS;
    int turn = 0;
    request((long long)blockIdx.x * ROWS + threadIdx.x / LANES);
    for (long long first = (long long)blockIdx.x * ROWS; first < N.T; first += step, turn ^= 1) {
        const long long row = first + threadIdx.x / LANES;
        const bool there = row < N.T;
        float s[CHUNKS][E], sq[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float d[E];
            IO::unpack(xr[c], s[c]);
            if (delta) {
                IO::unpack(dr[c], d);
#pragma unroll
                for (int e = 0; e < E; ++e) s[c][e] += d[e];
                const uint4 kept = IO::pack(s[c]);
                if (there && lane + LANES * c < groups) put(&sum[row * groups + lane + LANES * c], kept, stream);
                IO::unpack(kept, s[c]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) sq[0] += s[c][e] * s[c][e];
        }
        request(row + step);
        sum_row<LANES, 1>(sq, sums, turn);
        const float r = rsqrtf(sq[0] * inv_d + N.eps);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int g = lane + LANES * c;
#pragma unroll
            for (int e = 0; e < E; ++e) s[c][e] = s[c][e] * r * w[c][e];
            if constexpr (!CODED) {
                if (there && g < groups) put(&reinterpret_cast<uint4 *>(out)[row * groups + g], IO::pack(s[c]), stream);
            } else {
                // GROUP lanes hold the channels of a scale: all of them have groups of the row, or none
                float most = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) most = larger(most, fabsf(s[c][e]));
                most = row_largest<GROUP>(most);
                float scale = most * (1.f / kE4m3Most), inv = kE4m3Most / most;
                if (scale < 0x1p-126f) scale = inv = 0.f;                      // nothing, or next to nothing: codes of zero
                if (!there || g >= groups) continue;
                if (lane % GROUP == 0) scales[row * (N.D / kNormGroup) + g / GROUP] = scale;
                uint32_t code[E / 4];
#pragma unroll
                for (int e = 0; e < E; e += 4) code[e / 4] = e4m3_encode4(s[c][e] * inv, s[c][e + 1] * inv, s[c][e + 2] * inv, s[c][e + 3] * inv, 1.f);
                if constexpr (E == 8) reinterpret_cast<uint2 *>(out)[row * groups + g] = make_uint2(code[0], code[1]);
                else reinterpret_cast<uint32_t *>(out)[row * groups + g] = code[0];
            }
        }
    }
}

// A workgroup's sums of the weights' gradient are in 32 bits (at most kNormChain rows); k_norm_weights adds the workgroups' in 64.
template <typename IO, int LANES, int CHUNKS, bool WEIGHTS>
__global__ __launch_bounds__((kGroupThreads<LANES>)) void k_norm_backward(NormRows N, NormGrads G, uint4 *gx, float *partial, bool stream) {
    constexpr int E = IO::E, ROWS = kGroupThreads<LANES> / LANES;
    __shared__ float sums[2][kGroupThreads<LANES> / 64][2];
    const int lane = threadIdx.x % LANES, groups = N.D / E;
    const float inv_d = 1.f / (float)N.D;
    float w[CHUNKS][E], gw[CHUNKS][E];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        load_weights<IO>(N.w, (long long)(lane + LANES * c) * E, lane + LANES * c < groups, w[c]);
#pragma unroll
        for (int e = 0; e < E; ++e) gw[c][e] = 0.f;
    }
    const uint4 *x = reinterpret_cast<const uint4 *>(N.x), *dy = reinterpret_cast<const uint4 *>(G.dy), *dsum = reinterpret_cast<const uint4 *>(G.dsum);
    uint4 xr[CHUNKS], yr[CHUNKS], sr[CHUNKS];
    auto request = [&](long long row) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int g = lane + LANES * c;
            xr[c] = yr[c] = sr[c] = make_uint4(0, 0, 0, 0);
            if (row < N.T && g < groups) {
                xr[c] = x[row * (N.x_stride / E) + g];
                yr[c] = dy[row * (G.dy_stride / E) + g];
                if (dsum) sr[c] = dsum[row * (G.dsum_stride / E) + g];
            }
        }
    };
    const long long step = (long long)gridDim.x * ROWS;
    int turn = 0;
    request((long long)blockIdx.x * ROWS + threadIdx.x / LANES);
    for (long long first = (long long)blockIdx.x * ROWS; first < N.T; first += step, turn ^= 1) {
        const long long row = first + threadIdx.x / LANES;
        const bool there = row < N.T;
        uint4 xs[CHUNKS], ys[CHUNKS], ss[CHUNKS];
        float both[2] = {0.f, 0.f};                                            // sum s^2, sum h s
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            xs[c] = xr[c]; ys[c] = yr[c]; ss[c] = sr[c];
            float s[E], g[E];
            IO::unpack(xs[c], s);
            IO::unpack(ys[c], g);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                both[0] += s[e] * s[e];
                both[1] += g[e] * w[c][e] * s[e];
            }
        }
        request(row + step);
        sum_row<LANES, 2>(both, sums, turn);
        const float r = there ? rsqrtf(both[0] * inv_d + N.eps) : 0.f, m = both[1] * r * inv_d;      // m = mean(h u); rows behind the last add nothing
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float s[E], g[E], d[E];
            IO::unpack(xs[c], s);
            IO::unpack(ys[c], g);
            if (dsum) IO::unpack(ss[c], d);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float u = s[e] * r;
                if (WEIGHTS) gw[c][e] += g[e] * u;
                g[e] = r * (g[e] * w[c][e] - u * m);
                if (dsum) g[e] += d[e];
            }
            if (there && lane + LANES * c < groups) put(&gx[row * groups + lane + LANES * c], IO::pack(g), stream);
        }
    }
    if constexpr (WEIGHTS) {
        if constexpr (ROWS > 1) {                                              // the workgroup's waves, in their order
            __shared__ float others[ROWS - 1][LANES * CHUNKS * E];
            const int slot = threadIdx.x / LANES;
            if (slot > 0)
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int e = 0; e < E; ++e) others[slot - 1][(c * E + e) * LANES + lane] = gw[c][e];
            __syncthreads();
            if (slot > 0) return;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e)
#pragma unroll
                    for (int o = 0; o < ROWS - 1; ++o) gw[c][e] += others[o][(c * E + e) * LANES + lane];
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (lane + LANES * c < groups) {
                float *to = partial + (long long)blockIdx.x * N.D + (long long)(lane + LANES * c) * E;
#pragma unroll
                for (int e = 0; e < E; e += 4) *reinterpret_cast<float4 *>(to + e) = make_float4(gw[c][e], gw[c][e + 1], gw[c][e + 2], gw[c][e + 3]);
            }
    }
}

// Sixteen channels a workgroup, sixteen threads each, in a fixed order.
__global__ __launch_bounds__(256) void k_norm_weights(const float *partial, int rows, int D, float *gw) {
    __shared__ double sums[16][16];
    const int c = threadIdx.x & 15, part = threadIdx.x >> 4, i = blockIdx.x * 16 + c;
    double s = 0.0;
    if (i < D) {
#pragma unroll 8
        for (int r = part; r < rows; r += 16) s += partial[(long long)r * D + i];
    }
    sums[part][c] = s;
    __syncthreads();
    if (part || i >= D) return;
#pragma unroll
    for (int p = 1; p < 16; ++p) s += sums[p][c];
    gw[i] = (float)s;
}

// Threads of a row: a wave while that leaves each no more than two groups, then as many as it has groups, up to 1024.
int row_threads(int groups) { return groups <= 128 ? 64 : groups <= 256 ? 256 : groups <= 512 ? 512 : 1024; }
int group_threads(int groups) { return std::max(256, row_threads(groups)); }
int row_slots(int groups) { return group_threads(groups) / row_threads(groups); }

}  // namespace

hipError_t load_kernels_norm() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, reinterpret_cast<const void *>(k_norm_weights));
}

#define SPECTRE_NORM_CHUNKS(IO, CALL)                                              \
    if (groups <= 64) CALL(IO, 64, 1);                                             \
    else if (groups <= 128) CALL(IO, 64, 2);                                       \
    else if (groups <= 256) CALL(IO, 256, 1);                                      \
    else if (groups <= 512) CALL(IO, 512, 1);                                      \
    else if (groups <= 1024) CALL(IO, 1024, 1);                                    \
    else CALL(IO, 1024, 2)

hipError_t launch_norm(const NormRows &n, int io, void *sum, void *y, float *scales, hipStream_t st) {
    const int size = io == SPECTRE_BF16 ? 2 : 4, groups = n.D * size / 16, slots = row_slots(groups);
    const int blocks = (int)std::min<long long>(((long long)n.T + slots - 1) / slots, 2048 * 256 / group_threads(groups));
    const bool stream = (size_t)n.T * n.D * size > kL2Bytes;
    auto launch = [&](auto kernel) { kernel<<<blocks, group_threads(groups), 0, st>>>(n, (uint4 *)sum, y, scales, stream); };
#define CALL(IO, LANES, CHUNKS) (scales ? launch(k_norm<IO, LANES, CHUNKS, true>) : launch(k_norm<IO, LANES, CHUNKS, false>))
    if (io == SPECTRE_BF16) { SPECTRE_NORM_CHUNKS(Bf16Group, CALL); }
    else { SPECTRE_NORM_CHUNKS(F32Group, CALL); }
#undef CALL
    return hipGetLastError();
}

// 16 waves a compute unit, more workgroups where each would have more than kNormChain rows.  (Half of them: 16384 rows of 2048 bf16 channels, forward and backward, 105.6
// instead of 108.2 us, but 5000 of 8192 151 instead of 124.)
int norm_backward_blocks(int T, int groups, bool weights) {
    const int slots = row_slots(groups);
    if (T == 0) return 0;
    // one workgroup, whose sums are the weights' gradient: no other launch (8 rows of 2048, forward and backward, 19.4 us; 9 rows, with it, 24.1).  Without
    // that gradient there is none to save: 8 rows of 16384 7.9 us, by one workgroup 17.2
    if (weights && T <= 8 * slots) return 1;
    const long long most = std::max(1024ll * 256 / group_threads(groups), ((long long)T + kNormChain - 1) / kNormChain);
    return (int)std::min<long long>(((long long)T + slots - 1) / slots, most);
}

hipError_t launch_norm_backward(const NormRows &n, const NormGrads &g, int io, void *gx, float *gw, float *partial, hipStream_t st) {
    const int size = io == SPECTRE_BF16 ? 2 : 4, groups = n.D * size / 16, blocks = norm_backward_blocks(n.T, groups, gw != nullptr);
    const bool stream = (size_t)n.T * n.D * size > kL2Bytes;
    auto launch = [&](auto kernel) { kernel<<<blocks, group_threads(groups), 0, st>>>(n, g, (uint4 *)gx, blocks == 1 ? gw : partial, stream); };
#define CALL(IO, LANES, CHUNKS) (gw ? launch(k_norm_backward<IO, LANES, CHUNKS, true>) : launch(k_norm_backward<IO, LANES, CHUNKS, false>))
    if (n.T > 0) {
        if (io == SPECTRE_BF16) { SPECTRE_NORM_CHUNKS(Bf16Group, CALL); }
        else { SPECTRE_NORM_CHUNKS(F32Group, CALL); }
    }
#undef CALL
    if (gw && blocks != 1) k_norm_weights<<<(n.D + 15) / 16, 256, 0, st>>>(partial, n.T > 0 ? blocks : 0, n.D, gw);
    return hipGetLastError();
}

}  // namespace spectre
