// Norm and rotation of new tokens' heads, keys and values into pages of 8 bits.
//
// Each block of 16 tokens of a key head has a scale for its keys and one for its values, a power of two: the smallest s with max |x| <= 448 s over the finite
// ones.  A power of two costs a number of eight bits no accuracy (its spacing goes with its size) and makes growth harmless: tokens that join others in a
// block keep the larger of both scales, and codes of the smaller one are exact under the larger (but for subnormals), so a block that fills
// token by token ends as if it had come at once.  What is coded are the 32-bit results of norm and rotation, rounded once.
//
// A workgroup has the new tokens of one block (they are one sequence's), all or some of the heads: queries as in the other types, then two key
// heads (d = 128: one) at a time: 16 tokens' rows in the threads, their largest magnitudes through the wave and LDS, keys stored eight bytes a lane, values
// turned in LDS into groups of 16 tokens a channel.
//
// What bounds it: for few tokens a chain of loads (sequence, length, page, users, rows), about 5 us, and the launch (one token 5.4 us); for some thousands the vector
// unit, busy in two thirds of the cycles (angles, norm, turn); for many memory.  19 sequences of up to 900 new tokens, 16 + 4 heads, d = 128: 11.2 us (30 MB, 2.7 TB/s); 16384 tokens of
// 32 + 8 heads, d = 64: 40.6 us (185 MB, 4.5 TB/s); 32768: 84 us (4.4 TB/s).
// Measured and not taken: the first key head's rows asked for before the queries are worked on (15.5 instead of 15.1 us), queries and key heads in the same workgroups
// (13.0 instead of 11.2).
#include <algorithm>

#include "e4m3.h"
#include "heads_dev.h"

namespace spectre {
namespace {

typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));

// The largest of a wave's numbers, none of them NaN, in all lanes.
__device__ __forceinline__ float wave_largest(float x) {
    x = fmaxf(x, dpp<0xB1>(x));
    x = fmaxf(x, dpp<0x4E>(x));
    x = fmaxf(x, dpp<0x141>(x));
    x = fmaxf(x, dpp<0x140>(x));
    const u32x2_t a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const u32x2_t b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ float finite_size(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;                   // false for NaN, too
}

// At the largest scale the largest numbers would round to 2^128.
__device__ __forceinline__ void cut(float (&x)[8], float scale) {
    if (scale < kMostScale) return;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (fabsf(x[e]) > kCut && fabsf(x[e]) < INFINITY) x[e] = copysignf(kCut, x[e]);
}

template <int D, bool AXES, int TURN>
__global__ __launch_bounds__(kThreads) void k_append8(HeadParams P, HeadRows X, const int *positions, uint4 *q_out, KvView kv, const int *start, const int *seqs, int B,
                                                       int q_parts) {
    constexpr int TOKENS = kKvBlock, LANES = D / 8, ROWS = kThreads / LANES, HEADS = ROWS / TOKENS, WAVES = LANES * TOKENS / 64;    // key heads at once; waves of each
    constexpr int VROW = D / 4 + D / 16;             // words of a token's coded values in LDS: four tokens on are a quarter or half of the banks on
    __shared__ float2 turns[TOKENS][kMostHalf];
    __shared__ int pos[kAxesOf<AXES>][TOKENS];
    __shared__ float weights[2][D];
    __shared__ float most[kThreads / 64][2];
    __shared__ __align__(16) uint32_t coded[HEADS][TOKENS][VROW];
    Run run;
    if (!find_run<TOKENS>(kv, start, seqs, B, X.T, blockIdx.x, &run)) return;
    const FirstTurn first_angle = first_turn<AXES>(P);
    fill_positions<AXES, TOKENS>(P, AXES ? positions : nullptr, X.T, run.first, run.index, run.count, pos);
    for (int i = threadIdx.x; i < D; i += kThreads) {
        weights[0][i] = P.wq ? P.wq[i] : 1.f;
        weights[1][i] = P.wk ? P.wk[i] : 1.f;
    }
    const int p = run.index >> kv.page_log, slot = run.index & ((1 << kv.page_log) - 1), had = slot & (TOKENS - 1);       // tokens that the block has already
    const int page = p < kv.M ? kv.table[(long long)run.seq * kv.M + p] : -1;
    __syncthreads();
    fill_turns<AXES, true>(P, first_angle, pos, run.count, turns);
    __syncthreads();
    const bool in_pool = (unsigned)page < (unsigned)kv.P;
    const int users = in_pool ? kv.refs[page] : 0;   // a page with several users holds another sequence's tokens, too

    // parts of the heads: the first q_parts have queries, the others key heads; 0: each part has some of both
    const int q_part = blockIdx.y, q_step = q_parts ? q_parts : gridDim.y, k_part = blockIdx.y - q_parts, k_step = gridDim.y - q_parts;
    if (q_part < q_step) {   // queries, in the order (head, token), tokens padded to a power of two, so that a thread stays with one token and one group of channels
        int tl = 0;
        while ((1 << tl) < run.count) ++tl;
        const int token = (threadIdx.x / LANES) & ((1 << tl) - 1), first = (threadIdx.x / LANES) >> tl, step = ROWS >> tl;
        const bool there = token < run.count;
        Lane<Bf16Group, D> L;
        L.set(P, turns[there ? token : 0], 1.f);
        const long long t = run.first + token;
        const uint4 *q = reinterpret_cast<const uint4 *>(X.q);
        constexpr int AHEAD = 4;
        for (int h0 = first + q_part * AHEAD * step; h0 - first < X.H; h0 += AHEAD * step * q_step) {
            uint4 raw[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int h = h0 + i * step;
                raw[i] = make_uint4(0, 0, 0, 0);
                if (there && h < X.H) raw[i] = q[(t * X.q_stride + h * D) / 8 + L.lane];
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int h = h0 + i * step;
                const uint4 o = head_row<Bf16Group, D, TURN>(P, L, P.wq ? weights[0] : nullptr, raw[i]);
                if (there && h < X.H) q_out[(t * X.H + h) * LANES + L.lane] = o;
            }
        }
    }
    if (!in_pool || k_part < 0) return;
    if (users > 1) {
        if (threadIdx.x == 0) atomicOr(&kv.status[0], SPECTRE_KV_SHARED);
        return;
    }

    const int at = (threadIdx.x / LANES) % TOKENS, sub = threadIdx.x / (LANES * TOKENS), wave = threadIdx.x >> 6;     // this thread's token of the block
    const bool there = at >= had && at - had < run.count;
    Lane<Bf16Group, D> L;
    L.set(P, turns[there ? at - had : 0], 1.f);
    const long long t = run.first + at - had;
    const uint4 *k = reinterpret_cast<const uint4 *>(X.k), *v = reinterpret_cast<const uint4 *>(X.v);
    for (int h0 = HEADS * k_part; h0 < X.Hkv; h0 += HEADS * k_step) {
        const int h = h0 + sub;
        const bool mine = h < X.Hkv;
        const long long head = (long long)page * X.Hkv + (mine ? h : 0);
        uint4 kr = make_uint4(0, 0, 0, 0), vr = kr;
        if (there && mine) {
            kr = k[(t * X.k_stride + h * D) / 8 + L.lane];
            vr = v[(t * X.v_stride + h * D) / 8 + L.lane];
        }
        float2 *const scales = reinterpret_cast<float2 *>(kv.scales) + (head << (kv.page_log - kKvBlockLog)) + (slot >> kKvBlockLog);
        uint2 *const keys = reinterpret_cast<uint2 *>((char *)kv.k + (head << kv.page_log) * D + (((L.lane >> 1) << kv.page_log) + slot - had + at) * 16ll) + (L.lane & 1);
        float2 was = make_float2(0.f, 0.f);
        uint2 old = make_uint2(0, 0);
        if (had) {
            was = *scales;
            if (at < had && mine) old = *keys;
        }
        float x[8], y[8];
        head_channels<Bf16Group, D, TURN>(P, L, P.wq ? weights[1] : nullptr, kr, x);
        Bf16Group::unpack(vr, y);
        float mk = 0.f, mv = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mk = fmaxf(mk, there ? finite_size(x[e]) : 0.f);
            mv = fmaxf(mv, finite_size(y[e]));
        }
        mk = wave_largest(mk);
        mv = wave_largest(mv);
        if ((threadIdx.x & 63) == 0) {
            most[wave][0] = mk;
            most[wave][1] = mv;
        }
        asm volatile("s_waitcnt vmcnt(0)" : "+v"(was.x), "+v"(was.y) : : "memory");        // everybody has the block's scales before one thread writes the new ones
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            mk = fmaxf(mk, most[WAVES * sub + w][0]);
            mv = fmaxf(mv, most[WAVES * sub + w][1]);
        }
        const float2 scale = make_float2(fmaxf(e4m3_scale(mk), was.x), fmaxf(e4m3_scale(mv), was.y));
        if (there && mine) {
            cut(x, scale.x);
            cut(y, scale.y);
            *keys = e4m3_encode8(x, scale.x);
            *reinterpret_cast<uint2 *>(&coded[sub][at][2 * L.lane]) = e4m3_encode8(y, scale.y);
        } else if (at < had && mine && scale.x != was.x) {
            *keys = make_uint2(e4m3_rescale4(old.x, was.x, scale.x), e4m3_rescale4(old.y, was.x, scale.x));
        }
        if (mine && at == 0 && L.lane == 0) *scales = scale;
        __syncthreads();
        // values: four channels of four tokens a thread
        const int i = threadIdx.x % (LANES * TOKENS), c = i >> 2, quad = i & 3;
        if (i >= D || !mine) continue;
        const int from = max(0, min(4, had - 4 * quad)), end = max(0, min(4, had + run.count - 4 * quad));               // the new ones of these tokens
        const bool grown = from > 0 && scale.y != was.y;
        if (end <= from && !grown) continue;
        uint32_t w[4], u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = coded[sub][4 * quad + j][c];
        const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);     // channels 0 and 1 of two tokens each
        const uint32_t e = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), f = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);     // 2 and 3
        u[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        u[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        u[2] = __builtin_amdgcn_perm(f, e, 0x05040100u);
        u[3] = __builtin_amdgcn_perm(f, e, 0x07060302u);
        uint32_t *to = reinterpret_cast<uint32_t *>((char *)kv.v + (head << kv.page_log) * D + ((slot >> kKvBlockLog) * D + 4 * c) * 16ll) + quad;
        if (from == 0 && end == 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) to[4 * j] = u[j];
            continue;
        }
        // tokens in front of the new ones keep their values, what lies behind stays as it is
        const uint32_t before = (uint32_t)((1ull << (8 * from)) - 1), fresh = (uint32_t)((1ull << (8 * end)) - 1) & ~before;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t now = to[4 * j], again = grown ? e4m3_rescale4(now, was.y, scale.y) : now;
            to[4 * j] = (u[j] & fresh) | (again & before) | (now & ~(fresh | before));
        }
    }
}

}  // namespace

hipError_t load_kernels_append8() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, reinterpret_cast<const void *>(k_append8<64, false, kHalves>));
}

hipError_t launch_heads_append8(const spectre_heads &P, const HeadRows &x, const KvView &kv, const int *positions, const int *start, const int *seqs, int B, void *q_out,
                                hipStream_t st) {
    // As many workgroups as run at once, no more: each forms the angles of its tokens.  One or two for a block's queries and up to four for its key heads, or one for all.
    // 19 sequences' turns (202 blocks), with 8 parts 13.3 us, 6 (two and four) 11.4, 5 (one and four) 12.5; a prompt of 4096 (258 blocks) 15.7, 15.1 and 13.2.
    // Of the blocks of single tokens half are there.
    const int blocks = x.T / kKvBlock + 2 * B, heads = P.d == 64 ? 2 : 1, parts = std::min(6, 1300 / std::min(blocks, x.T));
    const int q_parts = parts < 2 ? 0 : parts < 6 ? 1 : 2, k_parts = std::max(1, std::min(parts - q_parts, (x.Hkv + heads - 1) / heads));
    auto launch = [&](auto kernel) { kernel<<<dim3(blocks, q_parts + k_parts), kThreads, 0, st>>>(head_params(P), x, positions, (uint4 *)q_out, kv, start, seqs, B, q_parts); };
    const int turn = turn_of(P);
#define CALL(D, AXES) (turn == kHalves ? launch(k_append8<D, AXES, kHalves>) : turn == kPairs ? launch(k_append8<D, AXES, kPairs>) : launch(k_append8<D, AXES, kAnyTurn>))
    if (P.d == 64) positions ? CALL(64, true) : CALL(64, false);
    else positions ? CALL(128, true) : CALL(128, false);
#undef CALL
    return hipGetLastError();
}

}  // namespace spectre
