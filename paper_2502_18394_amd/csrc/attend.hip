// Attention of each sequence's new tokens over its pages.
//
// Query i of n new ones, in a sequence of m tokens with them, stands at p = m - n + i and sees the keys j <= p (with a window: j > p - window):
// o = sum_j e^(s_j - M) v_j / sum_j e^(s_j - M), s_j = scale q . k_j, lse = M + log sum.  One pass over the keys with a running maximum and sum,
// both in fp32, as are scores and outputs until they are stored.
//
// The heads that share a key head and the new tokens are one list of rows, (token, head of the group): they read the same keys.  All products are
// formed transposed, S^T = K Q^T and O^T = V^T P^T, so that a row of scores lies in one lane (and its mate 32 or 16 lanes on): the softmax needs almost no
// exchange, and what a lane holds of P^T after S^T is what the second product wants of it, without a move.  For that the keys of a bf16 tile are
// given to the matrix instruction in an order in which each lane ends up with runs of 8.
// Probabilities go to the matrix cores in the type of the rows.  Of few rows, where memory leaves the matrix cores idle, a bf16 probability goes as two terms, itself rounded and
// the rest: outputs are off by their own rounding (1.64e-3 over all, 2.1e-3 with one term; 32 sequences of up to 32768 tokens 186 us, with one 185).  In tiles, which the matrix
// cores and the vector unit bound, it goes as one, rounded to half a step of 2^-8: errors of independent signs that average out like the values they weigh, 2.2e-3
// where the output's rounding alone is 1.65e-3 (an 8192-token prompt 336 us, with two terms 449; 16 tokens over 1000 for 90 sequences, d = 128, 41 and 49).
// The sum in the denominator is of the unrounded ones.
// Keys that nobody of the row's may see take no part whatever lies there: their scores are replaced, not shifted, and values that are infinite or NaN are
// taken out of the tiles where rows see different keys and added for the rows that do see them.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "e4m3.h"
#include "paged.h"

namespace spectre {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kLog2E = 1.4426950408889634f;
// The maximum follows only when a score is this far above it, in powers of two: until then probabilities grow to 2^8, which costs neither fp32 nor bf16
// any digit, and the outputs need not be rescaled.
constexpr float kLag = 8.f;

// 16 bytes a lane from its address into LDS, lane after lane from `to` on (the same in every lane of the wave).
template <bool STREAM>
__device__ __forceinline__ void to_lds(const void *from, uint4 *to) {
    constexpr int kNonTemporal = STREAM ? 2 : 0;
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, kNonTemporal);
}

__device__ __forceinline__ void to_lds4(const float *from, float *to) {     // the same of 4 bytes
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 4, 0, 0);
}

struct AttendK {
    KvView kv;
    AttendArgs a;
    int G, tiles, few_rows;                        // heads of a key head; tiles of a sequence; the rows up to which a sequence is the business of `few`
    int few_splits, tile_splits, slots;            // parts of a sequence's keys, at most; of either kind
    int part_keys;                                 // of a part of a tile's rows, at least
    int few_blocks, tile_blocks;                   // workgroups of each kind, where both are in one launch
    bool few_stream, tile_stream;                  // pages are read past the memory-side cache
    float c;                                       // scale * log2(e)
    // Places of partial results: `slots` for every row, or, where that would be too many (`packed`), as many as each row has parts: first those of few rows, few_tokens
    // tokens a sequence (0: every token of the batch has them), then those of tiles' rows, tile_places in all.
    bool packed;
    int few_tokens;
    long long few_places, tile_places;
    float *part;                                   // [places][d]
    float2 *stat;                                  // [places]: maximum in powers of two, sum
    int *count;                                    // [T * H] parts of the row's keys, 0: the output is written
    unsigned *first;                               // [T * H] the row's first place, if `packed`
};

struct Seq {
    int from, n, m, row;                           // first new token, new tokens, tokens, row of the table
    // parts that the keys of a tile's rows are divided into, of part_keys keys or more
    __device__ __forceinline__ int parts(const AttendK &k, int part_keys) const {
        const int keys = k.a.window ? min(m, k.a.window + n) : m;
        return max(1, min(k.tile_splits, (keys + part_keys - 1) / part_keys));
    }
};
__device__ __forceinline__ Seq sequence(const AttendK &k, int b) {
    Seq s;
    s.from = k.a.start[b];
    const int to = min(k.a.start[b + 1], k.a.T);
    s.n = s.from >= 0 ? max(to - s.from, 0) : 0;
    s.row = k.a.seqs ? k.a.seqs[b] : b;
    s.m = 0;
    if ((unsigned)s.row < (unsigned)k.kv.S) s.m = min(max(k.kv.lens[s.row], 0), k.kv.M << k.kv.page_log);
    else s.row = 0;
    return s;
}

// Length of parts and the tokens x parts of the sequences in front of sequence b, where places are shared out: to the sequences that have more than one part, in turn.  If
// all of them together want more places than there are, parts become longer until they fit.  Every workgroup of a sequence finds the same (a wave looks at
// 64 sequences at once).
struct Room {
    int part_keys, before;
};
__device__ __forceinline__ long long wave_sum(long long x) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m, 64);
    return x;
}
__device__ __forceinline__ Room room_of(const AttendK &k, int b) {
    const int lane = threadIdx.x & 63, B = k.a.B;
    int part_keys = k.part_keys;
    auto want = [&](const Seq &s) -> long long {
        const int parts = s.n * k.G > k.few_rows ? s.parts(k, part_keys) : 1;
        return parts > 1 ? (long long)s.n * parts : 0;
    };
    Seq mine = sequence(k, min(lane, B - 1));
    if (lane >= B) mine.n = 0;
    for (;; part_keys += part_keys / 8 + 1) {                    // ends where every sequence is one part
        long long all = want(mine);
        for (int i = lane + 64; i < B; i += 64) all += want(sequence(k, i));
        if (wave_sum(all) * k.a.H <= k.tile_places) break;
    }
    long long before = lane < b ? want(mine) : 0;
    for (int i = lane + 64; i < b; i += 64) before += want(sequence(k, i));
    return Room{part_keys, (int)wave_sum(before)};
}

// Rows from `r` on of a sequence with more new tokens than the launch is sized for: nobody takes them, and the join leaves them as they are.
__device__ __forceinline__ void left_out(const AttendK &k, const Seq &s, int h, int r, int threads) {
    for (r += threadIdx.x; r < s.n * k.G; r += threads) {
        const int token = r / k.G;
        k.count[(long long)(s.from + token) * k.a.H + h * k.G + (r - token * k.G)] = 0;
    }
}

// Which sequence and key head a workgroup works on: all of them in turn, for each `rest` (tile, part) turned on by eight.  Eight keep a pair on one XCD, whose L2 then has its
// keys; without the turn the workgroups of a long sequence come at a fixed distance, often a multiple of what an XCD deals out at a time, and
// land on the same few compute units (24 ragged sequences, d = 128: 302 instead of 137 us).
__device__ __forceinline__ int turned_pair(int block, int rest, int pairs) { return (int)((block - (long long)rest * pairs + 8ll * rest) % pairs); }

// E, kBytes: of rows and of the matrix cores' operands.  PE: elements of a page's 16-byte groups.  kStepKeys: of a wave's step through few rows' keys.
struct Bf16Mma {
    static constexpr int E = 8, kBytes = 2, PE = 8, kPageBytes = 2;
    static constexpr bool kCoded = false;
    static constexpr int kTileKeys = 64, kStepKeys = 32;
    typedef uint16_t elem_t;
    // 32 rows of A (keys, channels) x 32 columns: one group of 8 of the contraction a lane
    __device__ static __forceinline__ void mma32(f32x16_t &acc, uint4 a, uint4 b) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    }
    __device__ static __forceinline__ void mma16(f32x4_t &acc, uint4 a, uint4 b) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    }
    // key of row r of a 32-row tile, and of accumulator r in half h of the wave: runs of 8 a lane
    __device__ static __forceinline__ int key_of_row(int r) { return 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3); }
    __device__ static __forceinline__ constexpr int key_of_acc(int r) { return 16 * (r >> 3) + (r & 7); }   // + 8 h
    static constexpr int kHalf = 8;
    static constexpr int kChunks = 2;                                          // groups of P a lane holds of 32 keys
    __device__ static __forceinline__ uint4 pack(const float *p) {
        return make_uint4(IoBf16::pack(make_float2(p[0], p[1])), IoBf16::pack(make_float2(p[2], p[3])), IoBf16::pack(make_float2(p[4], p[5])),
                          IoBf16::pack(make_float2(p[6], p[7])));
    }
    // what pack() left of the numbers
    __device__ static __forceinline__ uint4 pack_rest(const float *p, uint4 g) {
        const uint32_t w[4] = {g.x, g.y, g.z, g.w};
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = p[2 * i] - __uint_as_float(w[i] << 16);
            x[2 * i + 1] = p[2 * i + 1] - __uint_as_float(w[i] & 0xffff0000u);
        }
        return pack(x);
    }
    __device__ static __forceinline__ bool finite(uint32_t w) { return (w & 0x7f80u) != 0x7f80u && (w & 0x7f800000u) != 0x7f800000u; }
    __device__ static __forceinline__ uint32_t finite_only(uint32_t w) {
        return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
    }
    __device__ static __forceinline__ float value(elem_t e) { return __uint_as_float((uint32_t)e << 16); }
    // the first `n` elements of a group, zeros behind
    __device__ static __forceinline__ uint32_t keep(uint32_t w, int i, int n) { return 2 * i + 1 < n ? w : 2 * i < n ? w & 0xffffu : 0u; }
};
struct F32Mma {
    static constexpr int E = 4, kBytes = 4, PE = 4, kPageBytes = 4;
    static constexpr bool kCoded = false;
    static constexpr int kTileKeys = 32, kStepKeys = 16;
    typedef uint32_t elem_t;
    __device__ static __forceinline__ void mma32(f32x16_t &acc, uint4 a, uint4 b) {
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
    }
    __device__ static __forceinline__ void mma16(f32x4_t &acc, uint4 a, uint4 b) {
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
    }
    __device__ static __forceinline__ int key_of_row(int r) { return r; }
    __device__ static __forceinline__ constexpr int key_of_acc(int r) { return 8 * (r >> 2) + (r & 3); }    // + 4 h
    static constexpr int kHalf = 4;
    static constexpr int kChunks = 4;
    __device__ static __forceinline__ uint4 pack(const float *p) {
        return make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3]));
    }
    __device__ static __forceinline__ bool finite(uint32_t w) { return (w & 0x7f800000u) != 0x7f800000u; }
    __device__ static __forceinline__ uint32_t finite_only(uint32_t w) { return finite(w) ? w : 0u; }
    __device__ static __forceinline__ float value(elem_t e) { return __uint_as_float(e); }
    __device__ static __forceinline__ uint32_t keep(uint32_t w, int i, int n) { return i < n ? w : 0u; }
};

// Pages of 8 bits, rows of bf16: codes become bf16 numbers, exactly, on their way to the matrix cores, their block's scale with them.  A group is 16 channels of a
// key, or 16 keys of a channel: two operands.
struct E4m3Mma : Bf16Mma {
    static constexpr int PE = 16, kPageBytes = 1, kStepKeys = 64;
    static constexpr bool kCoded = true;
    __device__ static __forceinline__ uint32_t keep8(uint32_t w, int i, int n) {
        return n >= 4 * i + 4 ? w : n <= 4 * i ? 0u : w & ((1u << (8 * (n - 4 * i))) - 1u);
    }
    __device__ static __forceinline__ uint4 keep_codes(uint4 g, int n) { return make_uint4(keep8(g.x, 0, n), keep8(g.y, 1, n), keep8(g.z, 2, n), keep8(g.w, 3, n)); }
    __device__ static __forceinline__ uint32_t nan_bits(uint4 g) { return e4m3_nan_bits(g.x) | e4m3_nan_bits(g.y) | e4m3_nan_bits(g.z) | e4m3_nan_bits(g.w); }
    __device__ static __forceinline__ uint4 finite_codes(uint4 g) {
        return make_uint4(e4m3_finite_only(g.x), e4m3_finite_only(g.y), e4m3_finite_only(g.z), e4m3_finite_only(g.w));
    }
};
// Operand `half` of a group as it lies in a page.
template <typename IO>
__device__ __forceinline__ uint4 operand(uint4 g, int half, float scale) {
    if constexpr (IO::kCoded) return half ? e4m3_decode8(g.z, g.w, scale) : e4m3_decode8(g.x, g.y, scale);
    else return g;
}

template <typename IO>
__device__ __forceinline__ uint4 keep_first(uint4 g, int n) {
    return make_uint4(IO::keep(g.x, 0, n), IO::keep(g.y, 1, n), IO::keep(g.z, 2, n), IO::keep(g.w, 3, n));
}
template <typename IO>
__device__ __forceinline__ bool all_finite(uint4 g) { return IO::finite(g.x) && IO::finite(g.y) && IO::finite(g.z) && IO::finite(g.w); }
// The same of N groups of bf16: the largest of all magnitudes, two at a time.
template <int N>
__device__ __forceinline__ bool all_finite_bf16(const uint4 (&g)[N]) {
    typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
    u16x2_t most = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t w[4] = {g[i].x, g[i].y, g[i].z, g[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2_t, w[j] & 0x7fff7fffu));
    }
    return most[0] < 0x7f80 && most[1] < 0x7f80;
}
template <typename IO>
__device__ __forceinline__ uint4 finite_only(uint4 g) {
    return make_uint4(IO::finite_only(g.x), IO::finite_only(g.y), IO::finite_only(g.z), IO::finite_only(g.w));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// One row's statistics after scores whose largest is mx: true in any lane asks for a rescale by the factor that follow() returns.
__device__ __forceinline__ bool lags(float mx, float top, float lag) { return mx > top + lag; }
__device__ __forceinline__ float follow(float mx, float c, float *top) {
    const float next = fmaxf(*top, mx), f = next == *top ? 1.f : exp2_fast((*top - next) * c);
    *top = next;
    return f;
}
// -top * c, 0 while nothing has been seen (then every score is -inf, and 2^(-inf) = 0)
__device__ __forceinline__ float shift_of(float top, float c) { return top == -INFINITY ? 0.f : -top * c; }

// Values that are not finite, of keys base .. base + count - 1 of head h, for a row at `pos` whose lane holds channels channel(r), r < N.  The rows' finite
// parts have been added; a weight is above zero for every key a row sees, so what is added is the value itself.
template <typename IO, int D, int N, bool ONE_BY_ONE, typename Channel, typename Add>
__device__ __forceinline__ void add_not_finite(const KvView &kv, const Seq &s, int h, int base, int count, int pos, int from, Channel channel, Add add) {
    typedef typename IO::elem_t elem_t;
    const int *table = kv.table + (long long)s.row * kv.M;
#pragma unroll 1
    for (int key = base; key < base + count && key < s.m; ++key) {
        const int page = table[key >> kv.page_log], slot = key & ((1 << kv.page_log) - 1);
        if ((unsigned)page >= (unsigned)kv.P || key > pos || key <= from) continue;
        const long long head = (long long)page * kv.Hkv + h;
        const elem_t *v = reinterpret_cast<const elem_t *>(kv.v) + ((head << kv.page_log) + slot / IO::E * IO::E) * D + slot % IO::E;
        const uint8_t *codes = reinterpret_cast<const uint8_t *>(kv.v) + ((head << kv.page_log) + slot / IO::PE * IO::PE) * D + slot % IO::PE;
        float scale = 0.f;
        if constexpr (IO::kCoded) scale = kv.scales[2 * ((head << (kv.page_log - kKvBlockLog)) + (slot >> kKvBlockLog)) + 1];
#pragma unroll
        for (int r = 0; r < N; ++r) {
            float x;
            if constexpr (IO::kCoded) x = e4m3_decode1(codes[channel(r) * IO::PE], scale);
            else x = IO::value(v[channel(r) * IO::E]);
            if constexpr (N > 32 || ONE_BY_ONE) {
                // one condition at a time: 64 pairs of scalar registers are taken from the loop around otherwise (its addresses then live in lanes of a
                // vector register: 540 instead of 499 us for 2048 rows over 28672, d = 128; with 32 channels a lane the plain form is the faster one)
                add(r, isfinite(x) ? 0.f : x);
                __builtin_amdgcn_sched_barrier(0);
            } else if (!isfinite(x)) add(r, x);
        }
    }
}

template <typename IO>
__device__ __forceinline__ void store4(void *out, long long at, float4 x) {
    if constexpr (IO::kBytes == 2) {
        uint2 w;
        w.x = IoBf16::pack(make_float2(x.x, x.y));
        w.y = IoBf16::pack(make_float2(x.z, x.w));
        *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(out) + at) = w;
    } else {
        *reinterpret_cast<float4 *>(reinterpret_cast<float *>(out) + at) = x;
    }
}

// The larger, NaN if one is: gfx950 has it as one instruction of three operands, without the quieting that fmaxf asks for.
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// The larger of a lane's number and that of the lane 32 on.
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float max_halves(float x) {
    const u32x2_t y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return larger(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// The same for the lane 16 on (within its half).
__device__ __forceinline__ float max_quarters(float x) {
    const u32x2_t y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return larger(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

__device__ __forceinline__ float lse_of(float top2, float sum) { return sum == 0.f ? -INFINITY : (top2 + log2f(sum)) * 0.69314718055994531f; }
__device__ __forceinline__ float inverse(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }

// ---------------------------------------------------------------- many rows: tiles of 64 keys (fp32: 32) through LDS
// 32 rows a wave; a workgroup's waves share each tile, which goes from memory into LDS without registers (one tile ahead, two buffers, a barrier a tile).
// The layout of the pages is that of the operands, so LDS reads are runs of 16 bytes without conflicts.
//
// What bounds it at d = 64: per 64 keys and 32 rows a wave issues 16 products (32 clocks each on the matrix cores) and about 130 vector instructions
// that cannot be saved (32 each of scale-and-shift, 2^x, sum; 16 each of maximum and packing), 2^x taking two slots.  Measured on their own in that proportion with their
// LDS reads, products and vector work overlap only in part: 26.5 ns a product, against 17.5 for products alone and 15.7 for the rest alone.  The kernel takes 35.
// Counters of that kernel: matrix cores busy in 41 % of the cycles, the vector unit in 65 %, no LDS conflict.
// An 8192-token prompt, 32 heads: 302 to 341 us by the machine, 806 to 911 TFLOP/s (all-zero inputs, which draw less power, take 13 % less); 2048 tokens over 28672 534 to
// 595 us, 837 to 933 TFLOP/s.
// At d = 128 there are twice the products for the same vector work, two waves a SIMD: the same prompt with 16 heads 267 to 287 us, 958 to 1031 TFLOP/s, the same chunk 484 to 510,
// 978 to 1031 TFLOP/s.  A large matrix product of the library reaches 1326.
// Where a page holds a whole tile its address is scalar work and the lanes' offsets stay the same from tile to tile; pages of less than a tile give every lane its
// own address (which took 614 us where this took 540: 2048 over 28672, d = 128, pages of 64).
// Measured and not taken: two sets of 32 rows a wave (half the LDS reads, two waves a SIMD: 4 % slower), scores of the next tile formed between the steps of this tile's
// softmax within a wave (17 % slower, d = 128 1 % faster), two tiles a barrier (3 % slower), raised priority around the products (no difference), tiles through registers (4 % slower).
template <typename IO, int D>
constexpr int kTileGroups = IO::kTileKeys * D / IO::E;
// Groups of a tile as they lie in pages of 8 bits, on their way.  (d = 64: in registers the queries went to memory and were read again for every tile, which waited for all loads on
// their way: 1006 instead of 630 us.)
template <typename IO, int D>
constexpr int kRawGroups = IO::kCoded && D == 64 ? 8 * D + 8 * D / 4 : 0;    // and their scales
// Groups of queries that registers have no room for beside those tiles: all of them (2048 rows over 28672 594 us, with
// three of four 619).
template <typename IO, int D, int WAVES>
constexpr int kQueryGroups = kRawGroups<IO, D> && WAVES == 8 ? 4 * 64 * WAVES : 0;
struct TileLds {
    uint4 *sk0, *sv0, *sk1, *sv1;                   // kTileGroups each, arrays of their own: the compiler sees which loads a read need not wait for
    uint4 *raw, *query;                             // kRawGroups, kQueryGroups
    int *odd;                                       // [2] the last tile whose values were not all finite; [2]: tokens x parts in front of the sequence's places
};

template <typename IO, int D, int WAVES>
__device__ __forceinline__ void tile_of_rows(const AttendK &k, int block, TileLds lds) {
    constexpr int THREADS = 64 * WAVES, kTileRows = 32 * WAVES;
    constexpr int E = IO::E, KT = IO::kTileKeys, NK = KT / 32, GROUPS = kTileGroups<IO, D>, PER = GROUPS / THREADS, QG = D / (2 * E), DT = D / 32;
    uint4 *const sk0 = lds.sk0, *const sv0 = lds.sv0, *const sk1 = lds.sk1, *const sv1 = lds.sv1;
    int *const odd = lds.odd;
    const KvView &kv = k.kv;
    const int pairs = kv.Hkv * k.a.B, rest = block / pairs, pair = turned_pair(block, rest, pairs);
    const int h = pair % kv.Hkv, split = rest % k.tile_splits, tile = k.tiles - 1 - rest / k.tile_splits;   // long rows first
    const Seq s = sequence(k, pair / kv.Hkv);
    const int rows = s.n * k.G, r0 = tile * kTileRows;
    if (rows <= k.few_rows || r0 >= rows) return;
    int parts = s.parts(k, k.part_keys);
    if (split >= parts) return;
    if (k.packed && parts > 1) {
        const Room room = room_of(k, pair / kv.Hkv);
        parts = s.parts(k, __builtin_amdgcn_readfirstlane(room.part_keys));
        if (split >= parts) return;
        if (threadIdx.x == 0) odd[2] = room.before;          // for the end
        __syncthreads();
    }
    if (k.slots > 1 && split == 0 && tile == 0) left_out(k, s, h, k.tiles * kTileRows, THREADS);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int r = min(r0 + 32 * wave + (lane & 31), rows - 1), token = r / k.G, head = h * k.G + (r - token * k.G);
    const bool mine = r0 + 32 * wave + (lane & 31) < rows, busy = r0 + 32 * wave < rows;
    const int p0 = s.m - s.n, pos = p0 + token;
    const int lowest = k.a.window ? pos - k.a.window + 1 : 0;                  // the row sees the `span` keys from here on
    const unsigned span = (unsigned)max(pos - lowest + 1, 0);
    // what all rows of the workgroup, and of the wave, see
    const int first_pos = p0 + r0 / k.G, last_pos = p0 + min(r0 + kTileRows - 1, rows - 1) / k.G;
    const int wave_first = p0 + min(r0 + 32 * wave, rows - 1) / k.G, wave_last = p0 + min(r0 + 32 * wave + 31, rows - 1) / k.G;
    int t_lo = k.a.window ? max(0, first_pos - k.a.window + 1) / KT : 0, t_hi = last_pos >= 0 ? last_pos / KT + 1 : 0;
    if (parts > 1) {
        const int per = (max(t_hi - t_lo, 0) + parts - 1) / parts;
        t_lo += split * per;
        t_hi = min(t_hi, t_lo + per);
    }

    constexpr int QL = kQueryGroups<IO, D, WAVES> / THREADS;                   // of a row's groups, the last ones, in LDS
    uint4 q[QG];
    {
        const char *base = reinterpret_cast<const char *>(k.a.q) + ((s.from + token) * k.a.q_stride + head * D) * IO::kBytes;
#pragma unroll
        for (int i = 0; i < QG; ++i) {
            q[i] = reinterpret_cast<const uint4 *>(base)[2 * i + half];
            if (i >= QG - QL) lds.query[(i - (QG - QL)) * THREADS + threadIdx.x] = q[i];
        }
    }
    f32x16_t o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float top = -INFINITY, sum = 0.f;
    const float lag = kLag / k.c;

    const int mask = (1 << kv.page_log) - 1;
    const int *table = kv.table + (long long)s.row * kv.M;
    // page of this lane's key of tile t (every wave has all keys of a tile), -1 where there is none.  It is looked at only when its tile is requested: a
    // comparison here would wait for it, and with it for the tile requested before.
    auto page_of = [&](int t) {
        const int key = t * KT + (lane & (KT - 1));
        int p = -1;
        if (t < t_hi && key < s.m) p = table[key >> kv.page_log];
        return p;
    };
    const unsigned P = (unsigned)kv.P;
    // bytes of a page, and of this head and thread inside one: a 64-bit product a lane (keys) or a wave (values), 32-bit sums for the rest
    const unsigned page_bytes = (unsigned)kv.Hkv * (D * IO::kPageBytes) << kv.page_log, head_bytes = (unsigned)h * (D * IO::kPageBytes) << kv.page_log;
    const unsigned k_at = (threadIdx.x / KT * 16u) << kv.page_log, k_lane = k_at + (lane & (KT - 1)) * 16u;
    const char *const k_head = reinterpret_cast<const char *>(kv.k) + head_bytes, *const v_head = reinterpret_cast<const char *>(kv.v) + head_bytes;
    // Groups of a tile straight from memory into LDS, in the order they have there: a wave's 64 lanes write 1 KB from its first group on.  Absent keys leave
    // what lies there.
    const bool one_page = (1 << kv.page_log) >= KT;                          // a tile lies in one page: its address is scalar work
    auto copy_keys = [&](const char *kb, unsigned off, uint4 *to, auto stream) {
        unsigned k_next = ((unsigned)THREADS / KT * 16u) << kv.page_log;
        int wave_now = wave;
        asm volatile("" : "+s"(k_next), "+s"(wave_now));                      // opaque: its multiples are not kept in registers from tile to tile
#pragma unroll
        for (int i = 0; i < PER; ++i) to_lds<decltype(stream)::value>(kb + i * k_next + off, to + 64 * wave_now + THREADS * i);
    };
    auto copy_values = [&](const char *vb, uint4 *to, auto stream) {
        int wave_now = wave;
        asm volatile("" : "+s"(wave_now));
#pragma unroll
        for (int i = 0; i < PER; ++i) to_lds<decltype(stream)::value>(vb + i * (THREADS * 16u) + threadIdx.x * 16u, to + 64 * wave_now + THREADS * i);
    };
    auto request_keys = [&](int t, int page, uint4 *to) {
        if (one_page) {
            const unsigned p = (unsigned)__builtin_amdgcn_readfirstlane(page);
            if (p >= P) return;
            const char *kb = k_head + (unsigned long long)p * page_bytes + ((t * KT) & mask) * 16u;
            if (k.tile_stream) copy_keys(kb, k_lane, to, std::true_type());
            else copy_keys(kb, k_lane, to, std::false_type());
            return;
        }
        if ((unsigned)page >= P) return;
        const char *kb = k_head + (unsigned long long)(unsigned)page * page_bytes + (k_at + ((t * KT + (lane & (KT - 1))) & mask) * 16u);
        if (k.tile_stream) copy_keys(kb, 0u, to, std::true_type());
        else copy_keys(kb, 0u, to, std::false_type());
    };
    auto request_values = [&](int t, int page, uint4 *to) {
        if (one_page) {
            const unsigned p = (unsigned)__builtin_amdgcn_readfirstlane(page);
            if (p >= P) return;
            const char *vb = v_head + (unsigned long long)p * page_bytes + ((t * KT) & mask) / E * (D * 16u);
            if (k.tile_stream) copy_values(vb, to, std::true_type());
            else copy_values(vb, to, std::false_type());
            return;
        }
        int wave_now = wave;
        asm volatile("" : "+s"(wave_now));
#pragma unroll 1
        for (int i = 0; i < PER; ++i) {
            const int kg = (64 * wave_now + THREADS * i) / D * E;
            const unsigned p = (unsigned)__builtin_amdgcn_readlane(page, kg);
            const char *vb = v_head + (unsigned long long)p * page_bytes + (((t * KT + kg) & mask) / E) * (D * 16u);
            if (p < P) to_lds<false>(vb + threadIdx.x % D * 16u, to + 64 * wave_now + THREADS * i);
        }
    };
    // Pages of 8 bits are requested a tile ahead of being written to the tiles' LDS as bf16 numbers, which is a tile ahead of their use.  On their way they lie in LDS that only
    // the wave that asked for them reads (d = 128: in registers, of which it has enough, and LDS not).  A wave's 64 threads have the same 16 channels of a tile's
    // keys, or groups of one (d = 128: of half a) block of its values.  What stands for keys that are absent is what was there before: nobody's scores, and cleared values.
    // 2048 rows over 28672, 32 heads, d = 64: 585 to 600 us by the machine, 830 to 850 TFLOP/s, where pages of bf16 take 558 to 575.
    constexpr int CODED = IO::kCoded ? 8 * D / THREADS : 1;                  // groups a thread, keys' first
    constexpr bool RAW = kRawGroups<IO, D> > 0;
    uint4 code[CODED];
    float code_scale[CODED] = {};
    auto request_codes = [&](int t, int page) {
        if constexpr (IO::kCoded) {
            int lane = threadIdx.x;
            asm volatile("" : "+v"(lane));                                   // opaque: what is formed of it is not kept in registers from tile to tile
            lane &= 63;
#pragma unroll
            for (int i = 0; i < CODED; ++i) {
                const int u = 64 * wave + THREADS * i;
                const bool keys = u < 4 * D;
                const int kg = keys ? 0 : (u - 4 * D) / D;                   // block of values
                auto request = [&](const char *from, const float *scale) {
                    if constexpr (RAW) {
                        to_lds<false>(from, lds.raw + u);
                        to_lds4(scale, reinterpret_cast<float *>(lds.raw + 8 * D) + u);
                    } else {
                        code[i] = *reinterpret_cast<const uint4 *>(from);
                        code_scale[i] = *scale;
                    }
                };
                if (one_page || !keys) {                                     // scalar addresses
                    const int p = one_page ? __builtin_amdgcn_readfirstlane(page) : __builtin_amdgcn_readlane(page, 16 * kg);
                    if ((unsigned)p >= P) continue;
                    const int slot = (t * KT + 16 * kg) & mask;
                    const long long head = (long long)p * kv.Hkv + h;
                    const char *base = reinterpret_cast<const char *>(keys ? kv.k : kv.v) + (head << kv.page_log) * D;
                    const float *scale = kv.scales + 2 * ((head << (kv.page_log - kKvBlockLog)) + (slot >> kKvBlockLog));
                    if (keys) request(base + ((((u / KT) << kv.page_log) + slot) * 16u) + lane * 16u, scale + (lane >> 4) * 2);
                    else request(base + ((slot >> kKvBlockLog) * D + (u - 4 * D) % D) * 16u + lane * 16u, scale + 1);
                } else {
                    if ((unsigned)page >= P) continue;
                    const int slot = (t * KT + lane) & mask;
                    const long long head = (long long)page * kv.Hkv + h;
                    request(reinterpret_cast<const char *>(kv.k) + (head << kv.page_log) * D + (((u / KT) << kv.page_log) + slot) * 16u,
                            kv.scales + 2 * ((head << (kv.page_log - kKvBlockLog)) + (slot >> kKvBlockLog)));
                }
            }
        }
    };
    // Writes what has been requested of one tile, and requests tile t in its place.
    auto write_codes = [&](uint4 *sk, uint4 *sv, int t, int page) {
        if constexpr (IO::kCoded) {
            int at = threadIdx.x;
            asm volatile("" : "+v"(at));
            if constexpr (RAW) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
                for (int i = 0; i < CODED; ++i) {
                    code[i] = lds.raw[at + THREADS * i];
                    code_scale[i] = reinterpret_cast<const float *>(lds.raw + 8 * D)[at + THREADS * i];
                }
            }
            const int lane = at & 63;
#pragma unroll
            for (int i = 0; i < CODED; ++i) {
                const int u = 64 * wave + THREADS * i;
                uint4 *to = u < 4 * D ? sk + 2 * (u / KT) * KT + lane : sv + 2 * ((u - 4 * D) / D) * D + (u - 4 * D) % D + lane;
                to[0] = operand<IO>(code[i], 0, code_scale[i]);
                to[u < 4 * D ? KT : D] = operand<IO>(code[i], 1, code_scale[i]);
            }
            // behind the writes, which the compiler would have wait for what is on its way to LDS
            if constexpr (RAW) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // the codes have left their place
            request_codes(t, page);
        }
    };
    auto arrived = [&]() {
        if constexpr (!IO::kCoded) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's part has arrived ...
        __syncthreads();                                                    // ... and everybody's, and nobody reads the other buffers any more
    };
    const int back = k.a.window ? k.a.window : 1 << 30;
    // Tile t's values of no one's keys, and those that are not finite, where rows of the workgroup see different keys.
    auto clean = [&](int t, unsigned long long there, uint4 *sv, int *flag) {
        if (there == ~0ull && t * KT + KT - 1 <= first_pos && t * KT > last_pos - back) return;
        bool fine = true;
#pragma unroll 1
        for (int i = 0; i < PER; ++i) {
            const int kg = (64 * wave + THREADS * i) / D * E;
            uint4 x = sv[threadIdx.x + THREADS * i];
            x = keep_first<IO>(x, ((there >> kg) & 1) ? s.m - (t * KT + kg) : 0);
            if (!all_finite<IO>(x)) {
                fine = false;
                x = finite_only<IO>(x);
            }
            sv[threadIdx.x + THREADS * i] = x;
        }
        if (!fine) *flag = t;
        __syncthreads();
    };
    // Scores that the row does not see are replaced.
    auto hide = [&](int t, unsigned long long there, f32x16_t(&sc)[NK]) {
        if (there == ~0ull && t * KT + KT - 1 <= wave_first && t * KT > wave_last - back) return;
        const unsigned at0 = (unsigned)(t * KT + IO::kHalf * half - lowest);
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (at0 + (32 * n + IO::key_of_acc(i)) >= span) sc[n][i] = -INFINITY;
        if (there != ~0ull) {                                           // pages that are not there
            const unsigned long long mates = there >> (IO::kHalf * half);
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {                              // by bits: conditions would want a pair of scalar registers each
                    const int gone = (int)(~(unsigned)(mates >> (32 * n + IO::key_of_acc(i))) << 31) >> 31;
                    sc[n][i] = __int_as_float((__float_as_int(sc[n][i]) & ~gone) | ((int)0xff800000 & gone));
                }
        }
    };
    auto largest = [&](const f32x16_t(&sc)[NK]) {
        float mx = sc[0][0];
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = larger(mx, sc[n][i]);
        return mx;
    };
    auto keep_up = [&](float mx) {                                      // with the maximum mx of a tile's scores, of both halves
        if (!__ballot(IO::kCoded ? (mx - top) * k.c > kLag : lags(mx, top, lag))) return;     // no register for the lag, either
        const float f = follow(mx, k.c, &top);
        sum *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= f;
    };
    auto add_odd = [&](int t) {
        add_not_finite<IO, D, 16 * DT, false>(kv, s, h, t * KT, KT, pos, lowest - 1, [half](int i) { return 32 * (i / 16) + 8 * ((i % 16) / 4) + 4 * half + i % 4; },
                                       [&](int i, float x) { o[i / 16][i % 16] += x; });
    };
    const int krow = IO::key_of_row(lane & 31);
    auto scores = [&](const uint4 *sk, f32x16_t(&sc)[NK]) {
        uint4 ql[QL ? QL : 1];
        if constexpr (QL > 0) {
            int at = threadIdx.x;
            asm volatile("" : "+v"(at));
#pragma unroll
            for (int i = 0; i < QL; ++i) ql[i] = lds.query[i * THREADS + at];
        }
#pragma unroll
        for (int n = 0; n < NK; ++n) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[n][i] = 0.f;
            uint4 a[QG];
#pragma unroll
            for (int i = 0; i < QG; ++i) a[i] = sk[(2 * i + half) * KT + 32 * n + krow];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < QG; ++i) IO::mma32(sc[n], a[i], QL && i >= QG - QL ? ql[i - (QG - QL)] : q[i]);
        }
    };
    if (threadIdx.x < 2) odd[threadIdx.x] = -1;
    int page = page_of(t_lo), next = page_of(t_lo + 1);
    unsigned long long here = 0, soon = 0;               // which keys of this tile and the next are there (pages of 8 bits, whose page numbers are not kept so long)
    if (t_lo < t_hi) {
        if constexpr (IO::kCoded) {
            here = __ballot((unsigned)page < P);
            request_codes(t_lo, page);
            soon = __ballot((unsigned)next < P);
            write_codes(sk0, sv0, t_lo + 1, next);
            next = page_of(t_lo + 2);
        } else {
            request_keys(t_lo, page, sk0);
            request_values(t_lo, page, sv0);
        }
    }
    auto tile_step = [&](int t, uint4 *sk, uint4 *sv, uint4 *next_k, uint4 *next_v, int *flag) {
        const unsigned long long there = IO::kCoded ? here : __ballot((unsigned)page < P);      // bit = key of the tile (fp32: twice 32 keys)
        arrived();
        if constexpr (IO::kCoded) {
            here = soon;
            soon = __ballot((unsigned)next < P);
            write_codes(next_k, next_v, t + 2, next);
            next = page_of(t + 3);
        } else page = next;
        if (!IO::kCoded && t + 1 < t_hi) {
            request_keys(t + 1, page, next_k);
            request_values(t + 1, page, next_v);
            next = page_of(t + 2);
        }
        clean(t, there, sv, flag);
        if (!busy || t * KT > wave_last) return;
        f32x16_t sc[NK];
        scores(sk, sc);
        hide(t, there, sc);
        keep_up(max_halves(largest(sc)));
        const float shift = shift_of(top, k.c);
        float p[NK * 16];
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[16 * n + i] = exp2_fast(fmaf(sc[n][i], k.c, shift));
                sum += p[16 * n + i];
            }
#pragma unroll
        for (int g = 0; g < NK * IO::kChunks; ++g) {
            const uint4 pg = IO::pack(p + g * E);
#pragma unroll
            for (int d = 0; d < DT; ++d) IO::mma32(o[d], sv[(2 * g + half) * D + 32 * d + (lane & 31)], pg);
        }
        if (*flag == t) add_odd(t);
    };
    for (int t = t_lo; t < t_hi; t += 2) {
        tile_step(t, sk0, sv0, sk1, sv1, &odd[0]);
        if (t + 1 < t_hi) tile_step(t + 1, sk1, sv1, sk0, sv0, &odd[1]);
    }
    if (!mine) return;
    sum += __shfl_xor(sum, 32, 64);
    const long long at = (long long)(s.from + token) * k.a.H + head;
    const float top2 = top * k.c;
    if (k.slots > 1 && split == 0 && half == 0) k.count[at] = parts > 1 ? parts : 0;
    if (parts > 1) {
        long long place = at * k.slots;
        if (k.packed) {
            place = k.few_places + (long long)odd[2] * k.a.H + ((long long)token * k.a.H + head) * parts;
            if (split == 0 && half == 0) k.first[at] = (unsigned)place;
        }
        place += split;
        if (half == 0) k.stat[place] = make_float2(top2, sum);
        if (sum == 0.f) return;
        float *to = k.part + place * D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<float4 *>(to + 32 * d + 8 * i + 4 * half) = make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
        return;
    }
    const float inv = inverse(sum);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store4<IO>(k.a.out, at * D + 32 * d + 8 * i + 4 * half, make_float4(o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv));
    if (k.a.lse && half == 0) k.a.lse[at] = lse_of(top2, sum);
}

// ---------------------------------------------------------------- few rows: up to 16 of a key head (pages of 8 bits: 64), keys split over waves and workgroups
// Pages of 8 bits have steps of 64 keys, the same bytes: 32 sequences of up to 32768 tokens, 547 MB, 98 us and 5 of the join (5.6 TB/s; parts of 1024 and of 4096 keys 104), bf16 pages 181
// and 5.  Their codes become bf16 on the way to the matrix cores, two an instruction, the scale in it; the vector unit is busy in 44 % of the cycles.
// Every key and value is read once and multiplied with 16 columns of rows, empty ones among them: memory bounds it.  No LDS: a lane's loads are the operands (the
// layout of the pages), one step of 32 keys (fp32: 16) in registers, of which each half is requested again as soon as it has been used, so that four waves a SIMD
// keep up to 8 KB (d = 64) each on its way.  (Two steps in turn need twice the registers: 16 sequences of 4000 tokens, d = 128, 36 instead of 29 us.)
// A large pool is read past the memory-side cache, its pages come round again only when every other layer's have.  8 sequences of 32700 tokens, 537 MB:
// 89 us, 6.0 TB/s (cached 100); 32 of up to 32768, 1.09 GB, 185 us, 5.9 TB/s; a pool of 67 MB would lose (23.1 -> 24.2 us), one of 131 MB gains (33.2 -> 31.1).
// COLS groups of 16 rows share what is read and, of pages of 8 bits, what is converted; their queries lie in LDS, and a probability goes as one term, as in tiles.  Without a
// barrier between steps, and with every wave at work, a tile's way is the longer one up to 64 rows (d = 128: 48, whose registers leave one wave a SIMD): 64 sequences of
// 8 tokens over 8000, 32 rows, 112 us, as tiles 179; 64 of 16 over 2000, 64 rows, 36 and 60; d = 128, 32 of 5 over 4000, 40 rows, 26 and 32.5, but 64 rows (registers
// spilled) 48 and 34.5.  A second term (see above) costs more here, where the first one's registers are all there are: 32 rows over 8000 122 us instead of 111, 64 rows over 2000 55
// instead of 37 (it spills), 40 rows of d = 128 over 4000 27.3 instead of 25.3, for outputs that would be off by 1.65e-3, as those of up to 16 rows are, instead of 1.9e-3.
// Short parts take the longer the more code they go through once (kernels of 12.5, 14.8 and 17.2 KB, one step each: 7.6, 9.6 and 11.5 us): outputs are joined in one loop
// for all groups (16 windows of 5 tokens, 40 rows, d = 128: 21.3 us, group by group 23.1).
constexpr int kSection = 256;                      // page numbers in LDS at a time

template <typename IO, int D>
constexpr int kFewGroups = 16 * D / 4;              // of a wave's 16 rows of outputs
template <int ROWS>
struct FewLds {
    int *pages;                                     // [kSection + 2]
    float (*tops)[ROWS], (*sums)[ROWS];             // [waves][rows]
    f32x4_t *out0, *out1, *out2, *out3;             // kFewGroups for 16 rows of every fourth wave each
    uint4 *query;                                   // kFewQueries
};

// Operands of 16 rows' queries, of which there are COLS; more than one stay in LDS, where the waves share them.
template <typename IO, int D>
constexpr int kFewOperands = D / (4 * IO::PE) * (IO::PE == 16 ? 2 : 1);
template <typename IO, int D, int COLS>
constexpr int kFewQueries = COLS > 1 ? 64 * COLS * kFewOperands<IO, D> : 0;

template <typename IO, int D, int WAVES, int COLS>
__device__ __forceinline__ void few_rows(const AttendK &k, int block, FewLds<16 * COLS> lds) {
    constexpr int E = IO::E, PE = IO::PE, SK = IO::kStepKeys, KTILES = SK / 16, DT = D / 16, THREADS = 64 * WAVES;
    constexpr int GROUPS = D / (4 * PE), HALVES = PE == 16 ? 2 : 1, QG = kFewOperands<IO, D>;    // groups of a key a lane, operands of each
    int *const pages = lds.pages;
    const KvView &kv = k.kv;
    const int pairs = kv.Hkv * k.a.B, split = block / pairs, pair = turned_pair(block, split, pairs), h = pair % kv.Hkv;
    const Seq s = sequence(k, pair / kv.Hkv);
    const int rows = s.n * k.G;
    if (rows > k.few_rows && k.tiles == 0 && k.slots > 1 && split == 0) left_out(k, s, h, 0, THREADS);
    if (rows == 0 || rows > k.few_rows) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;
    const int p0 = s.m - s.n, mask = (1 << kv.page_log) - 1;
    int pos[COLS], lowest[COLS];                                              // row 16 g + col sees the `span` keys from `lowest` on
    unsigned span[COLS];
    uint4 q[COLS > QG ? COLS : QG];
#pragma unroll
    for (int g = 0; g < COLS; ++g) {
        const int r = min(16 * g + col, rows - 1), token = r / k.G, head = h * k.G + (r - token * k.G);
        pos[g] = p0 + token;
        lowest[g] = k.a.window ? pos[g] - k.a.window + 1 : 0;
        span[g] = (unsigned)max(pos[g] - lowest[g] + 1, 0);
        const char *base = reinterpret_cast<const char *>(k.a.q) + ((s.from + token) * k.a.q_stride + head * D) * IO::kBytes;
#pragma unroll
        for (int j = 0; j < QG; ++j) {
            const uint4 *from = reinterpret_cast<const uint4 *>(base) + HALVES * (4 * (j / HALVES) + quarter) + j % HALVES;
            if constexpr (COLS == 1) q[j] = *from;
            else if ((g * QG + j) % WAVES == wave) lds.query[64 * (g * QG + j) + lane] = *from;
        }
    }
    // this workgroup's keys: whole steps of all waves
    const int lo = k.a.window ? max(0, p0 - k.a.window + 1) & ~63 : 0, hi = s.m;
    const int chunk = ((max(hi - lo, 0) + k.few_splits - 1) / k.few_splits + WAVES * SK - 1) / (WAVES * SK) * (WAVES * SK);
    const int begin = min(lo + (long long)split * chunk, (long long)hi), end = min(hi, begin + chunk);
    const int all_from = k.a.window ? p0 + s.n - 1 - k.a.window : -1;         // every row sees the keys above it ...
    const int all_pos = p0;                                                   // ... up to this one

    f32x4_t o[COLS][DT];
    float top[COLS], sum[COLS];
#pragma unroll
    for (int g = 0; g < COLS; ++g) {
        top[g] = -INFINITY;
        sum[g] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[g][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const float lag = kLag / k.c;
    const int koff = E == 8 ? PE * (col >> 2) + (col & 3) : col;              // this lane's key of a step (bf16: and the one 4 on, 8 bits: the three)
    const unsigned page_bytes = (unsigned)kv.Hkv * (D * IO::kPageBytes) << kv.page_log, head_bytes = (unsigned)h * (D * IO::kPageBytes) << kv.page_log;
    const unsigned k_at = head_bytes + ((quarter * 16u) << kv.page_log), k_next = 64u << kv.page_log, v_at = head_bytes + col * 16u;
    const unsigned P = (unsigned)kv.P;

    auto load = [](const char *p, auto stream) {
        if constexpr (decltype(stream)::value) return __builtin_bit_cast(uint4, stream_load(reinterpret_cast<const float4 *>(p)));
        else return *reinterpret_cast<const uint4 *>(p);
    };
    uint4 kr[KTILES * GROUPS], vr[DT];
    float k_scale = 1.f, v_scale = 1.f;
    int vpage = -1;
    // scale of the block of this lane's keys (which = 0) or values
    auto scale_at = [&](int page, int key, int which) {
        if constexpr (IO::kCoded) return kv.scales[2 * ((((long long)page * kv.Hkv + h) << (kv.page_log - kKvBlockLog)) + ((key & mask) >> kKvBlockLog)) + which];
        else return 1.f;
    };
    // sections of keys whose page numbers fit LDS
    const int keys_a_section = kSection << kv.page_log;
    for (int sec = begin; sec < end; sec += keys_a_section) {
        const int sec_end = min(end, sec + keys_a_section), first = sec >> kv.page_log, count = ((sec_end - 1) >> kv.page_log) - first + 1;
        __syncthreads();
        for (int i = threadIdx.x; i < count; i += THREADS) pages[i] = kv.table[(long long)s.row * kv.M + first + i];
        __syncthreads();
        auto page_at = [&](int key) { return key < sec_end ? pages[(key >> kv.page_log) - first] : -1; };
        auto request_keys = [&](int base) {
            const int key = base + koff, page = page_at(base + (E == 8 ? PE * (col >> 2) : col));    // keys at and behind the end lie in its page, or in none
            const char *kb = reinterpret_cast<const char *>(kv.k) + (unsigned long long)(unsigned)page * page_bytes + k_at + (key & mask) * 16u;
            auto all = [&](auto stream) {
#pragma unroll
                for (int j = 0; j < GROUPS; ++j)
#pragma unroll
                    for (int t = 0; t < KTILES; ++t) kr[t * GROUPS + j] = load(kb + j * k_next + 64 * t, stream);
                k_scale = scale_at(page, key, 0);
            };
            if (__ballot((unsigned)page < P) == ~0ull) {                          // nothing to choose, nothing to clear
                if (k.few_stream) all(std::true_type());
                else all(std::false_type());
                return;
            }
#pragma unroll
            for (int i = 0; i < KTILES * GROUPS; ++i) kr[i] = make_uint4(0, 0, 0, 0);
            if ((unsigned)page < P) all(std::false_type());
        };
        auto request_values = [&](int base) {
            const int key = base + PE * quarter;
            vpage = page_at(key);                                                 // a block of 16 that begins behind the end has no page here: its scale, which nobody has written, is not asked for
            const char *vb = reinterpret_cast<const char *>(kv.v) + (unsigned long long)(unsigned)vpage * page_bytes + v_at + ((key & mask) / PE) * (D * 16u);
            auto all = [&](auto stream) {
#pragma unroll
                for (int d = 0; d < DT; ++d) vr[d] = load(vb + 256 * d, stream);
                v_scale = scale_at(vpage, key, 1);
            };
            if (__ballot((unsigned)vpage < P) == ~0ull) {
                if (k.few_stream) all(std::true_type());
                else all(std::false_type());
                return;
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) vr[d] = make_uint4(0, 0, 0, 0);
            if ((unsigned)vpage < P) all(std::false_type());
        };
        // the next step's keys are requested as soon as the scores have used these, its values behind the product with these
        int base = sec + SK * wave;
        if (base < sec_end) {
            request_keys(base);
            request_values(base);
        }
        for (; base < sec_end; base += WAVES * SK) {
            const bool more = base + WAVES * SK < sec_end;
            const bool absent = (unsigned)vpage >= P;                             // this lane's run of E keys, whose scores and values it holds
            const bool edge = __ballot(absent) != 0 || base + SK - 1 > all_pos || base <= all_from;
            f32x4_t sc[COLS][KTILES];
#pragma unroll
            for (int t = 0; t < KTILES; ++t) {
#pragma unroll
                for (int g = 0; g < COLS; ++g) sc[g][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if constexpr (COLS == 1) {
#pragma unroll
                    for (int j = 0; j < QG; ++j) IO::mma16(sc[0][t], operand<IO>(kr[t * GROUPS + j / HALVES], j % HALVES, k_scale), q[j]);
                }
            }
            if constexpr (COLS > 1) {
                int at = lane;
                asm volatile("" : "+v"(at));                                  // opaque: not kept in registers from step to step
#pragma unroll
                for (int j = 0; j < QG; ++j) {
#pragma unroll
                    for (int g = 0; g < COLS; ++g) q[g] = lds.query[64 * (g * QG + j) + at];
#pragma unroll
                    for (int t = 0; t < KTILES; ++t) {
                        const uint4 key = operand<IO>(kr[t * GROUPS + j / HALVES], j % HALVES, k_scale);
#pragma unroll
                        for (int g = 0; g < COLS; ++g) IO::mma16(sc[g][t], key, q[g]);
                    }
                }
            }
            if (more) request_keys(base + WAVES * SK);
            uint4 pg[COLS][HALVES], rest[HALVES];
#pragma unroll
            for (int g = 0; g < COLS; ++g) {
                float p[4 * KTILES];
                if (edge) {
                    const unsigned at = (unsigned)(base + PE * quarter - lowest[g]);
#pragma unroll
                    for (int t = 0; t < KTILES; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (absent || at + (4 * t + e) >= span[g]) sc[g][t][e] = -INFINITY;
                }
                float mx = sc[g][0][0];
#pragma unroll
                for (int t = 0; t < KTILES; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mx = larger(mx, sc[g][t][e]);
                mx = max_halves(max_quarters(mx));
                if (__ballot(lags(mx, top[g], lag))) {
                    const float f = follow(mx, k.c, &top[g]);
                    sum[g] *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[g][d] *= f;
                }
                const float shift = shift_of(top[g], k.c);
#pragma unroll
                for (int t = 0; t < KTILES; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[4 * t + e] = exp2_fast(fmaf(sc[g][t][e], k.c, shift));
                        sum[g] += p[4 * t + e];
                    }
#pragma unroll
                for (int x = 0; x < HALVES; ++x) {
                    pg[g][x] = IO::pack(p + 8 * x);
                    if constexpr (E == 8 && COLS == 1) rest[x] = IO::pack_rest(p + 8 * x, pg[g][x]);
                }
            }
            // two terms of a probability may be of different signs, or one of them zero: infinite values go their own way in every step
            bool look = edge, odd = false;
            if constexpr (IO::kCoded) {
                uint32_t nans = 0;
#pragma unroll
                for (int d = 0; d < DT; ++d) nans |= IO::nan_bits(vr[d]);
                look = look || __ballot(nans != 0) != 0;
            } else if constexpr (E == 8) look = look || __ballot(!all_finite_bf16<DT>(vr)) != 0;
            if constexpr (IO::kCoded) {
                if (look) {
                    const int have = s.m - (base + PE * quarter);
                    bool fine = true;
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        if (have < PE) vr[d] = IO::keep_codes(vr[d], have);
                        if (IO::nan_bits(vr[d])) {
                            fine = false;
                            vr[d] = IO::finite_codes(vr[d]);
                        }
                    }
                    odd = __ballot(!fine) != 0;
                }
            } else if (look) {
                const int have = s.m - (base + E * quarter);
                bool fine = true;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    if (have < E) vr[d] = keep_first<IO>(vr[d], have);
                    if (!all_finite<IO>(vr[d])) {
                        fine = false;
                        vr[d] = finite_only<IO>(vr[d]);
                    }
                }
                odd = __ballot(!fine) != 0;
            }
#pragma unroll
            for (int x = 0; x < HALVES; ++x) {
                if constexpr (IO::kCoded) {
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const uint4 v = operand<IO>(vr[d], x, v_scale);
#pragma unroll
                        for (int g = 0; g < COLS; ++g) {
                            IO::mma16(o[g][d], v, pg[g][x]);
                            if constexpr (COLS == 1) IO::mma16(o[g][d], v, rest[x]);
                        }
                    }
                } else {
#pragma unroll
                    for (int d = 0; d < DT; ++d) IO::mma16(o[0][d], vr[d], pg[0][0]);
                    if constexpr (E == 8) {
#pragma unroll
                        for (int d = 0; d < DT; ++d) IO::mma16(o[0][d], vr[d], rest[0]);
                    }
                }
            }
            if (more) request_values(base + WAVES * SK);
            if (odd)
#pragma unroll
                for (int g = 0; g < COLS; ++g)
                    add_not_finite<IO, D, 4 * DT, (COLS > 1)>(kv, s, h, base, SK, pos[g], lowest[g] - 1, [quarter](int n) { return 16 * (n / 4) + 4 * quarter + n % 4; },
                                                  [&](int n, float y) { o[g][n / 4][n % 4] += y; });
        }
    }

    // the waves' results, joined in a fixed order
    // rows turned, no two in one bank; every pointer by its name, so that accesses stay LDS accesses
    auto place = [&](int w, int r, int c) { return ((w >> 2) + (r >> 4) * (WAVES / 4)) * kFewGroups<IO, D> + (r & 15) * (D / 4) + (c ^ (r & 15)); };
    constexpr int of_wave = COLS * kFewGroups<IO, D>;                         // several: one array, four waves
    static_assert(COLS == 1 || WAVES == 4, "outputs' places");
#pragma unroll
    for (int g = 0; g < COLS; ++g) {
        sum[g] += __shfl_xor(sum[g], 16, 64);
        sum[g] += __shfl_xor(sum[g], 32, 64);
        if (quarter == 0) {
            lds.tops[wave][16 * g + col] = top[g];
            lds.sums[wave][16 * g + col] = sum[g];
        }
    }
#pragma unroll
    for (int g = 0; g < COLS; ++g)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int at = place(wave, 16 * g + col, 4 * d + quarter), which = wave & 3;
            if constexpr (COLS > 1) lds.out0[of_wave * wave + at] = o[g][d];
            else if (which == 0) lds.out0[at] = o[g][d];
            else if (which == 1) lds.out1[at] = o[g][d];
            else if (which == 2) lds.out2[at] = o[g][d];
            else lds.out3[at] = o[g][d];
        }
    __syncthreads();
    for (int x = threadIdx.x; x < rows * (D / 4); x += THREADS) {
        const int r = x / (D / 4), c = 4 * (x % (D / 4));
        float best = lds.tops[0][r], total = 0.f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) best = fmaxf(best, lds.tops[w][r]);
        f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = lds.tops[w][r] == best ? 1.f : exp2_fast((lds.tops[w][r] - best) * k.c);
            const int at = place(w, r, c / 4);
            total += f * lds.sums[w][r];
            if constexpr (COLS > 1) y += f * lds.out0[of_wave * w + at];
            else y += f * ((w & 3) == 0 ? lds.out0[at] : (w & 3) == 1 ? lds.out1[at] : (w & 3) == 2 ? lds.out2[at] : lds.out3[at]);
        }
        const int token = r / k.G, head = h * k.G + (r - token * k.G);
        const long long at = (long long)(s.from + token) * k.a.H + head;
        if (k.slots > 1 && split == 0 && c == 0) k.count[at] = k.few_splits > 1 ? k.few_splits : 0;
        if (k.few_splits > 1) {
            long long place = at * k.slots;
            if (k.packed) {
                place = (k.few_tokens ? ((long long)(pair / kv.Hkv) * k.few_tokens + token) * k.a.H + head : at) * k.few_splits;
                if (split == 0 && c == 0) k.first[at] = (unsigned)place;
            }
            place += split;
            *reinterpret_cast<f32x4_t *>(k.part + place * D + c) = y;
            if (c == 0) k.stat[place] = make_float2(best * k.c, total);
        } else {
            const float inv = inverse(total);
            store4<IO>(k.a.out, at * D + c, make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv));
            if (k.a.lse && c == 0) k.a.lse[at] = lse_of(best * k.c, total);
        }
    }
}

// ---------------------------------------------------------------- the launches: either kind, or both for a mixed batch
template <typename IO, int D, int COLS>
__global__ __launch_bounds__(256, COLS > 2 && D == 128 ? 1 : COLS > 1 ? 2 : D == 64 ? 4 : IO::kCoded ? 2 : 3) void k_attend_few(AttendK k) {
    __shared__ int pages[kSection + 2];
    __shared__ float tops[4][16 * COLS], sums[4][16 * COLS];
    __shared__ f32x4_t outs[4][kFewGroups<IO, D> * COLS];
    __shared__ uint4 query[kFewQueries<IO, D, COLS> ? kFewQueries<IO, D, COLS> : 1];
    few_rows<IO, D, 4, COLS>(k, blockIdx.x, FewLds<16 * COLS>{pages, tops, sums, outs[0], outs[1], outs[2], outs[3], query});
}

// Waves a SIMD that registers (and, of workgroups of four waves with pages of 8 bits, LDS) leave room for.
template <typename IO, int D, int WAVES>
constexpr int tile_waves_a_simd() { return IO::E == 8 && D == 64 ? (IO::kCoded && WAVES == 4 ? 3 : 4) : 2; }

template <typename IO, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (tile_waves_a_simd<IO, D, WAVES>())) void k_attend_tile(AttendK k) {
    __shared__ uint4 sk0[kTileGroups<IO, D>], sv0[kTileGroups<IO, D>], sk1[kTileGroups<IO, D>], sv1[kTileGroups<IO, D>];
    __shared__ uint4 raw[kRawGroups<IO, D> ? kRawGroups<IO, D> : 1], query[kQueryGroups<IO, D, WAVES> ? kQueryGroups<IO, D, WAVES> : 1];
    __shared__ int odd[3];
    tile_of_rows<IO, D, WAVES>(k, blockIdx.x, TileLds{sk0, sv0, sk1, sv1, raw, query, odd});
}

// The tiles of a batch's prompts, which arithmetic bounds, and behind them its single tokens, which memory bounds, where the tiles leave compute units free (before
// them, or dealt out evenly: 32 ragged sequences 258 and 261 instead of 234 us; two launches 310).
template <typename IO, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (tile_waves_a_simd<IO, D, WAVES>())) void k_attend_mixed(AttendK k) {
    __shared__ uint4 sk0[kTileGroups<IO, D>], sv0[kTileGroups<IO, D>], sk1[kTileGroups<IO, D>], sv1[kTileGroups<IO, D>];
    __shared__ uint4 raw[kRawGroups<IO, D> ? kRawGroups<IO, D> : 1], query[kQueryGroups<IO, D, WAVES> ? kQueryGroups<IO, D, WAVES> : 1];
    __shared__ int odd[3], pages[kSection + 2];
    __shared__ float tops[WAVES][16], sums[WAVES][16];
    static_assert(kTileGroups<IO, D> >= (WAVES / 4) * kFewGroups<IO, D>, "outputs of few rows fit where tiles lie");
    const int tiles = (k.tile_blocks + 7) & ~7, block = blockIdx.x;              // eights again, for the XCDs
    if (block >= tiles) {
        few_rows<IO, D, WAVES, 1>(k, block - tiles, FewLds<16>{pages, tops, sums, reinterpret_cast<f32x4_t *>(sk0), reinterpret_cast<f32x4_t *>(sv0), reinterpret_cast<f32x4_t *>(sk1),
                                                        reinterpret_cast<f32x4_t *>(sv1), nullptr});
    } else if (block < k.tile_blocks) {
        tile_of_rows<IO, D, WAVES>(k, block, TileLds{sk0, sv0, sk1, sv1, raw, query, odd});
    }
}

// ---------------------------------------------------------------- splits joined
// D / 4 lanes hold a row's channels; GROUPS such groups of a workgroup share the parts of one row.  Many rows have a group each; few rows (and then many
// parts) a workgroup each, where what counts is that all loads are on their way at once: the first parts' before the row's own number of them is known, as the
// row has room for the launch's largest number (with the number found first, from the row's sequence: one sequence of 32700 tokens 20.2 instead of 18.9 us in all,
// 16 windows of 5 tokens over 9000, d = 128, 36.7 instead of 34.0).
template <typename IO, int D, int GROUPS>
__global__ __launch_bounds__(256) void k_attend_join(AttendK k) {
    constexpr int LANES = D / 4, ROWS = 256 / (LANES * GROUPS), AT_ONCE = 4;
    __shared__ f32x4_t so[GROUPS > 1 ? GROUPS : 1][LANES];
    __shared__ float2 st[GROUPS > 1 ? GROUPS : 1];
    const int c = threadIdx.x % LANES, g = threadIdx.x / LANES % GROUPS;
    const long long rows = (long long)k.a.T * k.a.H, mine = (long long)blockIdx.x * ROWS + threadIdx.x / (LANES * GROUPS), row = min(mine, rows - 1);
    int splits = min(k.count[row], k.slots);
    if (mine >= rows || (int)(row / k.a.H) >= k.a.start[k.a.B]) splits = 0;    // behind the last sequence nothing was written
    long long place = row * k.slots;
    if (k.packed) {
        place = splits > 0 ? k.first[row] : 0;
        if (place + splits > k.few_places + k.tile_places) splits = 0;         // a row that no sequence has
    }
    const int last = (GROUPS > 1 && !k.packed ? k.slots : splits) - 1;
    const float2 *stat = k.stat + place;
    const float *part = k.part + place * D + 4 * c;
    float best = -INFINITY, total = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    int from = g;
    do {
        float2 x[AT_ONCE];
        f32x4_t y[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int s = from + i * GROUPS;
            x[i] = make_float2(0.f, 0.f);
            y[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (s <= last) {
                x[i] = stat[s];
                y[i] = *reinterpret_cast<const f32x4_t *>(part + (long long)s * D);
            }
        }
        float higher = best;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            if (from + i * GROUPS >= splits) x[i].y = 0.f;
            if (x[i].y != 0.f) higher = fmaxf(higher, x[i].x);                // a part whose sum is zero saw nothing and wrote nothing
        }
        if (higher != best) {
            const float f = exp2_fast(best - higher);
            total *= f;
            o *= f;
            best = higher;
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
            if (x[i].y != 0.f) {
                const float f = x[i].x == best ? 1.f : exp2_fast(x[i].x - best);
                total += f * x[i].y;
                o += f * y[i];
            }
        from += AT_ONCE * GROUPS;
    } while (from < splits);
    if constexpr (GROUPS > 1) {
        so[g][c] = o;
        if (c == 0) st[g] = make_float2(best, total);
        __syncthreads();
        if (g) return;
        for (int i = 1; i < GROUPS; ++i) best = fmaxf(best, st[i].x);
        total = 0.f;
        o = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < GROUPS; ++i) {
            const float2 x = st[i];
            if (x.y == 0.f) continue;
            const float f = x.x == best ? 1.f : exp2_fast(x.x - best);
            total += f * x.y;
            o += f * so[i][c];
        }
    }
    if (splits <= 0) return;
    const float inv = inverse(total);
    store4<IO>(k.a.out, row * D + 4 * c, make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv));
    if (k.a.lse && c == 0) k.a.lse[row] = lse_of(best, total);
}

}  // namespace

hipError_t load_kernels_attend() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, reinterpret_cast<const void *>(k_attend_join<Bf16Mma, 64, 1>));
}

// Up to this many rows a joining workgroup has one row, beyond it a row for each D / 4 lanes: 512 rows of 16 parts and more 17.3 instead of 19.6 us, the windows' 1280
// 34.0 instead of 36.9; 4096 of eight 64.2 where workgroups of their own take 67.9 (with the attention before them).
constexpr long long kWideRows = 2048;
// Where the sequences differ, the longest must not be one workgroup's work for as long as the others take together; every part costs its rows once through
// memory: 32 sequences of up to 512 new and 8500 tokens in all take 237 us with parts of 4096 keys, 245 with 2048, 248 with 8192.  Batches of many times more
// tiles than run at once even out by themselves: 48 of up to 2000 new tokens 825 with 8192, 887 with 4096.
constexpr long long kRaggedKeys = 4096;
constexpr long long kStreamBytes = 96ll << 20;
constexpr long long kMostThreads = (1ll << 32) - 1;
// Partial results: a place for every part of every row up to this many bytes (or to what sharing would take); beyond it rows of tiles share five places for two rows, or half as
// many bytes if that is more, and few rows have as many parts as this many bytes hold.  One chunk of 8192 tokens beside 31 decoding sequences, lengths of up to 131072,
// 32 heads, d = 128: 0.5 GB, where a place for every part would be 8.8.  Sharing is free until parts have to become longer (32 sequences of up to 1500 new tokens over
// 36000, 0.2 instead of 1.7 GB: 1885 us, before 1880; 40 over 20000, 0.4 instead of 1.6 GB: 1684, before 1672); then it costs the even end of the launch (20 of up to
// 4000 over 60000, d = 128, 0.4 instead of 4.6 GB: 7102, before 6786).
constexpr long long kPartBytes = 256ll << 20;

AttendPlan attend_plan(int d, int dtype, int B, int T, int H, int Hkv, int max_new, int max_len, int window) {
    AttendPlan p{};
    p.fits = true;
    if (T == 0 || B == 0) return p;                                // nothing to launch
    const int G = H / Hkv;
    max_new = std::min(max_new, T);
    const long long rows = (long long)max_new * G;
    const bool even = T == (long long)B * max_new;                 // every sequence has max_new tokens
    const long long len = window ? std::min<long long>(max_len, (long long)window + max_new) : max_len;
    // Up to 16 rows (pages of 8 bits: 64 or 48) need no tile.  Beyond, one tile does for the few rows of a mixed batch too (23 sequences of up to 5 tokens, 8 heads a key head: 39 instead of 73 us) until
    // the tiles of the others make it long.
    const int few_most = dtype == SPECTRE_E4M3 ? (d == 64 ? 64 : 48) : 16;
    p.few = rows <= few_most || (!even && G <= 16 && rows > 128);
    p.tile = rows > few_most;
    p.few_rows = !p.few ? 0 : p.tile ? 16 : (int)rows;
    p.few_splits = p.tile_splits = 1;
    const long long pairs = (long long)B * Hkv, place = 4 * d + 8;         // bytes of a part's results
    p.few_tokens = p.tile && p.few && (long long)B * (16 / G) < T ? 16 / G : 0;
    const long long few_rows = (long long)H * (p.few_tokens ? (long long)B * p.few_tokens : T);
    if (p.few) {
        // two workgroups a compute unit of at least 256 keys each: four of 128 cost the join what they gain (one sequence of 32700 tokens 21.9 instead of
        // 19.8 us, 64 of 2000, which need no join then, 48 instead of 43), one leaves the memory waiting (16 fp32 sequences of 4000: 52.7 instead of 47.5).
        // No part longer than 2048 keys, for sequences of different lengths (32 of up to 32768: 202 us, with 4096 205).
        long long s = std::max(p.few_rows > 16 ? 256 / pairs : (512 + pairs - 1) / pairs, (len + 2047) / 2048);
        // More than 16 rows without a tile: one workgroup a compute unit (48 sequences of 60 rows over 560 keys 15.6 us, with two 18.7; 4 of 24 over 8000, d = 128, 18.6 and
        // 20.0).  Few rows beside tiles have their two: they are a launch's last workgroups, and longer parts its tail (a chunk of 300 and 31 tokens over 2000 70.0 us, with
        // half the parts 80.6, fp32 119 and 143, pages of 8 bits 50.8 and 54.7; one of 2048 and three over 8192 191 and 187).
        s = std::min(s, (len + 255) / 256);
        s = std::min(s, std::max((512 + pairs - 1) / pairs, kPartBytes / (few_rows * (place + 4))));
        p.few_splits = (int)std::max(1ll, std::min(s, 256ll));
    }
    if (p.tile) {
        auto groups = [&](int waves) {
            const long long tiles = (rows + 32 * waves - 1) / (32 * waves), filled = ((long long)T * G + 32 * waves - 1) / (32 * waves);
            return Hkv * (even ? B * tiles : std::max(1ll, std::min(B * tiles, filled)));
        };
        // 256 rows a workgroup halve the keys' way through LDS (8192-token prompt, d = 128: 281 instead of 304 us); with fewer than a workgroup a compute unit
        // 128 fill the card better (512 tokens over 16000, d = 128: 88 instead of 100 us; a ragged fp32 batch 155 instead of 167), but half a workgroup is enough
        // where many keys are left to split (2048 over 28672, d = 128: 494 instead of 518 us; a 1024-token prompt of its own would lose, 44 instead of 34).
        // A ragged fp32 batch has 128: its products take longer than the keys' way.
        // So have rows that fit 128 (256 sequences of 32 tokens 30 instead of 37 us, 90 of 16 over 1000, d = 128, 41 instead of 54).
        const bool slow = dtype == SPECTRE_F32 && !even && rows > 128;
        p.tile_waves = groups(8) >= (even && len >= 8192 ? 128 : 256) && !slow && rows > 128 ? 8 : 4;
        p.tiles = (int)((rows + 32 * p.tile_waves - 1) / (32 * p.tile_waves));
        // workgroups that run at once, by their registers and LDS; keys are split where rows leave some of them free.  Of single tiles, which memory bounds, two a
        // compute unit are enough: the join costs more than a third and fourth gain (64 sequences of 8 tokens over 2000 48 instead of 55 us, 16 over 9000 53 instead
        // of 58; one a compute unit: 50 and 73).
        const long long slots = p.tile_waves == 8 || d == 128 || (rows <= 128 && dtype != SPECTRE_E4M3) ? 512 : dtype == SPECTRE_BF16 ? 1024 : 768;
        // Pages of 8 bits leave LDS for three workgroups of four waves a compute unit: 13 ragged sequences 47 us, with 1024 59, with 512 55; 7 of 17 tokens over 17721 60.0, with 512 63.4.
        // Parts of the longest sequence; the others' parts are as long.  With several tiles a sequence of a ragged batch they take different times, and
        // twice the parts even them out (fp32 batch of up to 397 new tokens 135 instead of 142 us; single tiles, bound by memory, lose: 25.0 -> 28.8).
        const long long all = groups(p.tile_waves), keys = all > 4 * slots ? 2 * kRaggedKeys : kRaggedKeys;
        long long s = std::max(1ll, (even || rows <= 128 ? 1 : 2) * slots / all);
        // fp32: four times, as long as parts have 768 keys or more (24 sequences of up to 300 new and 4300 tokens, 32 heads, d = 64: 428 us, with 1024 keys or more 459, with
        // 256 rows and twice the parts 535; 12 of up to 1500 new: 150, with parts down to 500 keys 160; bf16 with four times 133 instead of 111).
        if (slow) s = std::max(s, std::min(4 * slots / all, len / 768));
        if (!even) s = std::max(s, (len + keys - 1) / keys);
        s = std::max(1ll, std::min({s, len / 256, 64ll}));
        p.tile_splits = (int)s;
    }
    // A launch has fewer than 2^32 threads: batches of loose bounds get fewer parts, and what is too large even so none at all.
    const long long threads = p.tile ? 64 * p.tile_waves : 256;
    auto blocks = [&]() { return pairs * ((p.few ? p.few_splits : 0) + (long long)p.tile_splits * p.tiles) + 8; };
    while (blocks() * threads > kMostThreads && (p.few_splits > 1 || p.tile_splits > 1)) {
        p.few_splits = (p.few_splits + 1) / 2;
        p.tile_splits = (p.tile_splits + 1) / 2;
    }
    if ((long long)T * H * (d / 4) + 256 > kMostThreads) p.few_splits = p.tile_splits = 1;       // no join
    p.fits = blocks() * threads <= kMostThreads;
    p.part_keys = (int)((len + p.tile_splits - 1) / p.tile_splits);
    const long long most = std::max(p.few_splits, p.tile_splits), rows_all = (long long)T * H;
    if (most == 1) return p;
    const long long few = p.few_splits > 1 ? few_rows * p.few_splits : 0;
    const long long tile = p.tile_splits > 1 ? std::min(rows_all * p.tile_splits, std::max(5 * rows_all / 2, kPartBytes / 2 / place)) : 0;
    const long long all = rows_all * (most * place + 4), shared = (few + tile) * place + 8 * rows_all;
    p.packed = all > std::max(kPartBytes, shared);
    p.few_places = p.packed ? few : 0;
    p.tile_places = p.packed ? tile : rows_all * most;
    p.partial_bytes = (size_t)(p.packed ? shared : all);
    return p;
}

template <typename IO, int D>
void launch_mixed(int waves, int blocks, const AttendK &k, hipStream_t st) {
    if constexpr (IO::E == 8) {                    // the plan gives a ragged fp32 batch 128 rows
        if (waves == 8) {
            k_attend_mixed<IO, D, 8><<<blocks, 512, 0, st>>>(k);
            return;
        }
    }
    k_attend_mixed<IO, D, 4><<<blocks, 256, 0, st>>>(k);
}

template <typename IO, int D>
void launch_few(const AttendK &k, hipStream_t st) {
    if constexpr (IO::kCoded) {
        if (k.few_rows > 16) {
            if (k.few_rows <= 32) k_attend_few<IO, D, 2><<<k.few_blocks, 256, 0, st>>>(k);
            else if (k.few_rows <= 48) k_attend_few<IO, D, 3><<<k.few_blocks, 256, 0, st>>>(k);
            else if constexpr (D == 64) k_attend_few<IO, D, 4><<<k.few_blocks, 256, 0, st>>>(k);
            return;
        }
    }
    k_attend_few<IO, D, 1><<<k.few_blocks, 256, 0, st>>>(k);
}

hipError_t launch_attend(const KvView &kv, int layers, int d, int io, const AttendArgs &a, const AttendPlan &p, void *ws, hipStream_t st) {
    AttendK k;
    k.kv = kv;
    k.a = a;
    k.G = a.H / kv.Hkv;
    k.few_rows = p.few_rows;
    k.part_keys = p.part_keys;
    k.tiles = p.tiles;
    k.c = a.scale * kLog2E;
    const size_t places = (size_t)(p.few_places + p.tile_places);
    k.slots = std::max(p.few_splits, p.tile_splits);
    k.packed = p.packed;
    k.few_tokens = p.few_tokens;
    k.few_places = p.few_places;
    k.tile_places = p.tile_places;
    k.part = (float *)ws;
    k.stat = (float2 *)((char *)ws + places * d * 4);
    k.count = (int *)(k.stat + places);
    k.first = (unsigned *)(k.count + (size_t)a.T * a.H);
    const bool stream = 2 * kv.layer_bytes * layers > kStreamBytes;
    k.few_splits = p.few_splits;
    k.tile_splits = p.tile_splits;
    k.few_stream = stream;
    k.tile_stream = stream && p.tiles == 1;        // with several tiles of rows a tile of keys is read as often
    const int pairs = a.B * kv.Hkv;
    k.few_blocks = pairs * p.few_splits;
    k.tile_blocks = pairs * p.tile_splits * p.tiles;
    // rows' type and the pages'
    const bool coded = kv.layer_scales != 0;
#define SPECTRE_ATTEND_DISPATCH(CALL)                                 \
    if (coded && d == 64) { CALL(E4m3Mma, 64); }                      \
    else if (coded) { CALL(E4m3Mma, 128); }                           \
    else if (io == SPECTRE_BF16 && d == 64) { CALL(Bf16Mma, 64); }    \
    else if (io == SPECTRE_BF16) { CALL(Bf16Mma, 128); }              \
    else if (d == 64) { CALL(F32Mma, 64); }                           \
    else { CALL(F32Mma, 128); }
    if (p.few && p.tile) {
        const int blocks = ((k.tile_blocks + 7) & ~7) + k.few_blocks;
#define CALL(IO, D) launch_mixed<IO, D>(p.tile_waves, blocks, k, st)
        SPECTRE_ATTEND_DISPATCH(CALL)
#undef CALL
    } else if (p.few) {
#define CALL(IO, D) launch_few<IO, D>(k, st)
        SPECTRE_ATTEND_DISPATCH(CALL)
#undef CALL
    } else {
#define CALL(IO, D)                                                                        \
    if (p.tile_waves == 8) k_attend_tile<IO, D, 8><<<k.tile_blocks, 512, 0, st>>>(k);      \
    else k_attend_tile<IO, D, 4><<<k.tile_blocks, 256, 0, st>>>(k)
        SPECTRE_ATTEND_DISPATCH(CALL)
#undef CALL
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.few_splits > 1 || p.tile_splits > 1) {
        const long long rows = (long long)a.T * a.H;
#define CALL(IO, D)                                                                                                             \
    if (rows <= kWideRows) k_attend_join<IO, D, 1024 / D><<<(int)rows, 256, 0, st>>>(k);                                        \
    else k_attend_join<IO, D, 1><<<(int)((rows + 1024 / D - 1) / (1024 / D)), 256, 0, st>>>(k)
        if (io == SPECTRE_BF16 && d == 64) { CALL(Bf16Mma, 64); }
        else if (io == SPECTRE_BF16) { CALL(Bf16Mma, 128); }
        else if (d == 64) { CALL(F32Mma, 64); }
        else { CALL(F32Mma, 128); }
#undef CALL
    }
    return hipGetLastError();
}

}  // namespace spectre
