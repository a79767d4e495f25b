// Attention over the paged 4-bit cache (apnn_kv_attention).
//
// Scores are computed transposed, S^T = K Q^T: the 16 x 16 matrix instruction then leaves a lane with scores of one query
// row (its column) and, in groups of four, of tokens that are the contraction index of O^T = V^T P^T.  P goes from one
// instruction to the next in its registers; only V has to change places, which it does on its way through LDS
// (ds_read_b64_tr_b16).  A 4-bit group with its power of two is exact in 16 bits, so the conversion
// (v_cvt_scalef32_pk_*_fp4, two values an instruction) costs no accuracy: keys take the queries' type, values fp16.
#include "kv_cache.h"
#include "lane_util.h"
#include "lds_load.h"

namespace apnn {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

struct AttentionArgs {
    apnn_kv_attention_desc d;
    apnn_kv_cache c;
    float *parts;                                         // workspace
    int64_t tiles;                                        // tiles of max_q * group rows
    int page_shift, group;                                // query heads to a cache head
    int splits, part_rows;                                // of a tile's tokens; rows of a tile that there can be
    int tile_rows;                                        // 16 or 128
};

// 16-bit operand types of the scores
template <class T> struct Operand;
template <> struct Operand<_Float16> {
    typedef half8_t vec;
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 0>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, 0)); }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 1>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, 1)); }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 2>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, 2)); }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 3>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, 3)); }
    static __device__ __forceinline__ uint32_t bits(half2_t v) { return __builtin_bit_cast(uint32_t, v); }
    static __device__ __forceinline__ f32x4_t product(vec a, vec b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16_t product(vec a, vec b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<__bf16> {
    typedef bf16x8_t vec;
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 0>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0)); }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 1>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1)); }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 2>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2)); }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 3>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3)); }
    static __device__ __forceinline__ uint32_t bits(bf16x2_t v) { return __builtin_bit_cast(uint32_t, v); }
    static __device__ __forceinline__ f32x4_t product(vec a, vec b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16_t product(vec a, vec b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// Eight 4-bit codes -> eight operands.
template <class T> __device__ __forceinline__ u32x4_t values8(uint32_t w, float unit)
{
    using I = Operand<T>;
    return u32x4_t{I::two(w, unit, std::integral_constant<int, 0>{}), I::two(w, unit, std::integral_constant<int, 1>{}),
                   I::two(w, unit, std::integral_constant<int, 2>{}), I::two(w, unit, std::integral_constant<int, 3>{})};
}

// A row's scale as the conversions take it; 255 stands for NaN there too.
__device__ __forceinline__ float unit_of(uint32_t byte) { return __uint_as_float(byte << 23); }
// Values': no more than the largest power of two that a value has, whatever the byte, so that the weight 0 of an unseen token leaves nothing of it.
__device__ __forceinline__ float value_unit_of(uint32_t byte) { return unit_of(min(byte, 140u)); }

// A quarter's share of a row: channels [D / 4 * quarter, + D / 4).  In a matrix instruction lane l has quarter l / 16 of token
// l % 16; loaded neighbours lie side by side in the cache, lane l with quarter l % 4 of token l / 4.
template <int D> struct Share {
    static constexpr int words = D / 32;                  // 32-bit words of codes
    static constexpr int units = D == 96 || D == 256 ? 2 : 1;             // groups of 32 channels it reaches into
    static __device__ __forceinline__ int unit(int quarter, int word) { return (quarter * (D / 4) + 8 * word) / 32 - quarter * (D / 4) / 32; }
};
template <int D> struct Codes { uint32_t w[Share<D>::words]; };

// A share to LDS and back (word by word: a copy of the whole would keep it in memory).
template <int D> __device__ __forceinline__ void put_codes(char *to, const Codes<D> &c)
{
    if constexpr (D % 128 == 0)
#pragma unroll
        for (int s = 0; s < Share<D>::words; s += 4) *reinterpret_cast<u32x4_t *>(to + 4 * s) = u32x4_t{c.w[s], c.w[s + 1], c.w[s + 2], c.w[s + 3]};
    else
#pragma unroll
        for (int s = 0; s < Share<D>::words; ++s) *reinterpret_cast<uint32_t *>(to + 4 * s) = c.w[s];
}
template <int D> __device__ __forceinline__ void take_codes(const char *from, Codes<D> &c)
{
    if constexpr (D % 128 == 0)
#pragma unroll
        for (int s = 0; s < Share<D>::words; s += 4) {
            const u32x4_t w = *reinterpret_cast<const u32x4_t *>(from + 4 * s);
#pragma unroll
            for (int j = 0; j < 4; ++j) c.w[s + j] = w[j];
        }
    else
#pragma unroll
        for (int s = 0; s < Share<D>::words; ++s) c.w[s] = *reinterpret_cast<const uint32_t *>(from + 4 * s);
}

// Keys and values of 32 tokens as they lie in the cache.
template <int D> struct Fetched {
    Codes<D> k[2], v[2];
    uint8_t ku[2][Share<D>::units], vu[2][Share<D>::units];
    bool there[2];                                        // the page of these 16 tokens is one of the cache
};

// Bytes between rows of values in LDS: 32 more than the values, so that eight rows cover all banks.
template <int D> constexpr int kValueRow = 2 * D + 32;

// Over the four lanes that share a column (lane ^ 16, lane ^ 32).
__device__ __forceinline__ float column_max(float x)
{
    u32x2_t y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
    y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// Two queries times the scale's sign, -1, 0 or 1: exact, and 0 makes NaN of what is not finite.  The scores' factor is then positive, in powers of
// two: with 0 there, an unseen token's -inf would become NaN.
template <class T> __device__ __forceinline__ uint32_t times_sign(uint32_t w, float sign);
template <> __device__ __forceinline__ uint32_t times_sign<_Float16>(uint32_t w, float sign)
{
    const _Float16 s = static_cast<_Float16>(sign);
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, w) * half2_t{s, s});
}
template <> __device__ __forceinline__ uint32_t times_sign<__bf16>(uint32_t w, float sign)
{
    const bf16x2_t x = __builtin_bit_cast(bf16x2_t, w);
    return __builtin_bit_cast(uint32_t, bf16x2_t{static_cast<__bf16>(static_cast<float>(x[0]) * sign), static_cast<__bf16>(static_cast<float>(x[1]) * sign)});
}
__device__ __forceinline__ float sign_of(float scale) { return scale == 0.0f ? 0.0f : copysignf(1.0f, scale); }
__device__ __forceinline__ float factor_of(float scale)
{
    const float f = scale == 0.0f ? 1.0f : fabsf(scale) * 1.4426950408889634f;
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(f)));        // (one for the wave: a scalar register)
}

// What a block works on: 16 or 128 rows (queries x the heads that share a cache head, heads inside) of one sequence and cache head.
struct Rows {
    int64_t q0;                                           // first query row of the sequence
    int n, all, have;                                     // its queries, at most max_q of them and all; its tokens that the table can name
    int shift;                                            // query i sees have' = min(have, shift + i + 1) tokens
    int r0;                                               // first row of the tile
    int most;                                             // tokens that any of the rows sees
    bool any;
};

__device__ __forceinline__ int seen_by(const Rows &x, int i) { return min(max(x.shift + i + 1, 0), x.have); }

__device__ __forceinline__ Rows find_rows(const AttentionArgs &a, int64_t b, int64_t tile)
{
    Rows x = {};
    int64_t n = 1;
    x.q0 = b;
    if (a.d.q_start_dev) {
        x.q0 = a.d.q_start_dev[b];
        n = a.d.q_start_dev[b + 1] - x.q0;
    }
    if (x.q0 < 0 || x.q0 > a.d.tokens) return x;
    n = n < a.d.tokens - x.q0 ? n : a.d.tokens - x.q0;
    x.all = static_cast<int>(n);
    x.n = static_cast<int>(n < a.d.max_q ? n : a.d.max_q);
    if (tile * a.tile_rows >= int64_t(x.n) * a.group) return x;
    x.any = true;
    x.r0 = static_cast<int>(tile * a.tile_rows);
    const int len = a.d.len_dev[b], room = static_cast<int>(a.d.max_pages << a.page_shift);
    x.have = min(max(len, 0), room);
    x.shift = max(len, 0) - x.all;
    const int last = min((x.r0 + a.tile_rows - 1) / a.group, x.n - 1);
    x.most = seen_by(x, last);
    return x;
}

// The maximum of a row of which no weight is left, over the tokens from `begin` up to `end`: -inf if it sees none of them, and a number below every
// other if one is in a page of the cache (its scores are then all -inf: infinite queries, sums out of range).  A row of which -inf is the maximum of
// all its parts gets zeros, one whose weights sum to 0 all the same NaN.  The loops over tokens need not know; this is looked up behind them.
__device__ __forceinline__ float top_of_nothing(const AttentionArgs &a, int64_t seq, int begin, int end)
{
    for (int p = begin >> a.page_shift; p << a.page_shift < end; ++p) {
        const int page = a.d.page_dev[seq * a.d.max_pages + p];
        if (page >= 0 && page < a.c.pages) return -3.402823466e38f;
    }
    return -INFINITY;
}

// Tile, cache head and sequence of a block.  Heads and sequences change fastest: blocks go to the eight XCDs in turn, so that the
// tiles of one head find its codes in the L2 of the same XCD as long as heads x seqs is a multiple of 8; the tiles that see the
// most tokens come first.
struct Place {
    int64_t tile, seq;
    int head;
};
__device__ __forceinline__ Place place_of(const AttentionArgs &a, int64_t unit)
{
    const int64_t pairs = a.d.seqs * a.c.heads, turn = quotient(unit, pairs), pair = unit - turn * pairs, seq = quotient(pair, a.c.heads);
    return {a.tiles - 1 - turn, seq, static_cast<int>(pair - seq * a.c.heads)};
}

// A sequence's page numbers, by scalar loads (no kernel writes a page table).
typedef const __attribute__((address_space(4))) int32_t *PageTable;
__device__ __forceinline__ PageTable table_of(const AttentionArgs &a, int64_t seq)
{
    return reinterpret_cast<PageTable>(reinterpret_cast<uintptr_t>(a.d.page_dev + seq * a.d.max_pages));
}

// The maximum that weights refer to moves only when a score exceeds it by this, in powers of two: fp16 weights and fp32 sums have
// room for it, and accumulators are rarely rescaled.
constexpr float kSlack = 8.0f;

// Weights are 2^(score - maximum + kLift): at most 2^15, which fp16 holds, and as far above fp16's smallest step as that allows.  A weight
// keeps fp16's 11 bits down to 2^-21 of the largest one and is lost only below 2^-32 of it; without the lift, 2^-14 and 2^-25, tokens
// 17 nats below a single large one lost 44 % and at 17.4 everything, however many they were.  Weights' sums have the same factor.
//
// One fp16 number a weight: its rounding weighs as much as an fp16 result's own (rms error 2.9e-4 of the result, 2.05e-4 with exact
// weights) and an eighth of a bf16 result's.  What it leaves in a second fp16 number and a second product makes the error that of exact
// weights, but 48 x 8192 tokens take 65.1 us instead of 62.9, 2 x 131072 27.6 instead of 26.7, 1 x 500 5.92 instead of 5.64 and prompts 300
// instead of 223.
constexpr float kLift = 7.0f;

// Tokens of a split: a tile's tokens over `splits`, whole turns of the block's waves, and no fewer than pay for the joining.
constexpr int kTurn = 128, kLeastSplit = 256;
__host__ __device__ __forceinline__ int split_tokens(int most, int splits)
{
    const int each = ((most + splits - 1) / splits + kTurn - 1) / kTurn * kTurn;
    return each < kLeastSplit ? kLeastSplit : each;
}

// Parts of a tile's rows in the workspace: [tile of tiles x heads x seqs][split][row] of D sums, then maximum and sum of weights.
template <int D> __device__ __forceinline__ float *part_of(const AttentionArgs &a, int64_t unit, int split, int row)
{
    return a.parts + ((unit * a.splits + split) * a.part_rows + row) * (D + 4);
}

// 16 query rows of one cache head against one split of the sequence, the four waves taking 32 tokens each in turn.
//
// Bound by memory: (D / 2 + D / 32) 2 bytes a token and cache head.  Of codes not read just before, 103 MB take 25.8 us and 242 MB in contexts of
// every length up to 8192 58 (4.0, 4.2 TB/s); 430 to 860 MB in contexts of one length 4.7 to 5.3 TB/s.  A wave has the next 32 tokens' codes in flight, in
// registers, while it works on the current ones, and the page numbers of the 32 after those; four blocks of four waves fit
// a compute unit, 70 KB in flight.  LDS is only the way V is transposed, private to a wave: no barrier before the end.
template <class T, int D, bool SPLIT> __global__ __launch_bounds__(256, D == 256 ? 2 : 4) void kv_attention_kernel(AttentionArgs a, int64_t first)
{
    using Op = Operand<T>;
    constexpr int steps = D / 32, tokens = 32;
    constexpr int wave_bytes = tokens * kValueRow<D> > 64 * D ? tokens * kValueRow<D> : 64 * D;
    __shared__ alignas(16) char lds[4][wave_bytes];
    __shared__ float row_max[4][16], row_sum[4][16];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, quarter = lane >> 4;
    const int64_t id = first + blockIdx.x, unit = SPLIT ? quotient(id, a.splits) : id;
    const int split = SPLIT ? static_cast<int>(id - unit * a.splits) : 0;
    const Place place = place_of(a, unit);
    const int64_t b = place.seq;
    const int head = place.head;
    const Rows x = find_rows(a, b, place.tile);
    if (!x.any) return;
    int begin = 0, end = x.most;
    if (SPLIT) {
        const int each = split_tokens(x.most, a.splits);
        if (split && static_cast<int64_t>(split) * each >= x.most) return;
        begin = split * each;
        end = min(begin + each, x.most);
    }

    const int r = x.r0 + c, i = r / a.group;
    const bool live = i < x.n;
    // tokens that the row sees, from the first that a lane has scores of on; all rows see the tokens before `least`
    const int seen = (live ? seen_by(x, i) : 0) - 4 * quarter, least = seen_by(x, x.r0 / a.group);
    typename Op::vec q[steps];
    {
        const int qh = head * a.group + (live ? r - i * a.group : 0);
        const T *src = static_cast<const T *>(a.d.q_dev) + (x.q0 + (live ? i : 0)) * a.d.q_token_stride + qh * a.d.q_head_stride + quarter * (D / 4);
        const float sign = sign_of(a.d.scale);
#pragma unroll
        for (int s = 0; s < steps; ++s) {
            u32x4_t w;
            __builtin_memcpy(&w, src + 8 * s, 16);        // (however they are aligned)
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = times_sign<T>(w[j], sign);
            q[s] = __builtin_bit_cast(typename Op::vec, w);
        }
    }
    const float factor = factor_of(a.d.scale);
    const PageTable pages = table_of(a, b);
    char *const mine = lds[wave];
    const int token = lane >> 2, piece = lane & 3;        // as loaded
    const uint32_t code_at = lane * (D / 8), k_unit_at = c * (D / 32) + quarter * (D / 4) / 32, v_unit_at = token * (D / 32) + piece * (D / 4) / 32;
    // the way of keys from one to the other, in the place of the values that come after them; pieces swizzled against bank conflicts
    char *const key_to = mine + token * (D / 2) + (piece ^ (token >> 2)) * (D / 8);
    const char *const key_from = mine + c * (D / 2) + (quarter ^ (c >> 2)) * (D / 8);
    const int mask = (1 << a.page_shift) - 1;

    const auto page_of = [&](int t) { return pages[t < end ? t >> a.page_shift : 0]; };      // (there is a first page if there are tokens)
    const auto fetch = [&](Fetched<D> &f, int t0, int page0, int page1) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = t0 + 16 * u, page = u ? page1 : page0;
            f.there[u] = t < end && page >= 0 && page < a.c.pages;
            const int64_t row = ((static_cast<int64_t>(f.there[u] ? page : 0) * a.c.heads + head) << a.page_shift) + (t & mask);
            f.k[u] = *reinterpret_cast<const Codes<D> *>(a.c.k_codes_dev + row * (D / 2) + code_at);
            f.v[u] = *reinterpret_cast<const Codes<D> *>(a.c.v_codes_dev + row * (D / 2) + code_at);
#pragma unroll
            for (int y = 0; y < Share<D>::units; ++y) {
                // (the second group of a 96-channel share may be the first again)
                f.ku[u][y] = (a.c.k_scale_dev + row * (D / 32))[k_unit_at + (y ? Share<D>::unit(quarter, steps - 1) : 0)];
                f.vu[u][y] = (a.c.v_scale_dev + row * (D / 32))[v_unit_at + (y ? Share<D>::unit(piece, steps - 1) : 0)];
            }
        }
    };

    f32x4_t out[D / 16] = {};
    float top = -INFINITY, sum = 0.0f;                    // what the column's weights refer to; this lane's part of their sum
    const auto work = [&](const Fetched<D> &now, int t0) {
        Codes<D> keys[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) put_codes<D>(key_to + u * 8 * D, now.k[u]);
        lds_in_order();
#pragma unroll
        for (int u = 0; u < 2; ++u) take_codes<D>(key_from + u * 8 * D, keys[u]);
        lds_in_order();
        f32x4_t score[2] = {};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int s = 0; s < steps; ++s) {
                const bool second = Share<D>::units > 1 && Share<D>::unit(piece, s);
                const u32x4_t v = values8<_Float16>(now.v[u].w[s], value_unit_of(now.vu[u][second ? Share<D>::units - 1 : 0]));
                *reinterpret_cast<u32x4_t *>(mine + (16 * u + token) * kValueRow<D> + (piece * (D / 4) + 8 * s) * 2) = v;
            }
#pragma unroll
            for (int s = 0; s < steps; ++s) {
                const bool second = Share<D>::units > 1 && Share<D>::unit(quarter, s);
                const u32x4_t k = values8<T>(keys[u].w[s], unit_of(now.ku[u][second ? Share<D>::units - 1 : 0]));
                score[u] = Op::product(__builtin_bit_cast(typename Op::vec, k), q[s], score[u]);
            }
        }
        if (t0 + tokens > least || !now.there[0] || !now.there[1]) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int limit = now.there[u] ? seen - t0 - 16 * u : 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) score[u][j] = j < limit ? score[u][j] : -INFINITY;
            }
        }
        float best = fmaxf(score[0][0], score[1][0]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 1; j < 4; ++j) best = fmaxf(best, score[u][j]);
        best = column_max(best) * factor;
        if (__any(best > top + kSlack)) {
            const float higher = fmaxf(top, best), keep = __builtin_amdgcn_exp2f(top - (higher == -INFINITY ? 0.0f : higher));
            top = higher;
            sum *= keep;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) out[d] *= keep;
        }
        const float lift = kLift - (top == -INFINITY ? 0.0f : top);
        half8_t p;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float e = __builtin_amdgcn_exp2f(fmaf(score[u][j], factor, lift));
                sum += e;
                p[4 * u + j] = static_cast<_Float16>(e);
            }
        lds_in_order();                                   // this wave's values are in LDS
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            const char *from = mine + (4 * quarter + (c >> 2)) * kValueRow<D> + (16 * d + 4 * (c & 3)) * 2;
            half8_t v;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(from + 16 * u * kValueRow<D>));
#pragma unroll
                for (int j = 0; j < 4; ++j) v[4 * u + j] = __builtin_bit_cast(_Float16, static_cast<short>(y[j]));
            }
            out[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p, out[d], 0, 0, 0);
        }
        lds_in_order();
    };
    int t0 = begin + wave * tokens;
    if (t0 < end) {                                       // two sets of registers in turn
        Fetched<D> one, two;
        fetch(one, t0, page_of(t0), page_of(t0 + 16));
        int page0 = page_of(t0 + kTurn), page1 = page_of(t0 + kTurn + 16);
        for (;;) {
            fetch(two, t0 + kTurn, page0, page1);
            page0 = page_of(t0 + 2 * kTurn);
            page1 = page_of(t0 + 2 * kTurn + 16);
            work(one, t0);
            if ((t0 += kTurn) >= end) break;
            fetch(one, t0 + kTurn, page0, page1);
            page0 = page_of(t0 + 2 * kTurn);
            page1 = page_of(t0 + 2 * kTurn + 16);
            work(two, t0);
            if ((t0 += kTurn) >= end) break;
        }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (top == -INFINITY && live) top = top_of_nothing(a, b, begin + wave * tokens, min(end, seen + 4 * quarter));

    // the four waves' parts, joined on their common maximum
    if (quarter == 0) {
        row_max[wave][c] = top;
        row_sum[wave][c] = sum;
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4_t *>(mine + (c * D + ((16 * d + 4 * quarter) ^ (4 * c & 15))) * 4) = out[d];
    __syncthreads();
    for (int y = threadIdx.x; y < 16 * D / 4; y += 256) {
        const int row = y / (D / 4), ch = y % (D / 4) * 4, rr = x.r0 + row, ri = rr / a.group;
        if (ri >= x.n) continue;
        float m = row_max[0][row];
        for (int w = 1; w < 4; ++w) m = fmaxf(m, row_max[w][row]);
        const float base = m == -INFINITY ? 0.0f : m;
        float l = 0.0f;
        f32x4_t o = {};
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(row_max[w][row] - base);
            l += row_sum[w][row] * f;
            o += *reinterpret_cast<const f32x4_t *>(lds[w] + (row * D + (ch ^ (4 * row & 15))) * 4) * f;
        }
        if (SPLIT) {
            float *part = part_of<D>(a, unit, split, row);
            *reinterpret_cast<f32x4_t *>(part + ch) = o;
            if (ch == 0) {
                part[D] = m;
                part[D + 1] = l;
            }
        } else {
            const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
            T *to = static_cast<T *>(a.d.out_dev) + (x.q0 + ri) * a.d.out_token_stride + (head * a.group + (rr - ri * a.group)) * a.d.out_head_stride + ch;
            for (int j = 0; j < 4; ++j) to[j] = static_cast<T>(o[j] * inv);
        }
    }
}

// Two lanes that share a column of the 32 x 32 instruction (lane ^ 32).
__device__ __forceinline__ u32x2_t both_halves(float x) { return __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false); }

// Bytes between rows of keys and values in LDS of the kernel for many rows: of the paddings that fit, the ones with the fewest bank
// conflicts by the counters.
template <int D> constexpr int kManyKeyRow = 2 * D + 16;
template <int D> constexpr int kManyValueRow = 2 * D + 32;
template <int D> constexpr int kManyTile = 64 * (kManyKeyRow<D> + kManyValueRow<D>);

// 128 query rows of one cache head against one split of the sequence, 32 rows a wave, 64 tokens at a time.
//
// Bound by the matrix unit and the vector instructions of the softmax, which the three blocks of a compute unit (two where
// D = 256) overlap: 34 % and 39 % of the cycles with two blocks of two tiles each, 245 us for prompts of up to 2048 tokens on
// contexts of up to 4096, 32 heads on 8 of D = 128; 214 to 223 us over boxes (840 to 875 TFLOP/s; 229 in a kernel trace) as it is.  D = 128 spills
// up to four registers, D = 256 21 to 26 (two prompts of 4096, 16 heads on 4: 358 us, 768 TFLOP/s).  The tokens' codes are converted to LDS once for
// all rows, those of the next tile on their way meanwhile.  As for 16 rows, scores are computed transposed and the weights stay
// in their registers: the 32 x 32 instruction leaves a lane with tokens 8 (i / 4) + 4 half + i % 4 of its column, and the
// values are read in that order.
template <class T, int D, bool SPLIT> __global__ __launch_bounds__(256, D == 256 ? 2 : 3) void kv_attention_many_kernel(AttentionArgs a, int64_t first)
{
    using Op = Operand<T>;
    constexpr int steps = D / 16, tokens = 64, words = Share<D>::words, kAhead = 2;
    extern __shared__ __attribute__((aligned(16))) char many_lds[];      // keys, values, then [4] pages that are there
    uint8_t *const pages_there = reinterpret_cast<uint8_t *>(many_lds + kManyTile<D>);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, half = lane >> 5;
    const int64_t id = first + blockIdx.x, unit = SPLIT ? quotient(id, a.splits) : id;
    const int split = SPLIT ? static_cast<int>(id - unit * a.splits) : 0;
    const Place place = place_of(a, unit);
    const int head = place.head;
    const Rows x = find_rows(a, place.seq, place.tile);
    if (!x.any) return;
    int begin = 0, end = x.most;
    if (SPLIT) {
        const int each = split_tokens(x.most, a.splits);
        if (split && static_cast<int64_t>(split) * each >= x.most) return;
        begin = split * each;
        end = min(begin + each, x.most);
    }

    const int r = x.r0 + 32 * wave + c, i = r / a.group;
    const bool live = i < x.n;
    const int seen = live ? seen_by(x, i) : 0;
    // every row of the wave sees the tokens before `least`, none one from `mine` on
    const int wave_first = x.r0 + 32 * wave, rows = x.n * a.group;
    const int least = wave_first < rows ? seen_by(x, wave_first / a.group) : 0;
    const int mine = wave_first < rows ? seen_by(x, min((wave_first + 31) / a.group, x.n - 1)) : 0;
    typename Op::vec q[steps];
    {
        const int qh = head * a.group + (live ? r - i * a.group : 0);
        const T *src = static_cast<const T *>(a.d.q_dev) + (x.q0 + (live ? i : 0)) * a.d.q_token_stride + qh * a.d.q_head_stride + 8 * half;
        const float sign = sign_of(a.d.scale);
#pragma unroll
        for (int s = 0; s < steps; ++s) {
            u32x4_t w;
            __builtin_memcpy(&w, src + 16 * s, 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = times_sign<T>(w[j], sign);
            q[s] = __builtin_bit_cast(typename Op::vec, w);
        }
    }
    const float factor = factor_of(a.d.scale);
    const int32_t *pages = a.d.page_dev + place.seq * a.d.max_pages;
    const int mask = (1 << a.page_shift) - 1;

    // loader: thread 4 t + u has token t of a tile and channels [D / 4 u, + D / 4)
    const int token = threadIdx.x >> 2, quarter = threadIdx.x & 3;
    struct Row { Codes<D> k, v; uint8_t ku[Share<D>::units], vu[Share<D>::units]; bool there; };
    const auto page_of = [&](int t0) { return t0 + token < end ? pages[(t0 + token) >> a.page_shift] : -1; };
    const auto fetch = [&](int t0, int page) {
        Row f;
        const int t = t0 + token;
        f.there = t < end && page >= 0 && page < a.c.pages;
        const int64_t row = ((static_cast<int64_t>(f.there ? page : 0) * a.c.heads + head) << a.page_shift) + (t & mask);
        const int64_t code_at = row * (D / 2) + quarter * (D / 8), unit_at = row * (D / 32) + quarter * (D / 4) / 32;
        f.k = *reinterpret_cast<const Codes<D> *>(a.c.k_codes_dev + code_at);
        f.v = *reinterpret_cast<const Codes<D> *>(a.c.v_codes_dev + code_at);
#pragma unroll
        for (int y = 0; y < Share<D>::units; ++y) {
            const int64_t at = unit_at + (y ? Share<D>::unit(quarter, words - 1) : 0);
            f.ku[y] = a.c.k_scale_dev[at];
            f.vu[y] = a.c.v_scale_dev[at];
        }
        return f;
    };
    const auto convert = [&](const Row &f) {
        char *const k_to = many_lds + token * kManyKeyRow<D> + quarter * (D / 2);
        char *const v_to = many_lds + 64 * kManyKeyRow<D> + token * kManyValueRow<D> + quarter * (D / 2);
#pragma unroll
        for (int s = 0; s < words; ++s) {
            const bool second = Share<D>::units > 1 && Share<D>::unit(quarter, s);
            *reinterpret_cast<u32x4_t *>(k_to + 16 * s) = values8<T>(f.k.w[s], unit_of(f.ku[second ? Share<D>::units - 1 : 0]));
            *reinterpret_cast<u32x4_t *>(v_to + 16 * s) = values8<_Float16>(f.v.w[s], value_unit_of(f.vu[second ? Share<D>::units - 1 : 0]));
        }
        if ((threadIdx.x & 63) == 0) pages_there[token / 16] = f.there;
    };

    f32x16_t out[D / 32] = {};
    float top = -INFINITY, sum = 0.0f;                    // what the column's weights refer to; this lane's part of their sum
    Row next = {};
    int page = -1;
    if (begin < end) {
        next = fetch(begin, page_of(begin));
        page = page_of(begin + tokens);
    }
    for (int t0 = begin; t0 < end; t0 += tokens) {
        convert(next);
        next = fetch(t0 + tokens, page);
        page = page_of(t0 + 2 * tokens);                  // (a page number is there by the time its codes are asked for)
        __syncthreads();
        if (t0 < mine) {
            const char *const keys = many_lds, *const values = keys + 64 * kManyKeyRow<D>;
            // fragments are read kAhead instructions before they are multiplied (left to itself the compiler waits for each)
            f32x16_t score[2] = {};
            const auto key = [&](auto ic) {
                constexpr int i = decltype(ic)::value;    // step i / 2, tokens 32 (i % 2) ..
                return __builtin_bit_cast(typename Op::vec, *reinterpret_cast<const u32x4_t *>(keys + (32 * (i % 2) + c) * kManyKeyRow<D> + 32 * (i / 2) + 16 * half));
            };
            typename Op::vec k[kAhead];
            static_for<kAhead>([&](auto i) { k[i] = key(i); });
            static_for<2 * steps>([&](auto ic) {
                constexpr int i = decltype(ic)::value;
                score[i % 2] = Op::product(k[i % kAhead], q[i / 2], score[i % 2]);
                if constexpr (i + kAhead < 2 * steps) k[i % kAhead] = key(std::integral_constant<int, i + kAhead>{});
                __builtin_amdgcn_sched_barrier(0);
            });
            const auto value = [&](auto ic) {
                constexpr int i = decltype(ic)::value, s = i / (D / 32), d = i % (D / 32);       // tokens 16 s .., channels 32 d ..
                const char *from = values + (16 * s + 4 * half + (lane % 16 >> 2)) * kManyValueRow<D> + (32 * d + 16 * (lane / 16 % 2) + 4 * (lane % 4)) * 2;
                half8_t v;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(from + 8 * h * kManyValueRow<D>));
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[4 * h + j] = __builtin_bit_cast(_Float16, static_cast<short>(y[j]));
                }
                return v;
            };
            half8_t v[kAhead];
            static_for<kAhead>([&](auto i) { v[i] = value(i); });
            const uint32_t there = __builtin_amdgcn_readfirstlane(*reinterpret_cast<const uint32_t *>(pages_there));
            if (t0 + tokens > least || there != 0x01010101u) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {             // 16 tokens, of one page
                    const int limit = there >> (8 * g) & 1 ? seen - t0 - 16 * g - 4 * half : INT_MIN;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (8 * (j / 4) + j % 4 >= limit) score[g / 2][8 * (g % 2) + j] = -INFINITY;
                }
            }
            float best = score[0][0];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 16; ++j) best = fmaxf(best, score[u][j]);
            const u32x2_t two = both_halves(best);
            best = fmaxf(__uint_as_float(two[0]), __uint_as_float(two[1])) * factor;
            if (__any(best > top + kSlack)) {
                const float higher = fmaxf(top, best), base = higher == -INFINITY ? 0.0f : higher, keep = __builtin_amdgcn_exp2f(top - base);
                top = higher;
                sum *= keep;
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
#pragma unroll
                    for (int j = 0; j < 16; ++j) out[d][j] *= keep;
            }
            const float lift = kLift - (top == -INFINITY ? 0.0f : top);
            half8_t p[4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(score[u][j], factor, lift));
                    sum += e;
                    p[2 * u + j / 8][j % 8] = static_cast<_Float16>(e);
                }
            __builtin_amdgcn_sched_barrier(0);
            static_for<D / 8>([&](auto ic) {
                constexpr int i = decltype(ic)::value, s = i / (D / 32), d = i % (D / 32);
                out[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[i % kAhead], p[s], out[d], 0, 0, 0);
                if constexpr (i + kAhead < D / 8) v[i % kAhead] = value(std::integral_constant<int, i + kAhead>{});
                __builtin_amdgcn_sched_barrier(0);
            });
        }
        __syncthreads();
    }
    const u32x2_t two = both_halves(sum);
    sum = __uint_as_float(two[0]) + __uint_as_float(two[1]);
    if (!live) return;
    if (top == -INFINITY) top = top_of_nothing(a, place.seq, begin, min(end, seen));
    if (SPLIT) {
        float *part = part_of<D>(a, unit, split, 32 * wave + c);
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<f32x4_t *>(part + 32 * d + 8 * j + 4 * half) = f32x4_t{out[d][4 * j], out[d][4 * j + 1], out[d][4 * j + 2], out[d][4 * j + 3]};
        if (half == 0) {
            part[D] = top;
            part[D + 1] = sum;
        }
        return;
    }
    const float inv = top == -INFINITY ? 0.0f : 1.0f / sum;
    T *to = static_cast<T *>(a.d.out_dev) + (x.q0 + i) * a.d.out_token_stride + (head * a.group + (r - i * a.group)) * a.d.out_head_stride + 4 * half;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            T y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = static_cast<T>(out[d][4 * j + e] * inv);
            __builtin_memcpy(to + 32 * d + 8 * j, y, sizeof y);
        }
}

// Joins the splits' parts of a row: D / 4 lanes take its channels.  Where rows are few and splits many, a block takes one row and
// its teams of lanes further splits of it; else every team a row of its own.
template <class T, int D, bool MANY> __global__ __launch_bounds__(256) void kv_attention_join_kernel(AttentionArgs a, int64_t first)
{
    constexpr int lanes = D / 4, teams = 256 / lanes;
    __shared__ f32x4_t sums[MANY ? 1 : teams][lanes];
    __shared__ float tops[teams], weights[teams];
    const int team = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    if (MANY && team >= teams) return;
    const int64_t id = MANY ? (first + blockIdx.x) * teams + team : first + blockIdx.x, unit = quotient(id, a.part_rows);
    if (MANY && unit >= a.tiles * a.d.seqs * a.c.heads) return;
    const int row = static_cast<int>(id - unit * a.part_rows);
    const Place place = place_of(a, unit);
    const int head = place.head;
    const Rows x = find_rows(a, place.seq, place.tile);
    const int rr = x.r0 + row, ri = rr / a.group;
    if (!x.any || ri >= x.n) return;
    const int each = split_tokens(x.most, a.splits), parts = max(1, (x.most + each - 1) / each);
    float l = 0.0f, m = -INFINITY;
    f32x4_t o = {};
    // four parts asked for at once, each brought to the maximum so far
    for (int s = MANY ? 0 : team; s < parts; s += 4 * (MANY ? 1 : teams)) {
        float pm[4], pl[4];
        f32x4_t po[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int at = s + u * (MANY ? 1 : teams);
            const float *part = part_of<D>(a, unit, at < parts ? at : s, row);
            pm[u] = at < parts ? part[D] : -INFINITY;
            pl[u] = part[D + 1];
            po[u] = *reinterpret_cast<const f32x4_t *>(part + 4 * lane);
        }
        const float higher = fmaxf(fmaxf(fmaxf(pm[0], pm[1]), fmaxf(pm[2], pm[3])), m), base = higher == -INFINITY ? 0.0f : higher;
        const float keep = __builtin_amdgcn_exp2f(m - base);
        m = higher;
        l *= keep;
        o *= keep;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (s + u * (MANY ? 1 : teams) >= parts) continue;
            const float f = __builtin_amdgcn_exp2f(pm[u] - base);
            l += pl[u] * f;
            o += po[u] * f;
        }
    }
    if constexpr (!MANY) {
        if (team < teams) {
            sums[team][lane] = o;
            if (lane == 0) {
                weights[team] = l;
                tops[team] = m;
            }
        }
        __syncthreads();
        if (team) return;
        for (int s = 0; s < teams; ++s) m = fmaxf(m, tops[s]);
        const float base = m == -INFINITY ? 0.0f : m;
        o = f32x4_t{};
        l = 0.0f;
        for (int s = 0; s < teams; ++s) {
            const float f = __builtin_amdgcn_exp2f(tops[s] - base);
            o += sums[s][lane] * f;
            l += weights[s] * f;
        }
    }
    const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
    T *to = static_cast<T *>(a.d.out_dev) + (x.q0 + ri) * a.d.out_token_stride + (head * a.group + (rr - ri * a.group)) * a.d.out_head_stride + 4 * lane;
    T y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = static_cast<T>(o[j] * inv);
    __builtin_memcpy(to, y, sizeof y);
}

}  // namespace apnn

namespace {

int check_attention(const char *who, const apnn_kv_attention_desc *d, const apnn_kv_cache *c)
{
    using namespace apnn;
    if (const int rc = check_cache(who, c)) return rc;
    if (!d) return fail(APNN_ERR_INVALID_ARG, "%s: no description", who);
    if (d->type != APNN_F16 && d->type != APNN_BF16) return fail(APNN_ERR_UNSUPPORTED, "%s: queries of type %d, supported APNN_F16 and APNN_BF16", who, static_cast<int>(d->type));
    if (d->tokens < 0 || d->seqs < 0 || d->max_pages < 0 || d->max_q < 0 || d->q_heads < 0)
        return fail(APNN_ERR_INVALID_ARG, "%s: tokens = %lld, seqs = %lld, max_pages = %lld, max_q = %lld, q_heads = %d", who, (long long)d->tokens,
                    (long long)d->seqs, (long long)d->max_pages, (long long)d->max_q, d->q_heads);
    if (d->tokens > INT_MAX || d->seqs > INT_MAX || d->max_pages > INT_MAX || d->q_heads > (1 << 16))
        return fail(APNN_ERR_UNSUPPORTED, "%s: a size is too large", who);
    if (d->max_pages * c->page_size > (int64_t(1) << 30)) return fail(APNN_ERR_UNSUPPORTED, "%s: a table of more than 2^30 tokens", who);
    if (d->q_heads >= c->heads && d->tokens * (d->q_heads / c->heads) > (int64_t(1) << 30))
        return fail(APNN_ERR_UNSUPPORTED, "%s: %lld rows of %d heads for each cache head", who, (long long)d->tokens, d->q_heads / c->heads);
    if (d->q_heads < 1 || d->q_heads % c->heads) return fail(APNN_ERR_INVALID_ARG, "%s: %d query heads over %d cache heads", who, d->q_heads, c->heads);
    const double rows = static_cast<double>(d->q_start_dev ? (d->max_q < d->tokens ? d->max_q : d->tokens) : 1) * d->q_heads;
    if ((rows / 16 + c->heads) * d->seqs > 1e12) return fail(APNN_ERR_UNSUPPORTED, "%s: %lld sequences of up to %lld queries", who, (long long)d->seqs, (long long)d->max_q);
    if (!(fabsf(d->scale) <= 0x1p127f)) return fail(APNN_ERR_INVALID_ARG, "%s: scale = %g, at most 2^127 in magnitude", who, static_cast<double>(d->scale));
    if (!d->q_start_dev && d->tokens < d->seqs) return fail(APNN_ERR_INVALID_ARG, "%s: one query each for %lld sequences, %lld rows", who, (long long)d->seqs, (long long)d->tokens);
    return APNN_OK;
}

}  // namespace

namespace apnn {

// How a call is cut: tiles of 16 or 128 rows, and splits of their tokens where tiles are too few to fill the chip.  A compute unit
// holds four blocks of the one and two of the other; twice as many of the first leave room for sequences of different lengths.
struct AttentionPlan {
    int64_t max_q, tiles;
    int splits, part_rows, tile_rows;
    size_t bytes;
};

static AttentionPlan plan_attention(const apnn_kv_attention_desc &d, const apnn_kv_cache &c)
{
    AttentionPlan p = {};
    const int group = d.q_heads / c.heads;
    p.max_q = d.q_start_dev ? (d.max_q < d.tokens ? d.max_q : d.tokens) : 1;
    if (d.tokens == 0 || d.seqs == 0 || p.max_q == 0) return p;
    const int64_t rows = p.max_q * group, pairs = static_cast<int64_t>(c.heads) * d.seqs, room = d.max_pages * c.page_size;
    // 128 rows a block pay where blocks are enough without splits, or scores many (us, 16 and 128 rows; 32 heads on 8, D = 128: 1 x 256 queries
    // on 2048 tokens 24, 34; 1 x 1024 60, 57; 1 x 2048 80, 59; 4 x 1024 on 1024 95, 54; 1 x 128 on 32768 152, 104; 16 heads, D = 64: 1 x 2048
    // on 2048 26, 35; 8 x 500 on 500 24, 15)
    const bool many = rows >= 64 && (ceil_div(rows, 128) * pairs >= 384 || static_cast<double>(rows) * pairs * (room - p.max_q / 2) >= 4e7);
    const int forced = kv_rows_override();
    p.tile_rows = forced == 16 || forced == 128 ? forced : (many ? 128 : 16);
    p.tiles = ceil_div(rows, p.tile_rows);
    p.part_rows = static_cast<int>(rows < p.tile_rows ? rows : p.tile_rows);
    const int64_t blocks = p.tiles * pairs;
    // two blocks a compute unit in any case, more only while a split keeps 2048 tokens
    // (2 x 131072 tokens on 4 heads: 28, 30, 34, 44 us with 512, 1024, 2048, 4096 blocks; 48 x 8192 on 8: 92, 68, 65, 64)
    int64_t splits = 512 / blocks, most = 2048 / blocks < room / 2048 ? 2048 / blocks : room / 2048;
    if (p.tile_rows == 16 && splits < most) splits = most;
    if (splits > ceil_div(room, kLeastSplit)) splits = ceil_div(room, kLeastSplit);
    // up to 1024 tokens the second kernel takes longer than it saves (32 x 1000 tokens on 8 heads: 10.5 us, split 15.3; 1 x 1000: 9.3, 9.7;
    // but 1 x 2000: 14.2, 9.7)
    if (p.tile_rows == 16 && room <= 1024) splits = 1;
    p.splits = splits < 1 ? 1 : static_cast<int>(splits);
    if (p.splits > 1) p.bytes = static_cast<size_t>(blocks) * p.splits * p.part_rows * (c.D + 4) * sizeof(float);
    return p;
}

}  // namespace apnn

extern "C" size_t apnn_kv_attention_workspace_bytes(const apnn_kv_attention_desc *desc, const apnn_kv_cache *cache)
{
    apnn::clear_error();
    if (check_attention("apnn_kv_attention_workspace_bytes", desc, cache) != APNN_OK) return 0;
    return apnn::plan_attention(*desc, *cache).bytes;
}

extern "C" int apnn_kv_attention(const apnn_kv_attention_desc *desc, const apnn_kv_cache *cache, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    using namespace apnn;
    clear_error();
    const char *who = "apnn_kv_attention";
    if (const int rc = check_attention(who, desc, cache)) return rc;
    const AttentionPlan plan = plan_attention(*desc, *cache);
    if (plan.tiles == 0) return APNN_OK;
    if (!desc->q_dev || !desc->out_dev || !desc->len_dev || (desc->max_pages && !desc->page_dev)) return fail(APNN_ERR_INVALID_ARG, "%s: null pointer", who);
    if (desc->q_dev == desc->out_dev) return fail(APNN_ERR_INVALID_ARG, "%s: out must not be q", who);
    if (!aligned_to(desc->q_dev, desc->type) || !aligned_to(desc->out_dev, desc->type)) return fail(APNN_ERR_ALIGNMENT, "%s: a pointer is not aligned to its type", who);
    if (!strides_fit(desc->tokens, desc->q_heads, cache->D, desc->q_token_stride, desc->q_head_stride, false) ||
        !strides_fit(desc->tokens, desc->q_heads, cache->D, desc->out_token_stride, desc->out_head_stride, true))
        return fail(APNN_ERR_INVALID_ARG, "%s: strides", who);
    if (plan.bytes && (!workspace_dev || workspace_bytes < plan.bytes))
        return fail(APNN_ERR_INVALID_ARG, "%s: a workspace of %zu bytes is needed, %zu given", who, plan.bytes, workspace_dev ? workspace_bytes : size_t(0));
    if (plan.bytes && !aligned16(workspace_dev)) return fail(APNN_ERR_ALIGNMENT, "%s: the workspace is not 16-byte aligned", who);
    AttentionArgs a = {};
    a.d = *desc;
    a.c = *cache;
    a.d.max_q = plan.max_q;
    if (cache->pages == 0) a.d.max_pages = 0;             // no page can be read
    a.parts = static_cast<float *>(workspace_dev);
    a.tiles = plan.tiles;
    a.page_shift = shift_of(cache->page_size);
    a.group = desc->q_heads / cache->heads;
    a.splits = plan.splits;
    a.part_rows = plan.part_rows;
    a.tile_rows = plan.tile_rows;
    const int64_t units = a.tiles * cache->heads * desc->seqs;
    const auto sliced = [](int64_t blocks, auto &&launch) {
        for (int64_t first = 0; first < blocks; first += kMaxBlocks) launch(first, static_cast<unsigned>(blocks - first < kMaxBlocks ? blocks - first : kMaxBlocks));
    };
    const auto go = [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        if (a.tile_rows == 128) {
            constexpr int bytes = kManyTile<D> + 16;
            if constexpr (bytes > 64 * 1024) {
                static std::atomic<uint64_t> granted[2];
                if (!all_of_lds(kv_attention_many_kernel<T, D, false>, granted[0]) || !all_of_lds(kv_attention_many_kernel<T, D, true>, granted[1]))
                    return fail(APNN_ERR_DEVICE, "%s: no %d bytes of LDS", who, bytes);
            }
            if (a.splits == 1) sliced(units, [&](int64_t first, unsigned blocks) { kv_attention_many_kernel<T, D, false><<<blocks, 256, bytes, as_stream(stream)>>>(a, first); });
            else sliced(units * a.splits, [&](int64_t first, unsigned blocks) { kv_attention_many_kernel<T, D, true><<<blocks, 256, bytes, as_stream(stream)>>>(a, first); });
        } else if (a.splits == 1) {
            sliced(units, [&](int64_t first, unsigned blocks) { kv_attention_kernel<T, D, false><<<blocks, 256, 0, as_stream(stream)>>>(a, first); });
        } else {
            sliced(units * a.splits, [&](int64_t first, unsigned blocks) { kv_attention_kernel<T, D, true><<<blocks, 256, 0, as_stream(stream)>>>(a, first); });
        }
        const int64_t rows = units * a.part_rows;
        if (a.splits > 1 && (rows >= 2048 || a.splits <= 8))
            sliced(ceil_div(rows, 256 / (D / 4)), [&](int64_t first, unsigned blocks) { kv_attention_join_kernel<T, D, true><<<blocks, 256, 0, as_stream(stream)>>>(a, first); });
        else if (a.splits > 1)
            sliced(rows, [&](int64_t first, unsigned blocks) { kv_attention_join_kernel<T, D, false><<<blocks, 256, 0, as_stream(stream)>>>(a, first); });
        return check_launch(who);
    };
    return by_channels(cache->D, [&](auto d) { return desc->type == APNN_F16 ? go(_Float16{}, d) : go(__bf16{}, d); });
}
