// Attention over the paged 4-bit cache (apnn_kv_attention).
//
// Scores are computed transposed, S^T = K Q^T: the 16 x 16 matrix instruction then leaves a lane with scores of one query
// row (its column) and, in groups of four, of tokens that are the contraction index of O^T = V^T P^T.  P goes from one
// instruction to the next in its registers; only V has to change places, which it does on its way through LDS
// (ds_read_b64_tr_b16).  A 4-bit group with its power of two is exact in 16 bits, so the conversion
// (v_cvt_scalef32_pk_*_fp4, two values an instruction) costs no accuracy: keys take the queries' type, values fp16.
#include "kv_cache.h"

namespace apnn {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

struct AttentionArgs {
    apnn_kv_attention_desc d;
    apnn_kv_cache c;
    int page_shift, group;                                // query heads to a cache head
    int64_t tiles;                                        // 16-row tiles of max_q * group rows
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
};
template <> struct Operand<__bf16> {
    typedef bf16x8_t vec;
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 0>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0)); }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 1>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1)); }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 2>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2)); }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float unit, std::integral_constant<int, 3>) { return bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3)); }
    static __device__ __forceinline__ uint32_t bits(bf16x2_t v) { return __builtin_bit_cast(uint32_t, v); }
    static __device__ __forceinline__ f32x4_t product(vec a, vec b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// Eight 4-bit codes -> eight operands.
template <class T> __device__ __forceinline__ u32x4_t values8(uint32_t w, float unit)
{
    using I = Operand<T>;
    return u32x4_t{I::two(w, unit, std::integral_constant<int, 0>{}), I::two(w, unit, std::integral_constant<int, 1>{}),
                   I::two(w, unit, std::integral_constant<int, 2>{}), I::two(w, unit, std::integral_constant<int, 3>{})};
}

// A row's scale as the conversions take it; 255 stands for NaN there too.
__device__ __forceinline__ float unit_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Geometry of a lane's share of a row: lane l of a wave has token l % 16 of 16 and channels [D / 4 * (l / 16), + D / 4).
template <int D> struct Share {
    static constexpr int words = D / 32;                  // 32-bit words of codes
    static constexpr int units = D == 96 || D == 256 ? 2 : 1;             // groups of 32 channels it reaches into
    static __device__ __forceinline__ int unit(int quarter, int word) { return (quarter * (D / 4) + 8 * word) / 32 - quarter * (D / 4) / 32; }
};

// Bytes between rows of values in LDS: 32 more than the values, so that eight rows cover all banks.
template <int D> constexpr int kValueRow = 2 * D + 32;

// 16 query rows of one cache head against the sequence, the four waves taking 32 tokens each in turn.
template <class T, int D> __global__ __launch_bounds__(256) void kv_attention_kernel(AttentionArgs a, int64_t first)
{
    using Op = Operand<T>;
    constexpr int steps = D / 32, tokens = 32;
    constexpr int wave_bytes = tokens * kValueRow<D> > 64 * D ? tokens * kValueRow<D> : 64 * D;
    __shared__ alignas(16) char lds[4][wave_bytes];
    __shared__ float row_max[4][16], row_sum[4][16];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, quarter = lane >> 4;
    const int64_t id = first + blockIdx.x, tile = id % a.tiles, rest = id / a.tiles;
    const int head = static_cast<int>(rest % a.c.heads);
    const int64_t b = rest / a.c.heads;
    if (b >= a.d.seqs) return;

    // the sequence: rows [q0, q0 + n), `have` tokens that the table can name
    int64_t q0 = b, n = 1;
    if (a.d.q_start_dev) {
        q0 = a.d.q_start_dev[b];
        n = a.d.q_start_dev[b + 1] - q0;
    }
    if (q0 < 0 || q0 > a.d.tokens) return;
    n = n < a.d.tokens - q0 ? n : a.d.tokens - q0;
    const int64_t all = n;                                // where the queries stand goes by all of them
    n = n < a.d.max_q ? n : a.d.max_q;
    const int64_t r0 = tile * 16;
    if (r0 >= n * a.group) return;
    const int64_t len = a.d.len_dev[b], room = a.d.max_pages << a.page_shift;
    const int64_t have = len < room ? (len > 0 ? len : 0) : room;

    const int64_t r = r0 + c, i = r / a.group;
    const bool live = i < n;
    const int64_t at = (live ? i : 0) + q0;
    const int qh = head * a.group + static_cast<int>(r - i * a.group);
    // tokens that the row of this lane's column sees, and the most any row of the tile sees
    int64_t seen = len - all + i + 1;
    seen = !live || seen < 0 ? 0 : (seen < have ? seen : have);
    const int64_t last = r0 + 15 < n * a.group ? (r0 + 15) / a.group : n - 1;
    int64_t most = len - all + last + 1;
    most = most < 0 ? 0 : (most < have ? most : have);

    typename Op::vec q[steps];
    {
        const T *src = static_cast<const T *>(a.d.q_dev) + at * a.d.q_token_stride + (live ? qh : head * a.group) * a.d.q_head_stride + quarter * (D / 4);
#pragma unroll
        for (int s = 0; s < steps; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) q[s][j] = src[8 * s + j];
    }
    const float factor = a.d.scale * 1.4426950408889634f; // scores in powers of two
    const int32_t *pages = a.d.page_dev + b * a.d.max_pages;
    char *const mine = lds[wave];

    f32x4_t out[D / 16] = {};
    float top = -INFINITY, sum = 0.0f;                    // of this lane's column: common to its four lanes, and this lane's part
    for (int64_t t0 = wave * tokens; t0 < most; t0 += 4 * tokens) {
        f32x4_t score[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t t = t0 + 16 * u;
            const int64_t page = t < most ? __builtin_amdgcn_readfirstlane(pages[t >> a.page_shift]) : -1;
            const bool there = page >= 0 && page < a.c.pages;
            const int64_t row = there ? ((page * a.c.heads + head) << a.page_shift) + (t & ((1 << a.page_shift) - 1)) + c : 0;
            uint32_t kw[steps] = {}, vw[steps] = {}, ku[Share<D>::units], vu[Share<D>::units];
#pragma unroll
            for (int x = 0; x < Share<D>::units; ++x) ku[x] = vu[x] = 127;
            if (there) {
#pragma unroll
                for (int s = 0; s < steps; ++s) {
                    kw[s] = reinterpret_cast<const uint32_t *>(a.c.k_codes_dev + row * (D / 2))[quarter * steps + s];
                    vw[s] = reinterpret_cast<const uint32_t *>(a.c.v_codes_dev + row * (D / 2))[quarter * steps + s];
                }
                const int64_t at_scale = row * (D / 32) + quarter * (D / 4) / 32;
#pragma unroll
                for (int x = 0; x < Share<D>::units; ++x) {
                    // (the second group of a 96-channel share may be the first again)
                    const int64_t where = at_scale + (x ? Share<D>::unit(quarter, steps - 1) : 0);
                    ku[x] = a.c.k_scale_dev[where];
                    vu[x] = t + c < have ? a.c.v_scale_dev[where] : 127;       // beyond the end: whatever it is, finite
                }
            }
            score[u] = f32x4_t{};
#pragma unroll
            for (int s = 0; s < steps; ++s) {
                const int x = Share<D>::units > 1 ? Share<D>::unit(quarter, s) : 0;
                const u32x4_t k = values8<T>(kw[s], unit_of(x ? ku[Share<D>::units - 1] : ku[0]));
                score[u] = Op::product(__builtin_bit_cast(typename Op::vec, k), q[s], score[u]);
                const u32x4_t v = values8<_Float16>(vw[s], unit_of(x ? vu[Share<D>::units - 1] : vu[0]));
                *reinterpret_cast<u32x4_t *>(mine + (16 * u + c) * kValueRow<D> + (quarter * (D / 4) + 8 * s) * 2) = v;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                score[u][j] = there && t + 4 * quarter + j < seen ? score[u][j] * factor : -INFINITY;
        }
        float best = top;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) best = fmaxf(best, score[u][j]);
        best = fmaxf(best, __shfl_xor(best, 16));
        best = fmaxf(best, __shfl_xor(best, 32));
        const float base = best == -INFINITY ? 0.0f : best, keep = __builtin_amdgcn_exp2f(top - base);
        top = best;
        half8_t p;
        float part = 0.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float e = __builtin_amdgcn_exp2f(score[u][j] - base);
                part += e;
                p[4 * u + j] = static_cast<_Float16>(e);
            }
        sum = sum * keep + part;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // this wave's values are in LDS (its accesses stay in order)
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            const char *from = mine + (4 * quarter + (c >> 2)) * kValueRow<D> + (16 * d + 4 * (c & 3)) * 2;
            half8_t v;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4_t *)(from + 16 * u * kValueRow<D>));
#pragma unroll
                for (int j = 0; j < 4; ++j) v[4 * u + j] = __builtin_bit_cast(_Float16, static_cast<short>(x[j]));
            }
            out[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p, out[d] * keep, 0, 0, 0);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // the four waves' parts, joined on their common maximum
    if (quarter == 0) {
        row_max[wave][c] = top;
        row_sum[wave][c] = sum;
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4_t *>(mine + (c * D + ((16 * d + 4 * quarter) ^ (4 * c & 15))) * 4) = out[d];
    __syncthreads();
    for (int x = threadIdx.x; x < 16 * D / 4; x += 256) {
        const int row = x / (D / 4), ch = x % (D / 4) * 4;
        const int64_t rr = r0 + row, ri = rr / a.group;
        if (ri >= n) continue;
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
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        T *to = static_cast<T *>(a.d.out_dev) + (q0 + ri) * a.d.out_token_stride + (head * a.group + (rr - ri * a.group)) * a.d.out_head_stride + ch;
        for (int j = 0; j < 4; ++j) to[j] = static_cast<T>(o[j] * inv);
    }
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
    if (d->q_heads < 1 || d->q_heads % c->heads) return fail(APNN_ERR_INVALID_ARG, "%s: %d query heads over %d cache heads", who, d->q_heads, c->heads);
    if (!(d->scale - d->scale == 0.0f)) return fail(APNN_ERR_INVALID_ARG, "%s: scale is not finite", who);
    if (!d->q_start_dev && d->tokens < d->seqs) return fail(APNN_ERR_INVALID_ARG, "%s: one query each for %lld sequences, %lld rows", who, (long long)d->seqs, (long long)d->tokens);
    return APNN_OK;
}

}  // namespace

extern "C" size_t apnn_kv_attention_workspace_bytes(const apnn_kv_attention_desc *desc, const apnn_kv_cache *cache)
{
    apnn::clear_error();
    if (check_attention("apnn_kv_attention_workspace_bytes", desc, cache) != APNN_OK) return 0;
    return 0;
}

extern "C" int apnn_kv_attention(const apnn_kv_attention_desc *desc, const apnn_kv_cache *cache, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    using namespace apnn;
    clear_error();
    const char *who = "apnn_kv_attention";
    if (const int rc = check_attention(who, desc, cache)) return rc;
    const int64_t max_q = desc->q_start_dev ? (desc->max_q < desc->tokens ? desc->max_q : desc->tokens) : 1;
    if (desc->tokens == 0 || desc->seqs == 0 || max_q == 0) return APNN_OK;
    if (!desc->q_dev || !desc->out_dev || !desc->len_dev || (desc->max_pages && !desc->page_dev)) return fail(APNN_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned_to(desc->q_dev, desc->type) || !aligned_to(desc->out_dev, desc->type)) return fail(APNN_ERR_ALIGNMENT, "%s: a pointer is not aligned to its type", who);
    if (!strides_fit(desc->tokens, desc->q_heads, cache->D, desc->q_token_stride, desc->q_head_stride, false) ||
        !strides_fit(desc->tokens, desc->q_heads, cache->D, desc->out_token_stride, desc->out_head_stride, true))
        return fail(APNN_ERR_INVALID_ARG, "%s: strides", who);
    (void)workspace_dev;
    (void)workspace_bytes;
    AttentionArgs a = {*desc, *cache, shift_of(cache->page_size), desc->q_heads / cache->heads, 0};
    a.d.max_q = max_q;
    a.tiles = ceil_div(max_q * a.group, 16);
    const int64_t blocks = a.tiles * cache->heads * desc->seqs;
    const auto go = [&](auto t, auto d) {
        for (int64_t first = 0; first < blocks; first += kMaxBlocks)
            kv_attention_kernel<decltype(t), decltype(d)::value><<<static_cast<unsigned>(blocks - first < kMaxBlocks ? blocks - first : kMaxBlocks), 256, 0, as_stream(stream)>>>(a, first);
        return check_launch(who);
    };
    const auto of_type = [&](auto d) { return desc->type == APNN_F16 ? go(_Float16{}, d) : go(__bf16{}, d); };
    return by_channels(cache->D, of_type);
}
