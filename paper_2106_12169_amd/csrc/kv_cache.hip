// Writing the paged 4-bit cache (apnn_kv_append) and reading it back (apnn_kv_read).
//
// A row is D channels of one (token, head); a team of lanes takes it, 8 channels a lane, so that a group of 32 channels
// with its common power of two is four neighbouring lanes.  The rotation is computed in 64 bits and rounded once: the
// codes then depend on the inputs alone, not on the order or contraction of 32-bit operations, which next to a border
// between two codes would decide a whole step.
#include "kv_cache.h"

namespace apnn {

int check_cache(const char *who, const apnn_kv_cache *c)
{
    if (!c) return fail(APNN_ERR_INVALID_ARG, "%s: no cache", who);
    if (c->D != 64 && c->D != 96 && c->D != 128 && c->D != 256) return fail(APNN_ERR_UNSUPPORTED, "%s: D = %d, supported 64, 96, 128, 256", who, c->D);
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
        return fail(APNN_ERR_UNSUPPORTED, "%s: pages of %d tokens, supported 16, 32, 64, 128, 256", who, c->page_size);
    if (c->heads < 1 || c->heads > 1024) return fail(APNN_ERR_UNSUPPORTED, "%s: %d heads, supported 1..1024", who, c->heads);
    if (c->pages < 0 || c->pages > INT_MAX) return fail(APNN_ERR_INVALID_ARG, "%s: %lld pages", who, (long long)c->pages);
    if (c->pages && (!c->k_codes_dev || !c->k_scale_dev || !c->v_codes_dev || !c->v_scale_dev)) return fail(APNN_ERR_INVALID_ARG, "%s: null cache pointer", who);
    if (!aligned16(c->k_codes_dev) || !aligned16(c->k_scale_dev) || !aligned16(c->v_codes_dev) || !aligned16(c->v_scale_dev))
        return fail(APNN_ERR_ALIGNMENT, "%s: a cache array is not 16-byte aligned", who);
    return APNN_OK;
}

struct AppendArgs {
    apnn_kv_cache c;
    apnn_kv_tokens t;
    int page_shift;
};

// What the rotation makes of channels c0 .. c0 + 7 of a row, in 64 bits, rounded once.
struct Rotation {
    enum Kind { NONE, PAIRS, HALVES, ODD } kind;          // not reached; pairs of neighbours; halves of 8 channels in a row; else
    int c0, rot;
    __device__ __forceinline__ Rotation(int c, int r, bool interleaved) : kind(c >= r ? NONE : interleaved ? PAIRS : r % 16 == 0 ? HALVES : ODD), c0(c), rot(r) {}
    __device__ __forceinline__ int half() const { return rot >> 1; }
    __device__ __forceinline__ bool first() const { return c0 < half(); }
    __device__ __forceinline__ int other() const { return first() ? c0 + half() : c0 - half(); }     // HALVES: where the pairs' other halves begin
};

// y: the channels; z: the other halves of their pairs (HALVES); angles: rot / 2 cosines, rot / 2 sines.
template <class T> __device__ __forceinline__ void rotate(const Rotation &r, const T *x, const float *angles, float (&y)[8], const float (&z)[8])
{
    const int half = r.half();
    if (r.kind == Rotation::PAIRS) {
        // four pairs; where the rotation ends among them, the angles of the last four, moved up, and none
        const int i = min(r.c0 >> 1, max(half - 4, 0)), by = (r.c0 >> 1) - i;
        float cs[4], sn[4];
        if (half >= 4) {
            __builtin_memcpy(cs, angles + i, 16);
            __builtin_memcpy(sn, angles + half + i, 16);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                cs[j] = j < half ? angles[j] : 1.0f;
                sn[j] = j < half ? angles[half + j] : 0.0f;
            }
        }
        if (by) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = j + by;
                cs[j] = k < 4 ? (k == 1 ? cs[1] : k == 2 ? cs[2] : cs[3]) : 1.0f;
                sn[j] = k < 4 ? (k == 1 ? sn[1] : k == 2 ? sn[2] : sn[3]) : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const double a = y[2 * j], b = y[2 * j + 1], c = cs[j], d = sn[j];
            const bool reached = (r.c0 >> 1) + j < half;  // (what is not keeps its value, whatever its neighbour is)
            y[2 * j] = reached ? static_cast<float>(a * c - b * d) : y[2 * j];
            y[2 * j + 1] = reached ? static_cast<float>(b * c + a * d) : y[2 * j + 1];
        }
    } else if (r.kind == Rotation::HALVES) {
        float cs[8], sn[8];
        const int i = r.first() ? r.c0 : r.other();
        load8(angles + i, cs);
        load8(angles + half + i, sn);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            y[j] = static_cast<float>(static_cast<double>(y[j]) * cs[j] + static_cast<double>(z[j]) * (r.first() ? -sn[j] : sn[j]));
    } else if (r.kind == Rotation::ODD) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = r.c0 + j, i = c < half ? c : c - half;
            if (c >= r.rot) continue;
            const double own = y[j], pair = static_cast<float>(x[c < half ? c + half : i]), cs = angles[i], sn = angles[half + i];
            y[j] = static_cast<float>(own * cs + pair * (c < half ? -sn : sn));
        }
    }
}

// Codes of 8 channels (one 32-bit word) and the scale byte of their group; all lanes of the group call it together.
__device__ __forceinline__ uint32_t codes8(const float (&y)[8], int &byte)
{
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(y[j]) & 0x7FFFFFFFu);
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
    // top = m 2^E with m in [1, 2): the least e with top < 7 2^e = 1.75 2^(e + 2)
    int e = static_cast<int>(top >> 23) - 127 - 2 + ((top & 0x7FFFFFu) >= 0x600000u ? 1 : 0);
    e = min(max(e, -23), 13);
    byte = e + 127;
    const float unit = __uint_as_float(static_cast<uint32_t>(byte) << 23);
    uint32_t w = 0;                                       // the instruction rounds half to even code and stops at 6
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], unit, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], unit, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], unit, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], unit, 3);
    return w;
}

__device__ __forceinline__ bool finite8(const float (&y)[8])
{
    bool ok = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) ok = ok && (__float_as_uint(y[j]) & 0x7FFFFFFFu) < 0x7F800000u;
    return ok;
}

// TEAM lanes (the power of two that holds D / 8) take one row: of a cache head, key and value, or of a query head.
//
// Bound by vector instructions (64 % of the cycles; the rotation's conversions to and from 64 bits lead) and by the way from a
// token's slot and position to its angles: what does not wait for the position is asked for at once, angles are read 16 bytes at a
// time.  8000 tokens, 8 cache and 32 query heads of D = 64, half of the channels rotated in neighbouring pairs: 22 us; four heads
// a team, with a quarter of the look-ups, 52.
template <class T, int D, int TEAM> __global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a, int64_t first)
{
    const int64_t item = first + static_cast<int64_t>(blockIdx.x) * (256 / TEAM) + threadIdx.x / TEAM;
    const int heads = a.c.heads + a.t.q_heads, part = threadIdx.x % TEAM;
    const bool mine = part * 8 < D;
    const int c0 = mine ? part * 8 : 0;
    const int64_t token = quotient(item, heads);
    const int h = static_cast<int>(item - token * heads);
    if (token >= a.t.tokens) return;                      // (a whole team, as below)
    const bool is_query = h >= a.c.heads;
    const Rotation r(c0, a.t.rot, a.t.interleaved);
    const T *x = is_query ? static_cast<const T *>(a.t.q_dev) + token * a.t.q_token_stride + (h - a.c.heads) * a.t.q_head_stride
                          : static_cast<const T *>(a.t.k_dev) + token * a.t.k_token_stride + h * a.t.k_head_stride;
    const int64_t slot = a.t.slot_dev[token], at = a.t.rot ? a.t.position_dev[token] : 0;
    float y[8], z[8] = {}, v[8] = {};
    load8(x + c0, y);
    if (r.kind == Rotation::HALVES) load8(x + r.other(), z);
    if (!is_query) load8(static_cast<const T *>(a.t.v_dev) + token * a.t.v_token_stride + h * a.t.v_head_stride + c0, v);
    __builtin_amdgcn_sched_barrier(0);
    if (slot < 0 || slot >= a.c.pages << a.page_shift || at < 0 || (a.t.rot && at >= a.t.table_rows)) return;
    rotate(r, x, a.t.table_dev + at * a.t.rot, y, z);
    if (is_query) {
        __builtin_amdgcn_wave_barrier();                  // in place: every lane of the team, all of one wave, has read its pairs
        if (mine) store8(y, static_cast<T *>(a.t.q_out_dev) + token * a.t.q_out_token_stride + (h - a.c.heads) * a.t.q_out_head_stride + c0);
        return;
    }
    int bad = !(finite8(y) && finite8(v));
    for (int d = 1; d < TEAM; d <<= 1) bad |= __shfl_xor(bad, d);
    if (bad)
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = v[j] = 0.0f;
    int ky, vy;
    const uint32_t kw = codes8(y, ky), vw = codes8(v, vy);
    if (!mine) return;
    const int64_t row = cache_row(slot, h, a.c.heads, a.page_shift);
    reinterpret_cast<uint32_t *>(a.c.k_codes_dev)[row * (D / 8) + part] = kw;
    reinterpret_cast<uint32_t *>(a.c.v_codes_dev)[row * (D / 8) + part] = vw;
    if (part % 4 == 0) {
        a.c.k_scale_dev[row * (D / 32) + part / 4] = static_cast<uint8_t>(bad ? 255 : ky);
        a.c.v_scale_dev[row * (D / 32) + part / 4] = static_cast<uint8_t>(vy);
    }
}

struct ReadArgs {
    apnn_kv_cache c;
    const int64_t *slot;
    int64_t n;
    void *k, *v;
    int page_shift;
};

// 8 channels of a key row and of a value row a thread.  Bound by memory (8000 tokens of 8 heads, D = 64, to fp16: 7.4 us).
template <class T, int D> __global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a, int64_t first)
{
    const int64_t item = first + static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, line = quotient(item, D / 8);
    const int part = static_cast<int>(item - line * (D / 8));
    const int64_t at = quotient(line, a.c.heads);
    if (at >= a.n) return;
    const int64_t slot = a.slot[at];
    const bool there = slot >= 0 && slot < a.c.pages << a.page_shift;
    const int64_t row = there ? cache_row(slot, static_cast<int>(line - at * a.c.heads), a.c.heads, a.page_shift) : 0;
    const uint32_t key_scale = there ? a.c.k_scale_dev[row * (D / 32) + part / 4] : 0;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        T *out = static_cast<T *>(which ? a.v : a.k);
        if (!out) continue;
        uint32_t w = 0, byte = 127;
        if (there) {
            w = reinterpret_cast<const uint32_t *>(which ? a.c.v_codes_dev : a.c.k_codes_dev)[row * (D / 8) + part];
            byte = which ? a.c.v_scale_dev[row * (D / 32) + part / 4] : key_scale;
            if (key_scale == 255) byte = 255;
        }
        const float unit = __uint_as_float(byte == 255 ? 0x7FC00000u : byte << 23);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t code = w >> (4 * j), low = code & 7;
            // magnitudes in halves: 0 1 2 3 4 6 8 12
            const float half = static_cast<float>(low < 4 ? low : (low < 6 ? 2 * low - 4 : 4 * low - 16));
            y[j] = (code & 8 ? -0.5f : 0.5f) * half * unit;
        }
        store8(y, out + line * D + part * 8);
    }
}

}  // namespace apnn

extern "C" int apnn_kv_append(const apnn_kv_cache *cache, const apnn_kv_tokens *t, void *stream)
{
    using namespace apnn;
    clear_error();
    const char *who = "apnn_kv_append";
    if (const int rc = check_cache(who, cache)) return rc;
    if (!t) return fail(APNN_ERR_INVALID_ARG, "%s: no tokens", who);
    if (!known_type(t->type)) return fail(APNN_ERR_INVALID_ARG, "%s: unknown type %d", who, static_cast<int>(t->type));
    if (t->tokens < 0 || t->q_heads < 0) return fail(APNN_ERR_INVALID_ARG, "%s: tokens = %lld, q_heads = %d", who, (long long)t->tokens, t->q_heads);
    if (t->tokens > INT_MAX || t->q_heads > (1 << 16)) return fail(APNN_ERR_UNSUPPORTED, "%s: tokens = %lld, q_heads = %d", who, (long long)t->tokens, t->q_heads);
    if (t->rot < 0 || t->rot > cache->D || t->rot % 2) return fail(APNN_ERR_INVALID_ARG, "%s: rot = %d of %d channels", who, t->rot, cache->D);
    if (t->tokens == 0) return APNN_OK;
    if (!t->k_dev || !t->v_dev || !t->slot_dev || (t->q_heads && (!t->q_dev || !t->q_out_dev))) return fail(APNN_ERR_INVALID_ARG, "%s: null pointer", who);
    if (t->rot && (!t->table_dev || !t->position_dev || t->table_rows < 0)) return fail(APNN_ERR_INVALID_ARG, "%s: a rotation needs a table and positions", who);
    if (!aligned_to(t->k_dev, t->type) || !aligned_to(t->v_dev, t->type) || (t->q_heads && (!aligned_to(t->q_dev, t->type) || !aligned_to(t->q_out_dev, t->type))))
        return fail(APNN_ERR_ALIGNMENT, "%s: a pointer is not aligned to its type", who);
    const int64_t n = t->tokens, D = cache->D;
    if (!strides_fit(n, cache->heads, D, t->k_token_stride, t->k_head_stride, false) || !strides_fit(n, cache->heads, D, t->v_token_stride, t->v_head_stride, false) ||
        (t->q_heads && (!strides_fit(n, t->q_heads, D, t->q_token_stride, t->q_head_stride, false) ||
                        !strides_fit(n, t->q_heads, D, t->q_out_token_stride, t->q_out_head_stride, true))))
        return fail(APNN_ERR_INVALID_ARG, "%s: strides", who);
    if (t->q_heads && t->q_dev == t->q_out_dev && (t->q_token_stride != t->q_out_token_stride || t->q_head_stride != t->q_out_head_stride))
        return fail(APNN_ERR_INVALID_ARG, "%s: queries rotated in place need the same strides", who);
    const AppendArgs a = {*cache, *t, shift_of(cache->page_size)};
    const int64_t rows = t->tokens * (cache->heads + t->q_heads);
    return by_type(t->type, [&](auto type) {
        return by_channels(cache->D, [&](auto d) {
            constexpr int D = decltype(d)::value, team = D == 96 ? 16 : D / 8;
            in_slices(rows * team, [&](int64_t first, unsigned blocks) {
                kv_append_kernel<decltype(type), D, team><<<blocks, 256, 0, as_stream(stream)>>>(a, first / team);
            });
            return check_launch(who);
        });
    });
}

extern "C" int apnn_kv_read(const apnn_kv_cache *cache, const int64_t *slot_dev, int64_t n, void *k_out_dev, void *v_out_dev, apnn_dtype type, void *stream)
{
    using namespace apnn;
    clear_error();
    const char *who = "apnn_kv_read";
    if (const int rc = check_cache(who, cache)) return rc;
    if (!known_type(type)) return fail(APNN_ERR_INVALID_ARG, "%s: unknown type %d", who, static_cast<int>(type));
    if (n < 0) return fail(APNN_ERR_INVALID_ARG, "%s: n = %lld", who, (long long)n);
    if (n > INT_MAX) return fail(APNN_ERR_UNSUPPORTED, "%s: n = %lld", who, (long long)n);
    if (n == 0 || (!k_out_dev && !v_out_dev)) return APNN_OK;
    if (!slot_dev) return fail(APNN_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned16(k_out_dev) || !aligned16(v_out_dev)) return fail(APNN_ERR_ALIGNMENT, "%s: an output is not 16-byte aligned", who);
    const ReadArgs a = {*cache, slot_dev, n, k_out_dev, v_out_dev, shift_of(cache->page_size)};
    return by_type(type, [&](auto t) {
        return by_channels(cache->D, [&](auto d) {
            constexpr int D = decltype(d)::value;
            in_slices(n * cache->heads * (D / 8), [&](int64_t first, unsigned blocks) {
                kv_read_kernel<decltype(t), D><<<blocks, 256, 0, as_stream(stream)>>>(a, first);
            });
            return check_launch(who);
        });
    });
}
