// 8-bit codes with a scale for each row (apnn_quantize_tokens).
//
//   a = max_k |x_k|, scale = a / 127, code_k = 127 x_k / a to the nearest integer, half to even.
//
// The quotient is decided exactly.  127 x / a is a rational whose distance from a half integer is either 0 or at least
// 2^-33: |254 x - (2n + 1) a| is a multiple of the last place of x, which is at least a 2^-32 wherever the tie n + 1/2 is
// within reach, over 2 a.  A 64-bit product with the rounded 127 / a is off by less than 2^-45, so the product rounded
// to a multiple of 2^-36 is the tie where there is one and on the right side of it where there is none.
#include "dense.h"

#include <type_traits>

namespace apnn {

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }     // compare like the values, infinities and NaN on top

// What a row's largest magnitude makes of it.
struct RowScale {
    double inv;                                           // 127 / a, 0 for a row of zeros or with something that is not finite
    float scale;
};
__device__ __forceinline__ RowScale row_scale(uint32_t top)
{
    const float a = __uint_as_float(top);
    if (top >= 0x7F800000u) return {0.0, __uint_as_float(0x7FC00000u)};
    return {top ? 127.0 / static_cast<double>(a) : 0.0, a / 127.0f};
}

__device__ __forceinline__ int code_of(float x, double inv)
{
    constexpr double grid = 3.0 * 32768.0;                // 1.5 * 2^16: sums with it are multiples of 2^-36
    const double r = static_cast<double>(x) * inv;
    return static_cast<int>(__builtin_rint((r + grid) - grid));
}

// Codes of eight elements, 8 bytes; none (inv 0) where the row has nothing to tell apart.
__device__ __forceinline__ void store_codes(const float (&x)[8], double inv, int8_t *to)
{
    uint32_t w[2] = {0, 0};
    if (inv != 0.0)
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j / 4] |= static_cast<uint32_t>(code_of(x[j], inv) & 0xFF) << (8 * (j % 4));
    *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
}

// Eight elements of a row of K from k on, zeros beyond its end.
template <class T> __device__ __forceinline__ void load_row8(const T *x, int k, int K, float (&y)[8])
{
    if (k + 8 <= K) load8(x + k, y);
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = k + j < K ? static_cast<float>(x[k + j]) : 0.0f;
}

// THREADS threads a row, UNITS times 8 elements a thread, held in registers between the maximum and the codes.  Bound by
// memory: the row is read once and its codes written once (6000 x 5003 fp32: 30 us, 5 TB/s).
template <class T, int THREADS, int UNITS>
__global__ __launch_bounds__(256) void quantize_tokens_kernel(const T *__restrict__ src, int64_t rows, int K, int64_t ld, int pitch,
                                                              int8_t *__restrict__ codes, float *__restrict__ scale, int64_t first)
{
    __shared__ uint32_t part[4];
    const int64_t row = first + static_cast<int64_t>(blockIdx.x) * (256 / THREADS) + threadIdx.x / THREADS;
    if (row >= rows) return;                              // (a whole wave, or the whole block)
    const T *x = src + row * ld;
    const int thread = threadIdx.x % THREADS;
    float y[UNITS][8];
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) load_row8(x, (u * THREADS + thread) * 8, K, y[u]);
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(y[u][j]));
    for (int d = 32; d; d >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), d)));
    if constexpr (THREADS == 256) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
        __syncthreads();
        top = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    const RowScale s = row_scale(top);
    if (thread == 0) scale[row] = s.scale;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int k = (u * THREADS + thread) * 8;
        if (k < pitch) store_codes(y[u], s.inv, codes + row * pitch + k);
    }
}

// Rows of any length, a block a row, read twice.
template <class T>
__global__ __launch_bounds__(256) void quantize_tokens_long_kernel(const T *__restrict__ src, int64_t rows, int K, int64_t ld, int pitch,
                                                                   int8_t *__restrict__ codes, float *__restrict__ scale, int64_t first)
{
    __shared__ uint32_t part[4];
    const int64_t row = first + blockIdx.x;
    if (row >= rows) return;
    const T *x = src + row * ld;
    uint32_t top = 0;
    float y[8];
    for (int k = threadIdx.x * 8; k < K; k += 2048) {
        load_row8(x, k, K, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(y[j]));
    }
    for (int d = 32; d; d >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), d)));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    const RowScale s = row_scale(max(max(part[0], part[1]), max(part[2], part[3])));
    if (threadIdx.x == 0) scale[row] = s.scale;
    for (int k = threadIdx.x * 8; k < pitch; k += 2048) {
        load_row8(x, k, K, y);
        store_codes(y, s.inv, codes + row * pitch + k);
    }
}

}  // namespace apnn

extern "C" int64_t apnn_token_pitch(int64_t K) { return K < 0 || K > INT64_MAX - 15 ? 0 : apnn::round_up(K, 16); }

extern "C" int apnn_quantize_tokens(const void *src_dev, apnn_dtype type, int64_t rows, int64_t K, int64_t ld,
                                    int8_t *codes_dev, float *scale_dev, void *stream)
{
    using namespace apnn;
    clear_error();
    if (!known_type(type)) return fail(APNN_ERR_INVALID_ARG, "apnn_quantize_tokens: unknown type %d", static_cast<int>(type));
    if (rows < 0 || K < 0 || ld < K) return fail(APNN_ERR_INVALID_ARG, "apnn_quantize_tokens: rows = %lld, K = %lld, ld = %lld", (long long)rows, (long long)K, (long long)ld);
    if (K > (int64_t(1) << 30)) return fail(APNN_ERR_UNSUPPORTED, "apnn_quantize_tokens: K = %lld", (long long)K);
    if (rows && ld > INT64_MAX / 8 / rows) return fail(APNN_ERR_INVALID_ARG, "apnn_quantize_tokens: %lld rows of stride %lld", (long long)rows, (long long)ld);
    if (rows == 0) return APNN_OK;
    if ((K && (!src_dev || !codes_dev)) || !scale_dev) return fail(APNN_ERR_INVALID_ARG, "apnn_quantize_tokens: null pointer");
    if (!aligned_to(src_dev, type)) return fail(APNN_ERR_ALIGNMENT, "apnn_quantize_tokens: src is not aligned to its type");
    if (!aligned16(codes_dev)) return fail(APNN_ERR_ALIGNMENT, "apnn_quantize_tokens: codes are not 16-byte aligned");
    const int pitch = static_cast<int>(apnn_token_pitch(K));
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        const T *src = static_cast<const T *>(src_dev);
        // a wave a row up to 2048 codes, a block up to 16384, as few registers as hold it
        const auto go = [&](auto threads, auto units) {
            constexpr int n = decltype(threads)::value, u = decltype(units)::value;
            for (int64_t first = 0; first < rows; first += kMaxBlocks / 4)
                quantize_tokens_kernel<T, n, u><<<static_cast<unsigned>(ceil_div(rows - first < kMaxBlocks / 4 ? rows - first : kMaxBlocks / 4, 256 / n)), 256, 0, as_stream(stream)>>>(
                    src, rows, static_cast<int>(K), ld, pitch, codes_dev, scale_dev, first);
        };
        using std::integral_constant;
        if (pitch <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
        else if (pitch <= 1024) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
        else if (pitch <= 2048) go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
        else if (pitch <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
        else if (pitch <= 8192) go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
        else if (pitch <= 16384) go(integral_constant<int, 256>{}, integral_constant<int, 8>{});
        else
            for (int64_t first = 0; first < rows; first += kMaxBlocks / 4)
                quantize_tokens_long_kernel<T><<<static_cast<unsigned>(rows - first < kMaxBlocks / 4 ? rows - first : kMaxBlocks / 4), 256, 0, as_stream(stream)>>>(
                    src, rows, static_cast<int>(K), ld, pitch, codes_dev, scale_dev, first);
        return check_launch("apnn_quantize_tokens");
    });
}
