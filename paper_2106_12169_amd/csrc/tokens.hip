// 8-bit codes with a scale for each row (apnn_quantize_tokens).
//
//   a = max_k |x_k|, scale = a / 127, code_k = 127 x_k / a to the nearest integer, half to even.
//
// The quotient is decided exactly.  127 x / a is a rational whose distance from a half integer is either 0 or at least
// 2^-33: |254 x - (2n + 1) a| is a multiple of the last place of x, which is at least a 2^-32 wherever the tie n + 1/2 is
// within reach, over 2 a.  A 64-bit product with the rounded 127 / a is off by less than 2^-45, so the product rounded
// to a multiple of 2^-36 is the tie where there is one and on the right side of it where there is none.
#include "dense.h"

namespace apnn {

// One block a row: the maximum in a first pass, the codes in a second.
template <class T>
__global__ __launch_bounds__(256) void quantize_tokens_kernel(const T *__restrict__ src, int64_t rows, int K, int64_t ld, int pitch,
                                                              int8_t *__restrict__ codes, float *__restrict__ scale, int64_t first)
{
    __shared__ uint32_t part[4];
    const int64_t row = first + blockIdx.x;
    if (row >= rows) return;
    const T *x = src + row * ld;
    uint32_t top = 0;                                     // magnitudes compare like their bits, infinities and NaN on top
    for (int k = threadIdx.x; k < K; k += 256) top = max(top, __float_as_uint(static_cast<float>(x[k])) & 0x7FFFFFFFu);
    for (int d = 32; d; d >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), d)));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(part[0], part[1]), max(part[2], part[3]));
    const bool finite = top < 0x7F800000u;
    const float a = __uint_as_float(top);
    const double inv = finite && top ? 127.0 / static_cast<double>(a) : 0.0;
    if (threadIdx.x == 0) scale[row] = finite ? a / 127.0f : __uint_as_float(0x7FC00000u);
    int8_t *c = codes + row * pitch;
    for (int k = threadIdx.x; k < pitch; k += 256) {
        int code = 0;
        if (k < K && inv != 0.0) {
            constexpr double grid = 3.0 * 32768.0;        // 1.5 * 2^16: sums with it are multiples of 2^-36
            const double r = static_cast<double>(static_cast<float>(x[k])) * inv;
            code = static_cast<int>(__builtin_rint((r + grid) - grid));
        }
        c[k] = static_cast<int8_t>(code);
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
    if (K > INT_MAX - 1024) return fail(APNN_ERR_UNSUPPORTED, "apnn_quantize_tokens: K = %lld", (long long)K);
    if (rows && ld > INT64_MAX / 8 / rows) return fail(APNN_ERR_INVALID_ARG, "apnn_quantize_tokens: %lld rows of stride %lld", (long long)rows, (long long)ld);
    if (rows == 0) return APNN_OK;
    if ((K && (!src_dev || !codes_dev)) || !scale_dev) return fail(APNN_ERR_INVALID_ARG, "apnn_quantize_tokens: null pointer");
    if (!aligned_to(src_dev, type)) return fail(APNN_ERR_ALIGNMENT, "apnn_quantize_tokens: src is not aligned to its type");
    if (!aligned16(codes_dev)) return fail(APNN_ERR_ALIGNMENT, "apnn_quantize_tokens: codes are not 16-byte aligned");
    const int pitch = static_cast<int>(apnn_token_pitch(K));
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        for (int64_t first = 0; first < rows; first += kMaxBlocks / 4) {
            const int64_t n = rows - first < kMaxBlocks / 4 ? rows - first : kMaxBlocks / 4;
            quantize_tokens_kernel<T><<<static_cast<unsigned>(n), 256, 0, as_stream(stream)>>>(
                static_cast<const T *>(src_dev), rows, static_cast<int>(K), ld, pitch, codes_dev, scale_dev, first);
        }
        return check_launch("apnn_quantize_tokens");
    });
}
