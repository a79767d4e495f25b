// Products of 8-bit codes with a scale for each token and each output channel (apnn_gemm_scaled).
//
//   Y[m][n] = x_scale[m] w_scale[n] sum_k X[m][k] W[n][k] + bias[n]
//
// The sum is exact in int32 (K 2^14 < 2^31 is checked); it is scaled in 64 bits, where no product of a sum and two
// scales loses digits, overflows or vanishes, and rounded once to 32 bits and once to the result's type.
#include "dense.h"

namespace apnn {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));

struct ScaledGemm {
    const int8_t *X, *W;
    const float *x_scale, *w_scale, *bias;
    void *Y;
    int64_t M, N, ldy;
    int pitch;                                            // bytes of a row of X and W
};

template <class T> __device__ __forceinline__ T scaled(int acc, double sx, double sw, double bias)
{
    return static_cast<T>(static_cast<float>(static_cast<double>(acc) * sx * sw + bias));
}

// 64 x 64 outputs a block, 32 x 32 a wave, operands straight from memory.
template <class T> __global__ __launch_bounds__(256) void gemm_scaled_kernel(ScaledGemm p, int64_t first)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, half = lane >> 5;
    const int64_t tile = first + blockIdx.x, across = (p.N + 63) / 64;
    const int64_t m0 = tile / across * 64 + (wave >> 1) * 32, n0 = tile % across * 64 + (wave & 1) * 32;
    const int64_t m = m0 + r < p.M ? m0 + r : p.M - 1, n = n0 + r < p.N ? n0 + r : p.N - 1;
    const int8_t *x = p.X + m * p.pitch, *w = p.W + n * p.pitch;
    i32x16_t acc = {};
    for (int k = 16 * half; k < p.pitch + 16 * half; k += 32) {
        i32x4_t a = {}, b = {};
        if (k < p.pitch) {
            a = *reinterpret_cast<const i32x4_t *>(x + k);
            b = *reinterpret_cast<const i32x4_t *>(w + k);
        }
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc, 0, 0, 0);
    }
    const int64_t col = n0 + r;
    if (col >= p.N) return;
    const double sw = p.w_scale[col], bias = p.bias ? p.bias[col] : 0.0f;
    for (int i = 0; i < 16; ++i) {
        const int64_t row = m0 + 8 * (i / 4) + 4 * half + i % 4;
        if (row < p.M) static_cast<T *>(p.Y)[row * p.ldy + col] = scaled<T>(acc[i], p.x_scale[row], sw, bias);
    }
}

}  // namespace apnn

extern "C" int apnn_gemm_scaled(const int8_t *X_dev, const float *x_scale_dev, const int8_t *W_dev, const float *w_scale_dev,
                                const float *bias_dev, void *Y_dev, apnn_dtype type, int64_t M, int64_t N, int64_t K, int64_t ldy, void *stream)
{
    using namespace apnn;
    clear_error();
    if (!known_type(type)) return fail(APNN_ERR_INVALID_ARG, "apnn_gemm_scaled: unknown type %d", static_cast<int>(type));
    if (M < 0 || N < 0 || K < 0 || ldy < N)
        return fail(APNN_ERR_INVALID_ARG, "apnn_gemm_scaled: M = %lld, N = %lld, K = %lld, ldy = %lld", (long long)M, (long long)N, (long long)K, (long long)ldy);
    if (K >= (int64_t(1) << 17)) return fail(APNN_ERR_OVERFLOW, "apnn_gemm_scaled: K 2^14 = %lld 2^14 does not fit int32", (long long)K);
    if (M == 0 || N == 0) return APNN_OK;
    if ((K && (!X_dev || !W_dev)) || !x_scale_dev || !w_scale_dev || !Y_dev) return fail(APNN_ERR_INVALID_ARG, "apnn_gemm_scaled: null pointer");
    if (!aligned16(X_dev) || !aligned16(W_dev)) return fail(APNN_ERR_ALIGNMENT, "apnn_gemm_scaled: codes are not 16-byte aligned");
    if (!aligned_to(Y_dev, type)) return fail(APNN_ERR_ALIGNMENT, "apnn_gemm_scaled: Y is not aligned to its type");
    if (M > INT_MAX || N > INT_MAX || ldy > INT64_MAX / 8 / M)
        return fail(APNN_ERR_UNSUPPORTED, "apnn_gemm_scaled: M = %lld, N = %lld, ldy = %lld", (long long)M, (long long)N, (long long)ldy);
    const ScaledGemm p = {X_dev, W_dev, x_scale_dev, w_scale_dev, bias_dev, Y_dev, M, N, ldy, static_cast<int>(apnn_token_pitch(K))};
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        const int64_t tiles = ceil_div(N, 64) * ceil_div(M, 64);
        for (int64_t first = 0; first < tiles; first += kMaxBlocks)
            gemm_scaled_kernel<T><<<static_cast<unsigned>(tiles - first < kMaxBlocks ? tiles - first : kMaxBlocks), 256, 0, as_stream(stream)>>>(p, first);
        return check_launch("apnn_gemm_scaled");
    });
}
