// Products of 8-bit codes with a scale for each token and each output channel (apnn_gemm_scaled).
//
//   Y[m][n] = x_scale[m] w_scale[n] sum_k X[m][k] W[n][k] + bias[n]
//
// The sum is exact in int32 (K 2^14 < 2^31 is checked).  It is scaled in fp32 by the scales' mantissas and then by the sum
// of their exponents, so that no intermediate overflows or vanishes: four roundings of 2^-24 before the result's own.
// Both kernels take W as the matrix instruction's rows: a lane then ends with neighbouring channels of one token.
#include "dense.h"
#include "lane_util.h"
#include "lds_load.h"

namespace apnn {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

struct ScaledGemm {
    const int8_t *X, *W;
    const float *x_scale, *w_scale, *bias;
    void *Y;
    int64_t ldy;
    int M, N, pitch;                                      // pitch: bytes of a row of X and W
    int across, tiles;                                    // tiles of a row of tiles, of the result
    bool wide;                                            // rows of Y can be written 16 bytes at a time
};

struct Scale {
    float part;                                           // 0.5 <= |part| < 1, or what has no exponent
    int exponent;
};
__device__ __forceinline__ Scale scale_of(float s) { return {__builtin_amdgcn_frexp_mantf(s), __builtin_amdgcn_frexp_expf(s)}; }
__device__ __forceinline__ float scaled(int acc, Scale x, Scale w, float bias)
{
    return __builtin_amdgcn_ldexpf(static_cast<float>(acc) * x.part * w.part, x.exponent + w.exponent) + bias;
}

// Tile of a block: blocks go to the eight XCDs in turn; each XCD gets a run of neighbouring tiles, walked in panels of four
// rows of tiles, so that what its compute units read together stays in its own L2.
__device__ __forceinline__ void tile_of(const ScaledGemm &p, int id, int &tm, int &tn)
{
    const int xcd = id & 7, each = p.tiles >> 3, more = p.tiles & 7;
    const int t = xcd * each + min(xcd, more) + (id >> 3);
    const int down = p.tiles / p.across, panel = t / (4 * p.across), rows = min(4, down - 4 * panel), in = t - 4 * panel * p.across;
    tm = 4 * panel + in % rows;
    tn = in / rows;
}

// 64 F x 64 F outputs a block, 32 F x 32 F a wave, K in chunks of 128 bytes, two of them in LDS.
//
// Bound by the matrix unit (F = 4: 256 accumulators, one wave a SIMD).  A chunk is loaded straight to LDS while the one
// before it is multiplied, its 16-byte pieces swizzled by row so that fragment reads meet no bank twice; the fragments of a
// step are read while the step before it is multiplied, one read or load behind each matrix instruction.
template <class T, int F> __global__ __launch_bounds__(256, F == 4 ? 1 : 2) void gemm_scaled_tile_kernel(ScaledGemm p)
{
    constexpr int EDGE = 64 * F, CHUNK = 128, SIDE = EDGE * CHUNK, STEPS = CHUNK / 32, LOADS = 2 * F;   // loads of a wave, chunk and operand
    extern __shared__ __attribute__((aligned(16))) char gemm_lds[];      // [2 buffers][W, X][EDGE][CHUNK]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, half = lane >> 5;
    const int wn = wave & 1, wm = wave >> 1;
    int tm, tn;
    tile_of(p, blockIdx.x, tm, tn);
    const int m0 = tm * EDGE, n0 = tn * EDGE;

    // loader: a wave's load u covers rows 16 F wave + 8 u .. + 7 of the tile, lane l row l / 8, piece (l % 8) ^ (l / 8)
    const v4u_t from[2] = {make_raw_desc(p.W + static_cast<int64_t>(n0) * p.pitch, static_cast<uint32_t>(min(EDGE, p.N - n0)) * p.pitch),
                           make_raw_desc(p.X + static_cast<int64_t>(m0) * p.pitch, static_cast<uint32_t>(min(EDGE, p.M - m0)) * p.pitch)};
    const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)gemm_lds));
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const uint32_t row_at = static_cast<uint32_t>(wave * 16 * F + (lane >> 3)) * p.pitch + piece;
    const int chunks = (p.pitch + CHUNK - 1) / CHUNK;
    const auto load = [&](int chunk, int buf, auto uc) {
        constexpr int u = decltype(uc)::value, side = u / LOADS, v = u % LOADS;
        // (beyond the row's end, or the last chunk: out of the descriptor's range, so zeros)
        const uint32_t at = chunk * CHUNK + piece < p.pitch ? row_at + chunk * CHUNK : 0x80000000u;
        load_to_lds_16(from[side], lds_base + (2 * buf + side) * SIDE + (wave * 16 * F + 8 * v) * CHUNK, at + static_cast<uint32_t>(8 * v) * p.pitch, 0);
    };

    // fragments of a step: rows 32 (F w + f) + r, piece (2 step + half) ^ (r % 8)
    const int frag_at = r * CHUNK + ((half ^ (r & 7)) << 4);
    i32x4_t fw[2][F], fx[2][F];
    const auto read = [&](int buf, auto sc, auto fc) {
        constexpr int s = decltype(sc)::value, f = decltype(fc)::value;
        const int at = 2 * buf * SIDE + (frag_at ^ (32 * s)) + (f % F) * 32 * CHUNK;
        if constexpr (f < F) fw[s & 1][f] = *reinterpret_cast<const i32x4_t *>(gemm_lds + at + wn * 32 * F * CHUNK);
        else fx[s & 1][f - F] = *reinterpret_cast<const i32x4_t *>(gemm_lds + at + SIDE + wm * 32 * F * CHUNK);
    };

    i32x16_t acc[F][F] = {};
    using I0 = std::integral_constant<int, 0>;
    constexpr int VMCNT0 = 0x0F70;
    static_for<2 * LOADS>([&](auto u) { load(0, 0, u); });
    static_for<2 * LOADS>([&](auto u) { load(1, 1, u); });
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS) : "memory");       // the first chunk has landed
    __syncthreads();
    if (chunks) static_for<2 * F>([&](auto f) { read(0, I0{}, f); });
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int buf = chunk & 1;
        static_for<STEPS>([&](auto sc) {
            constexpr int s = decltype(sc)::value, next = (s + 1) % STEPS;
            if constexpr (s == STEPS - 1) {
                __builtin_amdgcn_s_waitcnt(VMCNT0);       // the next chunk has landed, and everyone has read this one
                __syncthreads();
            }
            static_for<F * F>([&](auto qc) {
                constexpr int q = decltype(qc)::value;
                acc[q / F][q % F] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[s & 1][q / F], fx[s & 1][q % F], acc[q / F][q % F], 0, 0, 0);
                constexpr int reads = 2 * F * (q + 1) / (F * F) - 2 * F * q / (F * F);
                static_for<reads>([&](auto i) {
                    read(s == STEPS - 1 ? buf ^ 1 : buf, std::integral_constant<int, next>{}, std::integral_constant<int, 2 * F * q / (F * F) + decltype(i)::value>{});
                });
                if constexpr (s == STEPS - 1) {
                    constexpr int loads = 2 * LOADS * (q + 1) / (F * F) - 2 * LOADS * q / (F * F);
                    static_for<loads>([&](auto i) { load(chunk + 2, buf, std::integral_constant<int, 2 * LOADS * q / (F * F) + decltype(i)::value>{}); });
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    }
    __builtin_amdgcn_s_waitcnt(VMCNT0);                   // the loads beyond the last chunk are done with LDS
    __syncthreads();

    // results: 32 tokens at a time through LDS, so that whole runs of channels of a token leave together
    constexpr int ROW = 32 * F * static_cast<int>(sizeof(T)) + 16, REGION = 32 * (32 * F * 4 + 16);
    float *const wide_scale = reinterpret_cast<float *>(gemm_lds + 4 * REGION);      // [EDGE] mantissa, exponent, bias
    for (int i = threadIdx.x; i < EDGE; i += 256) {
        const int n = n0 + i;
        const Scale w = scale_of(n < p.N ? p.w_scale[n] : 0.0f);
        wide_scale[3 * i] = w.part;
        wide_scale[3 * i + 1] = __int_as_float(w.exponent);
        wide_scale[3 * i + 2] = p.bias && n < p.N ? p.bias[n] : 0.0f;
    }
    __syncthreads();
    char *const mine = gemm_lds + wave * REGION;
    static_for<F>([&](auto fm) {
        constexpr int b = decltype(fm)::value;
        const int mt = m0 + (wm * F + b) * 32;
        const Scale x = scale_of(mt + r < p.M ? p.x_scale[mt + r] : 0.0f);
        static_for<4 * F>([&](auto gc) {
            constexpr int g = decltype(gc)::value, f = g / 4;
            const int ch = f * 32 + 8 * (g % 4) + 4 * half;           // of the wave's channels
            T y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float *w = wide_scale + 3 * (wn * 32 * F + ch + j);
                y[j] = static_cast<T>(scaled(acc[f][b][4 * (g % 4) + j], x, Scale{w[0], __float_as_int(w[1])}, w[2]));
            }
            __builtin_memcpy(mine + r * ROW + ch * sizeof(T), y, sizeof y);
        });
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        constexpr int V = 16 / static_cast<int>(sizeof(T)), LANES = 32 * F / V;       // lanes of a row
#pragma unroll
        for (int i = 0; i < 32 * LANES / 64; ++i) {
            const int at = i * 64 + lane, row = at / LANES, ch = at % LANES * V, m = mt + row, n = n0 + wn * 32 * F + ch;
            if (m >= p.M || n >= p.N) continue;
            const Pack16<T> v = *reinterpret_cast<const Pack16<T> *>(mine + row * ROW + ch * sizeof(T));
            T *y = static_cast<T *>(p.Y) + m * p.ldy + n;
            if (p.wide && n + V <= p.N) *reinterpret_cast<Pack16<T> *>(y) = v;
            else
                for (int j = 0; j < V && n + j < p.N; ++j) y[j] = v.v[j];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    });
}

// Few tokens: 16 MT tokens x 16 NT channels a block, the block's waves sharing K in turns of 256 bytes.
//
// Bound by reading W once.  Lanes load fragments straight from memory, a load of 16 rows taking 64 neighbouring bytes of each
// and the four loads of a turn 256 (the order of K within a turn is free, the same for both operands).  The next turn is in
// flight while one is multiplied.  X comes from L2 again for each block: MT / NT bytes for each byte of W.
template <class T, int MT, int NT, int WAVES> __global__ __launch_bounds__(64 * WAVES) void gemm_scaled_few_kernel(ScaledGemm p)
{
    constexpr int TURN = 256;
    __shared__ i32x4_t sums[WAVES][NT][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, quarter = lane >> 4;
    const int n0 = static_cast<int>(blockIdx.x) % p.across * 16 * NT, m0 = static_cast<int>(blockIdx.x) / p.across * 16 * MT;
    const int8_t *w[NT], *x[MT];
#pragma unroll
    for (int i = 0; i < NT; ++i) w[i] = p.W + static_cast<int64_t>(min(n0 + 16 * i + r, p.N - 1)) * p.pitch + 16 * quarter;
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = p.X + static_cast<int64_t>(min(m0 + 16 * i + r, p.M - 1)) * p.pitch + 16 * quarter;
    i32x4_t acc[NT][MT] = {};
    struct Turn { i32x4_t a[4][NT], b[4][MT]; };
    const auto fetch = [&](int k) {
        Turn t;
        const bool whole = k + TURN <= p.pitch;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = whole || k + 16 * quarter + 64 * j < p.pitch;
            const int at = in ? k + 64 * j : -16 * quarter;            // (beyond the end: the row's first bytes, for nothing)
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                t.a[j][i] = *reinterpret_cast<const i32x4_t *>(w[i] + at);
                if (!in) t.a[j][i] = i32x4_t{};
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) t.b[j][i] = *reinterpret_cast<const i32x4_t *>(x[i] + at);
        }
        return t;
    };
    const auto multiply = [&](const Turn &t) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int l = 0; l < MT; ++l) acc[i][l] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t.a[j][i], t.b[j][l], acc[i][l], 0, 0, 0);
    };
    int k = wave * TURN;
    if (k < p.pitch) {
        Turn now = fetch(k);
        for (k += WAVES * TURN; k < p.pitch; k += WAVES * TURN) {
            const Turn next = fetch(k);
            multiply(now);
            now = next;
        }
        multiply(now);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int l = 0; l < MT; ++l) sums[wave][i][l][lane] = acc[i][l];
    __syncthreads();
    for (int t = threadIdx.x; t < NT * MT * 64; t += 64 * WAVES) {
        const int at = t & 63, l = t / 64 % MT, i = t / 64 / MT, m = m0 + 16 * l + (at & 15), n = n0 + 16 * i + 4 * (at >> 4);
        if (m >= p.M) continue;
        i32x4_t sum = sums[0][i][l][at];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += sums[v][i][l][at];
        const Scale sx = scale_of(p.x_scale[m]);
        T *y = static_cast<T *>(p.Y) + m * p.ldy + n;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n + j < p.N) y[j] = static_cast<T>(scaled(sum[j], sx, scale_of(p.w_scale[n + j]), p.bias ? p.bias[n + j] : 0.0f));
    }
}

template <class T, int F> int launch_tiles(ScaledGemm p, hipStream_t st)
{
    constexpr int edge = 64 * F, bytes = 4 * edge * 128;
    p.across = static_cast<int>(ceil_div(p.N, edge));
    p.tiles = p.across * static_cast<int>(ceil_div(p.M, edge));
    if constexpr (bytes > 64 * 1024) {
        static std::atomic<uint64_t> granted{0};
        if (!all_of_lds(gemm_scaled_tile_kernel<T, F>, granted)) return fail(APNN_ERR_DEVICE, "apnn_gemm_scaled: no %d bytes of LDS", bytes);
    }
    gemm_scaled_tile_kernel<T, F><<<static_cast<unsigned>(p.tiles), 256, bytes, st>>>(p);
    return check_launch("apnn_gemm_scaled");
}

template <class T, int MT, int NT> int launch_few(ScaledGemm p, hipStream_t st)
{
    p.across = static_cast<int>(ceil_div(p.N, 16 * NT));
    p.tiles = p.across * static_cast<int>(ceil_div(p.M, 16 * MT));
    gemm_scaled_few_kernel<T, MT, NT, 8><<<static_cast<unsigned>(p.tiles), 512, 0, st>>>(p);
    return check_launch("apnn_gemm_scaled");
}

template <class T> int launch_scaled(const ScaledGemm &p, hipStream_t st)
{
    if (p.M <= 16) return launch_few<T, 1, 1>(p, st);
    if (p.M <= 32) return launch_few<T, 2, 2>(p, st);
    if (p.M <= 48) return launch_few<T, 3, 2>(p, st);
    if (p.M <= 64) return launch_few<T, 4, 2>(p, st);
    const auto blocks = [&](int edge) { return ceil_div(p.M, edge) * ceil_div(p.N, edge); };
    if (blocks(256) >= 192) return launch_tiles<T, 4>(p, st);
    if (blocks(128) >= 192) return launch_tiles<T, 2>(p, st);
    return launch_tiles<T, 1>(p, st);
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
    if (M > (1 << 26) || N > (1 << 26) || M * N > (int64_t(1) << 35) || ldy > INT64_MAX / 8 / M)
        return fail(APNN_ERR_UNSUPPORTED, "apnn_gemm_scaled: M = %lld, N = %lld, ldy = %lld", (long long)M, (long long)N, (long long)ldy);
    ScaledGemm p = {X_dev, W_dev, x_scale_dev, w_scale_dev, bias_dev, Y_dev, ldy, static_cast<int>(M), static_cast<int>(N), static_cast<int>(apnn_token_pitch(K)), 0, 0, false};
    p.wide = aligned16(Y_dev) && ldy * size_of(type) % 16 == 0;
    return by_type(type, [&](auto t) { return launch_scaled<decltype(t)>(p, as_stream(stream)); });
}
