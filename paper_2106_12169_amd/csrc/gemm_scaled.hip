// Products of 8-bit codes with a scale for each token and each output channel (apnn_gemm_scaled).
//
//   Y[m][n] = x_scale[m] w_scale[n] sum_k X[m][k] W[n][k] + bias[n]
//
// The sum is exact in int32 (K 2^14 < 2^31 is checked).  It is scaled in fp32 by the scales' mantissas and then by the sum
// of their exponents, so that no intermediate overflows or vanishes: four roundings of 2^-24 before the result's own.
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
    bool stream;                                          // the result is too large to wait in L2 for its reader
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

// 64 F x 64 F outputs a block, 32 F x 32 F a wave, K in chunks of 128 bytes, STAGES of them in LDS.
//
// Bound by the matrix unit (F = 4: 256 accumulators, one wave a SIMD).  A chunk is loaded straight to LDS while the one
// before it is multiplied, its 16-byte pieces swizzled by row so that fragment reads meet no bank twice; the fragments of a
// step are read while the step before it is multiplied, one read or load behind each matrix instruction.
//
// The sums leave through LDS, 32 tokens at a time (a store to LDS takes them from the accumulators' half of the register file
// as they are), to lanes that keep the same channels for all tokens: those channels' scales stay in registers, and a lane
// stores 16 bytes, past L2 where the result is 16 MiB or more (33 MB: 18.1 us without the products, 13.9 so; 16.8 MB: 13.3, 10.9;
// 8.4 MB: 9.3, 8.8, left to L2 for its reader).  Its code is a loop: unrolled over the accumulators it was 72 KB that every launch fetched anew: 17 us of
// 4096 x 4096 outputs where this takes 9.  4096^3 in 64 us: 26 ns a matrix instruction with random codes, 17.6 with zeros, as the
// clock gives way to the power the products take.
template <class T, int F, int STAGES> __global__ __launch_bounds__(256, F == 4 ? 1 : 2) void gemm_scaled_tile_kernel(ScaledGemm p)
{
    constexpr int EDGE = 64 * F, CHUNK = 128, SIDE = EDGE * CHUNK, STEPS = CHUNK / 32, LOADS = 2 * F;   // loads of a wave, chunk and operand
    extern __shared__ __attribute__((aligned(16))) char gemm_lds[];      // [STAGES][W, X][EDGE][CHUNK]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, half = lane >> 5;
    const int wn = wave & 1, wm = wave >> 1;
    int tm, tn;
    tile_of(p, blockIdx.x, tm, tn);
    const int m0 = tm * EDGE, n0 = tn * EDGE;

    // loader: a wave's load u covers rows 16 F wave + 8 u .. + 7 of a side, lane l row l / 8, piece (l % 8) ^ (l / 8)
    const v4u_t from[2] = {make_raw_desc(p.W + static_cast<int64_t>(n0) * p.pitch, static_cast<uint32_t>(min(EDGE, p.N - n0)) * p.pitch),
                           make_raw_desc(p.X + static_cast<int64_t>(m0) * p.pitch, static_cast<uint32_t>(min(EDGE, p.M - m0)) * p.pitch)};
    const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)gemm_lds));
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const uint32_t row_at = static_cast<uint32_t>(wave * 16 * F + (lane >> 3)) * p.pitch + piece;
    const int chunks = (p.pitch + CHUNK - 1) / CHUNK;
    const auto load = [&](int chunk, int stage, auto uc) {
        constexpr int u = decltype(uc)::value, side = u / LOADS, v = u % LOADS;
        // (beyond the row's end, or the last chunk: out of the descriptor's range, so zeros)
        const uint32_t at = chunk * CHUNK + piece < p.pitch ? row_at + chunk * CHUNK : 0x80000000u;
        load_to_lds_16(from[side], lds_base + (2 * stage + side) * SIDE + (wave * 16 * F + 8 * v) * CHUNK, at + static_cast<uint32_t>(8 * v) * p.pitch, 0);
    };

    // fragments of a step: rows 32 (F w + f) + r, piece (2 step + half) ^ (r % 8)
    const int frag_at = r * CHUNK + ((half ^ (r & 7)) << 4);
    i32x4_t fw[2][F], fx[2][F];
    const auto read = [&](int stage, auto sc, auto fc) {
        constexpr int s = decltype(sc)::value, f = decltype(fc)::value;
        const int at = 2 * stage * SIDE + (frag_at ^ (32 * s)) + (f % F) * 32 * CHUNK;
        if constexpr (f < F) fw[s & 1][f] = *reinterpret_cast<const i32x4_t *>(gemm_lds + at + wn * 32 * F * CHUNK);
        else fx[s & 1][f - F] = *reinterpret_cast<const i32x4_t *>(gemm_lds + at + SIDE + wm * 32 * F * CHUNK);
    };

    i32x16_t acc[F][F] = {};
    using I0 = std::integral_constant<int, 0>;
    constexpr int VMCNT0 = 0x0F70;
    static_for<STAGES>([&](auto st) { static_for<2 * LOADS>([&](auto u) { load(decltype(st)::value, decltype(st)::value, u); }); });
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 1) * 2 * LOADS) : "memory");        // the first chunk has landed
    __syncthreads();
    if (chunks) static_for<2 * F>([&](auto f) { read(0, I0{}, f); });
    for (int chunk = 0, stage = 0; chunk < chunks; ++chunk) {
        const int after = stage + 1 == STAGES ? 0 : stage + 1;
        static_for<STEPS>([&](auto sc) {
            constexpr int s = decltype(sc)::value, next = (s + 1) % STEPS;
            if constexpr (s == STEPS - 1) {
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 2) * 2 * LOADS) : "memory");
                __syncthreads();                          // the next chunk has landed, and everyone has read this one
            }
            static_for<F * F>([&](auto qc) {
                constexpr int q = decltype(qc)::value;
                acc[q / F][q % F] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[s & 1][q / F], fx[s & 1][q % F], acc[q / F][q % F], 0, 0, 0);
                constexpr int reads = 2 * F * (q + 1) / (F * F) - 2 * F * q / (F * F);
                static_for<reads>([&](auto i) {
                    read(s == STEPS - 1 ? after : stage, std::integral_constant<int, next>{}, std::integral_constant<int, 2 * F * q / (F * F) + decltype(i)::value>{});
                });
                if constexpr (s == STEPS - 1) {
                    constexpr int loads = 2 * LOADS * (q + 1) / (F * F) - 2 * LOADS * q / (F * F);
                    static_for<loads>([&](auto i) { load(chunk + STAGES, stage, std::integral_constant<int, 2 * LOADS * q / (F * F) + decltype(i)::value>{}); });
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        stage = after;
    }
    __builtin_amdgcn_s_waitcnt(VMCNT0);                   // the loads beyond the last chunk are done with LDS
    __syncthreads();

    constexpr int V = 16 / static_cast<int>(sizeof(T)), LANES = 32 * F / V, ROW = 32 * F * 4 + 16, REGION = 32 * ROW + 32 * F * 4;
    char *const mine = gemm_lds + wave * REGION;
    float *const x_scale = reinterpret_cast<float *>(mine + 32 * ROW);   // of the wave's 32 F tokens
    const int mw = m0 + wm * 32 * F, n = n0 + wn * 32 * F + lane % LANES * V;
    float w[V], bias[V];
    bool far = false;                                     // a scale outside 2^-60 .. 2^60: the others can be multiplied as they are
#pragma unroll
    for (int j = 0; j < V; ++j) {
        w[j] = n + j < p.N ? p.w_scale[n + j] : 0.0f;
        bias[j] = p.bias && n + j < p.N ? p.bias[n + j] : 0.0f;
        far |= abs(scale_of(w[j]).exponent) > 60;
    }
#pragma unroll 1
    for (int i = lane; i < 32 * F; i += 64) {
        const float x = mw + i < p.M ? p.x_scale[mw + i] : 0.0f;
        x_scale[i] = x;
        far |= abs(scale_of(x).exponent) > 60;
    }
    far = __any(far);
    static_for<F>([&](auto fm) {
        constexpr int b = decltype(fm)::value;
        static_for<4 * F>([&](auto gc) {
            constexpr int g = decltype(gc)::value, f = g / 4;
            *reinterpret_cast<i32x4_t *>(mine + r * ROW + (f * 32 + 8 * (g % 4) + 4 * half) * 4) =
                i32x4_t{acc[f][b][4 * (g % 4)], acc[f][b][4 * (g % 4) + 1], acc[f][b][4 * (g % 4) + 2], acc[f][b][4 * (g % 4) + 3]};
        });
        lds_in_order();
        const char *from_lds = mine + lane / LANES * ROW + lane % LANES * V * 4;
        const float *x = x_scale + 32 * b + lane / LANES;
        constexpr int DOWN = 64 / LANES;                  // rows that lie between two of a lane's
        const auto leave = [&](int i, const T (&y)[V]) {
            const int m = mw + 32 * b + lane / LANES + i;
            T *const to = static_cast<T *>(p.Y) + m * p.ldy + n;
            if (m < p.M && n + V <= p.N) {
                if (p.stream) __builtin_nontemporal_store(__builtin_bit_cast(i32x4_t, y), reinterpret_cast<i32x4_t *>(to));
                else __builtin_memcpy(to, y, sizeof y);   // (wherever a row begins)
            } else if (m < p.M)
#pragma unroll
                for (int j = 0; j < V - 1; ++j)
                    if (n + j < p.N) to[j] = y[j];
        };
        if (far) {
#pragma unroll 1
            for (int i = 0; i < 32; i += DOWN) {
                T y[V];
#pragma unroll
                for (int j = 0; j < V; ++j) y[j] = static_cast<T>(scaled(reinterpret_cast<const int *>(from_lds + i * ROW)[j], scale_of(x[i]), scale_of(w[j]), bias[j]));
                leave(i, y);
            }
        } else {
            constexpr int AT_ONCE = 32 / DOWN < 4 ? 32 / DOWN : 4;
#pragma unroll 1
            for (int i = 0; i < 32; i += AT_ONCE * DOWN) {
                i32x4_t sum[AT_ONCE][V / 4];
                float xs[AT_ONCE];
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) {
                    xs[u] = x[i + u * DOWN];
#pragma unroll
                    for (int j = 0; j < V / 4; ++j) sum[u][j] = *reinterpret_cast<const i32x4_t *>(from_lds + (i + u * DOWN) * ROW + 16 * j);
                }
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) {
                    T y[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) y[j] = static_cast<T>(static_cast<float>(sum[u][j / 4][j % 4]) * xs[u] * w[j] + bias[j]);
                    leave(i + u * DOWN, y);
                }
            }
        }
        lds_in_order();
    });
}

// Few tokens: 16 MT tokens x 16 NT channels a block, the block's waves sharing K in turns of 128 bytes.
//
// Bound by reading W once.  Lanes of a fragment read straight from memory lie a row apart, which costs the address unit four
// times as long as neighbours do (M = 40, N = 10240, K = 5120: 35 us; 13.5 as it is), so a wave brings its turns through LDS: eight
// neighbours load a whole 128-byte line of a row, its pieces swizzled by row for the fragment reads.  A wave has LDS of its own, STAGES turns
// of it in flight, and waits for nobody before the sums are joined.  X comes from L2 for each block: MT / NT bytes for each
// byte of W; rows beyond M are out of the buffer's range and cost nothing.
template <class T, int MT, int NT, int WAVES, int STAGES> __global__ __launch_bounds__(64 * WAVES) void gemm_scaled_few_kernel(ScaledGemm p)
{
    constexpr int TURN = 128, STAGE = (NT + MT) * 16 * TURN;
    static_assert(STAGES * STAGE >= NT * MT * 1024, "the sums are joined in the same LDS");
    __shared__ alignas(16) char lds[WAVES][STAGES * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, quarter = lane >> 4;
    const int n0 = static_cast<int>(blockIdx.x) % p.across * 16 * NT, m0 = static_cast<int>(blockIdx.x) / p.across * 16 * MT;
    const v4u_t W = make_raw_desc(p.W + static_cast<int64_t>(n0) * p.pitch, static_cast<uint32_t>(min(16 * NT, p.N - n0)) * p.pitch);
    const v4u_t X = make_raw_desc(p.X + static_cast<int64_t>(m0) * p.pitch, static_cast<uint32_t>(min(16 * MT, p.M - m0)) * p.pitch);
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds[wave]));
    // loader: lane l has row l / 8 of 8, piece (l % 8) ^ (l / 8); reader: lane l row l % 16, piece 4 step + l / 16
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const uint32_t row_at = static_cast<uint32_t>(lane >> 3) * p.pitch + piece;
    const int frag_at = r * TURN + ((quarter ^ (r & 7)) << 4);
    const auto fetch = [&](int k, int stage) {
        const uint32_t at = k + piece < p.pitch ? row_at + k : 0x80000000u;       // beyond the row's end: out of range, so zeros
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) load_to_lds_16(W, base + stage * STAGE + i * 8 * TURN, at + static_cast<uint32_t>(8 * i) * p.pitch, 0);
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) load_to_lds_16(X, base + stage * STAGE + (2 * NT + i) * 8 * TURN, at + static_cast<uint32_t>(8 * i) * p.pitch, 0);
    };
    i32x4_t acc[NT][MT] = {};
    int k = wave * TURN, stage = 0;
#pragma unroll
    for (int s = 0; s < STAGES; ++s) fetch(k + s * WAVES * TURN, s);
    for (; k < p.pitch; k += WAVES * TURN) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 1) * 2 * (NT + MT)) : "memory"); // the oldest turn has landed
        i32x4_t w[2][NT], x[2][MT];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const char *from = lds[wave] + stage * STAGE + (frag_at ^ (64 * s));
#pragma unroll
            for (int i = 0; i < NT; ++i) w[s][i] = *reinterpret_cast<const i32x4_t *>(from + i * 16 * TURN);
#pragma unroll
            for (int i = 0; i < MT; ++i) x[s][i] = *reinterpret_cast<const i32x4_t *>(from + (NT + i) * 16 * TURN);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                  // and is in registers before its place is taken
        __builtin_amdgcn_sched_barrier(0);
        fetch(k + STAGES * WAVES * TURN, stage);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int l = 0; l < MT; ++l) acc[i][l] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[s][i], x[s][l], acc[i][l], 0, 0, 0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                                      // nothing is on its way to LDS any more
    i32x4_t *const sums = reinterpret_cast<i32x4_t *>(lds);              // [WAVES][NT][MT][64]
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int l = 0; l < MT; ++l) sums[((wave * NT + i) * MT + l) * 64 + lane] = acc[i][l];
    __syncthreads();
    for (int t = threadIdx.x; t < NT * MT * 64; t += 64 * WAVES) {
        const int at = t & 63, l = t / 64 % MT, i = t / 64 / MT, m = m0 + 16 * l + (at & 15), n = n0 + 16 * i + 4 * (at >> 4);
        if (m >= p.M) continue;
        i32x4_t sum = sums[t];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += sums[v * NT * MT * 64 + t];
        const Scale sx = scale_of(p.x_scale[m]);
        T *y = static_cast<T *>(p.Y) + m * p.ldy + n;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n + j < p.N) y[j] = static_cast<T>(scaled(sum[j], sx, scale_of(p.w_scale[n + j]), p.bias ? p.bias[n + j] : 0.0f));
    }
}

template <class T, int F, int STAGES> int launch_tiles(ScaledGemm p, hipStream_t st)
{
    constexpr int edge = 64 * F, bytes = STAGES * 2 * edge * 128;
    p.across = static_cast<int>(ceil_div(p.N, edge));
    p.tiles = p.across * static_cast<int>(ceil_div(p.M, edge));
    if constexpr (bytes > 64 * 1024) {
        static std::atomic<uint64_t> granted{0};
        if (!all_of_lds(gemm_scaled_tile_kernel<T, F, STAGES>, granted)) return fail(APNN_ERR_DEVICE, "apnn_gemm_scaled: no %d bytes of LDS", bytes);
    }
    gemm_scaled_tile_kernel<T, F, STAGES><<<static_cast<unsigned>(p.tiles), 256, bytes, st>>>(p);
    return check_launch("apnn_gemm_scaled");
}

template <class T, int MT, int NT, int WAVES, int STAGES> int launch_few(ScaledGemm p, hipStream_t st)
{
    p.across = static_cast<int>(ceil_div(p.N, 16 * NT));
    p.tiles = p.across * static_cast<int>(ceil_div(p.M, 16 * MT));
    gemm_scaled_few_kernel<T, MT, NT, WAVES, STAGES><<<static_cast<unsigned>(p.tiles), 64 * WAVES, 0, st>>>(p);
    return check_launch("apnn_gemm_scaled");
}

template <class T> int launch_scaled(const ScaledGemm &p, hipStream_t st)
{
    // Few tokens: the more channels a block has, the less often X is read, as long as most compute units get a block
    // (M = 40, N = 10240, K = 5120: 22.2, 21.2, 17.6, 19.3 us with 1 .. 4 tiles of channels; M = 64, N = K = 4096: 8.7, 9.8, -, 12.7).
    const int64_t units = ceil_div(p.N, 16);
    const auto few = [&](auto tokens, int wide) {
        constexpr int MT = decltype(tokens)::value;
        if (wide >= 4) return launch_few<T, MT, 4, 4, 1>(p, st);
        if (wide == 3) return launch_few<T, MT, 3, 4, 1>(p, st);
        if (wide == 2) return launch_few<T, MT, 2, 4, 1>(p, st);
        return launch_few<T, MT, 1, 4, MT == 4 ? 1 : 2>(p, st);
    };
    const int wide = static_cast<int>(units / 192), forced = scaled_tile_override();
    if (forced == 64) return launch_tiles<T, 1, 4>(p, st);
    if (forced == 128 || forced == 129) return forced == 128 ? launch_tiles<T, 2, 2>(p, st) : launch_tiles<T, 2, 4>(p, st);
    if (forced == 256) return launch_tiles<T, 4, 2>(p, st);
    // (one token, N = 1000: K = 12000 7.4 us with four waves a block, 5.7 with eight; K = 4096 3.9, 3.8; K = 1000 2.8, 3.0)
    if (p.M <= 16) return p.pitch >= 8192 ? launch_few<T, 1, 1, 8, 2>(p, st) : launch_few<T, 1, 1, 4, 2>(p, st);
    if (p.M <= 32) return few(std::integral_constant<int, 2>{}, wide);
    if (p.M <= 48) return few(std::integral_constant<int, 3>{}, wide);
    if (p.M <= 64 || forced == 16) return few(std::integral_constant<int, 4>{}, wide);
    // A few more: 64 tokens a block while that is about one block a compute unit and reads nothing often
    // (M = 256, N = 1000, K = 1999: 7.6 us, 64 x 64 tiles 9.6; M = 128, N = K = 4096: 10.3, 11.6; M = 200: 13.6, 12.1).
    const int64_t down = ceil_div(p.M, 64);
    const int64_t least = ceil_div(units * down, 320);
    if (least <= 4 && (down <= 2 || least == 1)) return few(std::integral_constant<int, 4>{}, static_cast<int>(least));
    // Tiles: rounds of blocks by what a round takes (us at K = 4096: 64-wide tiles 9 and 3 once, 128-wide 22 a block to a compute
    // unit and 38 two, 256-wide 67).
    const auto blocks = [&](int edge) { return ceil_div(p.M, edge) * ceil_div(p.N, edge); };
    const int64_t small = 3 + 9 * ceil_div(blocks(64), 256), middle = blocks(128) <= 256 ? 22 : 38 * ceil_div(blocks(128), 512), large = 67 * ceil_div(blocks(256), 256);
    if (large <= small && large <= middle) return launch_tiles<T, 4, 2>(p, st);
    if (small < middle) return launch_tiles<T, 1, 4>(p, st);
    return blocks(128) <= 256 ? launch_tiles<T, 2, 4>(p, st) : launch_tiles<T, 2, 2>(p, st);
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
    const ScaledGemm p = {X_dev, W_dev, x_scale_dev, w_scale_dev, bias_dev, Y_dev, ldy, static_cast<int>(M), static_cast<int>(N), static_cast<int>(apnn_token_pitch(K)), 0, 0,
                          M * N * size_of(type) >= (16 << 20) && aligned16(Y_dev) && ldy * size_of(type) % 16 == 0};
    return by_type(type, [&](auto t) { return launch_scaled<decltype(t)>(p, as_stream(stream)); });
}
