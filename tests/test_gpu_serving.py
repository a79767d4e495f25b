"""The operators of low-bit language models against their plain 64-bit forms (oracle/serving.py).

Codes are compared for equality: the quotient of the 8-bit codes and the rotation in front of the 4-bit ones are decided in
64 bits.  Rounded results may be off by half a step of their type, eps / 2 of the value, beside what the comment of each
bound derives."""
import numpy as np
import pytest
import torch

from oracle import serving as O
from paper_2106_12169_amd import binding as B

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def f64(t):
    return t.detach().cpu().double().numpy()


def close(got, want, dtype, slack=0.0, tiny=0.0):
    """|got - want| <= eps / 2 |want| + slack (array or number), with NaN where there is NaN."""
    got, want = f64(got), np.asarray(want)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    tol = torch.finfo(dtype).eps / 2 * np.abs(want) + slack + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps + tiny
    off = np.nan_to_num(np.abs(got - want) - tol, nan=0.0)
    assert (off <= 0).all(), f"{(off > 0).sum()} of {off.size} beyond the bound, the worst by {off.max():.3g}"


# ---- 8-bit codes ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows, K", [(1, 1), (3, 7), (2, 16), (5, 17), (16, 4096), (7, 1000), (33, 2051), (2, 8192), (3, 20011)])
def test_quantize_tokens(rows, K, dtype):
    g = rng(rows * 1000 + K)
    x = (normal(g, rows, K) * torch.exp(normal(g, rows, 1) * 3)).to(dtype)
    x[0, :: 3] = (x[0].abs().max() * 0.5).to(dtype)      # 63.5: a tie
    codes, scale = B.apnn_quantize_tokens(x)
    want, want_scale = O.quantize_tokens(f64(x))
    np.testing.assert_array_equal(codes.cpu().numpy(), want)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_scale)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_quantize_tokens_ties_go_to_the_even_code(dtype):
    """Every (n + 1/2) / 127 of a power of two times 127, exact in all three types up to n = 63 (7 bits), and next to them."""
    halves = torch.arange(-63, 64, device="cuda").float() + 0.5
    rows = torch.stack([torch.cat((halves, torch.tensor([127.0], device="cuda"))) * 2.0 ** e for e in (-3, 0, 5)]).to(dtype)
    codes, _ = B.apnn_quantize_tokens(rows)
    want = np.rint(halves.cpu().double().numpy()).astype(np.int8)
    for r in range(3):
        np.testing.assert_array_equal(codes[r, :127].cpu().numpy(), want)
    up = torch.nextafter(rows.float(), torch.full_like(rows.float(), np.inf))
    up[:, 127] = rows[:, 127].float()
    np.testing.assert_array_equal(B.apnn_quantize_tokens(up)[0].cpu().numpy(), O.quantize_tokens(f64(up))[0])


def test_quantize_tokens_extremes():
    x = torch.zeros((8, 40), device="cuda")
    x[1, 3], x[2, 4], x[3, 39] = float("nan"), float("inf"), float("-inf")
    x[4] = torch.finfo(F32).smallest_normal * torch.finfo(F32).eps * torch.arange(40, device="cuda")     # subnormal
    x[5], x[6, 0] = torch.finfo(F32).max, -1e-38
    x[7] = torch.linspace(-3e38, 3e38, 40)
    codes, scale = B.apnn_quantize_tokens(x)
    want, want_scale = O.quantize_tokens(f64(x))
    np.testing.assert_array_equal(codes.cpu().numpy(), want)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_scale)
    assert np.isnan(want_scale[1:4]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset, K, ld", [(0, 64, 96), (1, 64, 96), (3, 61, 67), (8, 4096, 4104), (5, 1, 9)])
def test_quantize_tokens_strides_and_alignment(offset, K, ld, dtype):
    base = normal(rng(K), 6, ld + 8, dtype=dtype)[:, offset:]
    x = base[:, :K]
    codes, scale = B.apnn_quantize_tokens(x)
    want, want_scale = O.quantize_tokens(f64(x))
    np.testing.assert_array_equal(codes.cpu().numpy(), want)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_scale)


def test_quantize_tokens_of_nothing():
    codes, scale = B.apnn_quantize_tokens(torch.empty((0, 5), device="cuda"))
    assert codes.shape == (0, 16) and scale.shape == (0,)
    codes, scale = B.apnn_quantize_tokens(torch.empty((3, 0), device="cuda"))
    assert codes.shape == (3, 0) and (scale == 0).all()


# ---- scaled products ------------------------------------------------------------------------------------------------------


def operands(M, N, K, seed=0, low=-127):
    g = rng(seed + M + 3 * N + 7 * K)
    pitch = B.apnn_token_pitch(K)
    X = torch.zeros((M, pitch), dtype=torch.int8, device="cuda")
    W = torch.zeros((N, pitch), dtype=torch.int8, device="cuda")
    X[:, :K] = torch.randint(low, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    W[:, :K] = torch.randint(low, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    return X, torch.rand(M, generator=g, device="cuda") * 0.1, W, torch.rand(N, generator=g, device="cuda") * 0.01, normal(g, N)


def check_product(got, X, xs, W, ws, bias, dtype):
    total = X.double() @ W.double().T                     # integers below 2^53: exact in any order
    want = total * xs.double()[:, None] * ws.double()
    slack = 3.01 * 2.0 ** -24 * want.abs()                # in fp32: the sum, and two products with the scales' mantissas
    if bias is not None:
        want = want + bias.double()
    slack = slack + 2.0 ** -24 * want.abs()               # the sum with the bias, in 32 bits on the way to 16
    close(got, want.cpu().numpy(), dtype, slack.cpu().numpy())


SIZES = [(1, 1, 1), (1, 64, 64), (1, 4096, 1024), (2, 100, 31), (5, 33, 4096), (16, 64, 16), (17, 48, 48), (31, 257, 640), (33, 1000, 500),
         (48, 512, 2048), (64, 128, 1000), (65, 129, 257), (100, 77, 20000), (128, 128, 128), (200, 333, 111), (257, 255, 4096),
         (512, 512, 64), (777, 1000, 1999), (1024, 1024, 1024), (300, 2048, 4112), (2049, 2047, 33), (4096, 24, 512), (3, 9000, 7000), (1, 40, 9000), (16, 100, 12001)]


@pytest.mark.parametrize("M, N, K", SIZES)
def test_gemm_scaled(M, N, K):
    X, xs, W, ws, bias = operands(M, N, K, low=-128)
    for dtype, b in ((F32, bias), (F16, None), (BF16, bias)):
        check_product(B.apnn_gemm_scaled(X, xs, W, ws, K, bias=b, dtype=dtype), X, xs, W, ws, b, dtype)


@pytest.mark.parametrize("form", [16, 64, 128, 129, 256])
@pytest.mark.parametrize("M, N, K", [(1, 1, 1), (5, 33, 300), (65, 70, 16), (130, 513, 129), (257, 255, 640), (300, 1000, 1999), (513, 256, 4096)])
def test_gemm_scaled_in_every_form(M, N, K, form):
    X, xs, W, ws, bias = operands(M, N, K, low=-128)
    B.apnn_debug_force("SCALED_TILE", form)
    for dtype, b in ((F32, bias), (F16, None), (BF16, bias)):
        check_product(B.apnn_gemm_scaled(X, xs, W, ws, K, bias=b, dtype=dtype), X, xs, W, ws, b, dtype)
    ws[N // 2], xs[M // 2] = 1e-30, 1e25                  # scales that cannot be multiplied as they are
    check_product(B.apnn_gemm_scaled(X, xs, W, ws, K, dtype=F32), X, xs, W, ws, None, F32)


def test_gemm_scaled_large():
    """Sizes that choose the widest tiles by themselves, whole rounds of them and a part of one; results of 16 MiB and more."""
    for M, N, K, dtype in ((4096, 4096, 320, BF16), (4000, 4100, 144, BF16), (2100, 2104, 64, F32), (8200, 1032, 48, F16)):
        X, xs, W, ws, bias = operands(M, N, K)
        check_product(B.apnn_gemm_scaled(X, xs, W, ws, K, bias=bias, dtype=dtype), X, xs, W, ws, bias, dtype)


def test_gemm_scaled_at_the_edge_of_int32():
    K = (1 << 17) - 1
    X = torch.full((3, B.apnn_token_pitch(K)), -128, dtype=torch.int8, device="cuda")
    X[:, K:] = 0
    W = X[:2].clone()
    W[1] = 127 * (X[1] != 0)
    one = torch.ones(3, device="cuda")
    got = B.apnn_gemm_scaled(X, one, W, one[:2], K, dtype=F32)
    assert (got[:, 0] == float(np.float32(K * 16384))).all() and (got[:, 1] == float(np.float32(-128 * 127 * K))).all()


@pytest.mark.parametrize("M, N, K", [(1, 300, 256), (40, 300, 256), (300, 260, 256)])
def test_gemm_scaled_into_a_strided_result(M, N, K):
    X, xs, W, ws, bias = operands(M, N, K)
    for dtype, pad, offset in ((F32, 4, 0), (BF16, 3, 1), (F16, 8, 8)):
        whole = torch.full((M + 2, N + pad + offset), 7.0, dtype=dtype, device="cuda")
        out = whole[1:M + 1, offset:offset + N]
        assert B.apnn_gemm_scaled(X, xs, W, ws, K, bias=bias, out=out) is out
        check_product(out, X, xs, W, ws, bias, dtype)
        out.fill_(7.0)
        assert (whole == 7.0).all()                       # nothing beside the result


def test_gemm_scaled_extremes():
    X, xs, W, ws, bias = operands(4, 40, 64)
    xs[0], xs[1], xs[2] = float("nan"), 1e38, 1e-38
    ws[:] = 1e-3
    ws[3], ws[4] = 1e-38, 1e30
    X[3] = 0
    got = B.apnn_gemm_scaled(X, xs, W, ws, 64, dtype=F32)
    want = (X.double() @ W.double().T * xs.double()[:, None] * ws.double()).float()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.isnan(got[0]).all()
    np.testing.assert_allclose(f64(got[1:]), f64(want[1:]), rtol=4.01 * 2.0 ** -24, atol=2.0 ** -149)
    empty = torch.zeros((4, 0), dtype=torch.int8, device="cuda")
    assert torch.equal(B.apnn_gemm_scaled(empty, xs[1:2].expand(4).contiguous(), empty, ws[:4], 0, bias=bias[:4], dtype=F32), bias[:4].expand(4, 4))
    assert B.apnn_gemm_scaled(X[:0], xs[:0], W, ws, 64).shape == (0, 40)


# ---- the 4-bit cache -------------------------------------------------------------------------------------------------------


def rotation(rot, rows=5000):
    inv = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    angle = np.arange(rows)[:, None] * inv
    return np.concatenate((np.cos(angle), np.sin(angle)), 1).astype(np.float32)


def held(cache):
    """The oracle's view of a cache's bytes: values [slots, heads, D]."""
    def values(codes, scale):
        codes, scale = (t.cpu().numpy().transpose(0, 2, 1, 3) for t in (codes, scale))
        nibbles = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
        x = O.decode4(nibbles, np.where(scale == 255, 0, scale.astype(np.int64) - 127))
        return x.reshape(-1, *x.shape[2:]), (scale == 255).any(-1).reshape(-1, scale.shape[2])
    k, nan = values(cache.k_codes, cache.k_scale)
    v, _ = values(cache.v_codes, cache.v_scale)
    k[nan] = v[nan] = np.nan
    return k, v


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D, heads, page, T", [(64, 1, 16, 1), (64, 3, 32, 50), (96, 2, 16, 33), (128, 8, 64, 100), (128, 1, 128, 3), (256, 2, 256, 40)])
def test_append_and_read(D, heads, page, T, dtype):
    g = rng(D + heads + T)
    pages = -(-T // page) + 2
    cache, want = B.KVCache.empty(pages, heads, page, D), O.Cache(pages, heads, page, D)
    for turn, (rot, interleaved) in enumerate(((0, False), (D, False), (D // 2, True), (20, False), (D - 2, True))):
        k, v = ((normal(g, T, heads, D) * torch.exp(normal(g, T, heads, D // 32).repeat_interleave(32, -1) * 3)).to(dtype) for _ in range(2))
        k[0, 0, :32], v[0, 0, 32:] = 0.0, 0.0
        q = normal(g, T, 2 * heads, D, dtype=dtype)
        slots = torch.randperm(pages * page, generator=g, device="cuda")[:T]
        if T > 2:
            slots[1] = -1                                 # padding
        table = rotation(rot)
        positions = torch.randint(0, 5000, (T,), generator=g, device="cuda", dtype=torch.int32)
        args = dict(positions=positions, table=torch.from_numpy(table).cuda(), interleaved=interleaved) if rot else {}
        q_out = torch.full_like(q, 9.0)
        B.apnn_kv_append(cache, k, v, slots, q=q, q_out=q_out, **args)
        at = positions.cpu().numpy()
        rk, rq = (O.rotate(f64(x), table, at, interleaved) if rot else f64(x) for x in (k, q))
        want.append(rk, f64(v), slots.cpu().numpy())
        got_k, got_v = held(cache)
        np.testing.assert_array_equal(got_k, want.k)
        np.testing.assert_array_equal(got_v, want.v)
        written = slots.cpu().numpy() >= 0
        close(q_out[torch.from_numpy(written).cuda()], rq[written], dtype)
        assert (q_out[~torch.from_numpy(written).cuda()] == 9.0).all()
        everything = torch.arange(-1, pages * page + 1, device="cuda")
        for out in (F32, F16, BF16):
            rk_, rv_ = B.apnn_kv_read(cache, everything, out)
            np.testing.assert_array_equal(f64(rk_)[1:-1], want.k)
            np.testing.assert_array_equal(f64(rv_)[1:-1], want.v)
            assert (rk_[[0, -1]] == 0).all() and (rv_[[0, -1]] == 0).all()


def test_append_borders_between_codes():
    """Every border and its neighbours, with the group's largest magnitude next to 7 * 2^e, over the whole range of e and beyond."""
    edges = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 6.5], np.float32)
    near = np.concatenate((edges, np.nextafter(edges, np.float32(9)), np.nextafter(edges, np.float32(-9))))
    rows = []
    for top in (3.5, np.nextafter(np.float32(3.5), np.float32(0)), np.nextafter(np.float32(7), np.float32(0)), 7.0, 6.0, 5.0):
        for e in (-140, -26, -24, -23, -22, -1, 0, 1, 12, 13, 14, 15, 100):
            for i in range(0, len(near), 31):
                g = np.zeros(32, np.float32)
                piece = near[i:i + 31]
                g[:len(piece)] = np.minimum(piece, np.float32(top)) * np.where(np.arange(len(piece)) % 2, -1, 1)
                g[31] = top
                rows.append(np.ldexp(g, e))
    x = np.stack(rows)
    x = np.concatenate((x, np.zeros((-len(x) % 2, 32), np.float32))).reshape(-1, 1, 64)
    T = len(x)
    cache, want = B.KVCache.empty(-(-T // 16), 1, 16, 64), O.Cache(-(-T // 16), 1, 16, 64)
    k = torch.from_numpy(x).cuda()
    B.apnn_kv_append(cache, k, k.flip(0).contiguous(), torch.arange(T, device="cuda"))
    want.append(x.astype(np.float64), x[::-1].astype(np.float64), np.arange(T))
    got_k, got_v = held(cache)
    np.testing.assert_array_equal(got_k, want.k)
    np.testing.assert_array_equal(got_v, want.v)
    assert np.abs(want.k).max() == 6 * 2.0 ** 13
    scales = cache.k_scale.cpu().numpy().reshape(-1)[:2 * T]
    assert scales.min() >= 104 and scales.max() == 140
    for out in (F16, BF16):
        np.testing.assert_array_equal(f64(B.apnn_kv_read(cache, torch.arange(T, device="cuda"), out)[0]), want.k[:T])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [2, 6, 12, 20, 30, 48])
def test_append_rotates_nothing_beyond_the_rotation(rot, interleaved):
    """Channels from rot on keep their values, next to infinities too."""
    D, T = 64, 5
    cache, g = B.KVCache.empty(1, 1, 16, D), rng(rot)
    q = normal(g, T, 3, D, dtype=BF16)
    q[:, :, rot + 1::4] = float("inf")
    k = normal(g, T, 1, D, dtype=BF16)
    table = rotation(rot, 50)
    positions = torch.arange(T, dtype=torch.int32, device="cuda") * 9
    out = B.apnn_kv_append(cache, k, k, torch.arange(T, device="cuda"), positions=positions, table=torch.from_numpy(table).cuda(), interleaved=interleaved, q=q)
    want = O.rotate(f64(q), table, positions.cpu().numpy(), interleaved)
    assert torch.equal(out[:, :, rot:], q[:, :, rot:])
    close(out[:, :, :rot], want[:, :, :rot], BF16)


def test_append_holds_what_is_not_finite_as_nan():
    g, D = rng(5), 128
    k, v = normal(g, 6, 2, D), normal(g, 6, 2, D)
    k[1, 0, 5], k[2, 1, 127], v[3, 0, 64], v[4, 1, 0] = float("nan"), float("inf"), float("-inf"), float("nan")
    cache, want = B.KVCache.empty(1, 2, 16, D), O.Cache(1, 2, 16, D)
    B.apnn_kv_append(cache, k, v, torch.arange(6, device="cuda"))
    want.append(f64(k), f64(v), np.arange(6))
    got_k, got_v = held(cache)
    np.testing.assert_array_equal(got_k, want.k)
    np.testing.assert_array_equal(got_v, want.v)
    rk, rv = B.apnn_kv_read(cache, torch.arange(6, device="cuda"))
    np.testing.assert_array_equal(f64(rk), want.k[:6])
    np.testing.assert_array_equal(f64(rv), want.v[:6])
    assert np.isnan(want.k).any() and (cache.v_scale.cpu() != 255).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rot", [0, 64, 40])
def test_append_strides_places_and_in_place_queries(rot, dtype):
    """q, k, v as views of one projection; slots and positions outside of cache and table are left out."""
    g, T, Hq, H, D = rng(7), 9, 4, 2, 64
    table = torch.from_numpy(rotation(64, 100)[:, list(range(rot // 2)) + list(range(32, 32 + rot // 2))].copy()).cuda()
    for odd in (0, 1):
        wide = normal(g, T, (Hq + 2 * H) * D + odd, dtype=dtype)[:, odd:].unflatten(1, (-1, D))
        q, k, v = wide[:, :Hq], wide[:, Hq:Hq + H], wide[:, Hq + H:]
        positions = torch.tensor([0, 99, 100, -1, 50, 3, 7, 8, 9], dtype=torch.int32, device="cuda")
        slots = torch.tensor([5, 32, 6, 7, 48, -1, 31, 0, 1 << 40], device="cuda")
        cache, want = B.KVCache.empty(3, H, 16, D), O.Cache(3, H, 16, D)
        left_out = (slots < 0) | (slots >= 48) | (((positions < 0) | (positions >= 100)) if rot else False)
        before_k, before_v, before_q = f64(k), f64(v), f64(q)
        args = dict(positions=positions, table=table) if rot else {}
        assert B.apnn_kv_append(cache, k, v, slots, q=q, q_out=q, **args) is q
        at = positions.clamp(0, 99).cpu().numpy()
        turn = (lambda x: O.rotate(x, table.cpu().numpy(), at, False)) if rot else (lambda x: x)
        want.append(turn(before_k), before_v, torch.where(left_out, -1, slots).cpu().numpy())
        got_k, got_v = held(cache)
        np.testing.assert_array_equal(got_k, want.k)
        np.testing.assert_array_equal(got_v, want.v)
        out = left_out.cpu().numpy()
        close(q[~left_out], turn(before_q)[~out], dtype)
        np.testing.assert_array_equal(f64(q)[out], before_q[out])
        np.testing.assert_array_equal(f64(k), before_k)   # beside the queries nothing of the projection changes


# ---- attention over the 4-bit cache ----------------------------------------------------------------------------------------


def filled(g, lens, heads, page, D, spare=3, offset=0.5):
    """A cache whose pages lie in any order, every byte of it set; the page table (its unused places outside the cache) and the values."""
    count = [-(-l // page) for l in lens]
    total = sum(count) + spare
    shape = (total, heads, page)
    random_bytes = lambda n: torch.randint(0, 256, shape + (n,), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    cache = B.KVCache(random_bytes(D // 2), random_bytes(D // 32), random_bytes(D // 2), random_bytes(D // 32))
    order = torch.randperm(total, generator=g, device="cuda").int()
    table = torch.full((len(lens), max(count + [1]) + 1), 1 << 30, dtype=torch.int32, device="cuda")
    at = 0
    for b, (l, c) in enumerate(zip(lens, count)):
        table[b, :c] = order[at:at + c]
        at += c
        if l:
            t = torch.arange(l, device="cuda")
            slots = table[b].long()[t // page] * page + t % page
            k, v = normal(g, l, heads, D, dtype=BF16) + offset, normal(g, l, heads, D, dtype=BF16)
            B.apnn_kv_append(cache, k, v, slots)
    return cache, table


def dense(cache, table, b, l):
    t = torch.arange(l, device="cuda")
    slots = table[b].long()[(t // cache.page_size).clamp(max=table.shape[1] - 1)] * cache.page_size + t % cache.page_size
    k, v = B.apnn_kv_read(cache, slots, F32)
    return f64(k), f64(v)


def check_attention(out, q, cache, table, lens, news, starts, scale, dtype):
    """Row by row against 64 bits.

    The bound: products of 16-bit numbers are exact in fp32, so a score of D terms is off by at most (D + 4) 2^-24 of the sum
    of its terms' magnitudes (accumulation in any order, the scale, the power-of-two base), which the exponential turns into the
    same error relative to the weight; v_exp_f32 adds at most 2^-22.  A weight is rounded to fp16, 2^-11 of it, or 2^-25 of the
    largest one where it is subnormal; the sum and the product accumulate at most the tokens' 2^-24 each.  The weights' errors
    count twice: in the sum and in what is divided by it."""
    G = q.shape[1] // cache.heads
    for b, (l, n) in enumerate(zip(lens, news)):
        k, v = dense(cache, table, b, l) if l else (np.zeros((0, cache.heads, cache.D)),) * 2
        rows = slice(starts[b], starts[b] + n)
        for h in range(q.shape[1]):
            want, spread, reach = O.attention(f64(q[rows, h]), k[:, h // G], v[:, h // G], l - n, scale)
            error = 2.0 ** -11 + 2 * ((cache.D + 4) * 2.0 ** -24 * reach + 2.0 ** -22 + 2 * l * 2.0 ** -24)
            big = np.abs(v[:, h // G]).max(initial=0.0)
            close(out[rows, h], want, dtype, error[:, None] * spread + l * 2.0 ** -25 * big)


@pytest.fixture(params=[16, 128], ids=["rows16", "rows128"])
def rows(request):
    """Both kernels, whatever the sizes would choose."""
    B.apnn_debug_force("KV_ROWS", request.param)


def attend(seed, lens, news, Hq, heads, D, page, dtype, ragged=None, scale=None, max_q=None):
    g = rng(seed)
    cache, table = filled(g, lens, heads, page, D)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    q = normal(g, starts[-1] + 2, Hq, D, dtype=dtype)     # two rows of padding
    scale = D ** -0.5 if scale is None else scale
    out = torch.full_like(q, 9.0)
    tensor = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    ragged = any(n != 1 for n in news) if ragged is None else ragged
    B.apnn_kv_attention(cache, q, tensor(lens), table, scale, q_start=tensor(starts) if ragged else None,
                        max_q=(max(news) if max_q is None else max_q) if ragged else None, out=out)
    check_attention(out, q, cache, table, lens, news, starts, scale, dtype)
    assert (out[starts[-1]:] == 9.0).all()
    return cache, table, q, out


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("Hq, heads", [(1, 1), (3, 3), (4, 1), (14, 2), (16, 1), (40, 2)])
def test_attention_of_single_tokens(D, Hq, heads, dtype, rows):
    attend(D + Hq, [1, 16, 17, 100, 333, 0, 31, 32, 33, 64], [1] * 10, Hq, heads, D, 16, dtype)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_attention_of_every_page_size(page, rows):
    attend(page, [page - 1, page, page + 1, 3 * page + 5], [1] * 4, 8, 2, 64, page, F16)
    attend(page + 1, [page - 1, page, page + 1, 3 * page + 5], [5, page, 40, 2 * page], 4, 2, 128, page, BF16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D, Hq, heads", [(64, 4, 4), (96, 6, 2), (128, 8, 2), (128, 7, 1), (256, 4, 1)])
def test_attention_of_prompts(D, Hq, heads, dtype, rows):
    attend(D * 3 + Hq, [70, 257, 1, 130, 40, 0, 200], [70, 100, 1, 129, 3, 0, 200], Hq, heads, D, 32, dtype)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_rows_that_see_nothing(dtype, rows):
    """More queries than tokens: the first ones stand before the cache begins and get zeros."""
    _, _, _, out = attend(3, [3, 0, 40, 1], [10, 5, 45, 200], 4, 2, 64, 16, dtype)
    assert (out[:7] == 0).all() and (out[7:10] != 0).any()
    assert (out[10:15] == 0).all() and (out[15:20] == 0).all() and (out[60:259] == 0).all()


@pytest.mark.parametrize("news", [1, 2, 3, 4, 8, 16])
def test_attention_of_a_few_tokens_on_long_contexts(news, rows):
    attend(news, [5000, 1200, 4096, 2047], [news, 1, news, news], 16, 2, 128, 64, BF16)
    attend(news + 50, [3000], [news], 8, 8, 64, 16, F16)


def test_attention_scales_and_far_scores(rows):
    """Scores far apart, negative scale, scale 0 (plain averages); one token with all of the weight."""
    for scale in (-0.3, 0.0, 3.0, 1e-30):
        attend(11, [300, 20], [1, 1], 4, 2, 64, 16, F16, scale=scale)
        attend(12, [300, 150], [100, 150], 4, 2, 64, 16, BF16, scale=scale)


def test_attention_max_q_and_one_query_each(rows):
    cache, table, q, out = attend(21, [50, 60, 70], [1, 1, 1], 4, 2, 64, 16, F16, ragged=False)
    lens = torch.tensor([50, 60, 70], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    for max_q in (1, 3, 5, None):
        again = B.apnn_kv_attention(cache, q, lens, table, 0.125, q_start=start, max_q=max_q)
        close(again[:3], f64(out[:3]), F16, 2.0 ** -10 * np.abs(f64(out[:3])))      # half a step of each and the weights' rounding
    cache, table, q, out = attend(22, [200, 90], [150, 20], 4, 2, 64, 16, BF16)
    start = torch.tensor([0, 150, 170], dtype=torch.int32, device="cuda")
    some = torch.full_like(q, 9.0)
    B.apnn_kv_attention(cache, q, torch.tensor([200, 90], dtype=torch.int32, device="cuda"), table, 0.125, q_start=start, max_q=33, out=some)
    close(some[:33], f64(out[:33]), BF16, 2.0 ** -7 * np.abs(f64(out[:33])) + 2.0 ** -10)
    assert (some[33:150] == 9.0).all() and (some[170:] == 9.0).all()    # queries beyond max_q are left as they were
    close(some[150:170], f64(out[150:170]), BF16, 2.0 ** -7 * np.abs(f64(out[150:170])) + 2.0 ** -10)


@pytest.mark.parametrize("news", [1, 40])
def test_attention_nan_reaches_only_queries_that_see_it(news, rows):
    g, D, page, l = rng(news), 64, 16, 200
    cache, table = filled(g, [l], 2, page, D)
    bad = l - max(1, news // 2)                           # seen by the later half of the queries
    k, v = normal(g, 1, 2, D), normal(g, 1, 2, D)
    v[0, 1, 7] = float("inf")                             # head 1's value only
    slot = table[0, bad // page].long() * page + bad % page
    B.apnn_kv_append(cache, k, v, slot.reshape(1))
    q = normal(g, news, 4, D, dtype=F16)
    q[0, 0, 3] = float("nan")
    start = torch.tensor([0, news], dtype=torch.int32, device="cuda")
    out = B.apnn_kv_attention(cache, q, torch.tensor([l], dtype=torch.int32, device="cuda"), table, 0.125, q_start=start, max_q=news)
    nan = torch.isnan(out).all(-1).cpu().numpy()
    assert (torch.isnan(out).any(-1).cpu().numpy() == nan).all()
    want = np.zeros((news, 4), bool)
    want[[l - news + i >= bad for i in range(news)], 2:] = True          # query heads 2, 3 read cache head 1
    want[0, 0] = True
    np.testing.assert_array_equal(nan, want)


@pytest.mark.parametrize("news", [1, 30])
def test_attention_skips_pages_outside_the_cache(news, rows):
    """A page index out of range counts as unseen, wherever it stands; so do tokens beyond the table."""
    g, D, page, l = rng(4), 128, 32, 300
    cache, table = filled(g, [l, l], 2, page, D)
    k, v = dense(cache, table, 0, l)
    q = normal(g, 2 * news, 4, D, dtype=BF16)
    for bad in (-1, cache.k_codes.shape[0], -(1 << 31), (1 << 31) - 1):
        damaged = table.clone()
        damaged[0, 2] = bad
        start = torch.tensor([0, news, 2 * news], dtype=torch.int32, device="cuda")
        lens = torch.tensor([l, l + 500], dtype=torch.int32, device="cuda")
        out = B.apnn_kv_attention(cache, q, lens, damaged[:, :10].contiguous(), 0.1, q_start=start, max_q=news)
        keep = np.r_[0:64, 96:l]
        for i in range(news):
            seen = keep[keep <= l - news + i]
            for h in range(4):
                want, spread, _ = O.attention(f64(q[i:i + 1, h]), k[seen, h // 2], v[seen, h // 2], len(seen) - 1, 0.1)
                close(out[i, h], want[0], BF16, 2.0 ** -10 * spread[0] + 1e-6)
        assert torch.isfinite(out[:news]).all()           # (the other sequence's table ends in tokens that nobody wrote)
    nothing = torch.full_like(table, -5)
    assert (B.apnn_kv_attention(cache, q, lens, nothing, 0.1, q_start=start, max_q=news) == 0).all()


@pytest.mark.parametrize("news", [1, 70])
def test_attention_strides(news, rows):
    g, D, Hq, H = rng(9), 64, 4, 2
    cache, table = filled(g, [200], H, 16, D)
    for odd in (0, 1):
        wide = normal(g, news, (Hq + 2 * H) * D + odd, dtype=F16)[:, odd:].unflatten(1, (-1, D))
        q = wide[:, :Hq]
        whole = torch.full((Hq, news, D + 8 + odd), 9.0, dtype=F16, device="cuda")
        out = whole[:, :, odd:odd + D].transpose(0, 1)
        start = torch.tensor([0, news], dtype=torch.int32, device="cuda")
        B.apnn_kv_attention(cache, q, torch.tensor([200], dtype=torch.int32, device="cuda"), table, 0.125, q_start=start, max_q=news, out=out)
        check_attention(out, q, cache, table, [200], [news], [0], 0.125, F16)
        out.fill_(9.0)
        assert (whole == 9.0).all()


def test_attention_with_a_workspace_that_is_kept():
    """One workspace for call after call, of the size asked for; and one that is too small is refused."""
    g, D = rng(79), 64
    cache, table = filled(g, [5000, 4000], 2, 64, D)
    need = B.apnn_kv_attention_workspace_bytes(cache, 2, 8, 2, table.shape[1])
    space = torch.full((need + 32,), 255, dtype=torch.uint8, device="cuda")
    for l in ([5000, 4000], [1, 3000], [0, 5]):
        q, lens = normal(g, 2, 8, D, dtype=F16), torch.tensor(l, dtype=torch.int32, device="cuda")
        out = B.apnn_kv_attention(cache, q, lens, table, 0.125, workspace=space[:need])
        assert torch.equal(out, B.apnn_kv_attention(cache, q, lens, table, 0.125))
        check_attention(out, q, cache, table, l, [1, 1], [0, 1], 0.125, F16)
    assert (space[need:] == 255).all()
    with pytest.raises(B.ApnnError, match="workspace"):
        B.apnn_kv_attention(cache, q, lens, table, 0.125, workspace=space[:need - 1])


@pytest.mark.parametrize("news", [1, 33])
def test_attention_of_queries_that_share_memory(news, rows):
    """One query row for all heads and tokens (strides 0) is only read; the result has memory of its own."""
    g, D = rng(80), 96
    cache, table = filled(g, [150], 2, 16, D)
    q = normal(g, 1, 1, D, dtype=BF16).expand(news, 6, D)
    start = torch.tensor([0, news], dtype=torch.int32, device="cuda")
    out = B.apnn_kv_attention(cache, q, torch.tensor([150], dtype=torch.int32, device="cuda"), table, 0.1, q_start=start, max_q=news)
    check_attention(out, q, cache, table, [150], [news], [0], 0.1, BF16)
    own = normal(g, news, 6, D, dtype=BF16)
    with pytest.raises(B.ApnnError, match="out must not be q"):
        B.apnn_kv_attention(cache, own, torch.tensor([150], dtype=torch.int32, device="cuda"), table, 0.1, q_start=start, max_q=news, out=own)


def test_attention_that_chooses_many_rows_itself():
    """Enough blocks of 128 rows, and enough scores, for that kernel to be taken (and joined from splits)."""
    attend(61, [150] * 64, [100] * 64, 8, 8, 64, 16, BF16)
    attend(62, [9000, 40], [260, 40], 32, 2, 64, 64, F16)


def test_attention_of_many_sequences(rows):
    lens = [(37 * b) % 90 for b in range(300)]
    attend(31, lens, [1] * 300, 2, 1, 64, 16, BF16)
    attend(32, lens[:60], [min(l, b % 5) for b, l in enumerate(lens[:60])], 2, 1, 64, 16, F16)


def test_attention_beyond_32_bits_of_offset(rows):
    """Pages whose bytes start past 2^32: a cache of 5 GB a side, most of it unused."""
    D, page, heads = 256, 256, 8
    pages = (5 << 30) // (heads * page * D // 2)
    cache = B.KVCache.empty(pages, heads, page, D)
    g = rng(41)
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    l = 3 * page - 7
    t = torch.arange(l, device="cuda")
    slots = table[0].long()[t // page] * page + t % page
    B.apnn_kv_append(cache, normal(g, l, heads, D, dtype=BF16), normal(g, l, heads, D, dtype=BF16), slots)
    for n in (1, 200):
        q = normal(g, n, heads, D, dtype=BF16)
        start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        out = B.apnn_kv_attention(cache, q, torch.tensor([l], dtype=torch.int32, device="cuda"), table, 0.0625, q_start=start, max_q=n)
        check_attention(out, q, cache, table, [l], [n], [0], 0.0625, BF16)


# ---- together --------------------------------------------------------------------------------------------------------------


def layer(x, weights, cache, slots, positions, table, lens, pages, start, max_q, Hq, H, D):
    """A quantised attention layer: project, append, attend, project."""
    (wqkv, sqkv, K), (wo, so, Ko) = weights
    codes, scale = B.apnn_quantize_tokens(x)
    y = B.apnn_gemm_scaled(codes, scale, wqkv, sqkv, K, dtype=x.dtype).unflatten(1, (Hq + 2 * H, D))
    q = B.apnn_kv_append(cache, y[:, Hq:Hq + H], y[:, Hq + H:], slots, positions=positions, table=table, q=y[:, :Hq])
    o = B.apnn_kv_attention(cache, q, lens, pages, D ** -0.5, q_start=start, max_q=max_q)
    codes, scale = B.apnn_quantize_tokens(o.flatten(1))
    return B.apnn_gemm_scaled(codes, scale, wo, so, Ko, dtype=x.dtype), q, o


def test_a_layer_of_a_prompt_and_then_token_by_token():
    """The operators as they are used: a prompt, then tokens one by one from a captured graph that is replayed with new
    inputs in place, every step checked against the 64-bit forms of what went into each operator, and against eager calls."""
    g, H, Hq, D, page, hidden, dtype = rng(77), 2, 8, 64, 16, 384, BF16
    weights = []
    for N, K in (((Hq + 2 * H) * D, hidden), (hidden, Hq * D)):
        weights.append((*B.apnn_quantize_tokens(normal(g, N, K) * 0.05), K))
    lens, slack = [37, 20, 5], 8
    pages = torch.arange(3 * 4, dtype=torch.int32, device="cuda").flip(0).reshape(3, 4).contiguous()
    caches = [B.KVCache.empty(12, H, page, D) for _ in range(2)]
    table = torch.from_numpy(rotation(D, 200)).cuda()
    place = lambda b, t: int(pages[b, t // page]) * page + t % page  # noqa: E731
    tensor = lambda v, t=torch.int32: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    x = normal(g, sum(lens), hidden, dtype=dtype)
    start = [0, 37, 57, 62]
    common = dict(Hq=Hq, H=H, D=D)
    for cache in caches:
        y, q, o = layer(x, weights, cache, tensor([place(b, t) for b in range(3) for t in range(lens[b])], torch.int64),
                        tensor([t for b in range(3) for t in range(lens[b])]), table, tensor(lens), pages, tensor(start), max(lens), **common)
        check_attention(o, q, cache, pages, lens, lens, start, D ** -0.5, dtype)
    # token by token: static buffers, one graph
    xs, slots, positions, now = normal(g, 3, hidden, dtype=dtype), tensor([0] * 3, torch.int64), tensor([0] * 3), tensor(lens)
    step = lambda cache: layer(xs, weights, cache, slots, positions, table, now, pages, None, None, **common)  # noqa: E731

    def advance(i):
        xs.copy_(normal(g, 3, hidden, dtype=dtype))
        slots.copy_(tensor([place(b, lens[b] + i) for b in range(3)], torch.int64))
        positions.copy_(tensor([lens[b] + i for b in range(3)]))
        now.copy_(tensor([lens[b] + i + 1 for b in range(3)]))

    advance(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[1])                                   # on another stream than the tensors' own
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(caches[1])
    for i in range(slack):
        advance(i)
        graph.replay()
        y, q, o = step(caches[0])
        torch.cuda.synchronize()
        for got, want in zip(captured, (y, q, o)):
            assert torch.equal(got, want)
        check_attention(o, q, caches[0], pages, [l + i + 1 for l in lens], [1] * 3, [0, 1, 2], D ** -0.5, dtype)
    for a, b in zip(vars(caches[0]).values(), vars(caches[1]).values()):
        assert torch.equal(a, b)


def test_two_graphs_on_two_streams_do_not_share_a_workspace():
    """Two captured attention calls that run at once, each against what it gives alone."""
    g, D = rng(78), 128
    cache, table = filled(g, [3000, 2500], 2, 64, D)
    lens = torch.tensor([3000, 2500], dtype=torch.int32, device="cuda")
    qs = [normal(g, 2, 8, D, dtype=F16) for _ in range(2)]
    alone = [B.apnn_kv_attention(cache, q, lens, table, 0.1) for q in qs]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for q in qs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(B.apnn_kv_attention(cache, q, lens, table, 0.1))
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for o, want in zip(outs, alone):
            assert torch.equal(o, want)


def test_the_binding_refuses_wrong_tensors():
    x = torch.zeros((4, 32), device="cuda")
    codes, scale = B.apnn_quantize_tokens(x)
    with pytest.raises(TypeError, match="float32, float16 or bfloat16"):
        B.apnn_quantize_tokens(x.int())
    with pytest.raises(ValueError, match="2 dimensions"):
        B.apnn_quantize_tokens(x, codes[0], scale)
    with pytest.raises(AssertionError, match="last dimension"):
        B.apnn_quantize_tokens(x.T)
    with pytest.raises(ValueError, match=r"codes: size \(4, 32\)"):
        B.apnn_quantize_tokens(x, codes[:3], scale)
    with pytest.raises(TypeError, match="x_scale"):
        B.apnn_gemm_scaled(codes, scale.double(), codes, scale, 32)
    with pytest.raises(ValueError, match="X: size"):
        B.apnn_gemm_scaled(codes, scale, codes, scale, 33)
    with pytest.raises(AssertionError, match="bias: a device tensor"):
        B.apnn_gemm_scaled(codes, scale, codes, scale, 32, bias=torch.zeros(4))
    with pytest.raises(B.ApnnError, match="ldy"):
        B.apnn_gemm_scaled(codes, scale, codes, scale, 32, out=torch.zeros(1, 4, device="cuda").expand(4, 4))
    cache = B.KVCache.empty(2, 2, 16, 64)
    k, slots, at = torch.zeros((3, 2, 64), device="cuda"), torch.arange(3, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="k: size"):
        B.apnn_kv_append(cache, k[:, :1], k, slots)
    with pytest.raises(TypeError, match="v: type"):
        B.apnn_kv_append(cache, k, k.half(), slots)
    with pytest.raises(TypeError, match="slots"):
        B.apnn_kv_append(cache, k, k, slots.int())
    with pytest.raises(ValueError, match="positions go with a table"):
        B.apnn_kv_append(cache, k, k, slots, positions=at)
    with pytest.raises(B.ApnnError, match="rot = 66"):
        B.apnn_kv_append(cache, k, k, slots, positions=at, table=torch.zeros((4, 66), device="cuda"))
    with pytest.raises(ValueError, match="v_scale: size"):
        B.apnn_kv_read(B.KVCache(cache.k_codes, cache.k_scale, cache.v_codes, cache.v_scale[:1]), slots)
    q, lens, pages = torch.zeros((3, 4, 64), device="cuda", dtype=F16), torch.ones(3, dtype=torch.int32, device="cuda"), torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    with pytest.raises(B.ApnnError, match="queries of type"):
        B.apnn_kv_attention(cache, q.float(), lens, pages, 1.0)
    with pytest.raises(ValueError, match="pages: size"):
        B.apnn_kv_attention(cache, q, lens, pages[:2], 1.0)
    with pytest.raises(ValueError, match="q_start: size"):
        B.apnn_kv_attention(cache, q, lens, pages, 1.0, q_start=lens)
    with pytest.raises(B.ApnnError, match="4 query heads|3 query heads"):
        B.apnn_kv_attention(cache, q[:, :3].contiguous(), lens, pages, 1.0)
    with pytest.raises(B.ApnnError, match="strides"):
        B.apnn_kv_attention(cache, q, lens, pages, 1.0, out=torch.zeros((3, 1, 64), device="cuda", dtype=F16).expand(3, 4, 64))
