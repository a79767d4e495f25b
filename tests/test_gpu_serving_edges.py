"""The operators of low-bit language models where sizes, scores, weights and cached bytes are unusual, against closed forms and 64 bits."""
import numpy as np
import pytest
import torch

from oracle import serving as O
from paper_2106_12169_amd import binding as B
from tests.test_gpu_serving import BF16, F16, F32, attend, check_product, close, dense, f64, filled, normal, operands, rng, rows  # noqa: F401  (rows: a fixture)

pytestmark = pytest.mark.gpu


def ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def sink_and_tail(l, heads, D, page, at):
    """A sequence whose token `at` has key 1 and value 0, all the others key 0 and value 1: every number of it is one of the cache."""
    pages = -(-l // page)
    cache = B.KVCache.empty(pages, heads, page, D)
    k, v = torch.zeros((l, heads, D), device="cuda"), torch.ones((l, heads, D), device="cuda")
    k[at], v[at] = 1.0, 0.0
    B.apnn_kv_append(cache, k, v, torch.arange(l, device="cuda"))
    return cache, torch.arange(pages, dtype=torch.int32, device="cuda").reshape(1, -1)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("l, D, at", [(20000, 64, 0), (20000, 128, 7777), (700, 96, 0), (3000, 256, 2999), (131072, 128, 0)])
def test_a_long_tail_of_small_weights(l, D, at, dtype, rows):
    """One token of value 0 with the largest weight and a tail e^-gap below it: the result is the tail's share.

    Scores are exact: products of 1 with 0 or 1.  In powers of two the gap is 1.4427 gap, off by at most 3 2^-24 of it (constant, scale,
    product), and v_exp_f32 adds 2^-22, to a tail weight w: 2^-21 w (1 + gap).  A weight is rounded by 2^-11 of it, or by 2^-32 of the largest
    one; sums of l terms of one sign are off by l 2^-24 of themselves at most, in any order.  Both count in the numerator and in the sum."""
    cache, pages = sink_and_tail(l, 2, D, 64, at)
    news = 70 if D == 64 else 3
    q = torch.ones((news, 4, D), dtype=dtype, device="cuda")
    for gap in (6.0, 10.0, 14.0, 16.0, 17.0, 17.5, 18.0):
        scale = float(np.float32(gap / D))
        out = B.apnn_kv_attention(cache, q, ints([l]), pages, scale, q_start=ints([0, news]), max_q=news)
        w = np.exp(-scale * D)
        for i in range(news):
            tail = l - news + i                           # tokens seen beside the sink
            if l - news + i < at:                         # (the sink is not seen yet: all weights are equal)
                want = 1.0
            else:
                want = tail * w / (1 + tail * w)
            rel = 2.0 ** -11 + 2 * (2.0 ** -21 * (1 + gap) + l * 2.0 ** -24)
            close(out[i], np.full((4, D), want), dtype, rel * want + l * 2.0 ** -32)


@pytest.mark.parametrize("news", [1, 40])
def test_scale_zero_is_the_average_whatever_the_queries(news, rows):
    """Finite queries of any size with scale 0: equal weights, so sums of values in fp32: l 2^-24 of the sum of magnitudes, twice."""
    l, D = 200, 64
    cache, table = filled(rng(50), [l], 2, 16, D)
    k, v = dense(cache, table, 0, l)
    for size in (1.0, 1e30, 3e38):
        q = (normal(rng(51), news, 4, D).clamp(-1, 1) * size).to(BF16)
        q[0, 1] = 0
        out = B.apnn_kv_attention(cache, q, ints([l]), table, 0.0, q_start=ints([0, news]), max_q=news)
        for i in range(news):
            seen = l - news + i + 1
            for h in range(4):
                close(out[i, h], v[:seen, h // 2].mean(0), BF16, 2 * l * 2.0 ** -24 * np.abs(v[:seen, h // 2]).mean(0))
    q[0, 2, 5], q[-1, 3, 0] = float("nan"), float("-inf")               # 0 times these is not 0
    out = B.apnn_kv_attention(cache, q, ints([l]), table, 0.0, q_start=ints([0, news]), max_q=news)
    want = np.zeros((news, 4), bool)
    want[0, 2] = want[-1, 3] = True
    np.testing.assert_array_equal(torch.isnan(out).all(-1).cpu().numpy(), want)
    np.testing.assert_array_equal(torch.isnan(out).any(-1).cpu().numpy(), want)


@pytest.mark.parametrize("l", [1, 40, 3000])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_queries_and_scores_beyond_range_give_nan(l, dtype, rows):
    """No number is the softmax of scores that are infinite or leave fp32's range, upwards or downwards; others in the batch are not touched,
    and a query that sees nothing still gets zeros."""
    D, H = 64, 2
    pages = -(-l // 64) + 1
    cache = B.KVCache.empty(pages, H, 64, D)
    k = torch.ones((l, H, D), device="cuda")
    B.apnn_kv_append(cache, k, k, torch.arange(l, device="cuda"))
    table = torch.arange(pages, dtype=torch.int32, device="cuda").reshape(1, -1)
    news = 3
    q = torch.ones((news, H, D), dtype=dtype, device="cuda")
    q[2, 0, 5], q[1, 1, 63] = float("-inf"), float("inf")
    out = B.apnn_kv_attention(cache, q, ints([l]), table, 0.125, q_start=ints([0, news]), max_q=news)
    want = torch.ones((news, H), device="cuda")
    want[2, 0] = want[1, 1] = float("nan")
    for i in range(news):
        if l - news + i + 1 <= 0:
            want[i] = 0
    assert torch.equal(torch.nan_to_num(out.float(), nan=7.0), torch.nan_to_num(want, nan=7.0)[:, :, None].expand(news, H, D))
    nothing = torch.full_like(table, -1)
    assert (B.apnn_kv_attention(cache, q, ints([l]), nothing, 0.125, q_start=ints([0, news]), max_q=news) == 0).all()
    q = torch.ones((1, H, D), dtype=dtype, device="cuda")
    for scale in (1e37, -1e37):                           # 64 of it is beyond fp32
        assert torch.isnan(B.apnn_kv_attention(cache, q, ints([l]), table, scale)).all()
    assert torch.equal(B.apnn_kv_attention(cache, q, ints([l]), table, 1e35), q)
    assert torch.equal(B.apnn_kv_attention(cache, q, ints([l]), table, -1e35), q)


def test_parts_without_a_number_join_with_those_that_have_one(rows):
    """Scores of -inf in one part of a context that is split and finite ones in another: the former have no weight; none at all gives NaN."""
    l, D = 6000, 64
    cache = B.KVCache.empty(l // 16, 1, 16, D)
    k, v = torch.zeros((l, 1, D), device="cuda"), torch.zeros((l, 1, D), device="cuda")
    k[:3000], k[3000:], v[:3000], v[3000:] = -6 * 2.0 ** 13, 1.0, 3.0, 2.0
    B.apnn_kv_append(cache, k, v, torch.arange(l, device="cuda"))
    table = torch.arange(l // 16, dtype=torch.int32, device="cuda").reshape(1, -1)
    q = torch.full((2, 2, D), 2.0 ** 115, dtype=BF16, device="cuda")   # -6 2^13 2^115 D: out of range; 2^115 D is not
    start = ints([0, 2])
    assert (B.apnn_kv_attention(cache, q, ints([l]), table, 2.0 ** -115, q_start=start, max_q=2) == 2).all()
    assert torch.isnan(B.apnn_kv_attention(cache, q, ints([3000]), table, 2.0 ** -115, q_start=start, max_q=2)).all()
    some = table.clone()
    some[0, :3000 // 16 + 1] = -1                         # tokens 0 .. 3007 are nowhere
    assert (B.apnn_kv_attention(cache, q, ints([3000]), some, 2.0 ** -115, q_start=start, max_q=2) == 0).all()
    assert (B.apnn_kv_attention(cache, q, ints([l]), some, 2.0 ** -115, q_start=start, max_q=2) == 2).all()


@pytest.mark.parametrize("l, news", [(300, 40), (300, 200), (3000, 4)])
def test_values_of_unseen_tokens_may_be_any_bytes(l, news, rows):
    """Value scale bytes that append never writes, in tokens that stand after the query: nothing of them reaches it."""
    D, page = 64, 16
    g = rng(60 + news)
    cache, table = filled(g, [l], 2, page, D)
    q = normal(g, news, 4, D, dtype=F16)
    run = lambda: B.apnn_kv_attention(cache, q, ints([l]), table, 0.125, q_start=ints([0, news]), max_q=news)  # noqa: E731
    good = run()
    first = l - news // 2                                 # tokens from here on: seen by the later queries only
    for t in range(first, l):
        at = int(table[0, t // page])
        cache.v_scale[at, :, t % page] = 255 if t % 2 else 150
    some = news - (l - first)                             # queries that see none of them
    assert some > 0
    got = run()
    assert torch.equal(got[:some], good[:some])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D, Hq, heads", [(96, 6, 2), (256, 4, 1), (64, 3, 3), (128, 8, 2)])
def test_long_contexts_of_every_size_of_head(D, Hq, heads, dtype, rows):
    """Parts of splits joined by both kernels that join, for every number of channels."""
    attend(100 + D, [9000, 1100, 5000], [1, 1, 1], Hq, heads, D, 64, dtype)        # up to 36 parts: a block to a row
    attend(200 + D, [6000, 1300], [40, 7], Hq, heads, D, 32, dtype)
    attend(300 + D, [2100] * 12, [1] * 12, 8 * (Hq // heads), 8, D, 16, dtype)      # 96 blocks, 5 parts: a team of lanes to a row


@pytest.mark.parametrize("D, heads", [(64, 2), (128, 4), (256, 1)])
def test_parts_beyond_one_pass_of_the_join(D, heads):
    """131072 tokens: more parts of a row than the teams of a block take at once."""
    attend(400 + D, [131072, 70000], [1, 1], 2 * heads, heads, D, 256, F16)


@pytest.mark.parametrize("D", [64, 96])
def test_splits_with_missing_pages_nan_and_nothing_to_see(D, rows):
    """On contexts that are split: a split made of missing pages, a NaN in a later split, sequences of which nothing is seen."""
    g, page, l, H = rng(70 + D), 64, 6000, 2
    cache, table = filled(g, [l, l], H, page, D)
    k, v = dense(cache, table, 0, l)
    q = normal(g, 4, 4, D, dtype=BF16)
    damaged = table.clone()
    damaged[0, 16:40] = -3                                # tokens 1024 .. 2559
    damaged[0, 70] = 1 << 30
    keep = np.r_[0:1024, 2560:4480, 4544:l]
    start = ints([0, 2, 4])
    out = B.apnn_kv_attention(cache, q, ints([l, 0]), damaged, 0.1, q_start=start, max_q=2)
    for i in range(2):
        seen = keep[keep <= l - 2 + i]
        for h in range(4):
            want, spread, _ = O.attention(f64(q[i:i + 1, h]), k[seen, h // 2], v[seen, h // 2], len(seen) - 1, 0.1)
            close(out[i, h], want[0], BF16, 2.0 ** -10 * spread[0] + 1e-6)
    assert (out[2:] == 0).all()
    bad = torch.randn(1, H, D, device="cuda")
    bad[0, 1, 3] = float("inf")
    t = l - 1                                             # seen by the second query only
    B.apnn_kv_append(cache, bad, bad, (table[0, t // page].long() * page + t % page).reshape(1))
    out = B.apnn_kv_attention(cache, q, ints([l, 1]), damaged, 0.1, q_start=start, max_q=2)
    nan = torch.isnan(out).all(-1).cpu().numpy()
    want = np.zeros((4, 4), bool)
    want[1, 2:] = True
    np.testing.assert_array_equal(nan, want)
    np.testing.assert_array_equal(torch.isnan(out).any(-1).cpu().numpy(), want)
    assert (out[2] == 0).all() and (out[3] != 0).any()
    assert (B.apnn_kv_attention(cache, q, ints([l, l]), torch.full_like(table, -1), 0.1, q_start=start, max_q=2) == 0).all()


# two, three and four tiles of channels a block with as many of tokens, sizes that end inside a tile
WIDE = [(20, 6150, 200), (40, 9300, 333), (17, 12301, 129), (48, 6200, 64), (33, 6145, 1000), (45, 12300, 130), (64, 6161, 100), (60, 9217, 65), (50, 12305, 47),
        (31, 9999, 77), (100, 2601, 77), (128, 5200, 300), (128, 7700, 300), (66, 5121, 500), (127, 10240, 33)]


@pytest.mark.parametrize("M, N, K", WIDE)
def test_few_tokens_against_wide_layers(M, N, K):
    """The forms that read the tokens less often, which need many channels; and nothing is written beside a strided result."""
    X, xs, W, ws, bias = operands(M, N, K, low=-128)
    for dtype, b in ((F32, bias), (F16, None), (BF16, bias)):
        check_product(B.apnn_gemm_scaled(X, xs, W, ws, K, bias=b, dtype=dtype), X, xs, W, ws, b, dtype)
    whole = torch.full((M + 2, N + 5), 7.0, dtype=BF16, device="cuda")
    out = whole[1:M + 1, 3:N + 3]
    B.apnn_gemm_scaled(X, xs, W, ws, K, bias=bias, out=out)
    check_product(out, X, xs, W, ws, bias, BF16)
    out.fill_(7.0)
    assert (whole == 7.0).all()


def test_inputs_that_require_gradients_are_refused():
    x = torch.randn(4, 32, device="cuda", requires_grad=True)
    with pytest.raises(RuntimeError, match="src: .*gradient"):
        B.apnn_quantize_tokens(x)
    with torch.no_grad():
        codes, scale = B.apnn_quantize_tokens(x)
    bias = torch.randn(4, device="cuda", requires_grad=True)
    with pytest.raises(RuntimeError, match="bias: .*gradient"):
        B.apnn_gemm_scaled(codes, scale, codes, scale, 32, bias=bias)
    assert not B.apnn_gemm_scaled(codes, scale, codes, scale, 32, bias=bias.detach()).requires_grad
    cache = B.KVCache.empty(1, 1, 16, 64)
    k = torch.randn(2, 1, 64, device="cuda")
    q = torch.randn(2, 1, 64, device="cuda", dtype=F16, requires_grad=True)
    with pytest.raises(RuntimeError, match="k: .*gradient"):
        B.apnn_kv_append(cache, k.requires_grad_(), k, torch.arange(2, device="cuda"))
    with pytest.raises(RuntimeError, match="q: .*gradient"):
        B.apnn_kv_attention(cache, q, ints([1, 2]), ints([[0], [0]]), 1.0)
    with torch.inference_mode():
        B.apnn_kv_attention(cache, q, ints([1, 2]), ints([[0], [0]]), 1.0, out=torch.empty_like(q))


def test_results_written_in_place_are_seen_by_autograd():
    """A tensor that a backward pass needs and a call has overwritten makes that pass fail instead of using the new values."""
    cache, w = B.KVCache.empty(1, 1, 16, 64), torch.randn(64, device="cuda", requires_grad=True)
    q, k = torch.randn(2, 1, 64, device="cuda"), torch.randn(2, 1, 64, device="cuda")
    y = (q * w).sum()
    table = torch.ones((4, 64), device="cuda")
    B.apnn_kv_append(cache, k, k, torch.arange(2, device="cuda"), q=q, q_out=q, table=table, positions=ints([1, 2]))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    out = torch.empty((2, 1, 64), device="cuda", dtype=F16)
    before = out._version
    B.apnn_kv_attention(cache, q.half(), ints([1, 2]), ints([[0], [0]]), 1.0, out=out)
    assert out._version == before + 1
