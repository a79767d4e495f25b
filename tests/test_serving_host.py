"""What the operators of low-bit language models refuse, without a GPU: the C entry points check before they touch the
device, the binding checks tensors before it calls them."""
import ctypes as C

import pytest
import torch

from paper_2106_12169_amd import binding as B

FAKE = 0x10000          # a 16-byte aligned non-null "device pointer" that must never be dereferenced
ARG, UNSUPPORTED, OVERFLOW, ALIGNMENT = 1, 2, 3, 4


def last():
    return B.lib().apnn_last_error().decode()


def cache(**over):
    d = dict(k_codes_dev=FAKE, k_scale_dev=FAKE, v_codes_dev=FAKE, v_scale_dev=FAKE, pages=4, heads=2, page_size=16, D=64)
    d.update(over)
    return B.KVCacheDesc(**d)


def tokens(**over):
    d = dict(tokens=3, type=2, k_dev=FAKE, v_dev=FAKE, k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64, slot_dev=FAKE)
    d.update(over)
    return B.KVTokensDesc(**d)


def attention(**over):
    d = dict(tokens=3, type=2, q_heads=4, q_dev=FAKE, out_dev=FAKE + 4096, q_token_stride=256, q_head_stride=64, out_token_stride=256, out_head_stride=64,
             seqs=3, q_start_dev=None, len_dev=FAKE, page_dev=FAKE, max_pages=2, max_q=1, scale=1.0)
    d.update(over)
    return B.KVAttentionDesc(**d)


def test_pitch():
    assert [B.apnn_token_pitch(k) for k in (0, 1, 16, 17, 4096, -1)] == [0, 16, 16, 32, 4096, 0]


@pytest.mark.parametrize("status, args", [
    (ARG, (FAKE, 3, 2, 8, 8, FAKE, FAKE)),              # no such type
    (ARG, (FAKE, 0, -1, 8, 8, FAKE, FAKE)),
    (ARG, (FAKE, 0, 2, -8, 8, FAKE, FAKE)),
    (ARG, (FAKE, 0, 2, 8, 7, FAKE, FAKE)),              # rows that overlap
    (ARG, (None, 0, 2, 8, 8, FAKE, FAKE)),
    (ARG, (FAKE, 0, 2, 8, 8, None, FAKE)),
    (ARG, (FAKE, 0, 2, 8, 8, FAKE, None)),
    (ALIGNMENT, (FAKE, 0, 2, 8, 8, FAKE + 8, FAKE)),
    (ALIGNMENT, (FAKE + 1, 1, 2, 8, 8, FAKE, FAKE)),
    (UNSUPPORTED, (FAKE, 0, 1, 1 << 31, 1 << 31, FAKE, FAKE)),
    (ARG, (FAKE, 0, 1 << 40, 8, 1 << 40, FAKE, FAKE)),  # no memory holds it
    (0, (None, 0, 0, 8, 8, None, None)),                # nothing to do
])
def test_quantize_tokens_refusals(status, args):
    assert B.lib().apnn_quantize_tokens(*args, None) == status
    assert bool(last()) == bool(status)


@pytest.mark.parametrize("status, over", [
    (ARG, dict(type=7)), (ARG, dict(M=-1)), (ARG, dict(N=-1)), (ARG, dict(K=-1)), (ARG, dict(ldy=7)),
    (OVERFLOW, dict(K=1 << 17)), (ARG, dict(X=None)), (ARG, dict(xs=None)), (ARG, dict(W=None)), (ARG, dict(ws=None)), (ARG, dict(Y=None)),
    (ALIGNMENT, dict(X=FAKE + 8)), (ALIGNMENT, dict(W=FAKE + 1)), (ALIGNMENT, dict(Y=FAKE + 1, type=2)), (UNSUPPORTED, dict(M=1 << 40, ldy=1 << 30)),
    (0, dict(M=0)), (0, dict(N=0, ldy=0)),
])
def test_gemm_scaled_refusals(status, over):
    a = dict(X=FAKE, xs=FAKE, W=FAKE, ws=FAKE, bias=None, Y=FAKE, type=0, M=4, N=8, K=32, ldy=8)
    a.update(over)
    assert B.lib().apnn_gemm_scaled(*a.values(), None) == status
    assert bool(last()) == bool(status)


BAD_CACHES = [(UNSUPPORTED, dict(D=80)), (UNSUPPORTED, dict(D=0)), (UNSUPPORTED, dict(page_size=8)), (UNSUPPORTED, dict(page_size=48)),
              (UNSUPPORTED, dict(page_size=512)), (UNSUPPORTED, dict(heads=0)), (UNSUPPORTED, dict(heads=2000)), (ARG, dict(pages=-1)),
              (ARG, dict(pages=1 << 31)), (ARG, dict(v_scale_dev=None)), (ALIGNMENT, dict(k_scale_dev=FAKE + 4))]


@pytest.mark.parametrize("status, over", BAD_CACHES)
def test_bad_caches_are_refused_by_every_entry_point(status, over):
    L, c = B.lib(), cache(**over)
    assert L.apnn_kv_append(C.byref(c), C.byref(tokens()), None) == status and last()
    assert L.apnn_kv_read(C.byref(c), FAKE, 3, FAKE, FAKE, 0, None) == status and last()
    assert L.apnn_kv_attention(C.byref(attention()), C.byref(c), None, 0, None) == status and last()
    assert L.apnn_kv_attention_workspace_bytes(C.byref(attention()), C.byref(c)) == 0 and last()


@pytest.mark.parametrize("status, over", [
    (ARG, dict(type=5)), (ARG, dict(tokens=-1)), (ARG, dict(q_heads=-1)), (UNSUPPORTED, dict(tokens=1 << 31)), (ARG, dict(rot=3)), (ARG, dict(rot=66)),
    (ARG, dict(rot=-2)), (ARG, dict(k_dev=None)), (ARG, dict(v_dev=None)), (ARG, dict(slot_dev=None)), (ARG, dict(q_heads=2)),
    (ARG, dict(rot=64)), (ARG, dict(rot=64, table_dev=FAKE)), (ARG, dict(rot=64, position_dev=FAKE)), (ALIGNMENT, dict(k_dev=FAKE + 1)),
    (ARG, dict(q_heads=4, q_dev=FAKE, q_out_dev=FAKE, q_token_stride=256, q_head_stride=64, q_out_token_stride=512, q_out_head_stride=64)),
    (ARG, dict(q_heads=4, q_dev=FAKE, q_out_dev=FAKE + 4096, q_token_stride=256, q_head_stride=64, q_out_token_stride=0, q_out_head_stride=64)),
    (ARG, dict(q_heads=4, q_dev=FAKE, q_out_dev=FAKE + 4096, q_token_stride=256, q_head_stride=64, q_out_token_stride=64, q_out_head_stride=64)),
    (ARG, dict(k_token_stride=-1)),
    (0, dict(tokens=0)),
])
def test_append_refusals(status, over):
    assert B.lib().apnn_kv_append(C.byref(cache()), C.byref(tokens(**over)), None) == status
    assert bool(last()) == bool(status)
    assert B.lib().apnn_kv_append(None, C.byref(tokens()), None) == ARG
    assert B.lib().apnn_kv_append(C.byref(cache()), None, None) == ARG


@pytest.mark.parametrize("status, args", [
    (ARG, (FAKE, 3, FAKE, FAKE, 9)), (ARG, (FAKE, -1, FAKE, FAKE, 0)), (ARG, (None, 3, FAKE, FAKE, 0)), (ALIGNMENT, (FAKE, 3, FAKE + 4, FAKE, 0)),
    (UNSUPPORTED, (FAKE, 1 << 31, FAKE, FAKE, 0)), (0, (None, 0, None, None, 0)), (0, (FAKE, 3, None, None, 0)),
])
def test_read_refusals(status, args):
    assert B.lib().apnn_kv_read(C.byref(cache()), *args, None) == status
    assert bool(last()) == bool(status)


@pytest.mark.parametrize("status, over", [
    (UNSUPPORTED, dict(type=0)), (UNSUPPORTED, dict(type=3)), (ARG, dict(tokens=-1)), (ARG, dict(seqs=-1)), (ARG, dict(max_pages=-1)), (ARG, dict(max_q=-1)),
    (ARG, dict(q_heads=3)), (ARG, dict(q_heads=0)), (ARG, dict(scale=float("inf"))), (ARG, dict(scale=float("nan"))), (ARG, dict(seqs=4)),
    (ARG, dict(q_dev=None)), (ARG, dict(out_dev=None)), (ARG, dict(len_dev=None)), (ARG, dict(page_dev=None)), (ALIGNMENT, dict(q_dev=FAKE + 1)),
    (ARG, dict(out_dev=FAKE)), (UNSUPPORTED, dict(max_pages=1 << 27)), (UNSUPPORTED, dict(tokens=1 << 30, q_start_dev=FAKE, max_q=1 << 20, seqs=1 << 30)),
    (UNSUPPORTED, dict(tokens=(1 << 30) + 1, q_heads=2, q_start_dev=FAKE)), (ARG, dict(max_pages=4096)),       # (the last one: a workspace is needed)
    (ARG, dict(out_head_stride=0)), (ARG, dict(out_token_stride=64)), (ARG, dict(q_token_stride=-256)),
    (0, dict(seqs=0)), (0, dict(tokens=0, seqs=0)), (0, dict(max_q=0, q_start_dev=FAKE)),
])
def test_attention_refusals(status, over):
    assert B.lib().apnn_kv_attention(C.byref(attention(**over)), C.byref(cache()), None, 0, None) == status
    assert bool(last()) == bool(status)
    assert B.lib().apnn_kv_attention(None, C.byref(cache()), None, 0, None) == ARG
    assert B.lib().apnn_kv_attention(C.byref(attention()), None, None, 0, None) == ARG


def test_workspace_sizes():
    """Splits of long contexts where blocks are few, and none where they are many or contexts short."""
    c = B.KVCache.empty(2, 2, 16, 64, "cpu")
    size = B.apnn_kv_attention_workspace_bytes
    assert size(c, 1, 4, 1, 64) == 0                                    # 1024 tokens
    assert size(c, 1, 4, 1, 4096) % ((64 + 4) * 4) == 0 and size(c, 1, 4, 1, 4096) > 0
    assert size(c, 5000, 4, 5000, 4096) == 0
    assert size(c, 0, 4, 0, 4096) == 0
    L, d = B.lib(), attention(max_pages=4096)
    need = L.apnn_kv_attention_workspace_bytes(C.byref(d), C.byref(cache()))
    assert need > 0
    assert L.apnn_kv_attention(C.byref(d), C.byref(cache()), FAKE, need - 1, None) == ARG and "workspace" in last()
    assert L.apnn_kv_attention(C.byref(d), C.byref(cache()), FAKE + 8, need, None) == ALIGNMENT


def test_the_binding_refuses_what_is_no_device_tensor():
    x = torch.zeros(2, 32)
    with pytest.raises(AssertionError, match="src: a device tensor"):
        B.apnn_quantize_tokens(x)
    with pytest.raises(TypeError, match="torch tensor"):
        B.native().quantize_tokens([1.0], x, x)
    with pytest.raises(TypeError, match="3 arguments expected, got 2"):
        B.native().quantize_tokens(x, x)
    c = B.KVCache.empty(2, 1, 16, 64, "cpu")
    assert (c.heads, c.page_size, c.D) == (1, 16, 64)
    with pytest.raises(AssertionError, match="k_codes: a device tensor"):
        B.apnn_kv_read(c, torch.zeros(1, dtype=torch.int64))
    with pytest.raises(B.ApnnError, match="pages of 24 tokens"):
        B.native().kv_attention_workspace(1, 24, 64, 1, 1, 1, 1, False, 1)


@pytest.mark.parametrize("at", [0, 1, 2, 4])
def test_sizes_beyond_32_bits_are_refused_and_not_cut_off(at):
    """heads, page size, channels and query heads of the workspace's size; 2^32 more than a size that is right, or less."""
    good = [2, 16, 64, 1, 4, 1, 4096, False, 1]
    assert B.native().kv_attention_workspace(*good) > 0
    for far in (1 << 32, -(1 << 32), 1 << 62):
        bad = list(good)
        bad[at] += far
        with pytest.raises(B.ApnnError):
            B.native().kv_attention_workspace(*bad)


@pytest.mark.parametrize("scale, status", [(1.5 * 2.0 ** 127, ARG), (-3e38, ARG), (2.0 ** 127, 0), (-(2.0 ** 127), 0), (1e-45, 0)])
def test_scales_that_leave_no_room_for_powers_of_two_are_refused(scale, status):
    """Scores are taken in powers of two: the scale times log2(e) has to be a number too."""
    d = attention(scale=scale, tokens=0, seqs=0)
    assert B.lib().apnn_kv_attention(C.byref(d), C.byref(cache()), None, 0, None) == status
    assert ("scale" in last()) == bool(status)
