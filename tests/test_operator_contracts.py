"""What the operators on pages, FP8 blocks and logits promise beside their results, as far as the host decides it: sizes beyond 32 bits, buffers that overlap or are
not dense, launches that do not fit, and what a failing call says."""
import ctypes as C

import pytest
import torch

from paper_2602_22732_amd import binding

I32, U8 = torch.int32, torch.uint8


@pytest.fixture
def anywhere(monkeypatch):
    """The binding's own checks on tensors that have a shape and no memory."""
    monkeypatch.setattr(binding, "_place", lambda *_: None)
    return lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="meta")


BIG = 2 ** 32  # a size of BIG + n would reach the library as n


def test_sizes_that_32_bits_do_not_hold(anywhere):
    z = anywhere
    bf16 = torch.bfloat16
    for x in (z(1, BIG + 128, dtype=bf16), z(BIG + 2, 3), z(2 ** 31, 1)):
        with pytest.raises(ValueError, match="32 bits"):
            binding.op_quantize_blocks(x)
    for M, N, K in ((BIG + 3, 4, 128), (3, BIG + 4, 128), (3, 4, BIG + 128), (1, 1, 2 ** 31)):
        with pytest.raises(ValueError, match="32 bits"):
            binding.op_linear_fp8_block(z(M, K, dtype=U8), z(-(-K // 128), M), z(N, K, dtype=U8), z(-(-K // 128), -(-N // 128)))
    for over in (dict(logits=z(BIG + 2, 8)), dict(logits=z(1, BIG + 8)), dict(history=z(2, BIG + 1, dtype=I32)), dict(bias=z(BIG + 1, 8)), dict(mask=z(BIG + 1, 1, dtype=I32))):
        with pytest.raises(ValueError, match="32 bits"):
            binding.op_adjust_logits(**dict(dict(logits=z(2, 8)), **over))


@pytest.mark.parametrize("sizes", [dict(N=BIG + 1), dict(H=BIG + 2), dict(B=BIG + 1), dict(max_pages=BIG + 1), dict(n_pages=BIG + 1), dict(H_kv=BIG + 1, H=BIG + 1), dict(page=BIG + 16), dict(dh=BIG + 16)])
def test_attention_sizes_that_32_bits_do_not_hold(anywhere, sizes):
    z, s = anywhere, dict(dict(N=1, H=2, B=1, max_pages=1, n_pages=1, H_kv=1, page=16, dh=16), **sizes)
    with pytest.raises(ValueError, match="32 bits"):
        binding.op_paged_attention(z(s["N"], s["H"], s["dh"]), z(s["n_pages"], s["H_kv"], s["page"], s["dh"]), z(s["n_pages"], s["H_kv"], s["dh"], s["page"]), z(s["B"], s["max_pages"], dtype=I32),
                                   z(s["B"] + 1, dtype=I32), z(s["B"], dtype=I32))


@pytest.mark.parametrize("kw", [dict(window=BIG + 5), dict(window=5, sinks=BIG), dict(window=-BIG + 5), dict(window=5, sinks=-BIG)])
def test_windows_that_32_bits_do_not_hold(anywhere, kw):
    z = anywhere
    with pytest.raises(ValueError, match="window"):
        binding.op_paged_attention(z(1, 2, 16), z(1, 1, 16, 16), z(1, 1, 16, 16), z(1, 1, dtype=I32), z(2, dtype=I32), z(1, dtype=I32), **kw)


def test_workspace_must_be_dense(anywhere):
    z = anywhere
    for workspace in (z(2, 1 << 20, dtype=U8)[:, ::2], z(1, dtype=U8).expand(1 << 24)):
        with pytest.raises(ValueError, match="workspace"):
            binding.op_paged_attention(z(1, 2, 64), z(9, 1, 16, 64), z(9, 1, 64, 16), z(1, 4096, dtype=I32), z(2, dtype=I32), z(1, dtype=I32), workspace=workspace)


K, M = 1 << 10, 1 << 20
# an attention call whose buffers lie 16 MB apart: bf16, 2 rows of 4 heads of 64 columns, 3 pages of 16 positions of 2 key heads
APART = dict(k=16 * M, v=32 * M, table=48 * M, q=64 * M, k_new=80 * M, v_new=96 * M, start=112 * M, len=128 * M, out=144 * M, ws=160 * M, q_stride=256, kv_stride=128, max_pages=4, n_pages=3, N=2)


def attention(**over):
    a = dict(APART, **over)
    cache = binding.PagedCacheDesc(a["k"], a["v"], a["table"], a["n_pages"], 16, a["max_pages"], 2, 64)
    return binding.lib().gr4ad_op_paged_attention(1, C.byref(cache), a["q"], a["q_stride"], a["k_new"], a["v_new"], a["kv_stride"], a["start"], a["len"], a["out"], 1, a["N"], 4, 0.1, 0, 0, a["ws"],
                                                  1 << 22, None)


ROW, PAGES = 4 * 64 * 2, 3 * 2 * 16 * 64 * 2  # bytes of a row of q, of an array of pages


@pytest.mark.parametrize("over", [
    dict(out=APART["q"]), dict(out=APART["q"] + 2 * ROW - 16), dict(out=APART["q"] - 2 * ROW + 16), dict(out=APART["q"] + 8 * K - 2 * ROW + 16, q_stride=4 * K), dict(out=APART["k_new"] + 16),
    dict(out=APART["v_new"] + 496), dict(out=APART["k"] + PAGES - 16), dict(out=APART["v"]), dict(v=APART["k"] + PAGES - 16), dict(out=APART["table"] - 16), dict(start=APART["out"] + 1000),
    dict(len=APART["out"]), dict(q=APART["v"] + 256), dict(k_new=APART["k"]), dict(max_pages=4096, ws=APART["q"] - 4 * K), dict(max_pages=4096, ws=APART["out"]), dict(max_pages=4096, ws=APART["k"] + 256),
    dict(table=APART["k"] + 16),
])
def test_attention_buffers_that_overlap(over):
    assert attention(**over) == -1
    assert b"overlap" in binding.lib().gr4ad_last_error(None)


@pytest.mark.parametrize("itemsize,entry", [(4, "gr4ad_op_adjust_logits"), (2, "gr4ad_op_adjust_logits_f16")])
def test_logits_that_overlap(itemsize, entry):
    rows, V, n = 3, 100, 300 * itemsize
    f = getattr(binding.lib(), entry)
    rules = binding.LogitRules(history=M, history_stride=5, bias=2 * M, n_bias=2, mask=3 * M, n_masks=2)
    for logits, out in ((8 * M, 8 * M + itemsize), (8 * M, 8 * M - n + itemsize), (8 * M, M), (8 * M, M + 56), (8 * M, 2 * M + 796), (8 * M, 3 * M + 28)):
        assert f(logits, out, rows, V, C.byref(rules), None) == -1
        assert b"overlap" in binding.lib().gr4ad_last_error(None)


def no_gpu():
    """Calls that no check refuses: only where no launch can follow."""
    if torch.cuda.is_available():
        pytest.skip("with a GPU these would launch on addresses that are none")


@pytest.mark.parametrize("over", [dict(out=APART["q"] + 2 * ROW), dict(out=APART["q"] - 2 * ROW), dict(out=APART["q"] + ROW, q_stride=4 * K), dict(out=APART["k"] + PAGES), dict(v=APART["k"] + PAGES),
                                  dict(ws=APART["q"]), dict(k_new=None, v_new=None, q=APART["v"] + 256), dict(v_new=APART["k_new"])])
def test_attention_buffers_side_by_side(over):
    no_gpu()
    assert attention(**over) == -4  # (as far as the launch)


def test_logits_side_by_side():
    no_gpu()
    for logits, out in ((8 * M, 8 * M), (8 * M, 8 * M + 1200), (8 * M, 8 * M - 1200)):
        assert binding.lib().gr4ad_op_adjust_logits(logits, out, 3, 100, C.byref(binding.LogitRules()), None) == -4


FAR = 1 << 42  # addresses whose buffers may have terabytes


def wide_attention(N, H, H_kv, dh, dtype=1, B=1, new=False):
    cache = binding.PagedCacheDesc(FAR, 2 * FAR, 3 * FAR, 2, 16, 1, H_kv, dh)
    L, row = binding.lib(), H * dh
    assert L.gr4ad_op_paged_attention_workspace_bytes(dtype, C.byref(cache), B, N, H, 0, 0) == 0
    return L.gr4ad_op_paged_attention(dtype, C.byref(cache), 4 * FAR, row, 5 * FAR if new else None, 6 * FAR if new else None, H_kv * dh, 7 * FAR, 8 * FAR, 9 * FAR, B, N, H, 0.1, 0, 0, None, 0, None)


@pytest.mark.parametrize("H,H_kv,dh", [(1 << 24, 1, 128), (1 << 27, 1 << 26, 16), (1 << 30, 1, 64)])
def test_rows_of_2_to_the_31_values(H, H_kv, dh):
    assert wide_attention(1, H, H_kv, dh) == -2
    assert b"2^31" in binding.lib().gr4ad_last_error(None)


# One launch takes fewer than 2^32 threads.  The first size that is too large, and one below it that is not.
@pytest.mark.parametrize("rows,n,block_rows,fits", [((1 << 28) - 15, 1, 1, False), ((1 << 28) - 16, 256, 1, True), ((1 << 28) - 16, 257, 1, False), ((1 << 30) + 1, 257, 128, False), ((1 << 30) + 1, 128, 128, True)])
def test_quantiser_launch(rows, n, block_rows, fits):
    if fits:
        no_gpu()
    assert binding.lib().gr4ad_op_quantize_blocks(1, FAR, n, 2 * FAR, 3 * FAR, rows, n, block_rows, None) == (-4 if fits else -2)
    assert fits or b"quantize_blocks" in binding.lib().gr4ad_last_error(None)


@pytest.mark.parametrize("M,N,K,fits", [(1, (1 << 27) - 15, 1, False), (1, (1 << 27) - 16, 1, True), (17, (1 << 29) - 63, 1, False), (64, (1 << 29) - 64, 1, True), (1 << 20, (1 << 19) + 1, 16, False),
                                        (1 << 20, (1 << 19) - 256, 16, True), (1 << 20, (1 << 18) + 1, 17, False), (1 << 20, (1 << 18) - 128, 17, True)])
def test_product_launch(M, N, K, fits):
    if fits:
        no_gpu()
    assert binding.lib().gr4ad_op_linear_fp8_block(FAR, 2 * FAR, 3 * FAR, 4 * FAR, None, 5 * FAR, M, N, K, 0, None) == (-4 if fits else -2)
    assert fits or b"linear_fp8_block" in binding.lib().gr4ad_last_error(None)


@pytest.mark.parametrize("rows,V,fits", [(1 << 26, 8, False), ((1 << 26) - 1, 8, True), (1 << 24, 4096, False), ((1 << 24) - 1, 4096, True)])
def test_logits_launch(rows, V, fits):
    if fits:
        no_gpu()
    assert binding.lib().gr4ad_op_adjust_logits_f16(FAR, 2 * FAR, rows, V, C.byref(binding.LogitRules()), None) == (-4 if fits else -2)
    assert fits or b"adjust_logits" in binding.lib().gr4ad_last_error(None)


@pytest.mark.parametrize("N,H,H_kv,dh,dtype,B,new,fits", [
    (1 << 25, 16, 16, 16, 0, 1, False, False), (1 << 24, 16, 16, 16, 0, 1, False, True),    # tiles of 32 rows
    (1 << 24, 16, 16, 16, 0, 1 << 24, False, False),                                         # of 16, a sequence each
    (1 << 26, 16, 16, 64, 1, 1, False, True),                                                # of 256
    (1 << 21, 1 << 8, 1 << 8, 32, 1, 1 << 14, False, True), (1 << 21, 1 << 8, 1 << 8, 32, 1, 1 << 14, True, False),  # of 128; with their pages' update, 2^16 tiles of 256 heads
])
def test_attention_launch(N, H, H_kv, dh, dtype, B, new, fits):
    if fits:
        no_gpu()
    assert wide_attention(N, H, H_kv, dh, dtype, B, new) == (-4 if fits else -2)
    assert fits or b"paged attention" in binding.lib().gr4ad_last_error(None)


def test_failing_launches_say_so():
    # every kind of launch without a GPU: the message is this call's and not an older one's
    no_gpu()
    L, rules = binding.lib(), C.byref(binding.LogitRules())
    calls = [("paged attention", lambda N=N, dh=dh, dtype=dtype, new=new: wide_attention(N, 16, 2, dh, dtype, 1, new)) for N, dh, dtype, new in ((1, 64, 0, False), (5, 32, 1, False), (10, 64, 1, True), (100, 128, 1, False), (2000, 64, 1, True))]
    calls += [("quantize_blocks", lambda: L.gr4ad_op_quantize_blocks(1, FAR, 8, 2 * FAR, 3 * FAR, 4, 8, 1, None))]
    calls += [("linear_fp8_block", lambda M=M, N=N, K=K: L.gr4ad_op_linear_fp8_block(FAR, 2 * FAR, 3 * FAR, 4 * FAR, None, 5 * FAR, M, N, K, 0, None))
              for M, N, K in ((4, 64, 128), (40, 20000, 128), (300, 300, 128), (2000, 2000, 128), (8192, 8192, 128), (300, 300, 130), (8192, 8192, 130))]
    calls += [("adjust_logits", lambda f=f: f(FAR, 2 * FAR, 3, 100, rules, None)) for f in (L.gr4ad_op_adjust_logits, L.gr4ad_op_adjust_logits_f16)]
    for name, call in calls:
        assert L.gr4ad_op_quantize_blocks(9, FAR, 8, FAR, FAR, 4, 8, 1, None) == -1 and b"dtype" in L.gr4ad_last_error(None)
        assert call() == -4
        said = L.gr4ad_last_error(None).decode()
        assert name in said and "hip" in said.lower(), said


def test_calls_without_rows(anywhere):
    # an idle step: nothing to do and nothing launched (there is no GPU behind these tensors)
    z = anywhere
    cache = (z(9, 2, 16, 64), z(9, 2, 64, 16), z(3, 4, dtype=I32), z(4, dtype=I32), z(3, dtype=I32))
    none = z(0, 4, 64)
    assert binding.op_paged_attention(none, *cache).shape == (0, 4, 64)
    assert binding.op_paged_attention(none, *cache, k_new=z(0, 2, 64), v_new=z(0, 2, 64), out=none) is none
    with pytest.raises(ValueError):
        binding.op_paged_attention(none, *cache, k_new=z(0, 3, 64), v_new=z(0, 2, 64))
    q, scale = binding.op_quantize_blocks(z(0, 300))
    assert q.shape == (0, 300) and scale.shape == (3, 0)
    assert binding.op_quantize_blocks(z(0, 300, dtype=torch.bfloat16), 128)[1].shape == (3, 0)
    c = binding.op_linear_fp8_block(q, scale, z(50, 300, dtype=U8), z(3, 1), out_dtype=torch.float16)
    assert c.shape == (0, 50) and c.dtype == torch.float16
    logits = z(0, 100)
    assert binding.op_adjust_logits(logits, history=z(0, 5, dtype=I32), repetition=z(0), bias=z(1, 100), out=logits) is logits
    assert binding.op_adjust_logits(z(2, 0, 100)).shape == (2, 0, 100)
    with pytest.raises(ValueError):
        binding.op_adjust_logits(logits, history=z(1, 5, dtype=I32))


def test_tables_without_rows(anywhere):
    # an empty table has no address, which the library takes for no rule at all: where every token was to be forbidden, all would be allowed
    z = anywhere
    for rule in (dict(mask=z(0, 4, dtype=I32)), dict(bias=z(0, 100))):
        with pytest.raises(ValueError, match="no rows"):
            binding.op_adjust_logits(z(2, 100), **rule)
