"""What gr4ad_op_paged_attention, gr4ad_op_quantize_blocks, gr4ad_op_linear_fp8_block and gr4ad_op_adjust_logits refuse, on the host: through the C ABI with
pointers that are never looked at, and through the binding with tensors that are not on a GPU."""
import ctypes as C

import pytest
import torch

from paper_2602_22732_amd import binding

P = 4096  # stands for an aligned device pointer
OK = dict(dtype=1, k=P, v=P, table=P, n_pages=4, page=16, max_pages=2, H_kv=2, dh=64, q=P, q_stride=256, k_new=P, v_new=P, kv_stride=128, start=P, len=P, out=P, B=1, N=1, H=4,
          scale=0.1, window=0, sinks=0, ws=P, ws_bytes=1 << 40)


def attention(**over):
    a = dict(OK, **over)
    cache = binding.PagedCacheDesc(a["k"], a["v"], a["table"], a["n_pages"], a["page"], a["max_pages"], a["H_kv"], a["dh"])
    L = binding.lib()
    return L.gr4ad_op_paged_attention(a["dtype"], C.byref(cache), a["q"], a["q_stride"], a["k_new"], a["v_new"], a["kv_stride"], a["start"], a["len"], a["out"], a["B"], a["N"], a["H"],
                                      a["scale"], a["window"], a["sinks"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("over,status,needle", [
    (dict(dtype=5), -1, "dtype"), (dict(B=0), -1, "positive"), (dict(N=0), -1, "positive"), (dict(H=0), -1, "positive"), (dict(n_pages=0), -1, "positive"),
    (dict(window=-1), -1, "window"), (dict(sinks=-1), -1, "sinks"), (dict(H=5), -1, "divisible"), (dict(dh=48, q_stride=4096), -2, "head width"), (dict(page=24), -2, "power of two"),
    (dict(page=8), -2, "page_size"), (dict(page=2048), -2, "page_size"), (dict(max_pages=1 << 28), -2, "2^30"), (dict(q=None), -1, "NULL"), (dict(out=None), -1, "NULL"),
    (dict(table=None), -1, "NULL"), (dict(k_new=None), -1, "both or neither"), (dict(scale=0.0), -1, "scale"), (dict(scale=float("nan")), -1, "scale"),
    (dict(scale=float("inf")), -1, "scale"), (dict(q_stride=255), -1, "strides"), (dict(kv_stride=127), -1, "strides"), (dict(q_stride=260), -1, "aligned"), (dict(q=P + 2), -1, "aligned"),
    (dict(kv_stride=129), -1, "aligned"), (dict(k_new=P + 2), -1, "aligned"), (dict(v=P + 8), -1, "aligned"), (dict(max_pages=4096, ws_bytes=16), -3, "workspace"),
    (dict(max_pages=4096, ws=None), -3, "workspace"), (dict(max_pages=4096, ws=P + 4), -3, "workspace"),
])
def test_attention_refuses(over, status, needle):
    assert attention(**over) == status
    assert needle in binding.lib().gr4ad_last_error(None).decode()


def test_attention_workspace():
    L = binding.lib()
    cache = binding.PagedCacheDesc(None, None, None, 4, 16, 4096, 2, 64)
    one = L.gr4ad_op_paged_attention_workspace_bytes(1, C.byref(cache), 1, 1, 4, 0, 0)
    assert one > 0 and L.gr4ad_op_paged_attention_workspace_bytes(1, C.byref(cache), 1, 2, 4, 0, 0) > one
    assert L.gr4ad_op_paged_attention_workspace_bytes(1, C.byref(cache), 0, 1, 4, 0, 0) == 0
    assert L.gr4ad_op_paged_attention_workspace_bytes(1, None, 1, 1, 4, 0, 0) == 0


@pytest.mark.parametrize("args,status", [
    ((0, None, 8, P, P, 1, 8, 1), -1), ((0, P, 8, None, P, 1, 8, 1), -1), ((0, P, 8, P, None, 1, 8, 1), -1), ((3, P, 8, P, P, 1, 8, 1), -1), ((0, P, 8, P, P, 0, 8, 1), -1),
    ((0, P, 7, P, P, 1, 8, 1), -1), ((0, P, 8, P, P, 1, 8, 64), -2), ((0, P + 2, 8, P, P, 1, 8, 1), -1), ((0, P, 8, P, P + 1, 1, 8, 1), -1), ((0, P, 2 ** 31 - 1, P, P, 2 ** 31 - 1, 2 ** 31 - 1, 1), -2),
    ((0, P, 2 ** 31 - 1, P, P, 1, 2 ** 31 - 1, 1), -2),
])
def test_quantize_refuses(args, status):
    assert binding.lib().gr4ad_op_quantize_blocks(*args, None) == status
    assert b"quantize_blocks" in binding.lib().gr4ad_last_error(None)


@pytest.mark.parametrize("args,status", [
    ((None, P, P, P, None, P, 1, 1, 1, 0), -1), ((P, None, P, P, None, P, 1, 1, 1, 0), -1), ((P, P, None, P, None, P, 1, 1, 1, 0), -1), ((P, P, P, None, None, P, 1, 1, 1, 0), -1),
    ((P, P, P, P, None, None, 1, 1, 1, 0), -1), ((P, P, P, P, None, P, 0, 1, 1, 0), -1), ((P, P, P, P, None, P, 1, 0, 1, 0), -1), ((P, P, P, P, None, P, 1, 1, 0, 0), -1),
    ((P, P, P, P, None, P + 1, 1, 1, 1, 0), -1), ((P, P + 2, P, P, None, P, 1, 1, 1, 0), -1), ((P, P, P, P, P + 2, P, 1, 1, 1, 0), -1), ((P, P, P, P, None, P, 2 ** 31 - 1, 1, 1, 0), -2),
    ((P, P, P, P, None, P, 2 ** 31 - 300, 2 ** 31 - 300, 128, 0), -2), ((P, P, P, P, None, P, 2 ** 31 - 300, 2 ** 31 - 300, 130, 0), -2),
])
def test_linear_refuses(args, status):
    assert binding.lib().gr4ad_op_linear_fp8_block(*args, None) == status
    assert b"linear_fp8_block" in binding.lib().gr4ad_last_error(None)


@pytest.mark.parametrize("over,rows,V,needle", [
    ({}, 0, 8, "rows"), ({}, 1, 0, "rows"), (dict(history=P), 1, 8, "history_stride"), (dict(repetition=P), 1, 8, "history"), (dict(presence=P), 1, 8, "history"),
    (dict(frequency=P), 1, 8, "history"), (dict(bias=P), 1, 8, "n_bias"), (dict(mask=P), 1, 8, "n_masks"),
])
def test_adjust_refuses(over, rows, V, needle):
    L = binding.lib()
    for entry in (L.gr4ad_op_adjust_logits, L.gr4ad_op_adjust_logits_f16):
        assert entry(P, P, rows, V, C.byref(binding.LogitRules(**over)), None) == -1
        assert needle in L.gr4ad_last_error(None).decode()
        assert entry(None, P, 1, 8, C.byref(binding.LogitRules()), None) == -1
        assert entry(P, P + 1, 1, 8, C.byref(binding.LogitRules()), None) == -1
        assert entry(P, P, 1, 8, None, None) == -1
        for size in ((1, 2 ** 30 + 1), (2 ** 31 - 1, 2 ** 30)):
            assert entry(P, P, *size, C.byref(binding.LogitRules()), None) == -2


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    z = torch.zeros
    with pytest.raises(ValueError, match="GPU"):
        binding.op_paged_attention(z(1, 1, 16), z(1, 1, 16, 16), z(1, 1, 16, 16), z(1, 1, dtype=torch.int32), z(2, dtype=torch.int32), z(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        binding.op_quantize_blocks(z(1, 8))
    with pytest.raises(ValueError, match="GPU"):
        binding.op_linear_fp8_block(z(1, 8, dtype=torch.uint8), z(1, 1), z(1, 8, dtype=torch.uint8), z(1, 1))
    with pytest.raises(ValueError, match="GPU"):
        binding.op_adjust_logits(z(1, 8))


@pytest.mark.gpu
def test_binding_refuses_types_shapes_and_strides():
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)  # noqa: E731
    i32 = dict(dtype=torch.int32)
    good = dict(q=z(3, 4, 64), k_pages=z(2, 2, 16, 64), v_pages=z(2, 2, 64, 16), page_table=z(1, 2, **i32), q_start=z(2, **i32), seq_len=z(1, **i32))
    binding.op_paged_attention(**good)
    for name, bad in [("q", z(3, 4, 64, dtype=torch.float16)), ("q", z(3, 64, 4).transpose(1, 2)), ("v_pages", z(2, 2, 16, 64)), ("k_pages", z(2, 2, 64, 16).transpose(2, 3)),
                      ("page_table", z(1, 2, dtype=torch.int64)), ("q_start", z(3, **i32)), ("seq_len", z(2, **i32)), ("q", z(3, 4, 64).cpu()), ("seq_len", z(1, **i32).cpu())]:
        with pytest.raises(ValueError):
            binding.op_paged_attention(**dict(good, **{name: bad}))
    with pytest.raises(ValueError):
        binding.op_paged_attention(**good, k_new=z(3, 2, 64), v_new=z(3, 2, 128)[:, :, :64])
    with pytest.raises(binding.Gr4adError, match="both or neither"):
        binding.op_paged_attention(**good, k_new=z(3, 2, 64))
    with pytest.raises(ValueError):
        binding.op_paged_attention(**good, out=z(3, 4, 64, dtype=torch.bfloat16))
    for kw in (dict(window=1 << 32), dict(window=4, sinks=1 << 31)):
        with pytest.raises(ValueError):
            binding.op_paged_attention(**good, **kw)
    with pytest.raises(ValueError):
        binding.op_quantize_blocks(z(4, 8).t())
    with pytest.raises(ValueError):
        binding.op_quantize_blocks(z(4, 8), block_rows=64)
    a, w = binding.op_quantize_blocks(z(4, 300)), binding.op_quantize_blocks(z(200, 300), 128)
    assert binding.op_linear_fp8_block(*a, *w).shape == (4, 200)
    for args in [(a[0], w[1], *w), (*a, w[0], a[1]), (*a, w[0][:, :200].contiguous(), w[1]), (a[0].view(torch.int8), a[1], *w)]:
        with pytest.raises(ValueError):
            binding.op_linear_fp8_block(*args)
    with pytest.raises(ValueError):
        binding.op_linear_fp8_block(*a, *w, out_dtype=torch.float32)
    x = z(4, 100)
    for kw in [dict(history=z(3, 5, **i32)), dict(history=z(4, 5, dtype=torch.int64)), dict(mask=z(1, 3, **i32)), dict(bias=z(1, 99)), dict(mask=z(1, 4, **i32), mask_row=z(5, **i32)),
               dict(out=z(4, 100, dtype=torch.float16)), dict(bias=z(100, 1).t().expand(2, 100))]:
        with pytest.raises(ValueError):
            binding.op_adjust_logits(x, **kw)
    with pytest.raises(ValueError):
        binding.op_adjust_logits(x.bfloat16())
