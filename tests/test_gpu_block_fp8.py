"""gr4ad_op_quantize_blocks and gr4ad_op_linear_fp8_block against their definitions: sizes with partial blocks and tiles, strided and misaligned rows, blocks of
zeros and of values that are no numbers."""
import numpy as np
import pytest
import torch

from paper_2602_22732_amd import binding
from test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


def blocks_of(x, block_rows):
    """(q, scale) by the definition, float32 operations on the CPU."""
    rows, n = x.shape
    rb, nb = -(-rows // block_rows), -(-n // 128)
    pad = torch.zeros(rb * block_rows, nb * 128)
    pad[:rows, :n] = x.float()
    pad = pad.view(rb, block_rows, nb, 128)
    amax = pad.abs().amax(dim=(1, 3))
    zero = amax < 2.0 ** -100
    inv = torch.where(zero, torch.ones(()), torch.full_like(amax, 448.0) / amax)  # (a number over a tensor would be rounded twice)
    q = (pad * inv[:, None, :, None]).to(F8).view(rb * block_rows, nb * 128)[:rows, :n]
    return q, torch.where(zero, torch.ones(()), amax / 448.0).t().contiguous()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,n", [(1, 1), (1, 128), (5, 127), (17, 130), (33, 1000), (128, 128), (200, 515), (300, 2048), (1, 16384)])
def test_quantize_blocks(dtype, block_rows, rows, n):
    g = torch.Generator().manual_seed(rows * 31 + n)
    x = torch.randn(rows, n, generator=g) * torch.exp(torch.empty(rows, 1).uniform_(-40, 40, generator=g))
    x[:, ::37] *= 50.0
    if rows > 4:
        x[3] = 0.0
        x[4] *= 1e-38
    x = x.to(dtype)
    wide = torch.full((rows, n + 3), float("nan"), dtype=dtype, device="cuda")   # rows that start anywhere
    wide[:, 1:n + 1] = x.cuda()
    want_q, want_s = blocks_of(x, block_rows)
    for xs in (x.cuda(), wide[:, 1:n + 1]):
        q, s = binding.op_quantize_blocks(xs, block_rows)
        assert q.shape == (rows, n) and s.shape == want_s.shape
        # the quotients are correctly rounded on both sides, the product and the conversion too: equal to the bit
        assert torch.equal(s.cpu(), want_s)
        assert torch.equal(q.cpu().view(F8).float(), want_q.float())


def test_quantize_blocks_with_values_that_are_no_numbers():
    x = torch.randn(4, 256).cuda()
    x[0, 5], x[1, 130] = float("nan"), float("inf")
    for block_rows in (1, 128):
        q, s = binding.op_quantize_blocks(x, block_rows)
        y = q.view(F8).float()
        assert torch.isnan(y[0, 5])
        if block_rows == 1:
            assert torch.isfinite(y[0, :5]).all() and torch.isfinite(s[0]).all()                   # a NaN stays where it is
            assert torch.isfinite(y[0, 128:]).all() and torch.isfinite(y[2:]).all() and torch.isfinite(y[1, :128]).all()
        assert torch.isnan(y[1, 128:] * (s[1, 1] if block_rows == 1 else s[1, 0])).any()           # an infinity shows in its block


def test_quantize_blocks_writes_nothing_outside():
    for block_rows in (1, 128):
        rows, n = 133, 390
        x = torch.randn(rows, n).cuda()
        gq, gs = Guarded(rows * n), Guarded(4 * 4 * -(-rows // block_rows))
        L = binding.lib()
        assert L.gr4ad_op_quantize_blocks(0, x.data_ptr(), n, gq.view.data_ptr(), gs.view.data_ptr(), rows, n, block_rows, None) == 0
        torch.cuda.synchronize()
        assert gq.intact() and gs.intact()


def random_e4m3(g, *shape):
    b = torch.randint(0, 256, shape, generator=g, dtype=torch.uint8)
    b[(b & 0x7F) == 0x7F] = 0x3A
    return b


SIZES = [(4099, 3000, 272), (4099, 3000, 256), (4096, 3100, 144), (4096, 3100, 128), (40, 16400, 300), (20, 8200, 200), (60, 9000, 128), (1100, 4100, 384), (1100, 4100, 400), (300, 900, 8320),
         (1, 1, 1), (1, 16, 128), (3, 50, 17), (16, 130, 256), (17, 1000, 1104), (33, 64, 4096), (64, 257, 515), (65, 66, 130), (100, 1000, 999), (130, 300, 1040),
         (517, 1000, 1104), (1500, 2100, 640), (2048, 2050, 384), (4099, 1030, 272), (2900, 2816, 144), (2100, 2070, 130)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("out,bias", [(torch.bfloat16, False), (torch.float16, True)])
def test_linear_fp8_block(M, N, K, out, bias):
    g = torch.Generator().manual_seed(M + N + K)
    A, W = random_e4m3(g, M, K), random_e4m3(g, N, K)
    nb, wb = -(-K // 128), -(-N // 128)
    sa = torch.exp(torch.empty(nb, M).uniform_(-3, 3, generator=g)) * 1e-3
    sw = torch.exp(torch.empty(nb, wb).uniform_(-3, 3, generator=g)) * 1e-3
    b = torch.randn(N, generator=g) if bias else None
    C = binding.op_linear_fp8_block(A.cuda(), sa.cuda(), W.cuda(), sw.cuda(), bias=None if b is None else b.cuda(), out_dtype=out)
    rows = torch.tensor(sorted(set(list(range(0, M, max(1, M // 29))) + list(range(max(0, M - 40), M)))))
    Ad = A[rows].view(F8).double() * sa.double().t()[rows].repeat_interleave(128, 1)[:, :K]
    Wd = W.view(F8).double() * sw.double().t().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    want, mag = Ad @ Wd.t(), Ad.abs() @ Wd.abs().t()
    if b is not None:
        want = want + b.double()
    # operands that span the whole format: a matrix instruction's sum of 128 products keeps a limited number of bits below the largest (2e-4 of the
    # magnitudes covers what the one-scale product shows on such operands; a dropped or doubled block would be 1/nb of them); then one rounding of the result
    tol = 2e-4 * mag + (want.abs() + 2e-4 * mag) * torch.finfo(out).eps / 2 + 2.0 ** -24
    far = (C.cpu()[rows].double() - want).abs() - tol
    assert (far <= 0).all(), float((far / mag).max())


def test_quantised_product_keeps_columns_apart():
    # a few columns 100 times as large: with one scale per row they would cost the others about seven bits; here only their blocks.  The definition's own
    # error (half an E4M3 step of each operand, 2^-4 relative and at least 2^-10 of the scale) bounds what comes out
    g = torch.Generator().manual_seed(3)
    M, N, K = 96, 200, 1000
    x = torch.randn(M, K, generator=g)
    x[:, 7] *= 100.0
    w = torch.randn(N, K, generator=g)
    (aq, sa), (wq, sw) = binding.op_quantize_blocks(x.cuda(), 1), binding.op_quantize_blocks(w.cuda(), 128)
    C = binding.op_linear_fp8_block(aq, sa, wq, sw, out_dtype=torch.float16).cpu().double()
    ax, aw = x.abs().double(), w.abs().double()
    ea = torch.maximum(ax * 2.0 ** -4, sa.cpu().double().t().repeat_interleave(128, 1)[:, :K] * 2.0 ** -10)
    ew = torch.maximum(aw * 2.0 ** -4, sw.cpu().double().t().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K] * 2.0 ** -10)
    bound = (ax + ea) @ ew.t() + ea @ aw.t()
    want = x.double() @ w.double().t()
    assert ((C - want).abs() <= bound * 1.001 + want.abs() * 2.0 ** -10).all()


def test_product_writes_nothing_outside():
    for M, N, K in [(5, 50, 77), (70, 77, 130), (300, 2100, 256), (4100, 2060, 256)]:
        gc = Guarded(M * N * 2)
        A, W = torch.full((M, K), 0x38, dtype=torch.uint8, device="cuda"), torch.full((N, K), 0x38, dtype=torch.uint8, device="cuda")   # ones
        nb = -(-K // 128)
        binding.op_linear_fp8_block(A, torch.ones(nb, M, device="cuda"), W, torch.ones(nb, -(-N // 128), device="cuda"), out=gc.typed(torch.bfloat16, (M, N)))
        torch.cuda.synchronize()
        assert gc.intact()
        assert (gc.typed(torch.bfloat16, (M, N)) == float(K)).all()   # K < 2^8 or K = 256: exact in bf16


@pytest.mark.parametrize("M,N", [(70, 300), (9, 300), (1100, 4100), (4100, 3100)])
def test_captured_product_and_quantiser(M, N):
    x, w = torch.randn(M, 640, device="cuda").bfloat16(), torch.randn(N, 640, device="cuda").bfloat16()
    wq, sw = binding.op_quantize_blocks(w, 128)

    def step():
        q, s = binding.op_quantize_blocks(x, 1)
        return binding.op_linear_fp8_block(q, s, wq, sw)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(4):
        x.copy_(torch.randn(M, 640, generator=torch.Generator().manual_seed(seed)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step())
        torch.cuda.synchronize()


def test_results_repeat_to_the_bit():
    x = torch.randn(700, 1500, device="cuda")
    wq, sw = binding.op_quantize_blocks(torch.randn(900, 1500, device="cuda"), 128)
    runs = []
    for _ in range(2):
        q, s = binding.op_quantize_blocks(x, 1)
        runs.append((q, s, binding.op_linear_fp8_block(q, s, wq, sw, out_dtype=torch.float16)))
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    np.testing.assert_array_equal(runs[0][2].cpu().numpy(), runs[1][2].cpu().numpy())


def test_rows_of_many_millions_of_values():
    M, N, K = 70, 3, 1 << 24
    A, W = torch.zeros(M, K, dtype=torch.uint8, device="cuda"), torch.zeros(N, K, dtype=torch.uint8, device="cuda")
    A[:, -300:] = 0x38                                          # 1.0
    A[66, 5] = 0x40                                             # 2.0
    W[1, :] = 0x38
    sa = torch.ones(K // 128, M, device="cuda")
    sa[-1] = torch.arange(M, device="cuda").float()
    out = binding.op_linear_fp8_block(A, sa, W, torch.ones(K // 128, 1, device="cuda"), out_dtype=torch.float16).float().cpu()
    want = torch.zeros(M, N)
    want[:, 1] = 172 + 128 * torch.arange(M).float()
    want[66, 1] += 2
    assert torch.equal(out, want.half().float())


@pytest.mark.parametrize("M,N,K", [(70, 300, 640), (1100, 4104, 256), (4100, 3104, 256), (5, 40, 256)])
def test_results_at_an_odd_place(M, N, K):
    x, w = torch.randn(M, K, device="cuda").bfloat16(), torch.randn(N, K, device="cuda").bfloat16()
    operands = (*binding.op_quantize_blocks(x), *binding.op_quantize_blocks(w, 128))
    want = binding.op_linear_fp8_block(*operands)
    room = torch.zeros(M * N + 8, device="cuda", dtype=torch.bfloat16)
    got = binding.op_linear_fp8_block(*operands, out=room[3:3 + M * N].view(M, N))
    assert torch.equal(got, want) and not room[:3].any() and not room[3 + M * N:].any()


@pytest.mark.parametrize("block_rows", [1, 128])
def test_large_quantised_outputs(block_rows):
    # beyond the size from which results pass the caches: the same as in parts
    x = torch.randn(2050, 4168, device="cuda").bfloat16()
    q, scale = binding.op_quantize_blocks(x, block_rows)
    for a, b in ((0, 1024), (1024, 2050)):
        qp, sp = binding.op_quantize_blocks(x[a:b], block_rows)
        assert torch.equal(q[a:b], qp) and torch.equal(scale[:, a // block_rows:-(-b // block_rows)], sp)
