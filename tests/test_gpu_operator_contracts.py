"""What the operators on pages, FP8 blocks and logits promise beside their results, on the GPU: first steps without a history, an output where another buffer lies, what the
per-kernel timing counts, and large products over many blocks."""
import pytest
import torch

from paper_2602_22732_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_a_first_step_has_no_history(dtype):
    g = torch.Generator().manual_seed(1)
    logits, bias = torch.randn(5, 300, generator=g).to(dtype).cuda(), torch.randn(1, 300, generator=g).cuda()
    ones = torch.ones(5, device="cuda")
    got = binding.op_adjust_logits(logits, history=torch.empty(5, 0, dtype=torch.int32, device="cuda"), history_len=torch.zeros(5, dtype=torch.int32, device="cuda"), repetition=2 * ones, presence=ones,
                                   frequency=ones, bias=bias)
    assert torch.equal(got, binding.op_adjust_logits(logits, bias=bias))


@pytest.fixture
def profile():
    binding.profile_enable(True)
    binding.profile_read()
    yield binding.profile_read
    binding.profile_enable(False)


@pytest.mark.parametrize("new,dtype,kind", [(1, torch.float32, "paged_attention"), (200, torch.float32, "paged_attention"), (200, torch.bfloat16, "paged_attention_staged")])
def test_work_counted_for_attention(profile, new, dtype, kind):
    # the timing counts the keys that a window leaves, and without one (the lengths are the device's) nothing: never the table, which is as long as a server's longest context
    H, H_kv, dh, page, pages = 8, 2, 64, 16, 4096
    q, k, v = (torch.zeros(*shape, device="cuda", dtype=dtype) for shape in ((new, H, dh), (20, H_kv, page, dh), (20, H_kv, dh, page)))
    table = torch.zeros(1, pages, dtype=torch.int32, device="cuda")
    args = (q, k, v, table, torch.tensor([0, new], dtype=torch.int32, device="cuda"), torch.tensor([300], dtype=torch.int32, device="cuda"))
    binding.op_paged_attention(*args, window=30, sinks=4)
    got = profile()[kind]
    assert got["launches"] == 1 and got["flops"] == 4.0 * new * (30 + 4) * H * dh
    assert got["bytes"] == dtype.itemsize * (2.0 * (30 + 4 + new - 1) * H_kv * dh + 2 * new * H * dh)
    binding.op_paged_attention(*args)
    got = profile()[kind]
    assert got["launches"] == 1 and got["flops"] == 0 and got["bytes"] == 0


def random_e4m3(g, *shape):
    b = torch.randint(0, 256, shape, generator=g, dtype=torch.uint8)
    b[(b & 0x7F) == 0x7F] = 0x3A
    return b


# Every kind of tile over many blocks of K: slots of local memory are filled anew from the third or fourth block on, and a wavefront takes the weights' scales for 64 blocks at a time.
@pytest.mark.parametrize("M,N,K,kind", [
    (4099, 3000, 1024, "256"), (4096, 3100, 1040, "256"), (4099, 3000, 8336, "256"), (4096, 3080, 8448, "256"), (4099, 2900, 16640, "256"), (1100, 4100, 8320, "128"), (1100, 4100, 8336, "128"),
    (2048, 3000, 1152, "128"), (300, 900, 8336, "64"), (517, 1000, 16400, "64"), (60, 500, 8321, "few"), (300, 900, 8321, "unaligned"), (2100, 2070, 8449, "unaligned"),
])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16])
def test_products_over_many_blocks(profile, M, N, K, kind, out):
    g = torch.Generator().manual_seed(M + N + K)
    A, W = random_e4m3(g, M, K), random_e4m3(g, N, K)
    nb, wb = -(-K // 128), -(-N // 128)
    sa = torch.exp(torch.empty(nb, M).uniform_(-3, 3, generator=g)) * 1e-3
    sw = torch.exp(torch.empty(nb, wb).uniform_(-3, 3, generator=g)) * 1e-3
    C = binding.op_linear_fp8_block(A.cuda(), sa.cuda(), W.cuda(), sw.cuda(), out_dtype=out)
    assert profile()["gemm_fp8_block_" + kind]["launches"] == 1
    rows = torch.tensor(sorted(set(list(range(0, M, max(1, M // 13))) + list(range(max(0, M - 20), M)))))
    cols = torch.tensor(sorted(set(list(range(0, N, max(1, N // 400))) + list(range(max(0, N - 40), N)))))
    Ad = A[rows].view(torch.float8_e4m3fn).double() * sa.double().t()[rows].repeat_interleave(128, 1)[:, :K]
    Wd = W[cols].view(torch.float8_e4m3fn).double() * sw.double().t()[cols // 128].repeat_interleave(128, 1)[:, :K]
    want, mag = Ad @ Wd.t(), Ad.abs() @ Wd.abs().t()
    # a matrix instruction's sum of 128 products keeps a limited number of bits below the largest (2e-4 of the magnitudes covers it), the blocks' sum adds nb steps of float32, and the
    # result is rounded once.  A block left out, or scaled as another, changes a sum of terms of both signs by about its magnitudes / (11 nb), 7e-4 of
    # them at nb = 130, and by several times that in some of the thousands of sums that are looked at.
    tol = (2e-4 + nb * 2.0 ** -24) * mag + want.abs() * torch.finfo(out).eps / 2 * (1 + 2e-4) + 2.0 ** -24
    far = (C.cpu()[rows][:, cols].double() - want).abs() - tol
    assert (far <= 0).all(), float((far / mag).max())
