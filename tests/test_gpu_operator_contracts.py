"""What the operators on pages, FP8 blocks and logits promise beside their results, on the GPU: first steps without a history, an output where another buffer lies, what the
per-kernel timing counts, and large products over many blocks."""
import pytest
import torch

from paper_2602_22732_amd import binding
from test_gpu_paged_attention import Case, check, same

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


@pytest.mark.parametrize("dtype,dh,group,news,staged", [
    (torch.bfloat16, 64, 4, [16, 16], False), (torch.bfloat16, 64, 4, [32, 1], True), (torch.bfloat16, 32, 1, [64], False), (torch.bfloat16, 32, 1, [65], True), (torch.bfloat16, 128, 16, [1, 1], False),
    (torch.bfloat16, 128, 17, [1], True), (torch.bfloat16, 128, 4, [1] * 3 + [40], True), (torch.bfloat16, 16, 4, [100], False), (torch.float32, 128, 4, [100], False),
])
def test_when_weights_are_rounded_once(profile, dtype, dh, group, news, staged):
    # The documented rule: bf16, 32 columns or more, and more than 64 rows (tokens times heads of a group) of a sequence on average, with 128 columns more than 16.
    H_kv, page, B, n = 2, 16, len(news), 128
    H, N, g = H_kv * group, sum(news), torch.Generator().manual_seed(dh + group)
    q, k, v = (torch.randn(*shape, generator=g).to(dtype) for shape in ((N, H, dh), (8 * B, H_kv, page, dh), (8 * B, H_kv, dh, page)))
    start = torch.tensor([0] + news).cumsum(0).to(torch.int32)
    out = binding.op_paged_attention(q.cuda(), k.cuda(), v.cuda(), torch.arange(8 * B, dtype=torch.int32, device="cuda").view(B, 8), start.cuda(), torch.full((B,), n, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert set(profile()) == {"paged_attention_staged" if staged else "paged_attention"}
    half = torch.finfo(dtype).eps / 2
    for b, m in enumerate(news):
        keys = k[8 * b:8 * b + 8].double().transpose(1, 2).flatten(0, 1).repeat_interleave(group, 1)                       # [n, H, dh]
        values = v[8 * b:8 * b + 8].double().permute(0, 3, 1, 2).flatten(0, 1).repeat_interleave(group, 1)
        for i in range(m):
            row, p = int(start[b]) + i, n - m + i
            x = (q[row].double()[None] * keys[:p + 1]).sum(-1) * dh ** -0.5
            w = torch.softmax(x, 0)[..., None]
            want, mag = (w * values[:p + 1]).sum(0), (w * values[:p + 1].abs()).sum(0)
            # float32: scores of dh terms and their exponentials, sums of p + 1; the result's rounding; a weight as one bf16 number is off by 2^-8, as two by 2^-16 of itself
            score = (dh + 8) * 2.0 ** -24 * (q[row].double().abs()[None] * keys[:p + 1].abs()).sum(-1).amax(0)[:, None] * dh ** -0.5
            tol = (2 * score + (p + 17) * 2.0 ** -24 + (0 if dtype == torch.float32 else 2.0 ** -8 if staged else 2.0 ** -16)) * mag + half * want.abs() * (1 + 2.0 ** -7)
            assert ((out[row].cpu().double() - want).abs() <= tol).all()


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


@pytest.mark.parametrize("dtype,m", [(torch.float32, 1), (torch.float32, 40), (torch.bfloat16, 1), (torch.bfloat16, 12), (torch.bfloat16, 40)])
def test_scores_of_minus_infinity(dtype, m):
    # such keys count as not seen; a row that sees no others is zero
    H, H_kv, dh, page, n = 4, 2, 64, 16, 90
    g = torch.Generator().manual_seed(m)
    q, k, v = (torch.randn(*shape, generator=g).to(dtype) for shape in ((m, H, dh), (6, H_kv, page, dh), (6, H_kv, dh, page)))
    q[..., 5] = 1.0
    table, start, lens = torch.arange(6, dtype=torch.int32).view(1, 6).cuda(), torch.tensor([0, m], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
    gone = torch.rand(96, generator=g) < 0.5
    for every in (False, True):
        dead = gone | every
        kk = k.transpose(1, 2).reshape(96, H_kv, dh).clone()
        kk[dead, :, 5] = -float("inf")
        out = binding.op_paged_attention(q.cuda(), kk.view(6, page, H_kv, dh).transpose(1, 2).contiguous().cuda(), v.cuda(), table, start, lens).cpu().double()
        if every:
            assert not out.any()
            continue
        vv = v.permute(0, 3, 1, 2).reshape(96, H_kv, dh).double().repeat_interleave(2, 1)
        for i in range(m):
            seen = ~dead & (torch.arange(96) <= n - m + i)
            x = (q[i].double()[None] * kk[seen].double().repeat_interleave(2, 1)).sum(-1) * dh ** -0.5
            w = torch.softmax(x, 0)[..., None]
            # scores of 64 terms of magnitude 3 at most on average, 1e-4 of them for float32 sums; bf16: a weight's and the result's rounding
            tol = 1e-4 + (2.0 ** -7 if dtype == torch.bfloat16 else 0) * (w * vv[seen].abs()).sum(0)
            assert ((out[i] - (w * vv[seen]).sum(0)).abs() <= tol).all()


@pytest.mark.parametrize("dtype,new", [("f32", [1, 1, 1]), ("f32", [3, 40, 1]), ("bf16", [1, 1, 1]), ("bf16", [3, 40, 1]), ("bf16", [100, 90, 120])])
def test_padded_tables(dtype, new):
    # entries behind a sequence's length may name any page, such as one that takes another sequence's new tokens in the same call
    for page in (16, 64):
        c = Case(dtype, 64, 4, 2, page, new=new, lens=[300, 130, 121], seed=31)
        busy = int(c.table[0, 299 // page])
        for b, n in enumerate(c.lens):
            c.table[b, -(-n // page):] = busy
        check(c)
        check(c, window=70, sinks=3)


@pytest.mark.parametrize("dtype,new", [("f32", [2, 1]), ("bf16", [2, 1]), ("bf16", [90, 80])])
def test_lengths_beyond_the_table(dtype, new):
    # counted as the table's: the new tokens are the last of the positions that it has
    c = Case(dtype, 64, 4, 2, 16, new=new, lens=[320, 100], seed=32)
    want, tol = c.expected()
    args = [t.cuda() for t in (c.q, c.k, c.v, c.table, torch.tensor(c.starts, dtype=torch.int32))]
    out = binding.op_paged_attention(*args, torch.tensor([2 ** 31 - 1, 100], dtype=torch.int32).cuda(), k_new=c.k_new.cuda(), v_new=c.v_new.cuda())
    assert ((out.cpu().double() - want).abs() <= tol).all()
    k, v = c.after()
    assert same(args[1].cpu(), k) and same(args[2].cpu(), v)
