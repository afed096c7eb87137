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


@pytest.mark.parametrize("new", [1, 200])
def test_work_counted_for_attention(profile, new):
    # the timing counts the keys that a window leaves, and without one (the lengths are the device's) nothing: never the table, which is as long as a server's longest context
    H, H_kv, dh, page, pages = 8, 2, 64, 16, 4096
    q, k, v = torch.zeros(new, H, dh, device="cuda"), torch.zeros(20, H_kv, page, dh, device="cuda"), torch.zeros(20, H_kv, dh, page, device="cuda")
    table = torch.zeros(1, pages, dtype=torch.int32, device="cuda")
    args = (q, k, v, table, torch.tensor([0, new], dtype=torch.int32, device="cuda"), torch.tensor([300], dtype=torch.int32, device="cuda"))
    binding.op_paged_attention(*args, window=30, sinks=4)
    got = profile()["paged_attention"]
    assert got["launches"] == 1 and got["flops"] == 4.0 * new * (30 + 4) * H * dh
    assert got["bytes"] == 4.0 * (2 * (30 + 4 + new - 1) * H_kv * dh + 2 * new * H * dh)
    binding.op_paged_attention(*args)
    got = profile()["paged_attention"]
    assert got["launches"] == 1 and got["flops"] == 0 and got["bytes"] == 0
