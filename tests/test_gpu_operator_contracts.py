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
