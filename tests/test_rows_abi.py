"""Host-side refusals of the operators on rows of logits that need no device."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding


def test_row_operators_refuse_a_null_context():
    L = binding.lib()
    assert L.dm_enable_score(None, 1, 1) == binding.EINVAL
    assert L.dropmatch_score(None, None, None, 1, 0, 1.0, None, None, None, None, None, None) == binding.EINVAL
    assert L.dropmatch_logprobs(None, None, 0, 8, 1, 8, None, 0, 1.0, None, None, None, None, None, None) == binding.EINVAL
    assert L.dropmatch_logprobs_grad(None, None, 0, 8, 1, 8, None, 1.0, None, None, None, 8, None) == binding.EINVAL
    assert L.dropmatch_distill(None, None, 0, 8, 1, 8, None, None, 1, 0, 1.0, None, None, None, 8, None) == binding.EINVAL


def test_binding_refuses_tensors_off_the_device():
    ctx = object.__new__(pk.Context)          # the argument checks come before any library call
    ctx._h, ctx.device, ctx.dtype, ctx.d = None, torch.device("cuda", 0), binding.BF16, 64
    x = torch.zeros((2, 8))
    with pytest.raises(TypeError):
        ctx.logprobs(x)
    with pytest.raises(TypeError):
        ctx.logprobs_grad(x, None, torch.zeros(2))
    with pytest.raises(TypeError):
        ctx.distill(x, torch.zeros((2, 1), dtype=torch.int32), torch.zeros((2, 1)))
    with pytest.raises(TypeError):
        ctx.score(torch.zeros((2, 64), dtype=torch.bfloat16))
