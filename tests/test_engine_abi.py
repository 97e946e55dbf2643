"""Host-side refusals of lossless verification, dropout on rows and 8-bit products that need no device."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding


def test_a_null_context_is_refused():
    L = binding.lib()
    assert L.dropmatch_verify_lossless(None, None, 0, 8, None, 0, 8, None, None, 1, 1, 1, 8, 1.0, 1.0, None, None, None, None,
                                       None, None) == binding.EINVAL
    assert L.dropmatch_dropout(None, None, 0, 8, 1, 1, 1, 8, 0.1, 1, 0, None, 8, None) == binding.EINVAL
    assert L.dropmatch_dropout_grad(None, None, 0, 8, 1, 1, 1, 8, 0.1, 1, 0, None, 8, None) == binding.EINVAL
    assert L.dropmatch_quantize_i8(None, None, 0, 16, 1, 16, None, 16, None, None) == binding.EINVAL
    assert L.dropmatch_matmul_i8(None, None, 16, None, 1, None, 16, None, 8, 16, None, 0, 8, None) == binding.EINVAL
    assert L.dropmatch_linear_i8(None, None, 0, 16, 1, None, 16, None, 8, 16, None, 16, None, None, 0, 8, None) == binding.EINVAL


def test_binding_refuses_tensors_off_the_device():
    ctx = object.__new__(pk.Context)          # the argument checks come before any library call
    ctx._h, ctx.device = None, torch.device("cuda", 0)
    x, tok = torch.zeros((2, 3, 8)), torch.zeros((2, 3), dtype=torch.int32)
    q, scale = torch.zeros((4, 16), dtype=torch.int8), torch.zeros(4)
    for call in (lambda: ctx.verify_lossless(x, tok, torch.zeros(2, 3), torch.zeros(2)),
                 lambda: ctx.verify_lossless(x[0], tok, torch.zeros(2, 3), torch.zeros(2)),
                 lambda: ctx.verify_lossless(x, tok[:, :1], torch.zeros(2, 1), torch.zeros(2)),
                 lambda: ctx.dropout(x, 4, 0.1, 1), lambda: ctx.dropout(x[0], 4, 0.1, 1),
                 lambda: ctx.dropout_grad(x[:, :, None], 0.1, 1), lambda: ctx.dropout_grad(x, 0.1, 1),
                 lambda: ctx.quantize_i8(x), lambda: ctx.matmul_i8(q, scale, q, scale), lambda: ctx.linear_i8(x, q, scale)):
        with pytest.raises(TypeError):
            call()


def test_references_agree_on_the_masks():
    """The vectorised keep flags of engine_ref.py are philox_ref.py's, row by row."""
    import engine_ref as ref
    from philox_ref import keep_bits
    import math
    flags = ref.keep_flags(2, 3, 2, 11, 0.3, 2 ** 40 + 5, seq_base=2 ** 32 - 1)
    thr = math.floor(ref.single(0.3) * 2.0 ** 32)
    for b in range(2):
        for t in range(3):
            for i in range(2):
                assert flags[b, t, i].tolist() == keep_bits(2 ** 40 + 5, 2 ** 32 - 1 + b, t, i, 11, thr).tolist()
