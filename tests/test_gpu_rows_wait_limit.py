"""What the calls on rows of logits, and the score kernel, do when one of their waits runs out.  The limit is set
to one clock cycle: nothing hangs and nothing faults."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding
from test_gpu_rows import make, teacher_for, tokens_for
from test_gpu_score import inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ERR_WAIT_ROW = 8


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(2000, 67), (1500, 9001), (300, 128256)])
def test_a_late_answer_is_reported_and_no_row_is_lost(dtype, rows, V):
    """Rows of one CTA and of clusters; a cluster that gave up on its request takes the row all the same."""
    x, g = make(rows, V, dtype)
    tok = tokens_for(rows, V, g)
    ones = torch.ones(rows, device=DEV)
    ids, v = teacher_for(x, 5, g, 1.0)
    ctx = pk.Context(0)
    calls = [lambda: {"grad": ctx.logprobs_grad(x, tok, ones, ones)},
             lambda: ctx.distill(x, ids, v, tail=binding.TAIL_BUCKET, grad=True)]
    if rows > 1000 and V > 9000:
        calls.append(lambda: ctx.logprobs(x, tok, n_top=5))      # ... long runs of rows of two batches and more
    try:
        for call in calls:
            want = call()
            assert ctx.device_error() == 0
            ctx.debug_set_wait_limit(1)
            got = call()
            assert ctx.device_error() == ERR_WAIT_ROW             # (reads and clears the word)
            for key in want:
                assert torch.equal(got[key], want[key]), key
            ctx.debug_set_wait_limit(0)
            again = call()
            assert ctx.device_error() == 0
            for key in want:
                assert torch.equal(again[key], want[key]), key
    finally:
        ctx.close()


@pytest.mark.parametrize("rows", [4, 200])
def test_score_reports_an_abandoned_wait_in_its_outputs(rows):
    """One CTA and a pair of CTAs per slice: no output may be mistaken for a result."""
    W, H = inputs(rows, 30000, 256, torch.bfloat16)
    tok = torch.zeros((rows,), dtype=torch.int32, device=DEV)
    ctx = pk.Context(0)
    try:
        ctx.set_head(W, max_rows=rows)
        ctx.enable_score(rows, 3)
        good = ctx.score(H, tok, n_top=3)
        assert ctx.device_error() == 0 and ctx.last_impl() == binding.IMPL_TCGEN05
        ctx.debug_set_wait_limit(1)               # the epilogue looks before the first tile can be there
        bad = ctx.score(H, tok, n_top=3)
        assert ctx.device_error() != 0
        for key in ("logprob", "lse", "entropy", "top_logprob"):
            assert torch.isnan(bad[key]).all(), key
        assert (bad["top_ids"] == -1).all()
        ctx.debug_set_wait_limit(0)
        again = ctx.score(H, tok, n_top=3)
        assert ctx.device_error() == 0
        for key in good:
            assert torch.equal(good[key], again[key]), key
    finally:
        ctx.close()
