"""dropmatch_score: hidden rows against the head, compared with the 64-bit statement on logits that are
computed in 64 bits.  Inputs lie on a grid on which every fp32 sum of products is exact, so that the
order of the alternatives, equal logits included, does not depend on the order of a summation."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding
import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def grid(shape, std, unit, dtype, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(shape, generator=g, device=DEV).mul_(std / unit).round_().clamp_(-255, 255)
    return (x * unit).to(dtype)


def inputs(rows, V, d, dtype, seed=1):
    if dtype == torch.float32:
        return grid((V, d), d ** -0.5, 2.0 ** -10, dtype, seed), grid((rows, d), d ** -0.5, 2.0 ** -10, dtype, seed + 1)
    return grid((V, d), 0.02, 2.0 ** -11, dtype, seed), grid((rows, d), 1.0, 2.0 ** -5, dtype, seed + 1)


def check(got, W, H, tokens, n_top, T, exact_order=True):
    x = H.double() @ W.double().T
    want = ref.logprobs(x, tokens, n_top, T)
    V, d = W.shape
    tol = ref.delta(V)     # on the grid the logits themselves are exact
    ref.same(got["lse"], want["lse"], tol + 4 * ref.U * want["lse"].abs())
    ref.same(got["entropy"], want["entropy"], tol * (1 + 2 * want["entropy"]))
    if tokens is not None:
        ref.same(got["logprob"], want["logprob"], tol + 4 * ref.U * want["logprob"].abs())
    if n_top:
        assert torch.equal(got["top_ids"], want["top_ids"])
        ref.same(got["top_logprob"], want["top_logprob"], tol + 4 * ref.U * want["top_logprob"].abs())


CASES = [  # rows, V, d, dtype, n_top
    (4, 4096, 256, torch.float32, 5), (1, 1, 8, torch.float32, 1), (9, 37, 64, torch.bfloat16, 37),
    (3, 999, 136, torch.bfloat16, 7), (1, 3000, 512, torch.bfloat16, 0), (1, 3000, 512, torch.bfloat16, 128),
    (17, 20000, 64, torch.bfloat16, 3), (61, 60000, 128, torch.bfloat16, 20), (257, 20000, 64, torch.bfloat16, 9),
    (600, 9001, 128, torch.bfloat16, 4), (1100, 5000, 64, torch.bfloat16, 1), (1, 128256, 4096, torch.bfloat16, 5),
    (40, 128256, 4096, torch.bfloat16, 0), (40, 151936, 1024, torch.bfloat16, 32), (300, 128256, 512, torch.bfloat16, 64),
]


@pytest.mark.parametrize("rows,V,d,dtype,n_top", CASES)
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_score(rows, V, d, dtype, n_top, T):
    W, H = inputs(rows, V, d, dtype)
    tok = torch.randint(0, V, (rows,), device=DEV, dtype=torch.int32)
    tok[::4] = -1
    ctx = pk.Context(0)
    try:
        ctx.set_head(W, max_rows=rows)
        ctx.enable_score(rows, n_top)
        got = ctx.score(H, tok, n_top=n_top, temperature=T)
        assert ctx.device_error() == 0
        check(got, W, H, tok, n_top, T)
        again = ctx.score(H, tok, n_top=n_top, temperature=T)
        for key in got:
            assert torch.equal(got[key], again[key]), key     # reproducible bit for bit
        few = ctx.score(H[:1], None)                          # fewer rows than reserved, no tokens, no alternatives
        check(few, W, H[:1], None, 0, 1.0)
        assert "logprob" not in few and "top_ids" not in few
    finally:
        ctx.close()


def test_score_ties_and_rows_behind_the_call():
    """A head of equal rows: every alternative ties, the lowest ids win; outputs of rows that are not
    part of the call are left alone."""
    V, d = 5000, 128
    W = torch.ones((V, d), dtype=torch.bfloat16, device=DEV) / 64
    W[4000] += 1.0 / 64
    H = torch.ones((3, d), dtype=torch.bfloat16, device=DEV)
    ctx = pk.Context(0)
    try:
        ctx.set_head(W, max_rows=64)
        ctx.enable_score(64, 6)
        got = ctx.score(H, None, n_top=6)
        assert got["top_ids"].tolist() == [[4000, 0, 1, 2, 3, 4]] * 3
        ids = torch.full((5, 6), -7, dtype=torch.int32, device=DEV)
        lp = torch.full((5, 6), 7.0, device=DEV)
        lse = torch.full((5,), 7.0, device=DEV)
        L = binding.lib()
        assert L.dropmatch_score(ctx._h, H.data_ptr(), None, 3, 6, 1.0, None, lse.data_ptr(), None, ids.data_ptr(),
                                 lp.data_ptr(), binding._stream(ctx.device)) == binding.OK
        assert torch.equal(ids[:3], got["top_ids"]) and (ids[3:] == -7).all() and (lp[3:] == 7.0).all() and (lse[3:] == 7.0).all()
        check(dict(got), W, H, None, 6, 1.0)
    finally:
        ctx.close()


def test_score_next_to_verify_and_in_a_graph():
    """Score, verify and score again on one context: neither disturbs the other; captured and replayed."""
    W, H = inputs(16, 30000, 256, torch.bfloat16)
    tok = torch.randint(0, 30000, (16,), device=DEV, dtype=torch.int32)
    draft = tok.view(4, 4)
    ctx = pk.Context(0)
    try:
        ctx.set_head(W, max_rows=128)
        before = ctx.verify_batched(H.view(4, 4, 256), draft, 8, 0.1, 11)
        ctx.enable_score(16, 5)
        a = ctx.score(H.view(4, 4, 256), draft, n_top=5)
        after = ctx.verify_batched(H.view(4, 4, 256), draft, 8, 0.1, 11)
        for key in before:
            assert torch.equal(before[key], after[key])
        assert a["top_ids"].shape == (4, 4, 5)
        plain = ctx.verify_batched_next(H.view(4, 4, 256), draft, 1, 0.1, 11)["plain"]
        assert torch.equal(a["top_ids"][..., 0], plain)        # the best alternative is the plain greedy token
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b = ctx.score(H.view(4, 4, 256), draft, n_top=5)
        for t in b.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for key in a:
            assert torch.equal(a[key], b[key]), key
        assert ctx.device_error() == 0
    finally:
        ctx.close()


def test_score_refusals_and_the_wait_limit():
    W, H = inputs(8, 30000, 256, torch.bfloat16)
    ctx = pk.Context(0)

    def refused(status, fn, *a, **k):
        with pytest.raises(pk.DropMatchError) as e:
            fn(*a, **k)
        assert e.value.status == status

    try:
        refused(binding.ENOHEAD, ctx.enable_score, 8, 1)
        ctx.set_head(W, max_rows=16)
        refused(binding.EWORKSPACE, ctx.score, H)
        refused(binding.EINVAL, ctx.enable_score, 17, 1)
        refused(binding.EINVAL, ctx.enable_score, 8, 129)
        refused(binding.EINVAL, ctx.enable_score, 0, 1)
        ctx.enable_score(4, 3)
        refused(binding.EWORKSPACE, ctx.score, H)
        refused(binding.EWORKSPACE, ctx.score, H[:4], None, n_top=4)
        refused(binding.EINVAL, ctx.score, H[:4], None, n_top=129)
        refused(binding.EINVAL, ctx.score, H[:4], None, temperature=0.0)
        for bad in (H.float(), H[0], H[:, :128].contiguous(), H.cpu()):
            with pytest.raises(TypeError):
                ctx.score(bad)
        assert ctx.score(H[:0], None, n_top=2)["top_ids"].shape == (0, 2)
        ctx.set_vocab_offset(8)
        refused(binding.EUNSUPPORTED, ctx.score, H[:4])
        ctx.set_vocab_offset(0)
        good = ctx.score(H[:4], None, n_top=2)
        ctx.debug_set_wait_limit(1)               # the first wait that is not satisfied at once runs out
        bad = ctx.score(H[:4], None, n_top=2)
        torch.cuda.synchronize()
        if ctx.device_error() != 0:
            assert torch.isnan(bad["lse"]).all() and torch.isnan(bad["entropy"]).all() and (bad["top_ids"] == -1).all()
        ctx.debug_set_wait_limit(0)
        again = ctx.score(H[:4], None, n_top=2)
        for key in good:
            assert torch.equal(good[key], again[key])
    finally:
        ctx.close()


def test_score_on_the_cuda_cores_and_without_early_start():
    """The kernel families agree on one head; switching programmatic stream serialization off changes nothing."""
    W, H = inputs(70, 20011, 192, torch.bfloat16)
    tok = torch.randint(0, 20011, (70,), device=DEV, dtype=torch.int32)
    ctx = pk.Context(0)
    try:
        ctx.set_head(W, max_rows=70)
        ctx.enable_score(70, 6)
        a = ctx.score(H, tok, n_top=6)
        assert ctx.last_impl() == binding.IMPL_TCGEN05 and ctx.last_launches() == 2
        ctx.set_pdl(False)
        b = ctx.score(H, tok, n_top=6)
        for key in a:
            assert torch.equal(a[key], b[key]), key
        ctx.set_impl(binding.IMPL_SIMT)
        c = ctx.score(H, tok, n_top=6)
        assert ctx.last_impl() == binding.IMPL_SIMT
        check(c, W, H, tok, 6, 1.0)
        ctx.set_impl(binding.IMPL_AUTO)
        ctx.enable_score(70, 0)                 # no alternatives: no room for the CUDA-core kernel's logits
        few = ctx.score(H, tok)
        for key in few:
            assert torch.equal(a[key], few[key]), key
        ctx.set_impl(binding.IMPL_SIMT)
        with pytest.raises(pk.DropMatchError) as e:
            ctx.score(H, tok)
        assert e.value.status == binding.EWORKSPACE
        ctx.enable_score(70, 0)                 # ... unless it is the family in force
        check(ctx.score(H, tok), W, H, tok, 0, 1.0)
    finally:
        ctx.close()


def test_score_workspace_is_counted_and_replaced():
    W, H = inputs(300, 9000, 64, torch.bfloat16)
    ctx = pk.Context(0)
    try:
        ctx.set_head(W, max_rows=300)
        base = ctx.workspace_bytes()
        ctx.enable_score(300, 8)
        one = ctx.workspace_bytes()
        assert one > base
        ctx.enable_score(300, 8)
        assert ctx.workspace_bytes() == one
        ctx.enable_score(10, 0)
        assert base < ctx.workspace_bytes() < one
        check(ctx.score(H[:10], None), W, H[:10], None, 0, 1.0)
        ctx.set_head(W, max_rows=300)           # drops it
        with pytest.raises(pk.DropMatchError) as e:
            ctx.score(H[:1])
        assert e.value.status == binding.EWORKSPACE
    finally:
        ctx.close()


@pytest.mark.parametrize("V", [47253, 77745, 103093, 128256])
def test_alternatives_after_calls_of_other_sizes(V):
    """Whatever earlier calls have left in the workspace: both cuts of the vocabulary, last tiles shorter than
    the others, fewer rows than before."""
    W, H = inputs(300, V, 64, torch.bfloat16)
    big = H * 16
    ctx = pk.Context(0)
    try:
        ctx.set_head(W, max_rows=300)
        ctx.enable_score(300, 40)
        for rows in (300, 27, 130, 128, 1, 257):
            ctx.score(big, None, n_top=40)
            ctx.score(big[:128], None, n_top=40)
            check(ctx.score(H[:rows], None, n_top=9), W, H[:rows], None, 9, 1.0)
    finally:
        ctx.close()
