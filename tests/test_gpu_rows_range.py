"""The operators on rows of logits at the ends of their range: large magnitudes, small temperatures, tails that are
nearly nothing, rows without a teacher.  Statements and error bounds are those of rows_ref.py."""
import math
import types

import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding
import rows_ref as ref
from test_gpu_rows import check_distill, check_grad, check_logprobs, make, teacher_for

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NINF = float("-inf")
DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
# rows of one CTA, rows shared by a cluster, rows that are read twice
LENGTHS = pytest.mark.parametrize("V", [1000, 40001, 500_003])


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    c.close()


def factors(rows, g):
    return torch.randn(rows, generator=g, device=DEV), torch.randn(rows, generator=g, device=DEV)


FILLS = [-1e9, -1.4e9, -1.6e9, -1e10, -1e12, -1e20, -1e30, 1e10, 1e30]


def large_rows(V, dtype):
    """One row of each fill, then each as the one entry among ordinary ones, then each among its double."""
    x, g = make(3 * len(FILLS), V, dtype)
    n = len(FILLS)
    for r, value in enumerate(FILLS):
        x[r] = value
        x[n + r, V // 3] = value
        x[2 * n + r] = 2 * value
        x[2 * n + r, V // 5::7] = value
    return x, g


@DTYPES
@LENGTHS
@pytest.mark.parametrize("T", [1.0, 0.37])
def test_statistics_of_large_logits(ctx, dtype, V, T):
    x, g = large_rows(V, dtype)
    tok = torch.full((x.shape[0],), V // 3, dtype=torch.int32, device=DEV)
    check_logprobs(ctx, x, tok, 5, T)
    check_logprobs(ctx, x, tok + 1, 0, T)
    for tail in (binding.TAIL_RENORM, binding.TAIL_BUCKET):
        ids = torch.randint(0, V, (x.shape[0], 6), generator=g, device=DEV, dtype=torch.int32)
        ids[::2, 1] = V // 3
        v = torch.log_softmax(torch.randn(ids.shape, generator=g, device=DEV), 1) - 0.5
        check_distill(ctx, x, ids, v, tail, T, None, grad=False)


@DTYPES
@LENGTHS
@pytest.mark.parametrize("T", [1.0, 0.37])
def test_gradients_at_large_logits(ctx, dtype, V, T):
    x, g = large_rows(V, dtype)
    rows = x.shape[0]
    tok = torch.full((rows,), V // 3, dtype=torch.int32, device=DEV)
    g_lp, g_h = factors(rows, g)
    for at in (tok, tok + 1):
        check_grad(ctx, x, at, g_lp, g_h, T)
        check_grad(ctx, x, at, g_lp, None, T)
    ids = torch.randint(0, V, (rows, 6), generator=g, device=DEV, dtype=torch.int32)
    ids[::2, 1] = V // 3
    v = torch.log_softmax(torch.randn(ids.shape, generator=g, device=DEV), 1) - 0.5
    w = torch.rand(rows, generator=g, device=DEV) + 0.1
    for tail in (binding.TAIL_RENORM, binding.TAIL_BUCKET):
        check_distill(ctx, x, ids, v, tail, T, w)


SMALL = pytest.mark.parametrize("exponent", [-26, -28, -30, -40, -66, -96])   # powers of two: 1 / T is exact


@DTYPES
@LENGTHS
@SMALL
def test_statistics_at_small_temperatures(ctx, dtype, V, exponent):
    """Ordinary logits are then a certain token, or equal ones."""
    T = 2.0 ** exponent
    x, g = make(4, V, dtype)
    tok = torch.tensor([0, V - 1, -1, 0], dtype=torch.int32, device=DEV)
    tok[3] = x[3].argmax()
    check_logprobs(ctx, x, tok, 5, T)
    ids, v = teacher_for(x, 8, g, T, pad=False)
    for tail in (binding.TAIL_RENORM, binding.TAIL_BUCKET):
        check_distill(ctx, x, ids, v, tail, T, None, grad=False)


@DTYPES
@LENGTHS
@SMALL
def test_gradients_at_small_temperatures(ctx, dtype, V, exponent):
    T = 2.0 ** exponent
    x, g = make(4, V, dtype)
    tok = torch.tensor([0, V - 1, -1, 0], dtype=torch.int32, device=DEV)
    tok[3] = x[3].argmax()
    g_lp, g_h = factors(4, g)
    check_grad(ctx, x, tok, g_lp, g_h, T)
    ids, v = teacher_for(x, 8, g, T, pad=False)
    for tail in (binding.TAIL_RENORM, binding.TAIL_BUCKET):
        check_distill(ctx, x, ids, v, tail, T)


def confident_rows(V, dtype, gap, at, T, masked):
    """The teacher's two tokens certain, everything else `gap` nats below them."""
    x = torch.full((3, V), -gap * T, device=DEV)
    if masked:
        x[:, 1::3] = NINF
    x[:, at] = 0.0
    x[:, at + 1] = -0.5 * T
    x = x.to(dtype)
    ids = torch.tensor([[at, at + 1]] * 3, dtype=torch.int32, device=DEV)
    v = torch.log(torch.full((3, 2), 0.25, device=DEV))
    return x, ids, v


@DTYPES
@LENGTHS
@pytest.mark.parametrize("T", [1.0, 0.1])
@pytest.mark.parametrize("masked", [False, True], ids=["all", "masked"])
def test_bucket_against_a_tail_that_is_nearly_nothing(ctx, dtype, V, T, masked):
    """A tail of 2^-126 of the row's mass and more is matched, however small its entries are; a smaller one counts
    as nothing: an infinite loss, and no share of the gradient.  No masked entry gets a NaN."""
    w = torch.tensor([1.0, 100.0, 1e-3], device=DEV)
    seen = set()
    for gap in (30.0, 45.0, 70.0, 80.0, 85.0, 86.5, 88.0, 90.0, 92.0, 95.0, 97.5, 99.0, 103.0, 110.0):
        for at in (3, V - 40):
            x, ids, v = confident_rows(V, dtype, gap, at, T, masked)
            _, _, _, p, _ = ref.stats(x.double(), T)
            pt = float(p[0, :at].sum() + p[0, at + 2:].sum())
            assert not 0.98 < pt * 2.0 ** 126 < 1.02
            there = pt > 2.0 ** -126
            seen.add(there)
            if there:
                check_distill(ctx, x, ids, v, binding.TAIL_BUCKET, T, w)
                check_distill(ctx, x, ids, v, binding.TAIL_BUCKET, T, w, grad=False)
                continue
            both = ctx.distill(x, ids, v, tail=binding.TAIL_BUCKET, temperature=T, weight=w, grad=True)
            only = ctx.distill(x, ids, v, tail=binding.TAIL_BUCKET, temperature=T, weight=w)
            assert (both["loss"] == math.inf).all() and (only["loss"] == math.inf).all()
            assert torch.isfinite(both["grad"]).all()
            want = p.clone()                                   # M = 1: the pull of the whole mass, less the teacher's q
            want[:, at:at + 2] -= 0.25
            want = want * w.double()[:, None] / T
            tol = 4 * ref.delta(V) * w.double()[:, None] / T + want.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else 0.0) + 1e-38
            ref.same(both["grad"], want, tol)
            assert (both["grad"][:, torch.arange(V, device=DEV) % 97 == 60].abs() <= 1e-30).all()
    assert seen == {False, True}


@DTYPES
@LENGTHS
def test_bucket_at_a_weight_that_overflows_the_share(ctx, dtype, V):
    """weight / T q_t / p_t beyond fp32, every gradient within it; masked entries get 0."""
    x, ids, v = confident_rows(V, dtype, 40.0, 3, 1.0, True)
    check_distill(ctx, x, ids, v, binding.TAIL_BUCKET, 1.0, torch.tensor([1e24, 1e28, 1.0], device=DEV))


@DTYPES
@LENGTHS
@pytest.mark.parametrize("tail", [0, 1], ids=["renorm", "bucket"])
def test_rows_without_a_teacher_count_for_nothing(ctx, dtype, V, tail):
    """Whatever they hold: a padded row's logits may be anything."""
    x, g = make(6, V, dtype)
    x[1] = float("nan")
    x[2, 7] = float("inf")
    x[3] = NINF
    ids, v = teacher_for(x, 5, g, 1.0, pad=False)
    ids[:4] = -1
    ids[2] = V
    v[1] = float("nan")
    w = torch.rand(6, generator=g, device=DEV) + 0.5
    for weight in (None, w):
        both = ctx.distill(x, ids, v, tail=tail, weight=weight, grad=True)
        assert (both["loss"][:4] == 0).all() and (both["grad"][:4] == 0).all()
        assert (ctx.distill(x, ids, v, tail=tail, weight=weight)["loss"][:4] == 0).all()
        check_distill(ctx, x[4:], ids[4:], v[4:], tail, 1.0, None if weight is None else weight[4:])
    y = x.clone()
    assert torch.equal(ctx.distill(y, ids, v, tail=tail, weight=w, grad=True, out=y)["grad"], both["grad"])


@LENGTHS
def test_loss_of_a_teacher_whose_tokens_are_masked_by_the_lowest_value(ctx, V):
    """Finite where the definition is: the weights of log p = -3.4e38 add up to the teacher's mass, not to a rounding
    error above it."""
    rows, k = 40, 33
    x, g = make(rows, V, torch.float32)
    ids = torch.stack([torch.randperm(V, generator=g, device=DEV)[:k] for _ in range(rows)]).to(torch.int32)
    x.scatter_(1, ids.long(), torch.finfo(torch.float32).min)
    v = torch.log_softmax(torch.randn((rows, k), generator=g, device=DEV) * 3, 1)
    want = ref.distill(x, ids, v, False, 1.0)[0].float().double()
    assert torch.isfinite(want).all()
    for grad in (False, True):
        got = ctx.distill(x, ids, v, tail=binding.TAIL_RENORM, grad=grad)["loss"]
        ref.same(got, want, 4 * ref.U * want.abs())


@DTYPES
def test_many_rows_with_and_without_a_teacher(ctx, dtype):
    """Rows of every kind one after the other in a cluster's walk: nothing of one reaches the next."""
    rows, V = 1500, 9001
    x, g = make(rows, V, dtype)
    ids, v = teacher_for(x, 7, g, 1.0)
    ids[::3] = -1
    x[::6] = float("nan")
    x[4::9] = -1e10
    x[7::9] = -90.0
    for r in range(7, rows, 9):
        ids[r] = torch.arange(7, device=DEV)
    x[7::9, :7] = 0.0
    v[7::9] = math.log(0.1)
    have = torch.ones(rows, dtype=torch.bool, device=DEV)
    have[::3] = False
    for tail in (binding.TAIL_RENORM, binding.TAIL_BUCKET):
        got = ctx.distill(x, ids, v, tail=tail, grad=True)
        assert (got["loss"][::3] == 0).all() and (got["grad"][::3] == 0).all()
        of_have = types.SimpleNamespace(distill=lambda *_, **__: {key: t[have] for key, t in got.items()})
        check_distill(of_have, x[have], ids[have], v[have], tail, 1.0)
    assert ctx.device_error() == 0
