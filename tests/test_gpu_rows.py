"""The operators on rows of logits (dropmatch_logprobs, _logprobs_grad, dropmatch_distill) against
plain 64-bit statements of them (rows_ref.py, which also derives the error bounds)."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding
import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NINF = float("-inf")


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    c.close()


def make(rows, V, dtype, seed=0, ld=None, offset=0, scale=3.0):
    """logits[rows,V] with row stride ld, starting `offset` entries into their buffer."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    ld = ld or V
    buf = torch.empty(offset + rows * ld, dtype=dtype, device=DEV).fill_(77.0)
    x = buf[offset:].view(rows, ld)[:, :V]
    x.copy_(torch.randn((rows, V), generator=g, device=DEV) * scale)
    return x, g


def tokens_for(rows, V, g):
    t = torch.randint(0, V, (rows,), generator=g, device=DEV, dtype=torch.int32)
    t[::5] = -1
    if rows > 3:
        t[3] = V
    return t


def check_logprobs(ctx, x, tokens, n_top, T):
    got = ctx.logprobs(x, tokens, n_top=n_top, temperature=T)
    want = ref.logprobs(x, tokens, n_top, T)
    V = x.shape[1]
    d = ref.delta(V)
    mag = torch.nan_to_num(want["lse"].abs(), posinf=0.0, neginf=0.0)
    ref.same(got["lse"], want["lse"], d + 4 * ref.U * mag)
    ref.same(got["entropy"], want["entropy"], d * (1 + 2 * torch.nan_to_num(want["entropy"])))
    if tokens is not None:
        ref.same(got["logprob"], want["logprob"], d + 4 * ref.U * torch.nan_to_num(want["logprob"].abs(), posinf=0.0))
    if n_top:
        assert torch.equal(got["top_ids"], want["top_ids"])
        ref.same(got["top_logprob"], want["top_logprob"], d + 4 * ref.U * torch.nan_to_num(want["top_logprob"].abs(), posinf=0.0))
    return got


SHAPES = [(1, 1, 1), (3, 2, 2), (5, 7, 3), (2, 255, 128), (4, 999, 16), (1, 4097, 5), (9, 5000, 0), (700, 1030, 4),
          (3, 32003, 100), (1, 128256, 20), (2, 151936, 128), (40, 128256, 8), (1300, 300, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,n_top", SHAPES)
@pytest.mark.parametrize("T", [1.0, 0.37])
def test_logprobs(ctx, rows, V, n_top, dtype, T):
    x, g = make(rows, V, dtype)
    check_logprobs(ctx, x, tokens_for(rows, V, g), n_top, T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("ld_more,offset", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_logprobs_strides_and_alignment(ctx, dtype, ld_more, offset):
    for rows, V in ((1, 9), (6, 1001), (2, 70001)):
        x, g = make(rows, V, dtype, ld=V + ld_more, offset=offset)
        check_logprobs(ctx, x, tokens_for(rows, V, g), min(V, 6), 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(12, 1000), (12, 40001)])
def test_logprobs_masks_and_ties(ctx, dtype, rows, V):
    x, g = make(rows, V, dtype)
    low = torch.finfo(dtype).min
    x[0] = NINF                                     # nothing left
    x[1] = NINF; x[1, V // 2] = 1.5                 # one token left
    x[2] = 0.25                                     # all equal
    x[3] = low                                      # the type's lowest value everywhere
    x[4] = low; x[4, 7] = 3.0; x[4, V - 1] = 2.0
    x[5] = NINF; x[5, ::97] = torch.linspace(-2, 2, len(x[5, ::97]), device=DEV).to(dtype)
    x[6] = torch.arange(V, device=DEV).to(dtype)    # sorted
    x[7] = torch.arange(V, 0, -1, device=DEV).to(dtype)
    x[8] = (torch.arange(V, device=DEV) % 3).to(dtype)   # three values
    x[9] = 0.0; x[9, ::2] = -0.0                    # equal whatever the sign
    x[10, :] = -30.0; x[10, V - 2] = 40.0           # near-certain
    tok = torch.full((rows,), V // 2, dtype=torch.int32, device=DEV)
    tok[10] = V - 2
    for n_top in (1, 20, 128):
        for T in (1.0, 0.5):
            check_logprobs(ctx, x, tok, n_top, T)


def test_logprob_of_a_near_certain_token_keeps_its_relative_precision(ctx):
    V = 32000
    x = torch.full((1, V), -12.0, device=DEV)
    x[0, 5] = 20.0
    tok = torch.tensor([5], dtype=torch.int32, device=DEV)
    got = ctx.logprobs(x, tok)
    rest = torch.tensor((V - 1), dtype=torch.float64).mul(torch.exp(torch.tensor(-32.0, dtype=torch.float64)))
    want = -torch.log1p(rest)
    assert abs(float(got["logprob"]) / float(want) - 1) < ref.delta(V)     # -4e-10: one minus it is 1 in fp32
    g = ctx.logprobs_grad(x, tok, torch.ones(1, device=DEV))
    assert abs(float(g[0, 5]) / float(rest / (1 + rest)) - 1) < 2 * ref.delta(V)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_nan_and_infinity_stay_in_their_row(ctx, dtype):
    x, g = make(6, 3001, dtype)
    x[1, 2000] = float("nan")
    x[3, 17] = float("inf")
    x[4, 5] = float("nan"); x[4, 6] = float("inf")
    tok = torch.full((6,), 3, dtype=torch.int32, device=DEV)
    got = check_logprobs(ctx, x, tok, 4, 1.0)
    assert got["top_ids"][1, 0] == 2000 and got["top_ids"][3, 0] == 17 and got["top_ids"][4, :2].tolist() == [5, 6]
    grad = ctx.logprobs_grad(x, tok, torch.ones(6, device=DEV))
    for r in range(6):
        assert torch.isnan(grad[r]).any() == (r in (1, 3, 4))


def check_grad(ctx, x, tokens, g_lp, g_h, T, out=None):
    want = ref.logprobs_grad(x, tokens, g_lp, g_h, T)
    V = x.shape[1]
    _, _, lp, p, H = ref.stats(x.double(), T)
    gl = g_lp.double().abs()[:, None] if g_lp is not None else 0.0
    gh = g_h.double().abs()[:, None] if g_h is not None else 0.0
    lp, p, H = torch.nan_to_num(lp, neginf=0.0), torch.nan_to_num(p), torch.nan_to_num(H)
    tol = 3 * ref.delta(V) * (gl * p + gh * p * (lp.abs() + H[:, None] + 1)) / T + 4 * ref.U * want.abs() + 1e-38
    if x.dtype == torch.bfloat16:
        tol = tol + want.abs() * 2.0 ** -8
    got = ctx.logprobs_grad(x, tokens, g_lp, g_h, temperature=T, out=out)
    ref.same(got, want, tol)
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 7), (5, 999), (2, 32003), (300, 4100), (7, 128256), (1, 300001)])
def test_logprobs_grad(ctx, rows, V, dtype):
    x, g = make(rows, V, dtype, ld=V + 3, offset=1)
    tok = tokens_for(rows, V, g)
    g_lp, g_h = torch.randn(rows, generator=g, device=DEV), torch.randn(rows, generator=g, device=DEV)
    check_grad(ctx, x, tok, g_lp, g_h, 1.0)
    check_grad(ctx, x, tok, g_lp, None, 0.6)
    check_grad(ctx, x, None, None, g_h, 1.7)


def test_gradients_agree_with_differences(ctx):
    """Central differences of the fp32 outputs' 64-bit references at the kernel's own inputs."""
    x, g = make(3, 50, torch.float32)
    tok = torch.tensor([4, 9, -1], dtype=torch.int32, device=DEV)
    g_lp, g_h = torch.tensor([0.7, -1.1, 2.0], device=DEV), torch.tensor([0.3, 0.0, -0.4], device=DEV)
    got = ctx.logprobs_grad(x, tok, g_lp, g_h, temperature=0.8)
    ids = torch.tensor([[1, 4], [9, 30], [-1, 2]], dtype=torch.int32, device=DEV)
    v = torch.log(torch.tensor([[0.5, 0.2], [0.1, 0.3], [0.9, 0.4]], device=DEV))
    w = torch.tensor([1.0, 0.5, 2.0], device=DEV)
    got_b = {b: ctx.distill(x, ids, v, tail=b, temperature=0.8, weight=w, grad=True)["grad"] for b in (0, 1)}

    def objective(xx):
        _, _, lp, _, entropy = ref.stats(xx, 0.8)
        given = lp.gather(1, tok.long().clamp(min=0)[:, None])[:, 0] * (tok >= 0)
        return (given * g_lp.double()).sum() + (entropy * g_h.double()).sum()

    def loss(xx, b):
        return (ref.distill(xx, ids, v, b, 0.8)[0] * w.double()).sum()

    h = 1e-5     # truncation h^2/6 |f'''| < 1e-10, rounding 1e-15 / h
    for r, c in ((0, 4), (0, 1), (1, 9), (1, 30), (2, 2), (2, 49)):
        a, b = x.double().clone(), x.double().clone()
        a[r, c] += h; b[r, c] -= h
        assert abs(float((objective(a) - objective(b)) / (2 * h)) - float(got[r, c])) < 1e-5
        for mode in (0, 1):
            assert abs(float((loss(a, mode) - loss(b, mode)) / (2 * h)) - float(got_b[mode][r, c])) < 1e-5


def test_grad_without_a_token_writes_nothing_else(ctx):
    """Rows that start off a 16-byte boundary and have no token: the entry in front of a row, which is the
    row before's last (or foreign memory), is left alone."""
    buf = torch.full((41,), 5.0, device=DEV)
    x, g = make(4, 7, torch.float32, ld=10, offset=1)
    out = buf[1:].view(4, 10)[:, :7]
    tok = torch.full((4,), -1, dtype=torch.int32, device=DEV)
    got = check_grad(ctx, x, tok, torch.ones(4, device=DEV), torch.ones(4, device=DEV), 1.0, out=out)
    assert got.data_ptr() == out.data_ptr() and buf[0] == 5.0 and (buf[1:].view(4, 10)[:, 7:] == 5.0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_grad_masked_rows_zero_factors_and_in_place(ctx, dtype):
    rows, V = 8, 5003
    x, g = make(rows, V, dtype, ld=V + 5)
    x[0] = NINF
    x[1] = NINF; x[1, 77] = 2.0
    x[2, 100:] = NINF
    x[3] = torch.finfo(dtype).min
    x[4] = float("nan")                              # a padded row: both factors 0
    tok = torch.full((rows,), 77, dtype=torch.int32, device=DEV)
    tok[6] = 3000                                    # ... of a masked token below
    x[6, 3000] = NINF
    g_lp, g_h = torch.randn(rows, generator=g, device=DEV), torch.randn(rows, generator=g, device=DEV)
    g_lp[4] = g_h[4] = 0.0
    want = ref.logprobs_grad(x, tok, g_lp, g_h, 1.0)
    got = check_grad(ctx, x, tok, g_lp, g_h, 1.0)
    assert (got[4] == 0).all() and (got[0] == 0).all()
    whole = torch.as_strided(x, (rows, V + 5), (V + 5, 1), x.storage_offset())
    pad = whole[:, V:].clone()
    again = ctx.logprobs_grad(x, tok, g_lp, g_h, out=x)          # in place: the same bits
    assert again.data_ptr() == x.data_ptr() and torch.equal(again, got)
    assert torch.equal(whole[:, V:], pad)                        # entries behind V are left alone
    assert want.shape == got.shape


def teacher_for(x, k, g, T, pad=True):
    z = x.float() / T + torch.randn(x.shape, generator=g, device=DEV)
    z = z.nan_to_num(nan=0.0, neginf=-50.0, posinf=50.0) if not torch.isfinite(z).all() else z
    lp, ids = torch.log_softmax(z, 1).topk(k, dim=1)
    ids = ids.to(torch.int32)
    if pad:
        ids[torch.rand(ids.shape, generator=g, device=DEV) < 0.1] = -1
        if k > 2:
            ids[0, 2] = x.shape[1]
    return ids.contiguous(), lp.contiguous()


def check_distill(ctx, x, ids, v, tail, T, weight=None, grad=True, loss=True, out=None):
    want, want_g = ref.distill(x, ids, v, tail == binding.TAIL_BUCKET, T, weight)
    V, k = x.shape[1], ids.shape[1]
    _, _, lp, p, _ = ref.stats(x.double(), T)
    got = ctx.distill(x, ids, v, tail=tail, temperature=T, weight=weight, loss=loss, grad=grad, out=out)
    d = ref.delta(V)
    if loss:   # every teacher token's log p and the tail's are off by delta and a few roundings; masses sum to 1
        big = torch.nan_to_num(lp, neginf=0.0).abs().amax(1)
        ref.same(got["loss"], want, 4 * d + 16 * ref.U * (big + 10) + 4 * ref.U * torch.nan_to_num(want.abs(), posinf=0.0))
    if grad:
        w = (weight.double().abs() if weight is not None else torch.ones_like(want))[:, None]
        i = ids.long()
        have = (i >= 0) & (i < V)
        q = torch.exp(torch.where(have, v.double(), torch.full_like(v, -1e9, dtype=torch.float64)))
        if tail == binding.TAIL_RENORM:
            q = q / q.sum(1, keepdim=True).clamp(min=1e-300)
        mag = p.scatter_add(1, i.clamp(0, V - 1), torch.where(have, q, torch.zeros_like(q)))
        # the tail's factor q_t / p_t: q_t carries the absolute rounding of the fp32 result of 1 - sum q
        seen = torch.zeros((x.shape[0], V + 1), dtype=torch.bool, device=DEV).scatter(1, torch.where(have, i, torch.full_like(i, V)), True)[:, :V]
        pt = torch.where(seen, torch.zeros_like(p), p).sum(1, keepdim=True)
        qt = (1 - q.sum(1, keepdim=True)).clamp(min=0)
        mag = mag + torch.where((tail == binding.TAIL_BUCKET) & (pt > 0) & ~seen, p / pt * qt, torch.zeros_like(p))
        tol = 4 * d * w * torch.nan_to_num(mag) / T + 4 * ref.U * want_g.abs() + 1e-38
        if x.dtype == torch.bfloat16:
            tol = tol + want_g.abs() * 2.0 ** -8
        ref.same(got["grad"], want_g, tol)
    return got


@pytest.mark.parametrize("tail", [0, 1], ids=["renorm", "bucket"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,k", [(1, 3, 1), (4, 9, 9), (3, 40, 17), (5, 999, 16), (2, 32003, 128), (260, 4100, 5),
                                      (9, 128256, 64), (1, 300001, 33)])
def test_distill(ctx, rows, V, k, dtype, tail):
    x, g = make(rows, V, dtype, ld=V + 1, offset=3)
    ids, v = teacher_for(x, k, g, 0.8)
    w = torch.rand(rows, generator=g, device=DEV)
    both = check_distill(ctx, x, ids, v, tail, 0.8, w)
    only = check_distill(ctx, x, ids, v, tail, 0.8, None, grad=False)
    assert torch.equal(torch.isinf(only["loss"]), torch.isinf(both["loss"]))
    check_distill(ctx, x, ids, v, tail, 1.0, None, loss=False)


@pytest.mark.parametrize("tail", [0, 1], ids=["renorm", "bucket"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_distill_edges(ctx, dtype, tail):
    rows, V, k = 12, 3001, 6
    x, g = make(rows, V, dtype)
    ids, v = teacher_for(x, k, g, 1.0, pad=False)
    ids[0] = -1                                      # no teacher
    x[1] = NINF                                      # no student
    x[2] = NINF; ids[2] = -1                         # neither
    ids[3, 1] = ids[3, 0]; ids[3, 4] = ids[3, 0]     # the same token three times
    v[4] = NINF; v[4, 2] = 0.0                       # a certain teacher
    x[5, ids[5, 0].long()] = NINF                    # a teacher token the student forbids: +inf
    v[6] += 1.0                                      # more than all of the mass
    x[7] = NINF; x[7, ids[7].long()] = torch.randn(k, generator=g, device=DEV).to(dtype)   # nothing outside the teacher's tokens
    x[8] = torch.finfo(dtype).min; x[8, 5] = 1.0
    x[9] = float("nan")                              # padding, weight 0
    x[10] = -20.0; x[10, ids[10].long()] = 20.0      # a tail of 1e-14
    w = torch.rand(rows, generator=g, device=DEV) + 0.1
    w[9] = 0.0
    if tail == binding.TAIL_BUCKET:
        v[7] -= torch.logsumexp(v[7], 0) + 0.5       # q_t > 0 against p_t = 0: +inf
    sel = [r for r in range(rows) if r != 9]
    got = check_distill(ctx, x[:9], ids[:9], v[:9], tail, 1.0, w[:9])
    assert got["loss"][0].abs() < 1e-5 and got["loss"][2].abs() < 1e-5 and torch.isinf(got["loss"][5])
    check_distill(ctx, x[10:], ids[10:], v[10:], tail, 1.0, w[10:])
    full = ctx.distill(x, ids, v, tail=tail, weight=w, grad=True)
    assert (full["grad"][9] == 0).all() and torch.isnan(full["loss"][9])
    assert len(sel) == rows - 1


def test_distill_in_place_and_other_alignment(ctx):
    x, g = make(5, 20001, torch.bfloat16, ld=20004)
    ids, v = teacher_for(x, 12, g, 1.0)
    got = ctx.distill(x, ids, v, tail=1, grad=True)
    other = torch.full((5 * 20007 + 1,), 9.0, dtype=torch.bfloat16, device=DEV)
    out = other[1:].view(5, 20007)[:, :20001]
    ctx.distill(x, ids, v, tail=1, grad=True, out=out)
    assert torch.equal(out, got["grad"]) and (other[1:].view(5, 20007)[:, 20001:] == 9.0).all() and other[0] == 9.0
    ctx.distill(x, ids, v, tail=1, grad=True, out=x)
    assert torch.equal(x, got["grad"])


def test_rows_far_apart(ctx):
    """Offsets past 2^32 bytes and 2^31 entries."""
    ld, V = 1_600_000_001, 4000
    buf = torch.empty(2 * ld + V, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (3, V), (ld, 1))
    small, g = make(3, V, torch.bfloat16)
    x.copy_(small)
    tok = torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV)
    a, b = ctx.logprobs(x, tok, n_top=3), ctx.logprobs(small, tok, n_top=3)
    for key in a:
        ref.same(a[key], b[key].double(), 2 * ref.delta(V) * 12)
    ones = torch.ones(3, device=DEV)
    want = ref.logprobs_grad(small, tok, ones, None, 1.0)
    got = ctx.logprobs_grad(x, tok, ones, out=x)
    ref.same(got, want, want.abs() * 2.0 ** -8 + 3 * ref.delta(V))


def test_leading_shapes_streams_and_graph(ctx):
    x, g = make(12, 2000, torch.bfloat16)
    x3 = x.view(3, 4, 2000)
    tok = tokens_for(12, 2000, g)
    flat, lead = ctx.logprobs(x, tok, n_top=4), ctx.logprobs(x3, tok.view(3, 4), n_top=4)
    for key in flat:
        assert torch.equal(flat[key].reshape(-1), lead[key].reshape(-1)) and lead[key].shape[:2] == (3, 4)
    assert torch.equal(ctx.logprobs(x3[:, 1:3].transpose(0, 1)[0], None)["lse"], flat["lse"].view(3, 4)[:, 1])
    with pytest.raises(TypeError):
        ctx.logprobs(x3.transpose(0, 1), None)
    ids, v = teacher_for(x, 8, g, 1.0)
    want = ctx.distill(x, ids, v, tail=1, grad=True)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = ctx.distill(x, ids, v, tail=1, grad=True)
    stream.synchronize()
    assert torch.equal(other["loss"], want["loss"]) and torch.equal(other["grad"], want["grad"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = ctx.distill(x, ids, v, tail=1, grad=True)
        rows = ctx.logprobs(x, tok, n_top=4)
    x.copy_(x.flip(0)); ids.copy_(ids.flip(0)); v.copy_(v.flip(0)); tok.copy_(tok.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(captured["loss"], want["loss"].flip(0)) and torch.equal(captured["grad"], want["grad"].flip(0))
    assert torch.equal(rows["top_ids"], flat["top_ids"].flip(0))


def test_no_rows(ctx):
    x = torch.empty((0, 100), device=DEV)
    i = torch.empty((0,), dtype=torch.int32, device=DEV)
    assert ctx.logprobs(x, i, n_top=3)["top_ids"].shape == (0, 3)
    assert ctx.logprobs_grad(x, i, torch.empty(0, device=DEV)).shape == (0, 100)
    assert ctx.distill(x, i.view(0, 1).expand(0, 4).contiguous(), torch.empty((0, 4), device=DEV), grad=True)["loss"].shape == (0,)


def test_refusals(ctx):
    x, g = make(4, 100, torch.float32)
    tok = tokens_for(4, 100, g)
    ids, v = teacher_for(x, 4, g, 1.0)

    def refused(status, fn, *a, **k):
        with pytest.raises(pk.DropMatchError) as e:
            fn(*a, **k)
        assert e.value.status == status

    for T in (0.0, -1.0, float("nan"), float("inf")):
        refused(binding.EINVAL, ctx.logprobs, x, tok, temperature=T)
        refused(binding.EINVAL, ctx.logprobs_grad, x, tok, torch.ones(4, device=DEV), temperature=T)
        refused(binding.EINVAL, ctx.distill, x, ids, v, temperature=T)
    refused(binding.EINVAL, ctx.logprobs, x, tok, n_top=101)
    refused(binding.EINVAL, ctx.logprobs, x.repeat(1, 2), tok, n_top=129)
    refused(binding.EINVAL, ctx.logprobs_grad, x, None, torch.ones(4, device=DEV))
    refused(binding.EINVAL, ctx.distill, x, ids, v, tail=2)
    refused(binding.EINVAL, ctx.distill, x, ids, v, loss=False, grad=False)
    big = torch.zeros((4, 129), dtype=torch.int32, device=DEV)
    refused(binding.EINVAL, ctx.distill, x, big, big.float())
    buf = torch.zeros(4 * 100 + 8, device=DEV)      # a gradient that overlaps the logits without being them
    refused(binding.EINVAL, ctx.logprobs_grad, buf[:400].view(4, 100), tok, torch.ones(4, device=DEV), out=buf[8:].view(4, 100))
    refused(binding.EINVAL, ctx.distill, buf[:400].view(4, 100), ids, v, grad=True, out=buf[8:].view(4, 100))
    for bad in (x.half(), x.cpu(), x[0], x[:, ::2], x[:1].expand(4, 100)):
        with pytest.raises(TypeError):
            ctx.logprobs(bad)
    for bad in (tok.long(), tok[:3], tok.cpu()):
        with pytest.raises(TypeError):
            ctx.logprobs(x, bad)
    with pytest.raises(TypeError):
        ctx.distill(x, ids, v.double())
    with pytest.raises(TypeError):
        ctx.distill(x, ids, v, weight=torch.ones(5, device=DEV))
    with pytest.raises(TypeError):
        ctx.distill(x, ids, v, out=torch.empty_like(x))
    with pytest.raises(TypeError):
        ctx.logprobs_grad(x, tok, torch.ones(4, device=DEV), out=torch.empty((4, 100), dtype=torch.bfloat16, device=DEV))
    assert ctx.device_error() == 0


@pytest.mark.parametrize("dtype,V", [(torch.float32, 500_003), (torch.bfloat16, 1_000_001), (torch.float32, 2_300_001)],
                         ids=["f32", "bf16", "f32_long"])
def test_rows_too_long_for_shared_memory(ctx, dtype, V):
    """Gradients of rows that are read twice, and the top entries of rows of many batches."""
    x, g = make(2, V, dtype)
    tok = tokens_for(2, V, g)
    check_logprobs(ctx, x, tok, 40, 1.0)
    g_lp, g_h = torch.randn(2, generator=g, device=DEV), torch.randn(2, generator=g, device=DEV)
    got = check_grad(ctx, x, tok, g_lp, g_h, 1.0)
    ids, v = teacher_for(x, 50, g, 1.0)
    both = check_distill(ctx, x, ids, v, binding.TAIL_BUCKET, 1.0)
    check_distill(ctx, x, ids, v, binding.TAIL_RENORM, 1.0)
    assert torch.equal(ctx.logprobs_grad(x.clone(), tok, g_lp, g_h), got)
    y = x.clone()
    assert torch.equal(ctx.distill(y, ids, v, tail=binding.TAIL_BUCKET, grad=True, out=y)["grad"], both["grad"])


def test_distill_refuses_rows_whose_marks_do_not_fit(ctx):
    x = torch.zeros((1, 13_000_000), dtype=torch.bfloat16, device=DEV)
    ids, v = torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.zeros((1, 1), device=DEV)
    with pytest.raises(pk.DropMatchError) as e:
        ctx.distill(x, ids, v, tail=binding.TAIL_BUCKET, grad=True)
    assert e.value.status == binding.EUNSUPPORTED
    assert abs(float(ctx.distill(x, ids, v)["loss"]) - 16.3805) < 1e-3      # log V: nothing to mark


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(5000, 67), (3001, 2049), (700, 40001)])
def test_many_rows_shared_out_between_clusters(ctx, dtype, rows, V):
    """Every row gets its gradient exactly once, whichever cluster takes it, with zero rows in between."""
    x, g = make(rows, V, dtype, ld=V + 1)
    tok = tokens_for(rows, V, g)
    g_lp, g_h = torch.randn(rows, generator=g, device=DEV), torch.randn(rows, generator=g, device=DEV)
    g_lp[::7] = 0.0
    g_h[::7] = 0.0
    check_grad(ctx, x, tok, g_lp, g_h, 1.0)
    ids, v = teacher_for(x, 9, g, 1.0)
    w = torch.rand(rows, generator=g, device=DEV)
    w[::5] = 0.0
    check_distill(ctx, x, ids, v, binding.TAIL_BUCKET, 1.0, w)
    check_distill(ctx, x, ids, v, binding.TAIL_RENORM, 1.0, w, loss=False)
    assert ctx.device_error() == 0


def test_two_calls_at_once(ctx):
    """Calls of one context on two streams share nothing."""
    x, g = make(300, 32003, torch.bfloat16)
    y, _ = make(200, 50001, torch.float32, seed=1)
    ids, v = teacher_for(x, 16, g, 1.0)
    jds, u = teacher_for(y, 16, g, 1.0)
    a, b = ctx.distill(x, ids, v, tail=1, grad=True), ctx.distill(y, jds, u, tail=1, grad=True)
    p, q = ctx.logprobs(x, None, n_top=9), ctx.logprobs(y, None, n_top=9)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    out = []
    for _ in range(5):
        with torch.cuda.stream(streams[0]):
            out.append((ctx.distill(x, ids, v, tail=1, grad=True), a))
            out.append((ctx.logprobs(x, None, n_top=9), p))
        with torch.cuda.stream(streams[1]):
            out.append((ctx.distill(y, jds, u, tail=1, grad=True), b))
            out.append((ctx.logprobs(y, None, n_top=9), q))
    torch.cuda.synchronize()
    for got, want in out:
        for key in want:
            assert torch.equal(got[key], want[key]), key


def test_teacher_to_student(ctx):
    """The operators together, as a draft head is trained: the target scores the hidden rows of a text, the
    draft's logits are pulled towards its top tokens, and the draft's log-probabilities are looked at."""
    V, d, rows, k = 4000, 128, 96, 32
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    target = (torch.randn((V, d), generator=g, device=DEV) * 0.3).to(torch.bfloat16)
    H = torch.randn((rows, d), generator=g, device=DEV).to(torch.bfloat16)
    c = pk.Context(0)
    try:
        c.set_head(target, max_rows=rows)
        c.enable_score(rows, k)
        T = 1.5
        teach = c.score(H, None, n_top=k, temperature=T)
        W = (torch.randn((V, d), generator=g, device=DEV) * 0.02).requires_grad_(True)
        hidden = H.float()
        weight = torch.full((rows,), 1.0 / rows, device=DEV)
        for _ in range(3):
            logits = hidden @ W.T
            res = c.distill(logits.detach(), teach["top_ids"], teach["top_logprob"], tail=binding.TAIL_BUCKET,
                            temperature=T, weight=weight, grad=True)
            want, want_g = ref.distill(logits.detach(), teach["top_ids"], teach["top_logprob"], True, T, weight)
            ref.same(res["loss"], want, 1e-4 * want.abs() + 1e-5)
            W.grad = None
            logits.backward(res["grad"])
            # the weight's gradient is the 64-bit one's
            exact = want_g.T @ hidden.double()
            assert float((W.grad.double() - exact).norm() / exact.norm()) < 1e-4
            with torch.no_grad():
                given = c.logprobs(logits, teach["top_ids"][:, 0].contiguous())
                check_logprobs(c, logits.detach(), teach["top_ids"][:, 0].contiguous(), 0, 1.0)
                assert given["logprob"].shape == (rows,)
                W -= 2.0 * W.grad
    finally:
        c.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [8200, 16391])
def test_many_rows_of_every_kind(ctx, dtype, V):
    """A run of rows long enough that CTAs take over rows of others, with rows in between that leave the
    usual path: masked, of equal entries (more than a list of candidates takes), NaN, one entry only."""
    rows = 1500
    x, g = make(rows, V, dtype, ld=V + 3)
    x[5::11] = NINF
    x[6::11] = 1.5
    x[7::11, 1:] = NINF
    x[8::11, ::2] = torch.finfo(dtype).min
    x[9::11, 100:] = NINF
    tok = tokens_for(rows, V, g)
    check_logprobs(ctx, x, tok, 5, 0.8)
    check_logprobs(ctx, x, tok, 100, 1.0)
    x[10::11, V // 2] = float("nan")
    got = check_logprobs(ctx, x, None, 0, 1.0)
    assert torch.isnan(got["lse"][10::11]).all() and not torch.isnan(got["lse"][9::11]).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(1200, 1001), (1200, 30011), (170, 128256)])
def test_many_rows_in_place(ctx, dtype, rows, V):
    """The next row is on its way while a row's gradient takes the place of its logits."""
    x, g = make(rows, V, dtype, ld=V + 2)
    tok = tokens_for(rows, V, g)
    g_lp, g_h = torch.randn(rows, generator=g, device=DEV), torch.randn(rows, generator=g, device=DEV)
    g_lp[::6] = 0.0
    g_h[::6] = 0.0
    ids, v = teacher_for(x, 33, g, 1.0)
    ids[:, 20] = ids[:, 3]                               # a token that is named twice
    w = torch.rand(rows, generator=g, device=DEV)
    w[::4] = 0.0
    x[::12] = float("nan")                               # padded rows: both factors 0, weight 0
    for call in (lambda at, out: ctx.logprobs_grad(at, tok, g_lp, g_h, out=out),
                 lambda at, out: ctx.distill(at, ids, v, tail=binding.TAIL_BUCKET, weight=w, grad=True, out=out)["grad"],
                 lambda at, out: ctx.distill(at, ids, v, weight=w, loss=False, grad=True, out=out)["grad"]):
        want = call(x, None)
        assert not torch.isnan(want).any() and (want[::12] == 0).all()
        whole = torch.as_strided(x, (rows, V + 2), (V + 2, 1), x.storage_offset()).clone()
        call(whole[:, :V], whole[:, :V])
        assert torch.equal(whole[:, :V], want) and (whole[:-1, V:] == 77.0).all()
    assert ctx.device_error() == 0


@pytest.mark.parametrize("tail", [0, 1], ids=["renorm", "bucket"])
def test_repeated_tokens_give_the_same_bits_every_time(ctx, tail):
    x, g = make(600, 5001, torch.bfloat16)
    ids = torch.randint(-1, 60, (600, 100), generator=g, device=DEV, dtype=torch.int32)
    v = torch.log_softmax(torch.randn((600, 100), generator=g, device=DEV), 1) - 0.3
    first = check_distill(ctx, x, ids, v, tail, 1.0)
    for _ in range(20):
        again = ctx.distill(x, ids, v, tail=tail, grad=True)
        assert torch.equal(again["grad"], first["grad"]) and torch.equal(again["loss"], first["loss"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=["nan", "inf"])
def test_nan_or_infinity_anywhere_in_a_row(ctx, dtype, value):
    """Wherever it stands, whatever comes after it: in rows shared by CTAs and in rows of one."""
    for rows, V in ((6, 40001), (700, 9001)):
        x, g = make(rows, V, dtype)
        for r, at in enumerate((0, 1, 1030, V // 2, V - 1)):
            x[r, at] = value
        check_logprobs(ctx, x, tokens_for(rows, V, g), 0, 1.0)
        ids, v = teacher_for(x, 6, g, 1.0, pad=False)
        for tail in (binding.TAIL_RENORM, binding.TAIL_BUCKET):
            loss = ctx.distill(x, ids, v, tail=tail)["loss"]
            both = ctx.distill(x, ids, v, tail=tail, grad=True)
            for got in (loss, both["loss"]):
                assert torch.isnan(got[:5]).all() and torch.isfinite(got[5:]).all()
            assert torch.isnan(both["grad"][:5]).any(1).all() and torch.isfinite(both["grad"][5:]).all()
            check_distill(ctx, x[5:], ids[5:], v[5:], tail, 1.0)


def test_a_tail_below_the_range_of_fp32(ctx):
    """Less than 1e-38 of the row's mass outside the teacher's tokens: an infinite loss, a finite gradient."""
    x = torch.full((3, 500), -400.0, device=DEV)
    x[:, :2] = 0.0
    x[2] = 0.0
    ids = torch.tensor([[0, 1]] * 3, dtype=torch.int32, device=DEV)
    v = torch.log(torch.full((3, 2), 0.25, device=DEV))
    res = ctx.distill(x, ids, v, tail=binding.TAIL_BUCKET, grad=True)
    assert torch.isinf(res["loss"][:2]).all() and (res["loss"][:2] > 0).all() and torch.isfinite(res["loss"][2])
    assert torch.isfinite(res["grad"]).all()
    assert torch.equal(ctx.distill(x, ids, v, tail=binding.TAIL_BUCKET)["loss"][:2], res["loss"][:2])
