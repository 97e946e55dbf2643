"""dropmatch_dropout and its gradient against a plain 64-bit statement (engine_ref.py, masks from the
tests' own generator)."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding
import engine_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED = 0x9E3779B97F4A7C15


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    c.close()


def rows_of(lead, d, dtype, ld=None, offset=0, fill=77.0):
    n = 1
    for k in lead:
        n *= k
    ld = ld or d
    buf = torch.full((offset + n * ld,), fill, dtype=dtype, device=DEV)
    return buf, buf[offset:].view(*lead, ld)[..., :d]


def want_dropout(x, keep, p):
    s = ref.single(1.0 / (1.0 - ref.single(p)))
    return torch.where(keep, (x.float().cpu() * torch.tensor(s))[:, :, None], torch.zeros(())).to(x.dtype)


def check(ctx, B, T, K, d, dtype, p=0.1, seq_base=0, more=0, offset=0, per_path=False):
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    keep = ref.keep_flags(B, T, K, d, p, SEED, seq_base, per_path)
    # forward: one product and one rounding, as in the definition: equal bits
    _, x = rows_of((B, T), d, dtype, d + more, offset)
    x.copy_(torch.randn((B, T, d), generator=g, device=DEV))
    buf, out = rows_of((B, T, K), d, dtype, d + 2 * more, 2 * offset)
    got = ctx.dropout(x, K, p, SEED, seq_base=seq_base, out=out)
    assert got is out
    assert torch.equal(got.cpu(), want_dropout(x, keep, p))
    out.fill_(77.0)
    assert bool((buf == 77.0).all())           # nothing between or behind the rows
    assert torch.equal(ctx.dropout(x, K, p, SEED, seq_base=seq_base).cpu(), want_dropout(x, keep, p))
    # gradient: K fp32 additions, the factor, one rounding
    _, gr = rows_of((B, T, K), d, dtype, d + more, offset)
    gr.copy_(torch.randn((B, T, K, d), generator=g, device=DEV))
    buf, out = rows_of((B, T), d, dtype, d + 3 * more, offset)
    got = ctx.dropout_grad(gr, p, SEED, seq_base=seq_base, out=out).double().cpu()
    masked = gr.double().cpu() * keep
    s = 1.0 / (1.0 - ref.single(p))
    want = masked.sum(2) * s
    tol = masked.abs().sum(2) * s * (K + 3) * ref.U + want.abs() * ref.half_step(dtype) * (1 + 2.0 ** -8)
    assert bool(((got - want).abs() <= tol).all())
    out.fill_(77.0)
    assert bool((buf == 77.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,K,d", [(1, 1, 1, 1), (2, 3, 2, 3), (1, 5, 8, 4096), (3, 7, 5, 79), (2, 2, 16, 130), (1, 3, 33, 256), (1, 2, 100, 515),
                                     (1, 1, 1024, 40), (2, 1, 17, 8192), (1, 300, 1, 1000), (40, 1, 3, 264)])
def test_dropout_and_gradient(ctx, B, T, K, d, dtype):
    check(ctx, B, T, K, d, DT[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("more,offset", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_strides_and_alignment(ctx, dtype, more, offset):
    for d in (1, 31, 256, 1001):
        check(ctx, 2, 3, 4, d, DT[dtype], more=more, offset=offset, seq_base=5)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -33, 1e-3, 0.5, 0.999, 1.0 - 2.0 ** -24])
def test_probabilities(ctx, p):
    check(ctx, 1, 4, 3, 515, torch.float32, p=p)
    check(ctx, 1, 4, 3, 512, torch.bfloat16, p=p)


def test_sequence_ids_wrap_and_masks_shared_over_positions(ctx):
    check(ctx, 3, 2, 2, 64, torch.float32, seq_base=2 ** 32 - 1)
    check(ctx, 3, 2, 2, 64, torch.float32, seq_base=2 ** 40 + 7)
    ctx.set_mask_mode(binding.MASK_PER_PATH)
    try:
        check(ctx, 3, 5, 2, 64, torch.bfloat16, seq_base=3, per_path=True)
    finally:
        ctx.set_mask_mode(binding.MASK_PER_POSITION)


def test_the_masks_are_those_of_the_verify_calls(ctx):
    B, T, K, d = 2, 3, 5, 200
    bits = ctx.debug_masks(B, T, K, d, 0.3, SEED, seq_base=9)
    got = ctx.dropout(torch.ones((B, T, d), device=DEV), K, 0.3, SEED, seq_base=9) != 0
    j = torch.arange(d, device=DEV)
    assert torch.equal(got, ((bits[..., j // 32] >> (j % 32)) & 1) == 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropped_nan_and_infinity_leave_no_trace(ctx, dtype):
    B, T, K, d = 1, 3, 4, 1000
    keep = ref.keep_flags(B, T, K, d, 0.5, SEED).to(DEV)
    for value in (float("nan"), float("inf")):
        x = torch.ones((B, T, d), dtype=DT[dtype], device=DEV)
        x[:, :, ::3] = value
        got = ctx.dropout(x, K, 0.5, SEED)
        assert bool((got[~keep] == 0).all()) and not bool(torch.signbit(got[~keep]).any())
        gr = torch.ones((B, T, K, d), dtype=DT[dtype], device=DEV)
        gr[~keep] = value
        assert torch.equal(ctx.dropout_grad(gr, 0.5, SEED).float(), keep.sum(2).float() * 2.0)


def test_in_place(ctx):
    for dtype, d in ((torch.float32, 1001), (torch.bfloat16, 1024), (torch.bfloat16, 77)):
        x = torch.randn((2, 9, d), device=DEV).to(dtype)
        want = ctx.dropout(x, 1, 0.2, 4)
        y = x.clone()
        ctx.dropout(y, 1, 0.2, 4, out=y[:, :, None])
        assert torch.equal(y, want[:, :, 0])
        z = x.clone()
        want = ctx.dropout_grad(x[:, :, None], 0.2, 4)
        ctx.dropout_grad(z[:, :, None], 0.2, 4, out=z)
        assert torch.equal(z, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_agrees_with_differences(ctx, dtype):
    """<dropout(x), g> is linear in x: its difference along any direction h is <h, dropout_grad(g)>; compared exactly in
    fp64 on whole numbers that every sum holds (scale 2 for p = 1/2)."""
    B, T, K, d = 2, 3, 6, 333
    g = torch.randint(-8, 9, (B, T, K, d), device=DEV).to(DT[dtype])
    x = torch.randint(-8, 9, (B, T, d), device=DEV).to(DT[dtype])
    h = torch.randint(-3, 4, (B, T, d), device=DEV).to(DT[dtype])
    value = lambda v: float((ctx.dropout(v, K, 0.5, 7).double() * g.double()).sum())
    slope = float((ctx.dropout_grad(g, 0.5, 7).double() * h.double()).sum())
    assert value(x + h) - value(x) == slope


def test_rows_do_not_depend_on_the_others(ctx):
    for K in (3, 40):
        x = torch.randn((4, 600, 520), device=DEV).bfloat16()
        g = torch.randn((4, 600, K, 520), device=DEV).bfloat16()
        y, z = ctx.dropout(x, K, 0.1, 5), ctx.dropout_grad(g, 0.1, 5)
        assert torch.equal(ctx.dropout(x[2:3], K, 0.1, 5, seq_base=2), y[2:3])
        assert torch.equal(ctx.dropout_grad(g[2:3], 0.1, 5, seq_base=2), z[2:3])


def test_rows_far_apart(ctx):
    """Offsets past 2^31 entries, of rows and of copies."""
    ld, d, K = 1 << 30, 100, 3
    x = torch.randn((1, 1, d), device=DEV).bfloat16()
    far = torch.empty(2 * ld + d, dtype=torch.bfloat16, device=DEV).as_strided((1, 1, K, d), (3 * ld, 3 * ld, ld, 1))
    want = ctx.dropout(x, K, 0.3, 3)
    assert torch.equal(ctx.dropout(x, K, 0.3, 3, out=far), want)
    assert torch.equal(ctx.dropout_grad(far, 0.3, 3), ctx.dropout_grad(want, 0.3, 3))


def test_streams_and_graph(ctx):
    x = torch.randn((2, 50, 1000), device=DEV)
    want = ctx.dropout(x, 4, 0.1, 5)
    back = ctx.dropout_grad(want, 0.1, 5)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = ctx.dropout(x, 4, 0.1, 5)
    s.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ctx.dropout(x, 4, 0.1, 5)
        z = ctx.dropout_grad(y, 0.1, 5)
    x2 = torch.randn_like(x)
    x.copy_(x2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, ctx.dropout(x2, 4, 0.1, 5)) and torch.equal(z, ctx.dropout_grad(y, 0.1, 5))
    assert not torch.equal(z, back)


def test_nothing_to_do(ctx):
    assert ctx.dropout(torch.empty((0, 3, 8), device=DEV), 4, 0.1, 1).shape == (0, 3, 4, 8)
    assert ctx.dropout_grad(torch.empty((2, 0, 4, 8), device=DEV), 0.1, 1).shape == (2, 0, 8)


@pytest.mark.parametrize("name", ["dropmatch_dropout", "dropmatch_dropout_grad"])
def test_refusals(ctx, name):
    fn = getattr(binding.lib(), name)
    one, many = torch.zeros((6, 40), device=DEV), torch.zeros((6 * 4, 40), device=DEV)
    a, b = (one, many) if name == "dropmatch_dropout" else (many, one)

    def call(**kw):
        v = dict(h=ctx._h, x=a.data_ptr(), dtype=binding.F32, ld=40, B=2, T=3, K=4, d=40, p=0.1, seed=1, seq=0, out=b.data_ptr(), ldo=40, s=None)
        v.update(kw)
        return fn(*v.values())

    assert call() == binding.OK
    for bad in (dict(h=None), dict(x=None), dict(x=a.data_ptr() + 2), dict(dtype=2), dict(ld=39), dict(B=-1), dict(T=-1), dict(K=0),
                dict(K=1025), dict(d=0), dict(p=1.0), dict(p=-0.1), dict(p=float("nan")), dict(out=None), dict(out=b.data_ptr() + 1),
                dict(ldo=39), dict(B=2 ** 20, T=2 ** 10), dict(out=a.data_ptr()), dict(out=a.data_ptr() + 160)):
        assert call(**bad) == binding.EINVAL, bad
    assert call(K=1, out=a.data_ptr(), ld=40, ldo=44) == binding.EINVAL       # in place needs one stride
    assert call(K=1, out=a.data_ptr()) == binding.OK
    assert call(d=2 ** 30 + 1, ld=2 ** 31, ldo=2 ** 31) == binding.EUNSUPPORTED
    assert call(B=0, x=None, out=None) == binding.OK
    x = torch.zeros((2, 3, 8), device=DEV)
    for bad in (x.cpu(), x.double(), x.half(), x[0], x.transpose(1, 2)[:, ::2]):
        with pytest.raises(TypeError):
            ctx.dropout(bad, 2, 0.1, 1)
        with pytest.raises(TypeError):
            ctx.dropout_grad(bad[:, :, None] if bad.dim() == 3 else bad, 0.1, 1)
    with pytest.raises(TypeError):
        ctx.dropout(x, 2, 0.1, 1, out=torch.zeros((2, 3, 3, 8), device=DEV))
    with pytest.raises(TypeError):
        ctx.dropout_grad(x[:, :, None], 0.1, 1, out=torch.zeros((2, 3, 8), dtype=torch.bfloat16, device=DEV))
