"""dropmatch_verify_lossless against a plain 64-bit statement of the rule (engine_ref.py)."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding
import engine_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NINF = float("-inf")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    c.close()


def rows_of(shape, dtype, ld, offset):
    B, R, V = shape
    buf = torch.full((offset + B * R * ld,), float("nan"), dtype=dtype, device=DEV)      # (what lies between rows is never read)
    return buf[offset:].view(B, R, ld)[:, :, :V]


def make(B, T, V, target="bf16", draft="bf16", bonus=1, seed=0, more=0, offset=0, ragged=False, scale=3.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn((B, T + 1, V), generator=g, device=DEV) * scale
    a = dict(target=rows_of((B, T + bonus, V), DT[target], V + more, offset))
    a["target"].copy_(x[:, :T + bonus])
    a["draft_logits"] = None
    if draft is not None:
        a["draft_logits"] = rows_of((B, T, V), DT[draft], V + 2 * more, 3 * offset)
        a["draft_logits"].copy_(x[:, :T] + 0.7 * torch.randn((B, T, V), generator=g, device=DEV))
    y = x[:, :T] - torch.log(-torch.log(torch.rand((B, T, V), generator=g, device=DEV).clamp(1e-7, 1 - 1e-7)))
    a["draft"] = y.argmax(2).to(torch.int32) if V and T else torch.zeros((B, T), dtype=torch.int32, device=DEV)
    a["u_accept"] = torch.rand((B, T), generator=g, device=DEV)
    a["u_next"] = torch.rand((B,), generator=g, device=DEV)
    a["draft_len"] = torch.randint(0, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32) if ragged else None
    return a


def check(ctx, a, T=1.0, Td=1.0):
    got = ctx.verify_lossless(**a, temperature=T, draft_temperature=Td)
    n, nxt, prob = ref.lossless(a["target"], a["draft"], a["u_accept"], a["u_next"], a["draft_logits"], a["draft_len"], T, Td)
    assert torch.equal(got["accept_len"].cpu(), n)
    assert torch.equal(got["next"].cpu(), nxt)
    p = got["accept_prob"].double().cpu()
    tol = ref.accept_tol(a["target"].shape[2], a["draft_logits"] is not None)
    assert torch.equal(torch.isnan(p), torch.isnan(prob))
    assert bool(((p - prob).abs().nan_to_num(0.0) <= tol * prob.nan_to_num(0.0) + 2.0 ** -126).all())
    return got


@pytest.mark.parametrize("draft", ["bf16", "f32", None])
@pytest.mark.parametrize("target", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,V,bonus,ragged", [(1, 1, 1, 1, False), (2, 3, 2, 0, False), (5, 4, 31, 1, True), (3, 2, 1000, 1, False),
                                                (9, 5, 4097, 0, True), (2, 40, 513, 1, True), (1, 5, 32003, 1, False)])
def test_lossless(ctx, B, T, V, bonus, ragged, target, draft):
    for seed in range(4):
        check(ctx, make(B, T, V, target, draft, bonus, seed=seed, ragged=ragged), T=1.0 if seed % 2 else 0.7, Td=1.3 if seed > 1 else 1.0)


@pytest.mark.parametrize("target,draft", [("bf16", "bf16"), ("f32", "f32"), ("bf16", None)])
def test_lossless_long_rows(ctx, target, draft):
    check(ctx, make(6, 3, 128256, target, draft, seed=5))
    check(ctx, make(3, 2, 151936, target, draft, seed=6, scale=0.01))      # nearly flat: every token within 1e-5 of the next


@pytest.mark.parametrize("target,draft", [("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("more,offset", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_lossless_strides_and_alignment(ctx, target, draft, more, offset):
    for V in (9, 1001, 20011):
        check(ctx, make(4, 3, V, target, draft, more=more, offset=offset, seed=V, ragged=True))


def test_one_token_per_sequence(ctx):
    for V in (1, 7, 5000):
        check(ctx, make(6, 0, V, "f32", None, seed=V))
        a = make(6, 2, V, seed=V)
        a["draft_len"] = torch.zeros((6,), dtype=torch.int32, device=DEV)
        got = check(ctx, a)
        assert int(got["accept_len"].sum()) == 0 and int(got["accept_prob"].abs().sum()) == 0


@pytest.mark.parametrize("draft", ["f32", None])
def test_draws_at_the_ends_of_the_unit_interval(ctx, draft):
    for u in (0.0, 1.0 - 2.0 ** -24):
        for V in (5, 3001):
            a = make(4, 3, V, "f32", draft, seed=V)
            a["u_next"].fill_(u)
            check(ctx, a)
            a["u_accept"].fill_(u)
            check(ctx, a)


@pytest.mark.parametrize("target,draft", [("f32", "f32"), ("bf16", "bf16"), ("f32", None)])
def test_decisions_next_to_the_border(ctx, target, draft):
    """u_accept one fp32 step around p / q: far inside what fp32 sums can tell apart."""
    B, T, V = 16, 4, 3000
    a = make(B, T, V, target, draft, seed=11)
    a["draft"] = torch.randint(0, V, (B, T), device=DEV, dtype=torch.int32)      # (drawn from p the ratio would often exceed 1)
    _, _, prob = ref.lossless(a["target"], a["draft"], a["u_accept"], a["u_next"], a["draft_logits"])
    near = prob.float()
    for step in range(-2, 3):
        u = near.clone()
        for _ in range(abs(step)):
            u = torch.nextafter(u, torch.full_like(u, 2.0 if step > 0 else -1.0))
        for t in range(T):
            v = torch.zeros_like(u)          # sure acceptance in front
            v[:, t:] = u[:, t:]
            a["u_accept"] = v.clamp(0.0, 1.0 - 2.0 ** -24).to(DEV)
            check(ctx, a)


def test_draws_next_to_the_border(ctx):
    """u_next one fp32 step around the cumulative sum of a token."""
    B, V = 64, 20000
    a = make(B, 0, V, "f32", None, seed=3, scale=1.0)
    for b in range(B):
        cum = torch.cumsum(ref.softmax64(a["target"][b, 0], 1.0), 0)
        at = cum[b * 311 % V].float()
        a["u_next"][b] = torch.nextafter(at, at + (1 if b % 2 else -1)).clamp(0, 1 - 2.0 ** -24) if b % 3 else at
    check(ctx, a)


@pytest.mark.parametrize("target", ["f32", "bf16"])
@pytest.mark.parametrize("draft", ["f32", "bf16", None])
def test_masks(ctx, target, draft):
    for V in (40, 9001):
        a = make(10, 3, V, target, draft, seed=V, ragged=False)
        x, low = a["target"], torch.finfo(DT[target]).min
        x[:, :, V // 2:] = NINF
        x[0, 0] = NINF                         # nothing allowed: rejected, nothing to draw
        x[1, 0, 1:] = NINF                     # one token allowed
        a["draft"][1, 0] = 0
        x[2, 0] = NINF
        x[2, 0, V - 1] = 3.0                   # the drafted token is forbidden
        a["draft"][2, 0] = 1
        x[3, 1:] = low                         # masked by the type's lowest value: a flat row
        a["u_accept"][3, 0] = 0.0
        a["draft"][4, 0] = V                   # no such token
        a["draft"][5, 0] = -7
        a["draft"][6, 1] = 2 ** 31 - 1
        if draft is not None:
            y = a["draft_logits"]
            y[:, :, V // 2:] = NINF
            y[7, 0] = NINF                     # a drafter that says nothing: q = 0, a token with p > 0 is accepted
            a["draft"][7, 0] = 3
            y[8, 0] = torch.finfo(DT[draft]).min
            a["draft"][8, 0] = V // 2 - 1
        check(ctx, a)
        check(ctx, a, T=0.4, Td=2.0)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("draft", ["f32", "bf16", None])
def test_nan_and_infinity_stay_in_their_sequence(ctx, draft, value):
    for V in (40, 9001):
        a = make(8, 3, V, "f32", draft, seed=V)
        a["u_accept"][:, :2] = 0.0
        a["target"][1, 0, V - 1] = value
        a["target"][2, 3, 0] = value           # the bonus row
        a["target"][3, 2, 7] = value
        a["target"][4, 1] = value
        a["target"][5, 1] = NINF
        a["target"][5, 1, 3] = value           # nothing else in the row
        if draft is not None:
            a["draft_logits"][6, 1, 5] = value
            a["draft_logits"][7, 0] = NINF
            a["draft_logits"][7, 0, 0] = value
        check(ctx, a)


def test_equal_distributions(ctx):
    """A drafter equal to the target: everything is accepted; where a token does not exist the draw is from p."""
    a = make(8, 4, 5003, "bf16", "bf16", seed=2)
    a["draft_logits"] = a["target"][:, :4].contiguous()
    a["u_accept"].fill_(1.0 - 2.0 ** -24)
    got = check(ctx, a)
    assert got["accept_len"].tolist() == [4] * 8
    a["draft"][:, 2] = -1
    assert check(ctx, a)["accept_len"].tolist() == [2] * 8


def test_large_logits_and_small_temperatures(ctx):
    for big, T in ((1e4, 1.0), (1e30, 1.0), (3.0, 1e-6), (3.0, 1e20)):
        a = make(6, 3, 2001, "f32", "f32", seed=4)
        a["target"] *= big
        a["draft_logits"] *= big
        check(ctx, a, T=T, Td=T)


@pytest.mark.parametrize("draft", ["f32", None])
def test_logits_spread_wider_than_fp64_reaches(ctx, draft):
    """The drafted token, or the entries that are looked at first, lie e^700 and more below the row's maximum."""
    for scale in (100.0, 400.0, 1000.0):
        a = make(8, 3, 2001, "f32", draft, seed=int(scale), scale=scale)
        a["u_accept"][::2] = 0.5
        check(ctx, a)
        a["draft"] = torch.randint(0, 2001, (8, 3), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV, dtype=torch.int32)
        check(ctx, a)
        a["target"][:, :, ::3] = NINF
        check(ctx, a)


def test_lengths_outside_the_draft_are_clamped(ctx):
    a = make(4, 3, 500, seed=8)
    a["draft_len"] = torch.tensor([-3, 9, 2 ** 31 - 1, 1], dtype=torch.int32, device=DEV)
    check(ctx, a)


def test_a_sequence_does_not_depend_on_the_others(ctx):
    a = make(7, 3, 9001, seed=9, ragged=True)
    whole = check(ctx, a)
    for b in range(7):
        one = {k: (v[b:b + 1].contiguous() if torch.is_tensor(v) else v) for k, v in a.items()}
        got = ctx.verify_lossless(**one)
        for k in got:
            assert torch.equal(got[k][0], whole[k][b])


def test_many_sequences(ctx):
    """More clusters than fit on the GPU at once."""
    a = make(700, 2, 4500, seed=10, ragged=True)
    check(ctx, a)


@pytest.mark.parametrize("descending", [False, True])
def test_rows_in_order(ctx, descending):
    """Every batch of a row above (below) all before it: sums must not be rounded anew with each."""
    for V, B, scale in ((300000, 8, 0.5), (300000, 8, 8.0), (40001, 30, 0.01)):
        a = make(B, 1, V, "f32", "f32", seed=V, scale=scale)
        for k in ("target", "draft_logits"):
            a[k].copy_(torch.sort(a[k], dim=2, descending=descending).values)
        check(ctx, a)
    # many positions, each read by one CTA alone
    a = make(300, 5, 20001, "bf16", "bf16", seed=3, scale=0.5)
    for k in ("target", "draft_logits"):
        a[k].copy_(torch.sort(a[k], dim=2, descending=descending).values)
    got = ctx.verify_lossless(**a)
    lp = torch.log_softmax(a["target"][:, :5].double(), 2) - torch.log_softmax(a["draft_logits"].double(), 2)
    want = lp.gather(2, a["draft"].long()[:, :, None])[:, :, 0].exp().clamp(max=1.0)
    assert bool(((got["accept_prob"].double() - want).abs() <= ref.accept_tol(20001, True) * want).all())


def test_streams_graph_and_two_calls_at_once(ctx):
    a, o = make(5, 4, 20001, seed=21), make(6, 3, 30011, "f32", "f32", seed=22)
    want_a, want_o = check(ctx, a), check(ctx, o)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(s1):
            got_a = ctx.verify_lossless(**a)
        with torch.cuda.stream(s2):
            got_o = ctx.verify_lossless(**o)
    torch.cuda.synchronize()
    for k in want_a:
        assert torch.equal(got_a[k], want_a[k]) and torch.equal(got_o[k], want_o[k])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = ctx.verify_lossless(**a)
    b = make(5, 4, 20001, seed=23)
    for k in a:
        if torch.is_tensor(a[k]):
            a[k].copy_(b[k])
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    want = check(ctx, a)
    for k in want:
        assert torch.equal(captured[k], want[k])


def test_rows_far_apart(ctx):
    """Row offsets past 2^31 entries."""
    V, ld = 1000, 1 << 30
    buf = torch.empty(3 * ld + V, dtype=torch.bfloat16, device=DEV)
    a = make(1, 3, V, seed=31)
    far = buf.as_strided((1, 4, V), (4 * ld, ld, 1))
    far.copy_(a["target"])
    a["target"] = far
    a["u_accept"].fill_(0.0)
    check(ctx, a)


def test_nothing_to_do(ctx):
    a = make(0, 3, 100)
    got = ctx.verify_lossless(**a)
    assert got["accept_len"].shape == (0,) and got["accept_prob"].shape == (0, 3)


def test_refusals(ctx):
    a = make(2, 3, 100)
    L, p = binding.lib(), lambda t: None if t is None else t.data_ptr()

    def call(**kw):
        v = dict(h=ctx._h, target=p(a["target"]), dtype=binding.BF16, ld=100, q=p(a["draft_logits"]), qd=binding.BF16, ldq=100,
                 draft=p(a["draft"]), dl=None, B=2, T=3, bonus=1, V=100, temp=1.0, tempd=1.0, ua=p(a["u_accept"]), un=p(a["u_next"]),
                 al=p(out["accept_len"]), nx=p(out["next"]), ap=p(out["accept_prob"]), s=None)
        v.update(kw)
        return L.dropmatch_verify_lossless(*v.values())

    out = ctx.verify_lossless(**a)
    assert call() == binding.OK
    for bad in (dict(h=None), dict(target=None), dict(target=p(a["target"]) + 1), dict(dtype=2), dict(dtype=-1), dict(ld=99), dict(q=p(a["draft_logits"]) + 1),
                dict(qd=7), dict(ldq=99), dict(draft=None), dict(B=-1), dict(T=-1), dict(bonus=2), dict(bonus=-1), dict(T=0, bonus=0),
                dict(V=0), dict(temp=0.0), dict(temp=-1.0), dict(temp=float("nan")), dict(temp=float("inf")), dict(tempd=0.0),
                dict(ua=None), dict(un=None), dict(al=None), dict(nx=None), dict(ap=None)):
        assert call(**bad) == binding.EINVAL, bad
    assert call(V=2 ** 30 + 1, ld=2 ** 31, ldq=2 ** 31) == binding.EUNSUPPORTED
    assert call(B=2 ** 26, T=2 ** 26) == binding.EUNSUPPORTED
    assert call(q=None, qd=9, ldq=0, tempd=-1.0) == binding.OK       # not looked at without draft logits
    torch.cuda.synchronize()
    for name, value in (("target", a["target"].cpu()), ("target", a["target"].double()), ("target", a["target"].transpose(1, 2)),
                        ("target", a["target"][:, :2]), ("draft", a["draft"].long()), ("draft", a["draft"][:1]),
                        ("draft_logits", a["draft_logits"][:, :2]), ("draft_logits", a["draft_logits"].half()),
                        ("u_accept", a["u_accept"][:, :2]), ("u_next", a["u_next"].double()), ("draft_len", torch.zeros(3, dtype=torch.int32, device=DEV))):
        with pytest.raises(TypeError):
            ctx.verify_lossless(**{**a, name: value})
