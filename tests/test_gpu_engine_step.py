"""The operators around a speculative engine's step, together as they are used: 8-bit heads whose logits are
verified against each other, and a draft head's training step under the verifier's dropout."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding
import engine_ref as ref
import rows_ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    assert c.device_error() == 0
    c.close()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,T,V,d", [(1, 1, 33, 64), (6, 3, 5003, 256), (40, 4, 3001, 200)])
def test_eight_bit_heads_and_lossless_verification(ctx, B, T, V, d, dtype):
    """Target and draft project through their 8-bit heads, the draft's tokens are drawn from its logits, verified, and the
    emitted tokens' log-probabilities looked at; eagerly and replayed from a graph on new hidden states."""
    g = gen(V)
    Wt, st = ctx.quantize_i8(torch.randn((V, d), generator=g, device=DEV) * 0.2)
    Wd, sd = ctx.quantize_i8(Wt.float() * st[:, None] + torch.randn((V, d), generator=g, device=DEV) * 0.02)
    H = torch.randn((B, T + 1, d), generator=g, device=DEV).to(dtype)
    noise = torch.rand((B, T, V), generator=g, device=DEV).clamp(1e-7, 1 - 1e-7)
    ua, un = torch.rand((B, T), generator=g, device=DEV), torch.rand((B,), generator=g, device=DEV)

    def step():
        target = ctx.linear_i8(H, Wt, st)
        draft_logits = ctx.linear_i8(H[:, :T].contiguous(), Wd, sd)
        draft = (draft_logits.float() - torch.log(-torch.log(noise))).argmax(2).to(torch.int32)
        out = ctx.verify_lossless(target, draft, ua, un, draft_logits=draft_logits)
        emitted = torch.cat([draft, torch.zeros_like(draft[:, :1])], 1)
        emitted.scatter_(1, out["accept_len"].long()[:, None], out["next"][:, None])
        return target, draft_logits, draft, out, emitted, ctx.logprobs(target, emitted)["logprob"]

    def check(target, draft_logits, draft, out, emitted, logprob):
        n, nxt, prob = ref.lossless(target, draft, ua, un, draft_logits)
        assert torch.equal(out["accept_len"].cpu(), n) and torch.equal(out["next"].cpu(), nxt)
        assert bool(((out["accept_prob"].double().cpu() - prob).abs() <= ref.accept_tol(V, True) * prob + 2.0 ** -126).all())
        q, scale = ref.quantize(H.reshape(-1, d))
        want = ((q @ Wt.double().T) * st.double() * scale[:, None]).view(B, T + 1, V)
        tol = want.abs() * (3 * ref.U + ref.half_step(dtype) * (1 + 2.0 ** -6)) + 2.0 ** -126
        assert bool(((target.double() - want).abs() <= tol).all())
        lp = torch.log_softmax(target.double(), 2).gather(2, emitted.long()[:, :, None])[:, :, 0]
        rows_ref.same(logprob, lp, rows_ref.delta(V) + 4 * ref.U * lp.abs())

    check(*step())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (1, 2):
        H.copy_(torch.randn(H.shape, generator=gen(seed), device=DEV).to(dtype))
        graph.replay()
        torch.cuda.synchronize()
        check(*captured)


@pytest.mark.parametrize("K", [1, 5, 40])
def test_training_step_under_the_verifiers_dropout(ctx, K):
    """Hidden rows -> K masked copies -> head -> distillation -> gradient of the hidden rows, against 64 bits."""
    B, T, d, V, k, p, seed = 2, 3, 96, 700, 16, 0.2, 77
    g = gen(K)
    x = torch.randn((B, T, d), generator=g, device=DEV)
    W = torch.randn((V, d), generator=g, device=DEV) * 0.2
    ids = torch.randint(0, V, (B, T, K, k), generator=g, device=DEV, dtype=torch.int32)
    val = torch.randn((B, T, K, k), generator=g, device=DEV)
    weight = torch.rand((B, T, K), generator=g, device=DEV)
    masked = ctx.dropout(x, K, p, seed)
    logits = masked @ W.T
    step = ctx.distill(logits, ids, val, tail=binding.TAIL_RENORM, weight=weight, grad=True)
    grad = ctx.dropout_grad(step["grad"] @ W, p, seed)

    keep = ref.keep_flags(B, T, K, d, p, seed).to(DEV)
    s = 1.0 / (1.0 - ref.single(p))
    x64 = x.double().requires_grad_(True)
    m64 = torch.where(keep, x64[:, :, None] * s, torch.zeros((), dtype=torch.float64, device=DEV))
    l64 = m64 @ W.double().T
    lp = torch.log_softmax(l64, 3)
    q = torch.zeros_like(lp).scatter_add(3, ids.long(), torch.softmax(val.double(), 3))
    loss = -(q.detach() * lp).sum(3)                  # the teacher's entropy is a constant
    want = torch.autograd.grad((loss * weight.double()).sum(), x64)[0]
    # bounds: the copies carry 2u (scale and product), the head's sums of d terms (d + 2)u of their magnitudes; that is an
    # absolute error of a logit, and with rows_ref.delta a relative one of its probability (the row's log-sum-exp moves
    # by as much); then V-term sums, K-term sums, the factor
    u = ref.U
    dl = weight.double()[..., None] * (lp.exp() - q)
    logit_err = ((d + 4) * u * (m64.abs() @ W.double().abs().T)).amax(3, keepdim=True)
    dl_err = weight.double()[..., None] * (lp.exp() * (2 * logit_err + rows_ref.delta(V)) * (1 + 2.0 ** -6) + q * 4 * u) + 4 * u * dl.abs()
    copy_err = dl_err @ W.double().abs() + (V + 2) * u * ((dl.abs() + dl_err) @ W.double().abs())
    copy = dl @ W.double()
    tol = s * ((copy_err * keep).sum(2) + (K + 4) * u * ((copy.abs() + copy_err) * keep).sum(2))
    assert bool(((grad.double() - want.detach()).abs() <= tol.detach()).all())
    # and the slope along a direction agrees with differences of the 64-bit loss
    h = torch.randn(x.shape, generator=g, device=DEV).double()
    eps = 1e-4

    def objective(v):
        m = torch.where(keep, v[:, :, None] * s, torch.zeros((), dtype=torch.float64, device=DEV))
        return float((-(q * torch.log_softmax(m @ W.double().T, 3)).sum(3) * weight.double()).sum())

    slope = (objective(x.double() + eps * h) - objective(x.double() - eps * h)) / (2 * eps)
    got = float((grad.double() * h).sum())
    # central differences: eps^2 / 6 times a third derivative, here below 1e3 |slope's terms|; rounding 1e-12 / eps
    assert abs(slope - got) <= float((tol.detach() * h.abs()).sum()) + 1e-5 * float((want.detach().abs() * h.abs()).sum())
