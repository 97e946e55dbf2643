"""dropmatch_verify_lossless over serving batches: numbers of sequences and vocabularies that give a draw each of its launch
shapes (clusters of 512 threads while four CTAs or more per sequence run side by side, of 256 beyond; at most 16 CTAs, each
with 2048 entries or more; six where sequences are drawn in turns)."""
import pytest
import torch

import paper_2603_03333_b200 as pk
import engine_ref as ref
from test_gpu_lossless import check, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("target,draft", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", None), ("f32", None)])
@pytest.mark.parametrize("B,T,V", [(17, 2, 33003), (33, 3, 12293), (40, 3, 40009), (64, 2, 24593), (77, 2, 16001), (110, 2, 12301), (113, 1, 20011),
                                   (210, 2, 12299), (250, 1, 30011)])
def test_serving_batches(ctx, B, T, V, target, draft):
    check(ctx, make(B, T, V, target, draft, seed=B, ragged=B % 2 == 1), T=0.8 if B % 3 else 1.0, Td=1.25 if B % 4 else 1.0)


@pytest.mark.parametrize("draft", ["f32", "bf16"])
def test_every_sequence_rejects(ctx, draft):
    """Draws from max(p - q, 0) in all of a batch's clusters."""
    for B, V in ((48, 20011), (100, 14001), (220, 12289)):
        a = make(B, 2, V, "f32", draft, seed=B)
        a["u_accept"].fill_(1.0 - 2.0 ** -24)
        a["draft"] = (a["draft_logits"].float() - a["target"][:, :2]).argmax(2).to(torch.int32)
        assert int(check(ctx, a)["accept_len"].max()) == 0


@pytest.mark.parametrize("descending", [False, True])
def test_rows_in_order_draw_by_draw(ctx, descending):
    a = make(300, 5, 20001, "bf16", "bf16", seed=3, scale=0.5)
    for k in ("target", "draft_logits"):
        a[k].copy_(torch.sort(a[k], dim=2, descending=descending).values)
    check(ctx, a)


@pytest.mark.parametrize("target,draft", [("bf16", "bf16"), ("f32", "f32"), ("bf16", None)])
def test_a_sequence_alone_and_in_a_large_batch(ctx, target, draft):
    """Decisions and draws are the same; accept_prob, whose sums are split by the number of rows in the call, up to its error."""
    a = make(96, 3, 40009, target, draft, seed=12, ragged=True)
    whole = check(ctx, a)
    tol = 2 * ref.accept_tol(40009, draft is not None)
    for b in range(0, 96, 7):
        got = ctx.verify_lossless(**{k: (v[b:b + 1].contiguous() if torch.is_tensor(v) else v) for k, v in a.items()})
        assert torch.equal(got["accept_len"][0], whole["accept_len"][b]) and torch.equal(got["next"][0], whole["next"][b])
        assert bool(((got["accept_prob"][0] - whole["accept_prob"][b]).abs() <= tol * whole["accept_prob"][b] + 2.0 ** -126).all())
