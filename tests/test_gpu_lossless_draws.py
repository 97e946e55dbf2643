"""Draws of dropmatch_verify_lossless where target and draft agree on most of the vocabulary, so that much of the mass lies
next to the border p = q that max(p - q, 0) is cut at.

What is compared.  Accepted lengths are equal.  The drawn token v is the first whose cumulative weight exceeds the
place u sum r.  Exponentials are good to e = 2^-42, so that p and q, each with its sum, are off by at most 2 e, a cumulative
sum of p - q by 4 e, and so is its total: the place is right up to 8 e / sum r.  An fp64 sum adds up at most V / 256 terms
in a thread (256 at least share a row) and some 32 over threads and CTAs; sums over p, q, and the two that make up a
cumulative sum and its total: less than 8 (V / 256 + 32) 2^-53 / sum r.  The statement is in 80-bit numbers.  A token is right iff its
own interval of the cumulative sum, widened by that, holds the place, and it has weight itself (more than half of
the 2^-40 p below which a difference counts as 0)."""
import numpy as np
import pytest
import torch

import paper_2603_03333_b200 as pk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NINF = float("-inf")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LAST = 1.0 - 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    c.close()


def residual(x, y):
    """p, max(p - q, 0) and its cumulative sum for one row of either model, as 80-bit numbers."""
    p, q = (np.exp((t := v.double().cpu().numpy().astype(np.longdouble)) - t.max()) for v in (x, y))
    p, q = p / p.sum(), q / q.sum()
    r = np.where(p - q < 2.0 ** -40 * p, 0, p - q)
    return p, q, np.cumsum(r)


def place_error(V, total):
    return float((8 * 2.0 ** -42 + 8 * (V / 256 + 32) * 2.0 ** -53) / total)


def check_rejected(ctx, x, y, token, u_next):
    """Rows x, y [B,V] of target and draft, the drafted token of each sequence rejected: the next token."""
    B, V = x.shape
    out = ctx.verify_lossless(x[:, None].contiguous(), token[:, None], torch.full((B, 1), LAST, device=DEV), u_next,
                              draft_logits=y[:, None].contiguous())
    assert out["accept_len"].tolist() == [0] * B
    got, wrong = out["next"].tolist(), []
    for b in range(B):
        p, q, cum = residual(x[b], y[b])
        total, v, u = cum[-1], got[b], float(u_next[b])
        assert total > 0
        tol = place_error(V, total)
        ok = 0 <= v < V and p[v] - q[v] >= 2.0 ** -41 * p[v]
        ok = ok and cum[v] / total >= u - tol and (v == 0 or cum[v - 1] / total <= u + tol)
        if not ok:
            wrong.append((b, u, int(np.searchsorted(cum, u * total, side="right")), v, float(total)))
    assert not wrong, (len(wrong), wrong[:5])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5000, 50000])
@pytest.mark.parametrize("apart", [0.0, 1e-8, 7.6e-8, 3e-7, 1e-6, -1e-8, -7.6e-8, -3e-7, -1e-6])
def test_two_logits_exchanged(ctx, dtype, V, apart):
    """Draft and target are equal but for two logits that change places, and a third that makes the sums of
    their exponentials differ by a share of `apart`: the bulk's p exceeds its q by that share."""
    B = 48
    x = torch.randn((B, V), generator=torch.Generator(device=DEV).manual_seed(V), device=DEV) * 2.0
    i, j, k = V // 2 + 7, V // 3, V // 5
    x[:, i], x[:, j], x[:, k] = 9.0, 3.0, 0.0
    x = x.to(DT[dtype])
    y = x.clone()
    y[:, i], y[:, j] = x[:, j], x[:, i]
    if apart != 0.0:
        mass = abs(apart) * torch.exp(x.double()).sum(1)
        if dtype == "f32":
            y[:, k] = torch.log1p(mass if apart > 0 else -mass).float()
        else:       # only one of the two models has the entry
            one, other = (y, x) if apart > 0 else (x, y)
            one[:, k], other[:, k] = torch.log(mass).to(DT[dtype]), NINF
    u = torch.arange(B, device=DEV, dtype=torch.float32) * 1e-6
    u[0], u[1] = 0.0, 2.0 ** -24
    check_rejected(ctx, x, y, torch.full((B,), j, dtype=torch.int32, device=DEV), u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("noise", [0.003, 0.01])
@pytest.mark.parametrize("B,V", [(4, 151936), (64, 151936), (16, 20011)])
def test_a_close_drafter(ctx, dtype, noise, B, V):
    """A drafter like a quantised copy of the target, all its p / q within a percent; u_next next to borders of the
    cumulative sum, beyond what the exponentials' error explains."""
    g = torch.Generator(device=DEV).manual_seed(B)
    x = torch.randn((B, V), generator=g, device=DEV)
    y = (x + noise * torch.randn((B, V), generator=g, device=DEV)).to(DT[dtype])
    x = x.to(DT[dtype])
    u = torch.empty((B,), device=DEV)
    for b in range(B):
        cum = residual(x[b], y[b])[2]
        tol, border = place_error(V, cum[-1]), cum[:-1] / cum[-1]
        single = border.astype(np.float32)
        off = np.abs(single - border)          # of the borders that lie just further than that from an fp32 number, one
        near = np.flatnonzero((off > 1.1 * tol) & (off < 2.0 * tol) & (single < 1))
        near = near if len(near) else np.flatnonzero((off > 1.1 * tol) & (single < 1))
        u[b] = float(single[near[b * 7919 % len(near)]])
    check_rejected(ctx, x, y, (y.double() - x.double()).argmax(1).to(torch.int32), u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_first_and_last_places_of_a_close_drafter(ctx, dtype):
    for noise in (1e-4, 0.003, 0.1):
        g = torch.Generator(device=DEV).manual_seed(3)
        x = torch.randn((24, 30011), generator=g, device=DEV)
        y = (x + noise * torch.randn(x.shape, generator=g, device=DEV)).to(DT[dtype])
        x = x.to(DT[dtype])
        y[:, 17] = x[:, 17] + 0.5          # (bf16 rows may be equal otherwise)
        u = torch.tensor([0.0, 2.0 ** -24, 2.0 ** -149, LAST], device=DEV).repeat(6)
        check_rejected(ctx, x, y, torch.full((24,), 17, dtype=torch.int32, device=DEV), u)
