"""dropmatch_dropout and its gradient on calls large enough that a lane takes two vectors of a row and a warp all
or several paths of its chunk, against the mask rule in plain integer operations."""
import math

import pytest
import torch

import paper_2603_03333_b200 as pk
import engine_ref as ref

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED = 0xD1B54A32D192ED03


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    c.close()


def keep_flags(B, T, K, d, p, seed, seq_base, device):
    """bool[B,T,K,d] of the mask rule: Philox4x32-10 in 64-bit integers (products modulo 2^64 hold both halves)."""
    low, dev = 0xFFFFFFFF, dict(dtype=torch.int64, device=device)
    c0 = torch.arange((d + 3) // 4, **dev)[None, None, None]
    c1 = torch.arange(K, **dev)[None, None, :, None]
    c2 = torch.arange(T, **dev)[None, :, None, None]
    c3 = ((torch.arange(B, **dev) + seq_base) & low)[:, None, None, None]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, c = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((c >> 32) & low) ^ c1 ^ k0, c & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), dim=-1).reshape(B, T, K, -1)[..., :d]
    return words >= math.floor(ref.single(p) * 2.0 ** 32)


def test_the_mask_rule_in_integers():
    for args in ((2, 3, 4, 21, 0.3, SEED, 2 ** 32 - 1), (1, 5, 2, 64, 0.05, 7, 2 ** 40 + 3)):
        assert torch.equal(keep_flags(*args, "cpu"), ref.keep_flags(*args))


def rows_of(lead, d, dtype, pad, offset):
    """Memory, and in it a view [*lead, d] with `pad` entries between its rows."""
    n = 1
    for k in lead:
        n *= k
    buf = torch.full((offset + n * (d + pad) + 5,), 77.0, dtype=dtype, device=DEV)
    view = buf[offset:offset + n * (d + pad)].view(*lead, d + pad)[..., :d]
    return buf, view


def compare(ctx, B, T, K, d, dtype, pad, offset, p=0.3, seq_base=11):
    g = torch.Generator(device=DEV).manual_seed(d)
    keep = keep_flags(B, T, K, d, p, SEED, seq_base, DEV)
    s = torch.tensor(ref.single(1.0 / (1.0 - ref.single(p))), device=DEV)
    x = rows_of((B, T), d, dtype, pad, offset)[1]
    x.copy_(torch.randn((B, T, d), generator=g, device=DEV))
    buf, out = rows_of((B, T, K), d, dtype, pad, offset)
    ctx.dropout(x, K, p, SEED, seq_base=seq_base, out=out)
    # one product and one rounding: equal bits
    assert torch.equal(out, torch.where(keep, (x.float() * s)[:, :, None], torch.zeros((), device=DEV)).to(dtype))
    out.fill_(77.0)
    assert bool((buf == 77.0).all())
    gr = rows_of((B, T, K), d, dtype, pad, offset)[1]
    gr.copy_(torch.randn((B, T, K, d), generator=g, device=DEV))
    buf, out = rows_of((B, T), d, dtype, pad, offset)
    ctx.dropout_grad(gr, p, SEED, seq_base=seq_base, out=out)
    masked = torch.where(keep, gr.double(), torch.zeros((), dtype=torch.float64, device=DEV))
    factor = 1.0 / (1.0 - ref.single(p))
    want = masked.sum(2) * factor
    # K additions and the product, its factor rounded, in fp32; one rounding to dtype
    tol = masked.abs().sum(2) * factor * (K + 3) * ref.U + want.abs() * ref.half_step(dtype) * (1 + 2.0 ** -8)
    assert bool(((out.double() - want).abs() <= tol).all())
    out.fill_(77.0)
    assert bool((buf == 77.0).all())


# (pads that make rows of either type whole 16-byte vectors, of none, and rows that start 16-byte aligned but for the offset)
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,pad", [("bf16", 1101, 3), ("bf16", 1101, 0), ("bf16", 1104, 0), ("bf16", 520, 0), ("f32", 701, 3), ("f32", 701, 0),
                                         ("f32", 702, 0), ("f32", 703, 0), ("f32", 704, 0), ("f32", 257, 3)])
@pytest.mark.parametrize("offset", [0, 1])
def test_two_vectors_a_lane(ctx, dtype, d, pad, offset):
    for B, T, K in ((3, 400, 1), (2, 600, 3), (1, 1200, 18)):
        compare(ctx, B, T, K, d, DT[dtype], pad, offset)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 264), ("bf16", 263), ("f32", 200), ("f32", 131)])
def test_several_paths_a_warp(ctx, dtype, d):
    """Rows of one vector a lane, and so few warps' worth of them that paths are dealt out in runs of two or more."""
    for T, K in ((1300, 7), (700, 9), (300, 40)):
        compare(ctx, 1, T, K, d, DT[dtype], 0, 0)
        compare(ctx, 1, T, K, d, DT[dtype], 5, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_paths_of_long_rows(ctx, dtype):
    """Gradient sums joined over two, four and eight warps, with two vectors a lane."""
    for T, K, d in ((300, 16, 4999), (260, 33, 4999), (240, 70, 5000)):
        compare(ctx, 1, T, K, d, DT[dtype], 0, 0)
