"""Plain 64-bit statements of lossless verification, of dropout on rows and of the projection through 8-bit
integers, and the error bounds of the CUDA path.

Lossless verification.  Accepted lengths and next tokens are those of 64-bit arithmetic: they are equal.
out_accept_prob is fp32: a term of a row's sum is 2^w, w = (x - m) log2(e)/T for a reference m of which the maximum is at
most the 2^20-fold, with three roundings in w (the difference, the rounded factor, the product: 3 |w| ln 2 u for
u = 2^-24) and one instruction of 2^-22 = 4u; |w| ln 2 averaged under the row's own distribution is at most ln V + 20 ln 2.
Seven additions per batch, batches joined with compensation; three joins (lanes, warps, CTAs) of one
exponential (4u and its own part of |w|) and at most 5 additions each.  A sum is off by at most
(3 (ln V + 14) + 4 + 7 + 30) u relative; p / q has two of them, two logarithms' worth of u, and one rounding.

Dropout.  x * s is one product and one rounding to the storage type; s = 1 / (1 - p) is rounded to fp32.  The gradient
adds up to K fp32 values (K u sum |g|), times s, rounded once.

8-bit integers.  Quantisation and integer sums are exact.  The sum's conversion to fp32, two products with scales and the
rounding to fp32 or bf16: (3 u + half a step) relative."""
import math

import numpy as np
import torch

from philox_ref import philox4x32_10

U = 2.0 ** -24


def single(x):
    return float(np.float32(x))


def accept_tol(V, with_q):
    one = (3 * (math.log(max(V, 2)) + 14) + 41) * U
    return one * (2 if with_q else 1) + 4 * U


def softmax64(x, T):
    """x[V] -> probabilities; all 0 for a row of nothing but -inf; NaN for a row with a NaN or +inf."""
    x = x.double()
    if bool(torch.isnan(x).any()) or bool((x == float("inf")).any()):
        return torch.full_like(x, float("nan"))
    m = x.max()
    if m == float("-inf"):
        return torch.zeros_like(x)
    e = torch.exp((x - m) / single(T))
    return e / e.sum()


def log_prob(x, j, T):
    """log of softmax64(x, T)[j], which may lie below what fp64 holds as a probability."""
    x = x.double()
    m = x.max()
    return float((x[j] - m) / single(T) - torch.log(torch.exp((x - m) / single(T)).sum()))


def lossless(target, draft, u_accept, u_next, draft_logits=None, draft_len=None, T=1.0, Td=1.0):
    """One Python loop per sequence and position; tensors on any device."""
    B, rows, V = target.shape
    n_draft = draft.shape[1]
    lens, nexts, prob = [], [], torch.zeros((B, n_draft), dtype=torch.float64)
    for b in range(B):
        length = n_draft if draft_len is None else min(n_draft, max(0, int(draft_len[b])))
        n, going = 0, True
        for t in range(length):
            x, u = int(draft[b, t]), float(u_accept[b, t])
            p = softmax64(target[b, t], T)
            q = softmax64(draft_logits[b, t], Td) if draft_logits is not None else None
            bad = bool(torch.isnan(p[0])) or (q is not None and bool(torch.isnan(q[0])))
            there = 0 <= x < V
            if bad:
                prob[b, t] = float("nan")
                ok = False
            elif not there or float(target[b, t, x]) == float("-inf"):
                ok = False                                    # p(x) = 0
            elif q is not None and float(draft_logits[b, t, x]) == float("-inf"):
                prob[b, t], ok = 1.0, True                    # q(x) = 0 < p(x)
            else:
                ratio = log_prob(target[b, t], x, T) - (0.0 if q is None else log_prob(draft_logits[b, t], x, Td))
                prob[b, t] = math.exp(min(0.0, ratio))
                ok = u == 0.0 or u < math.exp(min(ratio, 1.0))
            going = going and ok
            n += int(going)
        lens.append(n)
        if n >= rows:
            nexts.append(-1)
            continue
        p = softmax64(target[b, n], T)
        r = p
        if n < length:
            x = int(draft[b, n])
            if draft_logits is not None:
                r = p - softmax64(draft_logits[b, n], Td)
                r = torch.where(r < 2.0 ** -40 * p, torch.zeros_like(r), r)     # (a NaN stays)
            else:
                r = p.clone()
                if 0 <= x < V:
                    r[x] = 0.0
        if float(r.sum()) == 0:      # (a NaN in either row: nothing to draw from)
            r = p
        total = r.sum()
        if not float(total) > 0:
            nexts.append(-1)
            continue
        cum = torch.cumsum(r, 0)
        v = int((cum <= float(u_next[b]) * cum[-1]).sum())
        positive = torch.nonzero(r > 0)[:, 0]
        nexts.append(min(v, int(positive[-1])))
    return torch.tensor(lens, dtype=torch.int32), torch.tensor(nexts, dtype=torch.int32), prob


def keep_flags(B, T, K, d, p, seed, seq_base=0, per_path=False):
    """bool[B,T,K,d] of the mask rule, from the numpy generator."""
    quads = (d + 3) // 4
    b, t, i, j = np.meshgrid(np.arange(B), np.arange(T), np.arange(K), np.arange(quads), indexing="ij")
    if per_path:
        t = np.zeros_like(t)
    ctr = np.stack([j, i, t, (b + seq_base) & 0xFFFFFFFF], axis=-1).astype(np.uint64)
    key = np.array([seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF], dtype=np.uint64)
    words = philox4x32_10(ctr, np.broadcast_to(key, (*ctr.shape[:-1], 2)))
    thr = math.floor(single(p) * 2.0 ** 32)
    return torch.from_numpy((words.reshape(B, T, K, quads * 4)[..., :d] >= np.uint32(thr)))


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def quantize(x):
    """(q float64 holding whole numbers, scale float64): the definition, every rounding in its place."""
    x = x.double()
    bad = ~torch.isfinite(x).all(1)
    amax = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(1) if x.shape[1] else x.new_zeros(x.shape[0])
    scale = (amax / 127.0).float().clamp(min=2.0 ** -126).double()
    q = torch.round((torch.where(bad[:, None], torch.zeros_like(x), x) / scale[:, None]).float()).double()
    return q, torch.where(bad, torch.full_like(scale, float("nan")), scale)
