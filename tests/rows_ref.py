"""Plain 64-bit statements of the operators on rows of logits, and the error bounds of the CUDA path.

Bounds.  Let u = 2^-24 (half a step of fp32, relative).  A row's exponentials are 2^w with
w = (x - m) * log2(e)/T: two roundings and the rounding of the factor give w a relative error of 3u,
hence exp a relative error of 3u * |z| (z = w ln 2, at most Z in magnitude for entries that matter:
what lies below 2^-126 is dropped) plus 4u for the exponential instruction (two steps).  A thread adds
its V / 256 entries (or fewer) one after another and some 20 more additions join threads and blocks:
relative error of a sum of positive terms at most (V/256 + 20) u.  So sums, probabilities and
log-probabilities are off by at most
    delta = u * (V/256 + 24 + 6 Z)
relative (sums, probabilities) or absolute (log of a sum; a log-probability adds 2u * |z| for its own
z).  The entropy adds sum p |z| with the same relative error per term."""
import torch

U = 2.0 ** -24


def stats(x, T):
    """x[N,V] float64 -> z - max, lse, log p, p, entropy, with the conventions for masked rows."""
    m = x.amax(1, keepdim=True)
    dead = torch.isinf(m) & (m < 0)
    bad = torch.isnan(x).any(1, keepdim=True) | (x == float("inf")).any(1, keepdim=True)
    z = (x - torch.where(dead, torch.zeros_like(m), m)) / T
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    lp = torch.where(torch.isinf(z) & (z < 0), torch.full_like(z, float("-inf")), z - log_total)
    p = torch.where(dead, torch.zeros_like(e), e / total)
    lse = torch.where(dead, m, m / T + log_total)
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1, keepdim=True)
    nan = torch.full_like(m, float("nan"))
    lse, entropy = torch.where(bad, nan, lse), torch.where(bad, nan, entropy)
    lp = torch.where(bad, nan.expand_as(lp), lp)
    p = torch.where(bad, nan.expand_as(p), p)
    return z, lse[:, 0], lp, p, entropy[:, 0]


def logprobs(x, tokens, n_top, T):
    x = x.double()
    V = x.shape[1]
    z, lse, lp, p, entropy = stats(x, T)
    lse, lp = lse.float().double(), lp.float().double()      # what lies past fp32's range is infinite there
    out = dict(lse=lse, entropy=entropy)
    if tokens is not None:
        t = tokens.long()
        have = (t >= 0) & (t < V)
        given = lp.gather(1, t.clamp(0, V - 1)[:, None])[:, 0]
        out["logprob"] = torch.where(have, given, torch.zeros_like(given))
    if n_top:
        # NaN first, then decreasing, equal entries by id; -0 equals 0
        ids = torch.sort(x + 0.0, dim=1, descending=True, stable=True).indices[:, :n_top]
        out["top_ids"] = ids.to(torch.int32)
        out["top_logprob"] = lp.gather(1, ids)
    return out


def logprobs_grad(x, tokens, g_lp, g_h, T):
    x = x.double()
    N, V = x.shape
    _, _, lp, p, entropy = stats(x, T)
    t = tokens.long() if tokens is not None else torch.full((N,), -1, device=x.device)
    have = (t >= 0) & (t < V)
    gl = torch.where(have, g_lp.double(), 0.0) if g_lp is not None else torch.zeros(N, dtype=x.dtype, device=x.device)
    gh = g_h.double() if g_h is not None else torch.zeros(N, dtype=x.dtype, device=x.device)
    plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    g = -gl[:, None] * p - gh[:, None] * (plp + p * entropy[:, None])
    g.scatter_add_(1, t.clamp(0, V - 1)[:, None], gl[:, None])
    none = ((gl == 0) & (gh == 0)) | (x == float("-inf")).all(1)
    return torch.where(none[:, None], torch.zeros_like(g), g) / T


def distill(x, ids, v, bucket, T, weight=None):
    """-> loss[N], grad[N,V] (of sum weight * loss)."""
    x = x.double()
    N, V = x.shape
    _, _, lp, p, _ = stats(x, T)
    i = ids.long()
    have = (i >= 0) & (i < V)
    i = i.clamp(0, V - 1)
    v = torch.where(have, v.double(), torch.full_like(v, float("-inf"), dtype=torch.float64))
    if bucket:
        q = torch.exp(v)
    else:
        top = v.amax(1, keepdim=True)
        e = torch.exp(v - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = e.sum(1, keepdim=True)
        q = torch.where(total > 0, e / total, torch.zeros_like(e))
    mass = q.sum(1)
    term = q * (torch.log(q) - lp.gather(1, i))
    loss = torch.where(q > 0, term, torch.zeros_like(term)).sum(1)
    seen = torch.zeros((N, V + 1), dtype=torch.bool, device=x.device)
    seen = seen.scatter(1, torch.where(have, i, torch.full_like(i, V)), True)[:, :V]
    g = p * mass[:, None]
    if bucket:
        qt = torch.where(seen.all(1), torch.zeros_like(mass), (1.0 - mass).clamp(min=0.0))
        pt = torch.where(seen, torch.zeros_like(p), p).sum(1)
        dead = (x == float("-inf")).all(1)
        extra = qt * (torch.log(qt) - torch.log(pt))
        loss = loss + torch.where((qt > 0) & ~(dead & (mass == 0)), extra, torch.zeros_like(extra))
        in_tail = torch.where(pt[:, None] > 0, p * (qt / pt)[:, None], torch.zeros_like(p))
        g = p * (mass + qt)[:, None] - torch.where(seen, torch.zeros_like(p), in_tail)
    g = g.scatter_add(1, i, torch.where(have, -q, torch.zeros_like(q)))
    w = (weight.double() if weight is not None else torch.ones(N, dtype=x.dtype, device=x.device))[:, None]
    none = (w == 0) | (x == float("-inf")).all(1, keepdim=True)
    return loss, torch.where(none, torch.zeros_like(g), g * w / T)


def delta(V, Z=100.0):
    return U * (V / 256 + 24 + 6 * Z)


def same(got, want, tol):
    """Finite where the reference is, equal infinities and NaNs, and within tol (tensor or number)."""
    got = got.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fin = torch.isfinite(want)
    assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)])
    assert torch.isfinite(got[fin]).all()
    err = (got - want).abs()
    tol = torch.as_tensor(tol, dtype=torch.float64, device=got.device).expand_as(err)
    bad = fin & ~(err <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} out of tolerance, worst {float((err - tol)[fin].max()):.3g} over"
