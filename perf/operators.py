"""Measured cases of the vocabulary-row operators: scoring hidden states against the LM head, log
probabilities over rows of logits with their gradient, and distillation from a teacher's top tokens.

A case is a dict of plain values.  `run` computes it in plain torch operations, or, where `own` is
true, through the library's entry points; `exact` computes it in 64 bits from the definitions.

  score          H[N,d], W[V,d], tokens[N]      -> log-probability of the given token, entropy, log-sum-exp
                 and the top alternatives under Softmax(H W^T / temperature)
  logprobs       logits[N,V], tokens[N]         -> the same over logits in memory
  logprobs_grad  ... and the two upstream gradients -> the gradient of the logits
  distill        logits[N,V], the teacher's top ids and log-probabilities [N,k], row weights [N]
                 -> KL(teacher || student) of every row and, with `grad`, the logits' gradient
"""
import math

import torch

own = False

DEVICE = "cuda"
_handle = None


# ------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # the toy head (fp32, CUDA cores): four positions of a draft; the smallest call, all latency
        dict(name="score_toy", op="score", dtype="f32", rows=4, d=256, vocab=4096, top=5, temp=1.0),
        # one decoding step of one sequence on the Llama-3-8B head, five alternatives for the client
        dict(name="score_token_llama8b", op="score", dtype="bf16", rows=1, d=4096, vocab=128256, top=5, temp=1.0),
        # the positions of a drafted tree on the Qwen3-8B head, log-probabilities only (no alternatives)
        dict(name="score_tree_qwen8b", op="score", dtype="bf16", rows=61, d=4096, vocab=151936, top=0, temp=0.7),
        # teacher pass over a stretch of text on the Llama-3-70B head: 32 alternatives a position, odd row count
        dict(name="score_teacher_llama70b", op="score", dtype="bf16", rows=509, d=8192, vocab=128256, top=32, temp=1.0),
        # a sampler's own logits row, fp32, most of the vocabulary forbidden by a grammar
        dict(name="logprobs_token_masked", op="logprobs", dtype="f32", rows=1, vocab=128256, top=20, temp=1.0, masked=0.9),
        # evaluation of a text on a head of odd vocabulary size (rows start off 16-byte boundaries)
        dict(name="logprobs_odd_vocab", op="logprobs", dtype="bf16", rows=333, vocab=32003, top=8, temp=1.3, masked=0.0),
        # evaluation of a long text on the Qwen3-8B vocabulary
        dict(name="logprobs_text_qwen8b", op="logprobs", dtype="bf16", rows=2047, vocab=151936, top=5, temp=1.0, masked=0.0),
        # policy-gradient step of a draft model: gradient through log-probability and entropy, fp32 logits
        dict(name="logprobs_grad_f32", op="logprobs_grad", dtype="f32", rows=513, vocab=128256, temp=1.0, masked=0.0),
        # the same in bf16 on an odd vocabulary
        dict(name="logprobs_grad_odd_vocab", op="logprobs_grad", dtype="bf16", rows=1021, vocab=32003, temp=0.9, masked=0.0),
        # a few positions on a tiny vocabulary: the launch is the cost
        dict(name="distill_tiny", op="distill", dtype="bf16", rows=8, vocab=999, top=16, temp=1.0, tail="renorm", grad=True),
        # validation of a draft model: loss only, teacher's rest of the mass in one bucket
        dict(name="distill_loss_bucket", op="distill", dtype="f32", rows=97, vocab=151936, top=128, temp=2.0, tail="bucket", grad=False),
        # training step of a draft model on the Llama-3-8B vocabulary: loss and gradient
        dict(name="distill_step_llama8b", op="distill", dtype="bf16", rows=1024, vocab=128256, top=64, temp=1.0, tail="bucket", grad=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["score", "logprobs", "logprobs_grad", "distill"])
    temp = round(rng.uniform(0.5, 2.0), 2)
    if op == "score":
        if rng.random() < 0.25:     # heads of the CUDA-core path: fp32, or a hidden size that is no multiple of 64
            dtype = rng.choice(["f32", "bf16"])
            return dict(op=op, dtype=dtype, rows=_spread(rng, 1, 64), d=8 * _spread(rng, 1, 128),
                        vocab=_spread(rng, 200, 32768), top=rng.choice([0, 1, 7, 32]), temp=temp)
        return dict(op=op, dtype="bf16", rows=_spread(rng, 1, 509), d=64 * _spread(rng, 1, 128),
                    vocab=_spread(rng, 1000, 128256), top=rng.choice([0, 1, 5, 20, 64]), temp=temp)
    dtype = rng.choice(["f32", "bf16"])
    vocab = _spread(rng, 200, 200000)
    rows = _spread(rng, 1, max(1, min(4096, 150_000_000 // vocab)))
    if op == "logprobs":
        return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, top=rng.choice([0, 1, 5, 20, 100]), temp=temp,
                    masked=rng.choice([0.0, 0.0, 0.5, 0.95]))
    if op == "logprobs_grad":
        return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, temp=temp, masked=rng.choice([0.0, 0.0, 0.5]))
    return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, top=rng.choice([1, 5, 16, 64, 128]), temp=temp,
                tail=rng.choice(["renorm", "bucket"]), grad=rng.random() < 0.7)


# ------------------------------------------------------------------------------------- the inputs

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _grid(shape, std, unit, dtype, g):
    """N(0, std^2) on a grid of `unit`, at most 255 steps of it: exact in bf16, and every sum of
    products of two such arrays is exact in fp32 in any order, so that the order of the alternatives
    (equal logits included) is a property of the inputs and not of a summation order."""
    out = torch.empty(shape, dtype=dtype, device=DEVICE)
    step = max(1, (1 << 27) // shape[1])
    for r in range(0, shape[0], step):
        n = min(step, shape[0] - r)
        x = torch.randn((n, shape[1]), generator=g, device=DEVICE).mul_(std / unit).round_().clamp_(-255, 255)
        out[r:r + n] = x.mul_(unit).to(dtype)
    return out


def _logits(case, g):
    """Rows as a language model gives them: a broad bulk and a few dozen likely tokens; `masked` of
    the vocabulary is forbidden (-inf)."""
    n, v = case["rows"], case["vocab"]
    x = torch.randn((n, v), generator=g, device=DEVICE).mul_(2.0)
    likely = torch.randint(0, v, (n, min(48, v)), generator=g, device=DEVICE)
    boost = torch.rand(likely.shape, generator=g, device=DEVICE) * 14.0
    x.scatter_add_(1, likely, boost)
    if case.get("masked", 0.0) > 0:
        drop = torch.rand((n, v), generator=g, device=DEVICE) < case["masked"]
        drop[:, 0] = False
        x.masked_fill_(drop, float("-inf"))
    return x.to(_dtype(case))


def _tokens(case, g):
    """Given tokens, one row in sixteen without one (padding, -1)."""
    n, v = case["rows"], case["vocab"]
    t = torch.randint(0, v, (n,), generator=g, device=DEVICE, dtype=torch.int32)
    return t.masked_fill_(torch.rand((n,), generator=g, device=DEVICE) < 1 / 16, -1)


def _context():
    """One library context for the operators that need no head, as a program keeps it."""
    global _handle
    if _handle is None:
        import paper_2603_03333_b200 as pk
        _handle = pk.Context(0)
    return _handle


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    s = dict(case)
    n, v = case["rows"], case["vocab"]
    if case["op"] == "score":
        if case["dtype"] == "f32":
            W = _grid((v, case["d"]), case["d"] ** -0.5, 2.0 ** -10, torch.float32, g)
            H = _grid((n, case["d"]), case["d"] ** -0.5, 2.0 ** -10, torch.float32, g)
        else:
            W = _grid((v, case["d"]), 0.02, 2.0 ** -11, torch.bfloat16, g)
            H = _grid((n, case["d"]), 1.0, 2.0 ** -5, torch.bfloat16, g)
        s.update(W=W, H=H, tokens=_tokens(case, g))
        if own:     # the context with its head and workspace, which a serving program keeps
            import paper_2603_03333_b200 as pk
            s["ctx"] = pk.Context(0)
            s["ctx"].set_head(W, max_rows=n)
            s["ctx"].enable_score(n, case["top"])
        return s
    s["logits"] = _logits(case, g)
    if own:
        s["ctx"] = _context()
    if case["op"] in ("logprobs", "logprobs_grad"):
        s["tokens"] = _tokens(case, g)
        if case["op"] == "logprobs_grad":
            s["g_logprob"] = torch.randn((n,), generator=g, device=DEVICE)
            s["g_entropy"] = torch.randn((n,), generator=g, device=DEVICE) * 0.01
        return s
    # the teacher agrees with the student up to noise; one entry in sixteen is padding (-1)
    z = s["logits"].float() / case["temp"]
    z += torch.randn(z.shape, generator=g, device=DEVICE)
    lse = torch.logsumexp(z, 1, keepdim=True)
    val, ids = z.topk(min(case["top"], v), dim=1)
    pad = torch.rand(ids.shape, generator=g, device=DEVICE) < 1 / 16
    s["ids"] = ids.masked_fill(pad, -1).to(torch.int32)
    s["teacher"] = (val - lse).contiguous()
    s["weight"] = torch.rand((n,), generator=g, device=DEVICE) / n
    return s


# ------------------------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "score":
        return _rows_plain(s["H"].float() @ s["W"].float().T, s)
    if s["op"] == "logprobs":
        return _rows_plain(s["logits"].float(), s)
    if s["op"] == "logprobs_grad":
        return _grad_plain(s)
    return _distill_plain(s)


def _run_own(s):
    ctx = s["ctx"]
    if s["op"] == "score":
        return ctx.score(s["H"], s["tokens"], n_top=s["top"], temperature=s["temp"])
    if s["op"] == "logprobs":
        return ctx.logprobs(s["logits"], s["tokens"], n_top=s["top"], temperature=s["temp"])
    if s["op"] == "logprobs_grad":
        return ctx.logprobs_grad(s["logits"], s["tokens"], s["g_logprob"], s["g_entropy"], temperature=s["temp"])
    from paper_2603_03333_b200 import binding
    tail = binding.TAIL_BUCKET if s["tail"] == "bucket" else binding.TAIL_RENORM
    return ctx.distill(s["logits"], s["ids"], s["teacher"], tail=tail, temperature=s["temp"], weight=s["weight"],
                       grad=s["grad"])


def _stats_plain(x, temp):
    """Log-sum-exp, probabilities and log-probabilities of the rows of x / temp.  The largest entry
    is taken out of the sum: next to a near-certain token it is the rest that decides."""
    m, first = x.max(1, keepdim=True)
    z = (x - m) / temp
    e = torch.exp(z)
    rest = e.scatter(1, first, 0.0).sum(1, keepdim=True)
    log_total = torch.log1p(rest)
    return m / temp + log_total, e / (1.0 + rest), z - log_total


def _rows_plain(logits, s):
    lse, p, logp = _stats_plain(logits, s["temp"])
    tok = s["tokens"].long()
    given = logp.gather(1, tok.clamp(min=0)[:, None])[:, 0]
    out = dict(logprob=torch.where(tok >= 0, given, 0.0), lse=lse[:, 0],
               entropy=-(torch.where(p > 0, p * logp, 0.0)).sum(1))
    if s["top"] > 0:
        val, ids = torch.sort(logits, dim=1, descending=True, stable=True)   # equal logits: the lower id first
        ids = ids[:, :s["top"]]
        out["top_ids"] = ids.to(torch.int32)
        out["top_logprob"] = logp.gather(1, ids)
    return out


def _grad_plain(s):
    _, p, logp = _stats_plain(s["logits"].float(), s["temp"])
    plogp = torch.where(p > 0, p * logp, 0.0)
    entropy = -plogp.sum(1, keepdim=True)
    tok = s["tokens"].long()
    g_lp = torch.where(tok >= 0, s["g_logprob"], 0.0)[:, None]
    grad = -g_lp * p - s["g_entropy"][:, None] * (plogp + entropy * p)
    grad.scatter_add_(1, tok.clamp(min=0)[:, None], g_lp)
    return (grad / s["temp"]).to(s["logits"].dtype)


def _distill_plain(s):
    lse, p, logp = _stats_plain(s["logits"].float(), s["temp"])
    n, vocab = p.shape
    have = s["ids"] >= 0
    ids = s["ids"].long().clamp(min=0)
    # the teacher's few entries in 64 bits: the rest of its mass is one minus their sum
    v = torch.where(have, s["teacher"], float("-inf")).double()
    if s["tail"] == "renorm":
        top = v.amax(1, keepdim=True)
        e = torch.exp(v - torch.where(top > float("-inf"), top, 0.0))
        q = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        q = torch.exp(v)
    mass = q.sum(1, keepdim=True)
    loss = torch.where(q > 0, q * (torch.log(q) - logp.gather(1, ids).double()), 0.0).sum(1)
    if s["tail"] == "bucket":
        in_tail = torch.ones((n, vocab + 1), dtype=torch.bool, device=p.device)
        in_tail = in_tail.scatter_(1, torch.where(have, ids, vocab), False)[:, :vocab]
        pt = torch.where(in_tail, p, 0.0).sum(1, keepdim=True).double()
        qt = torch.where(in_tail.any(1, keepdim=True), (1.0 - mass).clamp(min=0.0), 0.0)
        loss = loss + torch.where(qt > 0, qt * (torch.log(qt) - torch.log(pt)), 0.0)[:, 0]
    out = dict(loss=loss.float())
    if s["grad"]:
        grad = p * mass.float()
        if s["tail"] == "bucket":
            grad = p * (mass + qt).float() - torch.where(in_tail, p * (qt / pt).float(), 0.0)
        grad.scatter_add_(1, ids, torch.where(have, -q, 0.0).float())
        out["grad"] = (grad * (s["weight"] / s["temp"])[:, None]).to(s["logits"].dtype)
    return out


# ------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    n, v = case["rows"], case["vocab"]
    el = 4 if case["dtype"] == "f32" else 2
    top = case.get("top", 0)
    if case["op"] == "score":     # W and H once, a token in and three numbers and the alternatives out for each row
        d = case["d"]
        return dict(bytes=(v * d + n * d) * el + n * (16 + 8 * top), flops=2.0 * n * v * d)
    if case["op"] == "logprobs":
        return dict(bytes=n * v * el + n * (16 + 8 * top), flops=4.0 * n * v)
    if case["op"] == "logprobs_grad":
        return dict(bytes=2 * n * v * el + n * 12, flops=8.0 * n * v)
    return dict(bytes=(2 if case["grad"] else 1) * n * v * el + n * (8 + 8 * top), flops=(8.0 if case["grad"] else 4.0) * n * v)


# ------------------------------------------------------------------------ the definitions, in 64 bits

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    rows = max(1, (1 << 27) // case["vocab"])     # a slab of rows at a time: 1 GB an array
    parts = []
    for r in range(0, case["rows"], rows):
        parts.append(_exact_rows(s, slice(r, r + rows)))
    if not isinstance(parts[0], dict):
        return torch.cat(parts)
    return {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_rows(s, r):
    if s["op"] == "score":
        H, W = s["H"][r].double(), s["W"]
        step = max(1, (1 << 27) // W.shape[1])
        x = torch.cat([H @ W[a:a + step].double().T for a in range(0, W.shape[0], step)], dim=1)
    else:
        x = s["logits"][r].double()
    if s["op"] in ("score", "logprobs"):
        d = torch.distributions.Categorical(logits=x / s["temp"], validate_args=False)
        tok = s["tokens"][r].long()
        lp = torch.log_softmax(x / s["temp"], dim=1)
        out = dict(logprob=torch.where(tok < 0, torch.zeros_like(lp[:, 0]), lp[torch.arange(len(tok), device=x.device), tok]),
                   lse=torch.logsumexp(x / s["temp"], dim=1), entropy=torch.special.entr(d.probs).sum(1))
        if s["top"] > 0:
            out["top_ids"] = None
            out["top_logprob"] = torch.topk(lp, s["top"], dim=1).values
        return out
    with torch.enable_grad():
        x.requires_grad_(True)
        lp = torch.log_softmax(x / s["temp"], dim=1)
        if s["op"] == "logprobs_grad":
            tok = s["tokens"][r].long()
            entropy = -(lp.exp() * lp.masked_fill(torch.isinf(lp), 0.0)).sum(1)
            given = lp[torch.arange(len(tok), device=x.device), tok.clamp(min=0)]
            objective = (given * s["g_logprob"][r].double() * (tok >= 0)).sum() + (entropy * s["g_entropy"][r].double()).sum()
            return torch.autograd.grad(objective, x)[0]
        have, ids = s["ids"][r] >= 0, s["ids"][r].long().clamp(min=0)
        v = s["teacher"][r].double()
        if s["tail"] == "renorm":
            q = torch.softmax(v.masked_fill(~have, float("-inf")), dim=1).nan_to_num(0.0)
        else:
            q = torch.where(have, v.exp(), torch.zeros_like(v))
        loss = (torch.special.xlogy(q, q) - q * lp.gather(1, ids)).sum(1)
        if s["tail"] == "bucket":
            seen = torch.zeros((x.shape[0], x.shape[1] + 1), dtype=torch.bool, device=x.device)
            seen.scatter_(1, torch.where(have, ids, torch.full_like(ids, x.shape[1])), True)
            seen = seen[:, :-1]
            rest = (1.0 - q.sum(1)).clamp(min=0.0)
            rest = torch.where(seen.all(1), torch.zeros_like(rest), rest)
            log_rest = torch.logsumexp(lp.masked_fill(seen, float("-inf")), dim=1)
            loss = loss + torch.where(rest > 0, torch.special.xlogy(rest, rest) - rest * log_rest, torch.zeros_like(rest))
        out = dict(loss=loss.detach())
        if s["grad"]:
            out["grad"] = torch.autograd.grad((loss * s["weight"][r].double()).sum(), x)[0]
        return out
