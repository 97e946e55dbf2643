"""Measured cases of the operators around an engine's speculative step: lossless verification of drafted
tokens, dropout with the verifier's masks and its gradient, and projections through a head held in
8-bit integers.

A case is a dict of plain values.  `run` computes it in plain torch operations, or, where `own` is
true, through the library's entry points; `exact` computes it in 64 bits from the definitions.

  lossless      target logits [B,T+1,V], draft logits [B,T,V] or none, drafted tokens [B,T], random numbers
                -> accepted length, next token, acceptance probability of every position
  dropout       x[B,T,d] -> K masked and rescaled copies of every row [B,T,K,d], masks from Philox counters
  dropout_grad  gradient of the copies [B,T,K,d] -> gradient of x[B,T,d]
  linear_i8     x[N,d], W[V,d] in 8-bit integers with a scale for each row -> x W^T [N,V]; x is quantised in the
                call, with a scale for each token
"""
import math

import torch

own = False

DEVICE = "cuda"
_handle = None


# ------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # the toy vocabulary, one short draft, fp32: the smallest call, all latency
        dict(name="lossless_toy", op="lossless", dtype="f32", batch=1, drafted=4, vocab=4096, q=True, ragged=False,
             masked=0.0, temp=1.0, draft_temp=1.0),
        # one sequence of an interactive session on the Llama-3-8B vocabulary
        dict(name="lossless_llama8b", op="lossless", dtype="bf16", batch=1, drafted=5, vocab=128256, q=True, ragged=False,
             masked=0.0, temp=0.75, draft_temp=1.0),
        # tokens proposed by lookup (no draft distribution), drafts of any length, a grammar forbids half the vocabulary
        dict(name="lossless_lookup_odd", op="lossless", dtype="f32", batch=47, drafted=3, vocab=32003, q=False, ragged=True,
             masked=0.5, temp=1.25, draft_temp=1.0),
        # a full serving batch on the Qwen3-8B vocabulary
        dict(name="lossless_batch_qwen8b", op="lossless", dtype="bf16", batch=96, drafted=7, vocab=151936, q=True, ragged=False,
             masked=0.0, temp=1.0, draft_temp=1.0),
        # the paths of one verify call on the Llama-3-8B head, as rows in memory
        dict(name="dropout_paths_llama8b", op="dropout", dtype="bf16", batch=1, drafted=5, paths=8, d=4096, p=0.1),
        # a training batch under eight paths
        dict(name="dropout_train_llama8b", op="dropout", dtype="bf16", batch=32, drafted=128, paths=8, d=4096, p=0.1),
        # plain dropout of fp32 activations, odd width
        dict(name="dropout_single_f32", op="dropout", dtype="f32", batch=4, drafted=1021, paths=1, d=5003, p=0.3),
        # backward of a few positions on the toy head
        dict(name="dropout_grad_toy", op="dropout_grad", dtype="f32", batch=1, drafted=4, paths=8, d=256, p=0.1),
        # backward of a training batch, hidden size of the Llama-3-70B head
        dict(name="dropout_grad_llama70b", op="dropout_grad", dtype="bf16", batch=16, drafted=61, paths=16, d=8192, p=0.1),
        # one decoding step on the Llama-3-8B head
        dict(name="linear_token_llama8b", op="linear_i8", dtype="bf16", rows=1, d=4096, vocab=128256, out="f32"),
        # the positions of a drafted tree on the Qwen3-8B head
        dict(name="linear_tree_qwen8b", op="linear_i8", dtype="bf16", rows=61, d=4096, vocab=151936, out="bf16"),
        # evaluation of a text on the Llama-3-70B head
        dict(name="linear_text_llama70b", op="linear_i8", dtype="bf16", rows=2047, d=8192, vocab=128256, out="bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["lossless", "dropout", "dropout_grad", "linear_i8"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "lossless":
        vocab, drafted = _spread(rng, 200, 200000), rng.randint(1, 8)
        batch = _spread(rng, 1, max(1, min(256, 100_000_000 // (vocab * (2 * drafted + 1)))))
        # temperatures are multiples of 1/64, which every type holds exactly
        return dict(op=op, dtype=dtype, batch=batch, drafted=drafted, vocab=vocab, q=rng.random() < 0.7,
                    ragged=rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.5, 0.95]),
                    temp=rng.randint(32, 128) / 64, draft_temp=rng.randint(32, 128) / 64)
    if op in ("dropout", "dropout_grad"):
        d, paths = _spread(rng, 16, 8192), _spread(rng, 1, 32)
        rows = _spread(rng, 1, max(1, min(8192, 60_000_000 // (d * paths))))
        batch = _spread(rng, 1, rows)
        return dict(op=op, dtype=dtype, batch=batch, drafted=max(1, rows // batch), paths=paths, d=d,
                    p=rng.choice([0.05, 0.1, 0.3, 0.5]))
    vocab, d = _spread(rng, 64, 128256), _spread(rng, 16, 8192)
    return dict(op=op, dtype=dtype, rows=_spread(rng, 1, 2047), d=d, vocab=vocab, out=rng.choice(["f32", "bf16"]))


# ------------------------------------------------------------------------------------- the inputs

def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


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
    if own:
        s["ctx"] = _context()
    if case["op"] == "lossless":
        _prepare_lossless(s, g)
    elif case["op"] == "dropout":
        s["x"] = torch.randn((case["batch"], case["drafted"], case["d"]), generator=g, device=DEVICE).to(_dtype(case["dtype"]))
        s["seed"], s["seq"] = int(seed) * 7919 + 13, int(seed) % 1000
    elif case["op"] == "dropout_grad":
        shape = (case["batch"], case["drafted"], case["paths"], case["d"])
        s["grad"] = (torch.randn(shape, generator=g, device=DEVICE) * 0.01).to(_dtype(case["dtype"]))
        s["seed"], s["seq"] = int(seed) * 7919 + 13, int(seed) % 1000
    else:
        _prepare_linear(s, g)
    return s


def _prepare_lossless(s, g):
    """Rows as a language model gives them: a broad bulk and a few dozen likely tokens; a drafter that agrees
    up to noise; drafted tokens drawn from it."""
    b, t, v = s["batch"], s["drafted"], s["vocab"]
    dtype = _dtype(s["dtype"])
    s["target"] = torch.empty((b, t + 1, v), dtype=dtype, device=DEVICE)
    s["draft_logits"] = torch.empty((b, t, v), dtype=dtype, device=DEVICE) if s["q"] else None
    s["draft"] = torch.empty((b, t), dtype=torch.int32, device=DEVICE)
    forbidden = torch.rand((v,), generator=g, device=DEVICE) < s["masked"]
    forbidden[0] = False
    for i in range(b):
        x = torch.randn((t + 1, v), generator=g, device=DEVICE).mul_(2.0)
        likely = torch.randint(0, v, (t + 1, min(48, v)), generator=g, device=DEVICE)
        x.scatter_add_(1, likely, torch.rand(likely.shape, generator=g, device=DEVICE) * 14.0)
        x.masked_fill_(forbidden, float("-inf"))
        y = x[:t] + torch.randn((t, v), generator=g, device=DEVICE) * 0.5
        s["target"][i] = x.to(dtype)
        if s["q"]:
            s["draft_logits"][i] = y.to(dtype)
        noise = torch.rand((t, v), generator=g, device=DEVICE).clamp_(1e-7, 1.0 - 1e-7)
        s["draft"][i] = (y / s["draft_temp"] - torch.log(-torch.log(noise))).argmax(1).to(torch.int32)
    s["u_accept"] = torch.rand((b, t), generator=g, device=DEVICE)
    s["u_next"] = torch.rand((b,), generator=g, device=DEVICE)
    s["draft_len"] = None
    if s["ragged"]:
        s["draft_len"] = torch.randint(0, t + 1, (b,), generator=g, device=DEVICE, dtype=torch.int32)
        s["draft"].masked_fill_(torch.arange(t, device=DEVICE)[None] >= s["draft_len"][:, None], -1)


def _prepare_linear(s, g):
    """Weights as a checkpoint holds them: 8-bit integers and a scale for each vocabulary entry; rows of W start
    on 16-byte boundaries."""
    v, d = s["vocab"], s["d"]
    store = torch.zeros((v, (d + 15) // 16 * 16), dtype=torch.int8, device=DEVICE)
    s["W"], s["w_scale"] = store[:, :d], torch.empty((v,), device=DEVICE)
    step = max(1, (1 << 27) // d)
    for r in range(0, v, step):
        n = min(step, v - r)
        q, scale = _quantize_plain(torch.randn((n, d), generator=g, device=DEVICE) * 0.02)
        s["W"][r:r + n], s["w_scale"][r:r + n] = q.to(torch.int8), scale
    s["x"] = torch.randn((s["rows"], d), generator=g, device=DEVICE).to(_dtype(s["dtype"]))


# ------------------------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "lossless":
        return _lossless_plain(s)
    if s["op"] == "dropout":
        keep = _keep_plain(s, s["batch"], s["drafted"])
        scale = 1.0 / (1.0 - _single(s["p"]))
        return torch.where(keep, s["x"].float()[:, :, None, :] * scale, 0.0).to(s["x"].dtype)
    if s["op"] == "dropout_grad":
        keep = _keep_plain(s, s["batch"], s["drafted"])
        scale = 1.0 / (1.0 - _single(s["p"]))
        return (torch.where(keep, s["grad"].float(), 0.0).sum(2) * scale).to(s["grad"].dtype)
    return _linear_plain(s)


def _run_own(s):
    ctx = s["ctx"]
    if s["op"] == "lossless":
        return ctx.verify_lossless(s["target"], s["draft"], s["u_accept"], s["u_next"], draft_logits=s["draft_logits"],
                                   draft_len=s["draft_len"], temperature=s["temp"], draft_temperature=s["draft_temp"])
    if s["op"] == "dropout":
        return ctx.dropout(s["x"], s["paths"], s["p"], s["seed"], seq_base=s["seq"])
    if s["op"] == "dropout_grad":
        return ctx.dropout_grad(s["grad"], s["p"], s["seed"], seq_base=s["seq"])
    return ctx.linear_i8(s["x"], s["W"], s["w_scale"], dtype=_dtype(s["out"]))


def _single(x):
    """The value that a single-precision argument takes."""
    return float(torch.tensor(x, dtype=torch.float32))


def _probs_plain(x, temp):
    """Softmax(x / temp) in 64 bits: decisions next to a border and places in long cumulative sums hang on it."""
    x = x.double()
    e = torch.exp((x - x.amax(-1, keepdim=True)) / temp)
    return e / e.sum(-1, keepdim=True)


def _lossless_plain(s):
    b, t, v = s["batch"], s["drafted"], s["vocab"]
    accept_prob = torch.zeros((b, t), dtype=torch.float32, device=DEVICE)
    accept_len = torch.empty((b,), dtype=torch.int32, device=DEVICE)
    following = torch.empty((b,), dtype=torch.int32, device=DEVICE)
    slab = max(1, (1 << 27) // (v * (t + 1)))      # sequences at a time: 1 GB an array
    for b0 in range(0, b, slab):
        r = slice(b0, b0 + slab)
        tok = s["draft"][r].long()
        n_seq = tok.shape[0]
        length = torch.full((n_seq,), t, device=DEVICE) if s["draft_len"] is None else s["draft_len"][r].long()
        here = torch.arange(t, device=DEVICE)[None] < length[:, None]
        at = tok.clamp(min=0)[:, :, None]
        p = _probs_plain(s["target"][r], s["temp"])
        px = p[:, :t].gather(2, at)[:, :, 0]
        if s["q"]:
            q = _probs_plain(s["draft_logits"][r], s["draft_temp"])
            qx = q.gather(2, at)[:, :, 0]
        else:
            q, qx = None, torch.ones_like(px)
        ratio = torch.where(qx > 0, px / qx, torch.where(px > 0, 1.0, 0.0)).clamp(max=1.0)
        accept_prob[r] = torch.where(here, ratio, 0.0).float()
        ok = here & (s["u_accept"][r].double() * qx < px)
        n = torch.cumprod(ok.long(), 1).sum(1)
        accept_len[r] = n.to(torch.int32)
        rows = torch.arange(n_seq, device=DEVICE)
        weight = p[rows, n]
        drawn_against = n < length
        pos = n.clamp(max=t - 1)
        if s["q"]:
            other = q[rows, pos]
        else:
            other = torch.zeros_like(weight).scatter_(1, at[rows, pos], 1.0)
        rest = torch.where(drawn_against[:, None], (weight - other).clamp(min=0.0), weight)
        weight = torch.where(rest.sum(1, keepdim=True) > 0, rest, weight)
        cum = torch.cumsum(weight, 1)
        following[r] = (cum <= s["u_next"][r].double()[:, None] * cum[:, -1:]).sum(1).clamp(max=v - 1).to(torch.int32)
    return dict(accept_len=accept_len, next=following, accept_prob=accept_prob)


def _keep_plain(s, b, t):
    """Keep flags [B,T,K,d]: element j of path i at position t of sequence s is dropped iff word j mod 4 of
    Philox4x32-10 at the counter (j / 4, i, t, s) under the key `seed` is below floor(p 2^32)."""
    k, d = s["paths"], s["d"]
    quads = (d + 3) // 4
    low = 0xFFFFFFFF
    dev = dict(dtype=torch.int64, device=DEVICE)
    c0 = torch.arange(quads, **dev)[None, None, None]
    c1 = torch.arange(k, **dev)[None, None, :, None]
    c2 = torch.arange(t, **dev)[None, :, None, None]
    c3 = ((torch.arange(b, **dev) + s["seq"]) & low)[:, None, None, None]
    k0, k1 = s["seed"] & low, (s["seed"] >> 32) & low
    for _ in range(10):
        a, c = c0 * 0xD2511F53, c2 * 0xCD9E8D57        # modulo 2^64: both halves are right
        c0, c1, c2, c3 = ((c >> 32) & low) ^ c1 ^ k0, c & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), dim=-1).reshape(b, t, k, quads * 4)[..., :d]
    return words >= math.floor(_single(s["p"]) * 2.0 ** 32)


def _quantize_plain(x):
    """Rows of x as 8-bit integers and a scale: the row's largest magnitude becomes 127."""
    x = x.float()
    scale = (x.abs().amax(1) / torch.tensor(127.0, device=x.device)).clamp(min=2.0 ** -126)
    return torch.round(x / scale[:, None]), scale


def _linear_plain(s):
    q, scale = _quantize_plain(s["x"])
    rows, v, d = s["rows"], s["vocab"], s["d"]
    out = torch.empty((rows, v), dtype=_dtype(s["out"]), device=DEVICE)
    step = max(1, (1 << 27) // max(d, rows))
    for r in range(0, v, step):
        # sums over 1024 products of 8-bit integers are whole numbers below 2^24: exact in 32 bits
        total = torch.zeros((rows, min(step, v - r)), dtype=torch.int32, device=DEVICE)
        for c in range(0, d, 1024):
            total += (q[:, c:c + 1024] @ s["W"][r:r + step, c:c + 1024].float().T).to(torch.int32)
        out[:, r:r + step] = (total.float() * s["w_scale"][None, r:r + step] * scale[:, None]).to(out.dtype)
    return out


# ------------------------------------------------------------------------ what a pass cannot do without

def _bytes(name):
    return 4 if name == "f32" else 2


def work(case):
    el = _bytes(case["dtype"])
    if case["op"] == "lossless":
        # the drafted positions' rows of both models (half of them where drafts end anywhere); not the bonus row,
        # which only a draft accepted in full needs
        n = case["batch"] * case["drafted"] * (0.5 if case["ragged"] else 1.0) * (2 if case["q"] else 1)
        return dict(bytes=n * case["vocab"] * el + case["batch"] * (case["drafted"] * 12 + 12), flops=4.0 * n * case["vocab"])
    if case["op"] in ("dropout", "dropout_grad"):
        n = case["batch"] * case["drafted"] * case["d"]
        return dict(bytes=n * (1 + case["paths"]) * el, flops=2.0 * n * case["paths"])
    rows, v, d = case["rows"], case["vocab"], case["d"]
    return dict(bytes=v * d + 4 * v + rows * d * el + rows * v * _bytes(case["out"]), flops=2.0 * rows * v * d)


# ------------------------------------------------------------------------ the definitions, in 64 bits

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "lossless":
        return _exact_lossless(s)
    if case["op"] == "linear_i8":
        return _exact_linear(s)
    p = float(torch.tensor(case["p"], dtype=torch.float32).double())
    parts = []
    for i in range(case["batch"]):
        keep = _exact_keep(s, i)
        if case["op"] == "dropout":
            parts.append(s["x"][i].double()[:, None] * keep / (1.0 - p))
        else:
            parts.append(torch.einsum("tkd,tkd->td", s["grad"][i].double(), keep) / (1.0 - p))
    return torch.stack(parts)


def _exact_lossless(s):
    t, v = s["drafted"], s["vocab"]
    lens, tokens, probs = [], [], []
    for i in range(s["batch"]):
        length = t if s["draft_len"] is None else int(s["draft_len"][i])
        lp = torch.log_softmax(s["target"][i].double() / s["temp"], dim=1)
        lq = torch.log_softmax(s["draft_logits"][i].double() / s["draft_temp"], dim=1) if s["q"] else None
        n, row = 0, torch.zeros((t,), dtype=torch.float64, device=DEVICE)
        going = True
        for j in range(length):
            x = int(s["draft"][i, j])
            ratio = float(torch.exp(lp[j, x] - (lq[j, x] if s["q"] else 0.0)))
            row[j] = min(1.0, ratio)
            going = going and float(s["u_accept"][i, j]) < ratio
            n += int(going)
        p = lp[n].exp()
        if n < length:
            q = lq[n].exp() if s["q"] else torch.nn.functional.one_hot(s["draft"][i, n].long(), v).double()
            p = torch.relu(p - q)
        cum = p.cumsum(0)
        lens.append(n)
        tokens.append(int(torch.searchsorted(cum, cum[-1] * float(s["u_next"][i]), right=True)))
        probs.append(row)
    to = dict(dtype=torch.int32, device=DEVICE)
    return dict(accept_len=torch.tensor(lens, **to), next=torch.tensor(tokens, **to), accept_prob=torch.stack(probs))


def _mul_32(a, const):
    """High and low word of a * const for 32-bit words, from products of 16-bit halves."""
    a0, a1, b0, b1 = a & 0xFFFF, a >> 16, const & 0xFFFF, const >> 16
    low = a0 * b0
    mid = a1 * b0 + (low >> 16)
    mid2 = a0 * b1 + (mid & 0xFFFF)
    return a1 * b1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)


def _exact_keep(s, i):
    """The keep flags of one sequence as numbers, [T,K,d]."""
    t, k, d = s["drafted"], s["paths"], s["d"]
    j = torch.arange((d + 3) // 4, device=DEVICE)
    x, y, z = (a.reshape(-1) for a in torch.meshgrid(torch.arange(t, device=DEVICE), torch.arange(k, device=DEVICE), j, indexing="ij"))
    words = [z, y, x, torch.full_like(z, (s["seq"] + i) % 2 ** 32)]
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32 % 2 ** 32]
    for _ in range(10):
        hi0, lo0 = _mul_32(words[0], 0xD2511F53)
        hi1, lo1 = _mul_32(words[2], 0xCD9E8D57)
        words = [hi1 ^ words[1] ^ key[0], lo1, hi0 ^ words[3] ^ key[1], lo0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    border = int(float(torch.tensor(s["p"], dtype=torch.float32).double()) * 2 ** 32)
    return (torch.stack(words, 1) >= border).double().reshape(t, k, -1)[:, :, :d]


def _exact_linear(s):
    x = s["x"].double()
    scale = (x.abs().amax(1) / 127.0).float().clamp(min=2.0 ** -126).double()
    q = (x / scale[:, None]).float().round().double()     # the quotient is rounded to 32 bits first: part of the definition
    parts = []
    step = max(1, (1 << 26) // s["d"])
    for r in range(0, s["vocab"], step):
        parts.append((q @ s["W"][r:r + step].double().T) * s["w_scale"][r:r + step].double())
    return torch.cat(parts, 1) * scale[:, None]
