"""The client's operators beside generation - scoring, and its ends of a fine-tuning step - as cases to be timed and compared.

Kinds of case (vocabularies and widths are those of the models in `synth.CONFIGS`, of `perf/cases.py` and of the tests):

  logprobs  log probabilities of given tokens, entropy of the distribution, the most likely alternatives
  distill   loss against a teacher's top logits and its gradient (one teacher token: cross-entropy)
  head      the gradient of the logits back through LM head and final LayerNorm, to the last block's output
  embed     the gradient of a batch's embedded tokens, one row for each different token
"""
import math

import torch

DEV = "cuda:0"
EPS = 1e-5
own = False


def _case(name, kind, **kw):
    return dict(kw, kind=kind, **({"name": name} if name else {}))


def listed():
    return [
        # a chat that shows the probability of each token it writes: one row per call, latency is everything
        _case("logprobs_chat", "logprobs", vocab=250880, rows=1, temperature=1.0, top_k=5),
        # the live branches of a beam search with a smaller vocabulary, whose rows begin at any alignment
        _case("logprobs_beams", "logprobs", vocab=50257, rows=12, temperature=0.8, top_k=20),
        # scoring documents: 1024 positions of a text at once
        _case("logprobs_score", "logprobs", vocab=250880, rows=1024, temperature=1.0, top_k=20),
        # prompt tuning with hard labels on one short example: cross-entropy is a teacher of one token
        _case("distill_labels", "distill", vocab=250880, rows=24, top=1, temperature=1.0),
        # a small vocabulary, an odd number of positions, long lists
        _case("distill_50257", "distill", vocab=50257, rows=701, top=128, temperature=2.0),
        # 4 sequences of 512 tokens: the largest of the loss
        _case("distill_batch", "distill", vocab=250880, rows=2048, top=64, temperature=2.0),
        # prompt tuning of a small model on one short example
        _case("head_small", "head", vocab=50257, hidden=1024, rows=16),
        # a short example with the 176B model: the matrix of 7.2 GB once
        _case("head_176b_24", "head", vocab=250880, hidden=14336, rows=24),
        # 3 sequences of 117 tokens, a vocabulary that no tile divides
        _case("head_351", "head", vocab=50257, hidden=2560, rows=351),
        # 4 sequences of 512 tokens of the 7B1-shaped model: the largest piece of work
        _case("head_batch", "head", vocab=250880, hidden=4096, rows=2048),
        # 16 prompt tokens in front of each of 8 sequences
        _case("embed_prompt", "embed", vocab=16, hidden=4096, rows=128, distinct=16),
        # 8 sequences of 512 tokens, the frequent words again and again
        _case("embed_batch", "embed", vocab=250880, hidden=4096, rows=4096, distinct=1300),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["logprobs", "distill", "head", "embed"], [0.25, 0.25, 0.25, 0.25])[0]
    vocab = _log_uniform(rng, 20000, 250880)
    if kind == "logprobs":
        return _case(None, kind, vocab=vocab, rows=_log_uniform(rng, 1, 1024), temperature=rng.choice([0.7, 1.0, 1.0]),
                     top_k=rng.choice([0, 1, rng.randint(2, 64)]))
    if kind == "distill":
        return _case(None, kind, vocab=vocab, rows=_log_uniform(rng, 1, 2048), top=rng.choice([1, _log_uniform(rng, 2, 256)]),
                     temperature=rng.choice([1.0, 2.0, 4.0]))
    hidden = 64 * _log_uniform(rng, 16, 224)
    if kind == "head":
        rows = min(_log_uniform(rng, 1, 2048), 2048 * 4096 * 250880 // (hidden * vocab))
        return _case(None, kind, vocab=vocab, hidden=hidden, rows=max(1, rows))
    rows = min(_log_uniform(rng, 1, 8192), 4096 * 4096 // hidden)
    return _case(None, kind, vocab=vocab, hidden=hidden, rows=rows, distinct=_log_uniform(rng, 1, rows))


# ---------------------------------------------------------------------------------------------- inputs

def _normal(shape, std, g, mean=0.0, dtype=torch.float32):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(mean, std, generator=g).to(dtype)


def _logits(rows, V, g):
    """fp32 [rows, V]: a broad floor and a few tokens that stand out, some of them by much."""
    x = _normal((rows, V), 2.0, g)
    at = torch.randint(0, V, (rows, 8), generator=g, device=DEV)
    x.scatter_(1, at, 6.0 + 9.0 * torch.rand((rows, 8), generator=g, device=DEV))
    return x, at


def _hidden(rows, hidden, g):
    """fp16 N(0, 1) with four feature dims whose magnitude is 20 to 60 in every row: the outlier features."""
    x = _normal((rows, hidden), 1.0, g)
    dims = torch.randperm(hidden, generator=g, device=DEV)[:4]
    sign = torch.where(torch.rand(4, generator=g, device=DEV) < 0.5, -1.0, 1.0)
    x[:, dims] = (20.0 + 40.0 * torch.rand((rows, 4), generator=g, device=DEV)) * sign
    return x.to(torch.float16)


def _embeddings(V, H, g):
    E = torch.empty((V, H), dtype=torch.float16, device=DEV)
    for v0 in range(0, V, 32768):
        E[v0:v0 + 32768] = _normal((min(32768, V - v0), H), 0.02, g, dtype=torch.float16)
    return E


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 11)
    kind, V, M, H = case["kind"], case["vocab"], case["rows"], case.get("hidden", 64)
    st = dict(case)
    E = _embeddings(V, H, g)
    vec = [_normal((H,), 0.02, g, mean=m, dtype=torch.float16) for m in (1.0, 0.0, 1.0, 0.0)]     # both LayerNorms
    st["E"], st["vec"] = E, vec
    if kind == "logprobs":
        st["logits"], at = _logits(M, V, g)
        col = torch.randint(0, 8, (M,), generator=g, device=DEV)
        tokens = at.gather(1, col[:, None])[:, 0].to(torch.int32)
        st["tokens"] = torch.where(torch.rand(M, generator=g, device=DEV) < 0.1, torch.full_like(tokens, -1), tokens)   # padding
    elif kind == "distill":
        K = case["top"]
        st["logits"], at = _logits(M, V, g)
        if K == 1:
            ids, vals = at[:, :1].clone(), torch.zeros((M, 1), device=DEV)
        else:
            vals, ids = (st["logits"] + _normal((M, V), 0.7, g)).topk(K, dim=1)
        short = torch.rand(M, generator=g, device=DEV) < 0.25                  # a quarter of the lists is shorter
        ids[short, K - K // 8:] = -1
        ids[torch.rand(M, generator=g, device=DEV) < 0.1] = -1                 # positions that are not trained on
        st["ids"], st["vals"] = ids.to(torch.int32).contiguous(), vals.contiguous()
        st["weight"] = 0.5 + torch.rand(M, generator=g, device=DEV)
    elif kind == "head":
        st["x"] = _hidden(M, H, g)
        q, at = _logits(M, V, g)                                               # a cross-entropy's gradient, q - [v = label]
        q.sub_(q.amax(1, keepdim=True)).exp_()
        q.div_(q.sum(1, keepdim=True))
        q.scatter_add_(1, at[:, :1], torch.full((M, 1), -1.0, device=DEV))
        q[torch.rand(M, generator=g, device=DEV) < 0.1] = 0.0                  # positions that are not trained on
        st["grad"] = q
    else:
        D = case["distinct"]
        some = torch.randperm(V, generator=g, device=DEV)[:D]
        rank = (torch.rand(M - D, generator=g, device=DEV) ** 3 * D).long().clamp_(max=D - 1)       # few tokens are frequent
        ids = some[torch.cat([torch.arange(D, device=DEV), rank])]
        st["ids"] = ids[torch.randperm(M, generator=g, device=DEV)].to(torch.int32)
        st["grad"] = _normal((M, H), 0.02, g, dtype=torch.float16)
        # what the caller keeps for the result; entries behind the last token stay as they are
        st["out"] = (torch.zeros(M, dtype=torch.int32, device=DEV), torch.zeros((M, H), device=DEV),
                     torch.zeros(1, dtype=torch.int32, device=DEV))
    if own:
        from paper_2209_01188_amd import binding
        st["client"] = binding.Client(E, *vec, max_rows=M)
        if kind == "head":
            st["store"] = torch.empty(binding.petals_client_lm_head_backward_bytes(st["client"].cfg, M), dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------------------------- one pass

def _own(st):
    c, kind = st["client"], st["kind"]
    if kind == "logprobs":
        logprob, entropy, top, top_logprob = c.logprobs(st["logits"], st["tokens"], st["temperature"], st["top_k"])
        return dict(logprob=logprob, entropy=entropy, **(dict(top=top, top_logprob=top_logprob) if st["top_k"] else {}))
    if kind == "distill":
        loss, grad = c.distill(st["logits"], st["ids"], st["vals"], st["temperature"], loss_grad=st["weight"])
        return dict(loss=loss, grad=grad)
    if kind == "head":
        return dict(grad_hidden=c.lm_head_backward(st["x"], st["grad"], store=st["store"]))
    tokens, grads, count = c.embed_backward(st["ids"], st["grad"], out=st["out"])
    return dict(tokens=tokens, grads=grads, count=count)


def _norm_backward(dy, x, gain):
    """Gradient of LayerNorm's input, fp32 rows."""
    xc = x - x.mean(1, keepdim=True)
    inv = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
    xh, d = xc * inv, dy * gain
    return inv * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))


def _plain_logprobs(st):
    x, K = st["logits"], st["top_k"]
    z = x / st["temperature"]
    z = z - z.amax(1, keepdim=True)
    e = z.exp()
    s = e.sum(1)
    lse = s.log()
    t = st["tokens"].long()
    logprob = torch.where(t >= 0, z.gather(1, t.clamp(min=0)[:, None])[:, 0] - lse, torch.zeros_like(lse))
    out = dict(logprob=logprob, entropy=lse - (e * z).sum(1) / s)
    if K:
        vals, ids = x.topk(min(K + 8, x.shape[1]), dim=1)        # some more, so that equal logits at the end are told apart
        ids, by = ids.sort(dim=1)
        vals, by = vals.gather(1, by).sort(dim=1, descending=True, stable=True)
        out["top"] = ids.gather(1, by)[:, :K].to(torch.int32)
        out["top_logprob"] = z.gather(1, out["top"].long()) - lse[:, None]
    return out


def _plain_distill(st):
    T, ids = st["temperature"], st["ids"].long()
    given = ids >= 0
    any_given = given.any(1)
    t = (st["vals"] / T).masked_fill(~given, -math.inf)
    t = torch.where(any_given[:, None], t - t.amax(1, keepdim=True), torch.zeros_like(t))
    p = t.exp() * given
    ps = p.sum(1, keepdim=True).clamp(min=1e-30)
    p = p / ps
    z = st["logits"] / T
    z = z - z.amax(1, keepdim=True)
    q = z.exp()
    s = q.sum(1, keepdim=True)
    logq = z.gather(1, ids.clamp(min=0)) - s.log()
    logp = torch.where(given, t - ps.log(), torch.zeros_like(t))
    loss = T * T * torch.where(given, p * (logp - logq), torch.zeros_like(p)).sum(1)
    scale = st["weight"] * T * any_given
    q.mul_(scale[:, None] / s)
    q.scatter_add_(1, ids.clamp(min=0), -p * scale[:, None])
    return dict(loss=loss, grad=q)


def _plain_head(st):
    da = st["grad"] @ st["E"].float()
    return dict(grad_hidden=_norm_backward(da, st["x"].float(), st["vec"][2].float()).to(torch.float16))


def _plain_embed(st):
    V, M, H = st["vocab"], st["rows"], st["hidden"]
    ids, order = st["ids"].long().clamp(0, V - 1).sort(stable=True)
    first = torch.ones(M, dtype=torch.int64, device=DEV)
    first[1:] = ids[1:] != ids[:-1]
    rank = first.cumsum(0) - 1
    tokens = torch.zeros(M, dtype=torch.int64, device=DEV).scatter_(0, rank, ids)
    sums = torch.zeros((M, H), device=DEV).index_add_(0, rank, st["grad"][order].float())
    grads = _norm_backward(sums, st["E"][tokens].float(), st["vec"][0].float())       # rows of zeros stay such
    return dict(tokens=tokens.to(torch.int32), grads=grads, count=(rank[-1:] + 1).to(torch.int32))


def run(st):
    if own:
        return _own(st)
    return dict(logprobs=_plain_logprobs, distill=_plain_distill, head=_plain_head, embed=_plain_embed)[st["kind"]](st)


# ------------------------------------------------------------------------------- the definitions in 64 bits

def _exact_rows(st, r):
    """logprobs and distill, of the rows of slice r."""
    T, lg = st["temperature"], st["logits"][r].double() / st["temperature"]
    logq = lg - torch.logsumexp(lg, 1, keepdim=True)
    q = logq.exp()
    if st["kind"] == "logprobs":
        t = st["tokens"][r].long()
        got = logq[torch.arange(t.numel(), device=DEV), t.clamp(min=0)]
        out = dict(logprob=torch.where(t < 0, 0.0, got), entropy=-(q * logq).sum(1))
        if st["top_k"]:
            top = st["logits"][r].sort(dim=1, descending=True, stable=True)[1][:, :st["top_k"]]
            out.update(top=top.to(torch.int32), top_logprob=logq.gather(1, top))
        return out
    ids, vals, w = st["ids"][r].long(), st["vals"][r].double() / T, st["weight"][r].double()
    p = torch.zeros_like(lg)
    on = ids >= 0
    row = torch.arange(ids.shape[0], device=DEV)[:, None].expand_as(ids)
    weights = torch.softmax(torch.where(on, vals, -math.inf), 1)
    p[row[on], ids[on]] = weights[on]
    some = on.any(1).double()
    loss = T * T * torch.where(on, weights * (weights.log() - logq.gather(1, ids.clamp(min=0))), 0.0).sum(1)
    return dict(loss=torch.where(some > 0, loss, 0.0), grad=(q - p) * (T * w * some)[:, None])


def exact(case, seed):
    st = prepare(case, seed)
    kind, M, H = case["kind"], case["rows"], case.get("hidden", 64)
    if kind in ("logprobs", "distill"):
        parts = [_exact_rows(st, slice(m, min(m + 64, M))) for m in range(0, M, 64)]
        return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if kind == "head":
        dy = torch.zeros((M, H), dtype=torch.float64, device=DEV)
        for v in range(0, case["vocab"], 16384):
            dy += st["grad"][:, v:v + 16384].double() @ st["E"][v:v + 16384].double()
        x, gain = st["x"].double(), st["vec"][2].double()
    else:
        tokens, place, count = torch.unique(st["ids"].long(), return_inverse=True, return_counts=True)
        n = tokens.numel()
        member = (torch.arange(n, device=DEV)[:, None] == place[None, :]).double()
        dy = member @ st["grad"].double()
        x, gain = st["E"][tokens].double(), st["vec"][0].double()
    # y = g xh + b with xh = (x - mean) / sqrt(var + eps): the Jacobian's product written out from its definition
    var = x.var(1, unbiased=False, keepdim=True) + EPS
    xh = (x - x.mean(1, keepdim=True)) / var.sqrt()
    u = dy * gain
    grad = (H * u - u.sum(1, keepdim=True) - xh * (u * xh).sum(1, keepdim=True)) / (H * var.sqrt())
    if kind == "head":
        return dict(grad_hidden=grad)
    return dict(tokens=torch.cat([tokens, tokens.new_zeros(M - n)]).to(torch.int32),
                grads=torch.cat([grad, grad.new_zeros((M - n, H))]),
                count=torch.tensor([n], dtype=torch.int32, device=DEV))


# ------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    M, V, H = case["rows"], case["vocab"], case.get("hidden", 64)
    if case["kind"] == "logprobs":
        return {"bytes": 4 * M * V + 12 * M + 8 * M * case["top_k"], "flops": 5 * M * V}
    if case["kind"] == "distill":
        return {"bytes": 8 * M * V + 8 * M * (1 + case["top"]), "flops": 6 * M * V}
    if case["kind"] == "head":
        return {"bytes": 2 * V * H + 4 * M * V + 4 * M * H + 4 * H, "flops": 2 * M * V * H + 10 * M * H}
    D = case["distinct"]
    return {"bytes": 2 * M * H + 6 * D * H + 8 * M, "flops": M * H + 10 * D * H}
