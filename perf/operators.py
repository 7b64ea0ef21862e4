"""The operators on a policy's logits, as measurable cases.

A row of logits per generated token goes through the binding as sampling and
training programs take it: log probabilities of the sampled tokens with the
entropy and the top alternatives (a decode step, the scoring of a rollout, a
teacher's answer), their gradient, the clipped policy loss with its gradient,
and the distillation loss over a teacher's top logits with its gradient.
Vocabularies and row counts are generic. Logits are spread like a trained
model's: most of the probability on a few candidates, tokens drawn from the
distribution, a share of the rows padding (token -1) where a batch is ragged.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# -------------------------------------------------------------------- cases --
def _case(path, rows, vocab, dtype="bf16", k=0, temperature=1.0, gap=0, pad=0.0, masked=0, entropy=True, grad=True, old=True):
    """``gap``: elements between rows; ``pad``: share of padding rows; ``masked``: vocabulary entries at -inf;
    ``entropy``: with the entropy's share of loss and gradient; ``grad``: the loss with its gradient; ``old``: with
    the sampling policy's log probabilities (else on-policy)."""
    return dict(path=path, rows=rows, vocab=vocab, dtype=dtype, k=k, temperature=temperature, gap=gap, pad=pad,
                masked=masked, entropy=entropy, grad=grad, old=old)


def listed():
    return [
        # one decode step of a prompt's eight live paths, 20 alternatives, some tokens not allowed (latency)
        dict(name="step_top20", **_case("score", 8, 128000, k=20, temperature=0.8, masked=1000)),
        # the sampling policy's log probabilities and entropy of a rollout's tokens
        dict(name="score_rollout", **_case("score", 4096, 131072, pad=0.1)),
        # a teacher's answers kept for distillation: fp32 logits, an odd vocabulary, 64 alternatives
        dict(name="teacher_top64", **_case("score", 1500, 100003, "f32", k=64)),
        # the gradient of one short segment's log probabilities (latency)
        dict(name="grad_segment", **_case("grad", 64, 32000, entropy=False)),
        # the gradient of a rollout's log probabilities and entropy
        dict(name="grad_rollout", **_case("grad", 4096, 131072, pad=0.1)),
        # fp16 logits of an odd vocabulary inside wider rows
        dict(name="grad_odd_f16", **_case("grad", 1000, 50001, "f16", gap=7, pad=0.05)),
        # the loss of one short segment, on-policy (latency)
        dict(name="policy_segment", **_case("policy", 16, 65537, old=False, entropy=False)),
        # a training step's micro batch of rollout tokens: the largest call
        dict(name="policy_batch", **_case("policy", 8192, 131072, pad=0.1)),
        # fp32 logits, odd vocabulary inside rows padded by the projection that made them
        dict(name="policy_f32", **_case("policy", 2000, 65537, "f32", gap=63, pad=0.1)),
        # distillation of one short segment (latency)
        dict(name="distill_segment", **_case("distill", 32, 32000, k=20, temperature=2.0)),
        # a distillation step's micro batch, 64 teacher logits a token
        dict(name="distill_batch", **_case("distill", 4096, 131072, k=64, pad=0.1)),
        # the held-out loss alone
        dict(name="distill_eval_f16", **_case("distill", 1000, 50001, "f16", k=100, grad=False)),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    most = 4096 * 131072
    while True:
        path = rng.choice(["score", "score", "grad", "policy", "policy", "distill", "distill"])
        rows, vocab = _log(rng, 1, 8192), _log(rng, 1000, 262144)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        k = 0
        if path == "score":
            k = rng.choice([0, 0, 1, 5, 20, 64, 128])
        elif path == "distill":
            k = _log(rng, 1, 256)
        if rows * vocab * SIZE[dtype] > 2 * most or (k and path == "score" and rows * vocab > most // 2):
            continue
        return _case(path, rows, vocab, dtype, k=k, temperature=rng.choice([1.0, 1.0, 0.7, 2.0]),
                     gap=rng.choice([0, 0, 0, 1, 7, 64]), pad=rng.choice([0.0, 0.0, 0.1]), masked=rng.choice([0, 0, 100]),
                     entropy=rng.random() < 0.6, grad=rng.random() < 0.75, old=rng.random() < 0.7)


# ------------------------------------------------------------------- inputs --
def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + stream * 7919 + 17) % (1 << 62))


def _wide(case):
    """[rows][vocab] inside rows of vocab + gap elements."""
    n, v, gap = case["rows"], case["vocab"], case["gap"]
    return torch.zeros((n, v + gap), dtype=TYPES[case["dtype"]], device=DEV)[:, :v]


def _logits(case, g):
    """N(0, 2.5^2) with eight candidates a row raised by 6 to 14; ``masked`` entries at the vocabulary's end at -inf."""
    n, v = case["rows"], case["vocab"]
    out = _wide(case)
    cand = torch.randint(0, v, (n, 8), generator=g, device=DEV)
    lift = 6 + 8 * torch.rand((n, 8), generator=g, device=DEV)
    step = max(1, (1 << 28) // v)
    for a in range(0, n, step):
        x = torch.randn((min(step, n - a), v), generator=g, device=DEV).mul_(2.5)
        x.scatter_add_(1, cand[a:a + step], lift[a:a + step])
        if case["masked"]:
            x[:, v - case["masked"]:] = -math.inf
        out[a:a + step].copy_(x)
    return out, cand


def _each(logits, temperature, f):
    """f of the rows' logits / temperature in 32 bits, some rows at a time."""
    step = max(1, (1 << 28) // logits.shape[1])
    parts = [f(logits[a:a + step].float() / temperature, slice(a, a + step)) for a in range(0, logits.shape[0], step)]
    return tuple(torch.cat(p) for p in zip(*parts))


def _known(logits, tokens, temperature):
    """lse, log probability of the token and entropy, which a program has from the forward pass."""
    def f(x, rows):
        lse = torch.logsumexp(x, -1)
        p = torch.exp(x - lse[:, None])
        h = lse - (p * torch.where(p > 0, x, 0.0)).sum(-1)
        lp = x.gather(1, tokens[rows, None].long().clamp(min=0))[:, 0] - lse
        return lse, lp, h
    return _each(logits, temperature, f)


def _tokens(case, logits, cand, g):
    """Mostly one of the candidates by its probability, else any allowed token; -1 where the row is padding."""
    n, v = case["rows"], case["vocab"]
    at = logits.gather(1, cand).float() / case["temperature"]
    gumbel = -torch.log(-torch.log(torch.rand((n, 8), generator=g, device=DEV).clamp(1e-7, 1 - 1e-6)))
    tok = cand.gather(1, (at + gumbel).argmax(-1, keepdim=True))[:, 0]
    other = torch.randint(0, v - case["masked"], (n,), generator=g, device=DEV)
    tok = torch.where(torch.rand(n, generator=g, device=DEV) < 0.1, other, tok)
    tok = torch.where(tok >= v - case["masked"], other, tok)
    pad = torch.rand(n, generator=g, device=DEV) < case["pad"]
    pad[0] = False
    return torch.where(pad, -1, tok).to(torch.int32)


def prepare(case, seed):
    g = _gen(seed, 1)
    n, v, k, t = case["rows"], case["vocab"], case["k"], case["temperature"]
    logits, cand = _logits(case, g)
    s = dict(case=case, logits=logits)
    f32 = lambda *shape: torch.zeros(shape, dtype=torch.float32, device=DEV)  # noqa: E731
    if case["path"] == "distill":
        # the teacher's k best of its own logits, near the student's; padding rows list none
        noise = _gen(seed, 2)
        step = max(1, (1 << 27) // v)
        best = []
        for a in range(0, n, step):
            x = logits[a:a + step].float()
            best.append((x + 1.5 * torch.randn(x.shape, generator=noise, device=DEV)).topk(k, -1))
        value, ids = (torch.cat([b[i] for b in best]) for i in (0, 1))
        pad = torch.rand(n, generator=noise, device=DEV) < case["pad"]
        pad[0] = False
        s["ids"] = torch.where(pad[:, None], -1, ids).to(torch.int32).contiguous()
        s["teacher"] = value.contiguous()
        s["weight"] = torch.full((n,), 1.0, device=DEV)
        s["loss"] = f32(n)
    else:
        s["tokens"] = _tokens(case, logits, cand, g)
        s["logp"], s["entropy"], s["lse"] = f32(n), f32(n), f32(n)
    if case["path"] == "score" and k:
        s["top_ids"], s["top_logp"] = torch.zeros((n, k), dtype=torch.int32, device=DEV), f32(n, k)
    if case["path"] == "grad":
        s["lse"], _, s["entropy"] = _known(logits, s["tokens"], t)
        s["dlogp"] = torch.randn(n, generator=g, device=DEV)
        s["dentropy"] = 0.1 * torch.randn(n, generator=g, device=DEV) if case["entropy"] else None
    if case["path"] == "policy":
        _, lp, _ = _known(logits, s["tokens"], t)
        if case["old"]:
            # some steps off-policy; ratios keep clear of the clip's edges, where rounding alone decides the gradient
            ratio = torch.exp(0.15 * torch.randn(n, generator=g, device=DEV))
            for edge in (0.8, 1.28):
                ratio = torch.where((ratio - edge).abs() < 1e-3, ratio + 4e-3, ratio)
            s["old_logp"] = lp - torch.log(ratio)
        else:
            s["old_logp"] = None
        s["advantage"] = torch.randn(n, generator=g, device=DEV)
        s["weight"] = 0.5 + torch.rand(n, generator=g, device=DEV)
        s["loss"] = f32(n)
    if case["path"] == "grad" or (case["path"] in ("policy", "distill") and case["grad"]):
        s["dlogits"] = _wide(case)
    return s


# --------------------------------------------------------------- plain form --
def _softmax(logits, temperature):
    """x, ln p, p and lse in 32 bits."""
    x = logits.float() / temperature
    m = x.amax(-1, keepdim=True)
    lse = m + torch.log(torch.exp(x - m).sum(-1, keepdim=True))
    lp = x - lse
    return x, lp, torch.exp(lp), lse[:, 0]


def _entropy(lp, p):
    return -torch.where(p > 0, p * lp, 0.0).sum(-1)


def _plain_score(s):
    case, k = s["case"], s["case"]["k"]
    live = s["tokens"] >= 0
    x, lp, p, lse = _softmax(s["logits"], case["temperature"])
    at = s["tokens"].long().clamp(min=0)[:, None]
    out = dict(logp=torch.where(live, lp.gather(1, at)[:, 0], 0.0), entropy=torch.where(live, _entropy(lp, p), 0.0),
               lse=torch.where(live, lse, 0.0))
    if k:
        # the order of the floats' bits with the lower id first among equals, as one integer key
        bits = (s["logits"].float() + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 32) + (case["vocab"] - torch.arange(case["vocab"], device=DEV))
        ids = key.topk(k, -1).indices
        top = lp.gather(1, ids)
        drop = (top == -math.inf) | ~live[:, None]
        out["top_ids"] = torch.where(drop, -1, ids).to(torch.int32)
        out["top_logp"] = torch.where(drop, -math.inf, top)
    return out


def _one(shape, at):
    return torch.arange(shape[1], device=DEV)[None, :] == at[:, None]


def _plain_grad(s):
    t = s["case"]["temperature"]
    live = (s["tokens"] >= 0)[:, None]
    lp = s["logits"].float() / t - s["lse"][:, None]
    p = torch.exp(lp)
    d = s["dlogp"][:, None] * (_one(p.shape, s["tokens"]).float() - p)
    if s["dentropy"] is not None:
        d = d - s["dentropy"][:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    return dict(dlogits=torch.where(live, d / t, 0.0).to(s["logits"].dtype))


CLIP_LOW, CLIP_HIGH, BETA = 0.2, 0.28, 0.01


def _plain_policy(s):
    case, t = s["case"], s["case"]["temperature"]
    live = s["tokens"] >= 0
    _, lps, p, _ = _softmax(s["logits"], t)
    lp = lps.gather(1, s["tokens"].long().clamp(min=0)[:, None])[:, 0]
    h = _entropy(lps, p)
    beta = BETA if case["entropy"] else 0.0
    a, w = s["advantage"], s["weight"]
    ratio = torch.exp(lp - s["old_logp"]) if case["old"] else torch.ones_like(lp)
    kept = ~(((a > 0) & (ratio > 1 + CLIP_HIGH)) | ((a < 0) & (ratio < 1 - CLIP_LOW)))
    loss = -torch.minimum(ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a) - beta * h
    out = dict(loss=torch.where(live, w * loss, 0.0), logp=torch.where(live, lp, 0.0), entropy=torch.where(live, h, 0.0))
    if case["grad"]:
        c = (w * torch.where(kept, -a * ratio, 0.0))[:, None]
        d = c * (_one(p.shape, s["tokens"]).float() - p)
        if beta:
            d = d + (w * beta)[:, None] * torch.where(p > 0, p * (lps + h[:, None]), 0.0)
        out["dlogits"] = torch.where(live[:, None], d / t, 0.0).to(s["logits"].dtype)
    return out


def _plain_distill(s):
    case, t = s["case"], s["case"]["temperature"]
    ids, w = s["ids"].long(), s["weight"]
    live = ids[:, 0] >= 0
    _, lp, p, _ = _softmax(s["logits"], t)
    q, lq = (f.view(len(w), -1) for f in _softmax(s["teacher"], t)[2:0:-1])
    at = ids.clamp(min=0)
    loss = torch.where(q > 0, q * (lq - lp.gather(1, at)), 0.0).sum(-1)
    out = dict(loss=torch.where(live, w * loss, 0.0))
    if case["grad"]:
        d = p.scatter_add(1, at, -q) * (w / t)[:, None]
        out["dlogits"] = torch.where(live[:, None], d, 0.0).to(s["logits"].dtype)
    return out


def run(s):
    case = s["case"]
    if not own:
        return {"score": _plain_score, "grad": _plain_grad, "policy": _plain_policy, "distill": _plain_distill}[case["path"]](s)
    import paper_2508_17445_gb300 as tp
    t = case["temperature"]
    if case["path"] == "score":
        tp.tp_token_logprobs(s["logits"], s["tokens"], s["logp"], s["entropy"], s["lse"], s.get("top_ids"), s.get("top_logp"),
                             temperature=t)
        names = ("logp", "entropy", "lse") + (("top_ids", "top_logp") if case["k"] else ())
    elif case["path"] == "grad":
        tp.tp_token_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["dlogits"], s["dlogp"], s["dentropy"],
                                      s["entropy"], temperature=t)
        names = ("dlogits",)
    elif case["path"] == "policy":
        tp.tp_policy_loss(s["logits"], s["tokens"], s["advantage"], s["loss"], s.get("dlogits"), s["old_logp"], s["weight"],
                          s["logp"], s["entropy"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                          entropy_coef=BETA if case["entropy"] else 0.0, temperature=t)
        names = ("loss", "logp", "entropy") + (("dlogits",) if case["grad"] else ())
    else:
        tp.tp_distill_loss(s["logits"], s["ids"], s["teacher"], s["loss"], s.get("dlogits"), s["weight"], temperature=t)
        names = ("loss",) + (("dlogits",) if case["grad"] else ())
    return {x: s[x] for x in names}


def work(case):
    """Every logit of a row that is not padding read once (and its gradient written once, padding rows' zeros too), and
    the rows' own numbers; about eight operations a logit for the statistics and six for the gradient."""
    n, v, k, e = case["rows"], case["vocab"], case["k"], SIZE[case["dtype"]]
    live = n * (1 - case["pad"])
    grad = case["path"] == "grad" or (case["path"] in ("policy", "distill") and case["grad"])
    size = live * v * e + (n * v * e if grad else 0)
    size += n * {"score": 16 + 8 * k, "grad": 20, "policy": 28, "distill": 8 + 8 * k}[case["path"]]
    flops = live * v * ((0 if case["path"] == "grad" else 8) + (6 if grad else 0))
    return {"bytes": size, "flops": flops}


# ----------------------------------------------------------- in 64 bits ------
def exact(case, seed):
    s = prepare(case, seed)
    n, v, k, t = case["rows"], case["vocab"], case["k"], case["temperature"]
    grad, path = "dlogits" in s, case["path"]
    out = {}
    step = max(1, (1 << 26) // v)
    whole = torch.zeros((n, v), dtype=torch.float64, device=DEV) if grad else None
    for a in range(0, n, step):
        r = slice(a, min(n, a + step))
        x = s["logits"][r].double() / t
        part = {}
        if path == "grad":
            lp = x - s["lse"][r].double()[:, None]
        else:
            lse = torch.logsumexp(x, -1)
            lp = x - lse[:, None]
        p = lp.exp()
        plp = torch.nan_to_num(p * lp, nan=0.0)  # 0 ln 0 = 0
        if path == "distill":
            ids = s["ids"][r].long()
            live = ids[:, 0] >= 0
            lq = torch.log_softmax(s["teacher"][r].double() / t, -1)
            w = s["weight"][r].double()
            part["loss"] = w * torch.nan_to_num(lq.exp() * (lq - lp.gather(1, ids.clamp(min=0))), nan=0.0).sum(-1)
            if grad:
                d = p.clone()
                d.scatter_add_(1, ids.clamp(min=0), -lq.exp())
                d *= (w / t)[:, None]
        else:
            tok = s["tokens"][r].long()
            live = tok >= 0
            hot = tok.clamp(min=0)[:, None]
            tlp = lp.gather(1, hot)[:, 0]
            if path == "grad":
                gl = s["dlogp"][r].double()
                d = -p * gl[:, None]
                d.scatter_add_(1, hot, gl[:, None])
                if s["dentropy"] is not None:
                    d -= s["dentropy"][r].double()[:, None] * (plp + p * s["entropy"][r].double()[:, None])
                d /= t
            else:
                h = -plp.sum(-1)
                part["logp"], part["entropy"] = tlp, h
            if path == "score":
                part["lse"] = lse
                if k:
                    part["top_logp"] = lp.topk(k, -1).values
            if path == "policy":
                adv, w = s["advantage"][r].double(), s["weight"][r].double()
                beta = BETA if case["entropy"] else 0.0
                ratio = (tlp - s["old_logp"][r].double()).exp() if case["old"] else torch.ones_like(tlp)
                inner, outer = ratio * adv, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
                part["loss"] = w * (-torch.minimum(inner, outer) - beta * h)
                if grad:
                    c = torch.where(inner <= outer, -w * inner, 0.0)
                    d = -p * c[:, None]
                    d.scatter_add_(1, hot, c[:, None])
                    d += (beta * w)[:, None] * (plp + p * h[:, None])
                    d /= t
        for name, y in part.items():
            if name == "top_logp":
                y = torch.where(live[:, None], y, -math.inf)
            else:
                y = torch.where(live, y, 0.0)
            out.setdefault(name, []).append(y)
        if grad:
            whole[r] = torch.where(live[:, None], d, 0.0)
    out = {name: torch.cat(y) for name, y in out.items()}
    if grad:
        out["dlogits"] = whole
    if path == "score" and k:
        out["top_ids"] = None
    return out
