"""The operators around the filter step, as measurable cases.

Before the step a trainer rescores prefixes: hidden states meet the output head
in 8-bit integers, and the logits give the log-probabilities of the recorded
tokens. After it, the packed batch's logits give log-probabilities again, these
the policy loss and its gradient, which goes back through the log-probabilities
to the logits; the weights' updates are orthogonalised.

Kinds of case:
  logprob  pace_token_logprob, with `grad` its backward pass too
  loss     pace_policy_loss on a packed batch
  i8       pace_quantize_rows of the tokens, then pace_matmul_i8 with weights
           that were quantised once
  ortho    pace_orthogonalize of a batch of updates

Where `own` is false the operators run in their plain form: elementary torch
operations in binary32, rounded once at the end."""
import math

import torch

own = False
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CLIP_LOW, CLIP_HIGH, DUAL_CLIP = 0.2, 0.28, 10.0
STEPS, COEFS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


def _logprob(name=None, rows=64, vocab=32768, dtype="bf16", top=0, grad=False, grad_entropy=False, masked=0.0, padded=0,
             temperature=1.0):
    return _named(name, kind="logprob", rows=rows, vocab=vocab, dtype=dtype, top=top, grad=grad,
                  grad_entropy=grad_entropy, masked=masked, padded=padded, temperature=temperature)


def _loss(name=None, n=64, tokens=70001, sigma=0.6, masked=False, weighted=False):
    return _named(name, kind="loss", n=n, tokens=tokens, sigma=sigma, masked=masked, weighted=weighted)


def _i8(name=None, m=1, n=4096, k=4096, dtype="bf16", out="bf16"):
    return _named(name, kind="i8", m=m, n=n, k=k, dtype=dtype, out=out)


def _ortho(name=None, batch=1, rows=256, cols=256, dtype="f32"):
    return _named(name, kind="ortho", batch=batch, rows=rows, cols=cols, dtype=dtype)


def _named(name, **c):
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # Rollouts being sampled: the log-probability of each new token, its entropy and the 20 best alternatives.
        _logprob("logprob_sample", rows=48, vocab=150000, top=20, temperature=0.7),
        # Prefixes rescored: a chunk of recorded tokens, one in four of them tool output that is not scored.
        _logprob("logprob_rescore", rows=4099, vocab=150000, masked=0.25, padded=11),
        # A small vocabulary trained in binary32 with an entropy bonus: forward, then backward.
        _logprob("logprob_train_f32", rows=1023, vocab=50021, dtype="f32", grad=True, grad_entropy=True),
        # A chunk of a training batch: forward, then backward.
        _logprob("logprob_train", rows=4096, vocab=150000, grad=True),
        # The policy loss of a small single-turn batch.
        _loss("loss_math", n=683, tokens=2533335, sigma=0.749, weighted=True),
        # The policy loss of a whole multi-turn batch with masked tool spans.
        _loss("loss_multiturn", n=1575, tokens=16892191, sigma=0.5, masked=True),
        # One token through a projection: the weights are read once.
        _i8("i8_token", m=1, n=16384, k=4096),
        # A chunk of prefix tokens through a projection.
        _i8("i8_prefix", m=4096, n=16384, k=4096),
        # The output head over an odd number of tokens.
        _i8("i8_head", m=1021, n=150000, k=2048),
        # Small square updates of one shape, as a batch: the products are short and launches count.
        _ortho("ortho_small", batch=24, rows=256, cols=256),
        # A tall update with odd sizes.
        _ortho("ortho_odd", rows=3001, cols=1000, dtype="bf16"),
        # A large projection's update.
        _ortho("ortho_large", rows=4096, cols=16384),
    ]


def _log_int(rng, a, b):
    v = int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    kind = rng.choice(["logprob", "logprob", "loss", "i8", "i8", "ortho"])
    if kind == "logprob":
        vocab = rng.choice([32000, 50021, 131072, 150000, _log_int(rng, 1000, 150000)])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        most = 4096 * 150000 // (2 if dtype == "f32" else 1) // vocab
        grad = rng.random() < 0.5
        return _logprob(rows=_log_int(rng, 1, min(8192, most)), vocab=vocab, dtype=dtype,
                        top=rng.choice([0, 1, 5, 20, 64]), grad=grad, grad_entropy=grad and rng.random() < 0.5,
                        masked=rng.choice([0.0, 0.25]), padded=rng.choice([0, 11]),
                        temperature=rng.choice([1.0, 0.7, 1.3]))
    if kind == "loss":
        n = _log_int(rng, 16, 3000)
        return _loss(n=n, tokens=n * rng.randint(300, 5600) + rng.randint(0, 63), sigma=rng.uniform(0.1, 0.8),
                     masked=rng.random() < 0.5, weighted=rng.random() < 0.5)
    if kind == "i8":
        k = rng.choice([1024, 2048, 4096, 8192, _log_int(rng, 64, 8192)])
        n = rng.choice([4096, 16384, 150000, _log_int(rng, 256, 16384)])
        m = _log_int(rng, 1, min(4096, 4096 * 16384 * 4096 // (n * k)))
        return _i8(m=m, n=n, k=k, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    rows, cols = _log_int(rng, 32, 4000), _log_int(rng, 32, 8000)
    if rng.random() < 0.5:
        rows, cols = (rows + 319) // 320 * 320, (cols + 319) // 320 * 320
    if rng.random() < 0.3:
        rows, cols = cols, rows
    batch = rng.randint(2, 24) if rows * cols <= 512 * 512 else 1
    return _ortho(batch=batch, rows=rows, cols=cols, dtype=rng.choice(["f32", "bf16"]))


# ---- inputs ------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    state = {"case": case, "kept": {}}
    state.update({"logprob": _prepare_logprob, "loss": _prepare_loss, "i8": _prepare_i8, "ortho": _prepare_ortho}[case["kind"]](case, g))
    return state


def _prepare_logprob(c, g):
    rows, vocab = c["rows"], c["vocab"]
    z = 2.5 * torch.randn(rows, vocab, generator=g, device=DEV)
    if c["padded"]:                                          # vocabulary entries that stand for no token
        z[:, vocab - c["padded"]:] = -math.inf
    u = torch.rand(rows, vocab, generator=g, device=DEV).clamp_(min=1e-30)
    ids = (z / c["temperature"] - u.log_().neg_().log_()).argmax(1).to(torch.int32)      # sampled tokens
    del u
    if c["masked"]:
        ids[torch.rand(rows, generator=g, device=DEV) < c["masked"]] = -1
    s = {"logits": z.to(DTYPES[c["dtype"]]), "ids": ids}
    if c["grad"]:
        s["g"] = torch.randn(rows, generator=g, device=DEV)
        s["gh"] = 0.01 * torch.randn(rows, generator=g, device=DEV) if c["grad_entropy"] else None
    return s


def _lengths(g, n, tokens, sigma):
    """n log-normal lengths of at least one token that add up to `tokens`."""
    w = torch.exp(sigma * torch.randn(n, generator=g, device=DEV, dtype=torch.float64).clamp(-3.0, 3.0))
    free = tokens - n
    L = (w * (free / w.sum())).floor().to(torch.int64)
    left = free - L.sum()
    L += left // n + (torch.arange(n, device=DEV) < left % n)
    return L + 1


def _prepare_loss(c, g):
    n, tokens = c["n"], c["tokens"]
    L = _lengths(g, n, tokens, c["sigma"])
    off = torch.zeros(n + 1, dtype=torch.int64, device=DEV)
    torch.cumsum(L, 0, out=off[1:])
    lp_b = (-1.2 + 0.8 * torch.randn(tokens, generator=g, device=DEV)).clamp(max=0.0)
    lp_n = (lp_b + 0.15 * torch.randn(tokens, generator=g, device=DEV)).clamp(max=0.0)
    s = {"off": off, "lp_b": lp_b, "lp_n": lp_n, "adv": torch.randn(n, generator=g, device=DEV), "tags": None, "weight": None}
    if c["masked"]:
        turn = torch.randint(0, 3, ((tokens + 499) // 500,), generator=g, device=DEV)      # spans of 500: one in three a tool's
        s["tags"] = torch.where(turn == 0, -1, 7).to(torch.int32).repeat_interleave(500)[:tokens].contiguous()
    if c["weighted"]:
        s["weight"] = L.float().reciprocal() * (tokens / n)
    return s


def _prepare_i8(c, g):
    x = torch.randn(c["m"], c["k"], generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(c["k"], generator=g, device=DEV))               # channels of different sizes
    w = 0.02 * torch.randn(c["n"], c["k"], generator=g, device=DEV)
    scale = w.abs().amax(1) / 127
    w8 = torch.round(w / scale[:, None]).clamp(-127, 127).to(torch.int8)
    return {"x": x.to(DTYPES[c["dtype"]]), "w": w8, "w_scale": scale}


def _prepare_ortho(c, g):
    b, r, k = c["batch"], c["rows"], c["cols"]
    low = max(1, min(r, k) // 8)                             # momentum: a few strong directions over noise
    u = torch.randn(b, r, k, generator=g, device=DEV)
    u += torch.bmm(torch.randn(b, r, low, generator=g, device=DEV), torch.randn(b, low, k, generator=g, device=DEV)) * (2.0 / math.sqrt(low))
    return {"update": (1e-3 * u).to(DTYPES[c["dtype"]])}


# ---- one pass ----------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2609_36830_amd as pace
        return {"logprob": _own_logprob, "loss": _own_loss, "i8": _own_i8, "ortho": _own_ortho}[kind](pace, state)
    return {"logprob": _plain_logprob, "loss": _plain_loss, "i8": _plain_i8, "ortho": _plain_ortho}[kind](state)


def _kept(state, make):
    """Outputs and workspace that a program keeps from step to step, made at the first one."""
    if not state["kept"]:
        state["kept"] = make()
    return state["kept"]


def _own_logprob(pace, s):
    c = s["case"]
    k = _kept(s, lambda: pace.token_logprob_buffers(c["rows"], c["vocab"], c["top"], DEV))
    logp, entropy, stats, top_ids, top_logp = pace.pace_token_logprob(
        s["logits"], s["ids"], temperature=c["temperature"], top_k=c["top"], buffers=k)
    out = {"logp": logp, "entropy": entropy}
    if c["top"]:
        out.update(top_ids=top_ids, top_logp=top_logp)
    if c["grad"]:
        k.setdefault("grad", torch.empty_like(s["logits"]))
        out["grad"] = pace.pace_token_logprob_backward(s["logits"], s["ids"], stats, s["g"], entropy=entropy,
                                                       grad_entropy=s["gh"], temperature=c["temperature"],
                                                       grad_logits_out=k["grad"])
    return out


def _own_loss(pace, s):
    c = s["case"]
    k = _kept(s, lambda: pace.policy_loss_buffers(c["n"], c["tokens"], DEV))
    grad, loss, kl, clipped = pace.pace_policy_loss(s["lp_n"], s["lp_b"], s["off"], s["adv"], tags=s["tags"],
                                                    weight=s["weight"], scale=1.0 / c["tokens"], clip_low=CLIP_LOW,
                                                    clip_high=CLIP_HIGH, dual_clip=DUAL_CLIP, buffers=k)
    return {"grad": grad, "loss": loss, "kl": kl, "clipped": clipped}


def _own_i8(pace, s):
    c = s["case"]
    k = _kept(s, lambda: pace.matmul_i8_buffers(c["m"], c["n"], c["k"], DTYPES[c["out"]], DEV))
    q, scale = pace.pace_quantize_rows(s["x"], q_out=k["q"], scale_out=k["scale"])
    out = pace.pace_matmul_i8(q, scale, s["w"], s["w_scale"], out=k["out"], workspace=k["workspace"])
    return {"out": out, "scale": scale}


def _own_ortho(pace, s):
    c = s["case"]
    k = _kept(s, lambda: pace.orthogonalize_buffers(c["batch"], c["rows"], c["cols"], DEV))
    return {"out": pace.pace_orthogonalize(s["update"], steps=STEPS, coefs=COEFS, eps=EPS, out=k["out"], workspace=k["workspace"])}


def _plain_logprob(s):
    c, ids, inv = s["case"], s["ids"], 1.0 / s["case"]["temperature"]
    live, t = ids >= 0, ids.clamp(min=0).to(torch.int64)
    z = s["logits"].float()
    d = (z - z.amax(1, keepdim=True)) * inv
    e = torch.exp(d)
    total = e.sum(1)
    ed = torch.where(e > 0, e * d, 0.0)
    log_total = torch.log(total)
    logp = d.gather(1, t[:, None])[:, 0] - log_total
    entropy = log_total - ed.sum(1) / total
    out = {"logp": torch.where(live, logp, 0.0), "entropy": torch.where(live, entropy, 0.0)}
    del ed
    if c["top"]:
        # One whole number for (logit descending, index ascending): the logit's bits in order, then the index from the end.
        bits = (z + 0.0).view(torch.int32).to(torch.int64)
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 31) + (c["vocab"] - 1 - torch.arange(c["vocab"], device=DEV))
        best = key.topk(c["top"], 1).values
        ids_top = c["vocab"] - 1 - (best & 0x7FFFFFFF)
        out["top_ids"] = torch.where(live[:, None], ids_top, -1).to(torch.int32)
        out["top_logp"] = torch.where(live[:, None], d.gather(1, ids_top) - log_total[:, None], -math.inf)
        del bits, key
    if c["grad"]:
        p = e / total[:, None]
        grad = -p * s["g"][:, None]
        grad.scatter_add_(1, t[:, None], s["g"][:, None])
        if s["gh"] is not None:
            grad -= torch.where(p > 0, p * (d - log_total[:, None] + entropy[:, None]), 0.0) * s["gh"][:, None]
        out["grad"] = torch.where(live[:, None], grad * inv, 0.0).to(s["logits"].dtype)
    return out


def _plain_loss(s):
    c, n = s["case"], s["case"]["n"]
    off, adv = s["off"], s["adv"]
    tr = torch.repeat_interleave(torch.arange(n, device=DEV), off[1:] - off[:-1], output_size=c["tokens"])
    a = adv[tr]
    w = (s["weight"] if s["weight"] is not None else torch.ones_like(adv)) / c["tokens"]
    w = w[tr]
    d = s["lp_n"] - s["lp_b"]
    r = torch.exp(d)
    lo, hi, dual = (torch.tensor(math.log(v), dtype=torch.float32, device=DEV) for v in (1 - CLIP_LOW, 1 + CLIP_HIGH, DUAL_CLIP))
    up, down, far = (a > 0) & (d > hi), (a < 0) & (d < lo), (a < 0) & (d > dual)
    rc = torch.where(up, 1 + CLIP_HIGH, torch.where(down, 1 - CLIP_LOW, torch.where(far, DUAL_CLIP, r)))
    cut = up | down | far
    loss = -w * a * rc
    grad = torch.where(cut, 0.0, -w * a * r)
    kl = torch.expm1(d) - d
    if s["tags"] is not None:
        live = s["tags"] != -1
        loss, grad, kl, cut = torch.where(live, loss, 0.0), torch.where(live, grad, 0.0), torch.where(live, kl, 0.0), cut & live
    total = lambda v: torch.segment_reduce(v, "sum", lengths=off[1:] - off[:-1])
    return {"grad": grad, "loss": total(loss), "kl": total(kl), "clipped": total(cut.float()).to(torch.int32)}


def _plain_i8(s):
    x = s["x"].float()
    most = x.abs().amax(1)
    q = torch.round(x * (127.0 / most)[:, None]).clamp(-127, 127)
    scale = most / 127.0
    acc = q @ s["w"].float().t()
    return {"out": (acc * (scale[:, None] * s["w_scale"][None, :])).to(DTYPES[s["case"]["out"]]), "scale": scale}


def _plain_ortho(s):
    x = s["update"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    a, b, c = COEFS
    for _ in range(STEPS):
        p = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * p + c * torch.bmm(p, p), x)
    if tall:
        x = x.transpose(1, 2).contiguous()
    return {"out": x.to(torch.bfloat16)}


# ---- what a pass cannot do without --------------------------------------------
def work(case):
    c = case
    if c["kind"] == "logprob":
        size = 4 if c["dtype"] == "f32" else 2
        live = c["rows"] * (1 - c["masked"])
        b = live * c["vocab"] * size + c["rows"] * (12 + 8 * c["top"])
        f = 6 * live * c["vocab"]
        if c["grad"]:
            b += live * c["vocab"] * size + c["rows"] * c["vocab"] * size + c["rows"] * 16
            f *= 2
        return {"bytes": b, "flops": f}
    if c["kind"] == "loss":
        return {"bytes": c["tokens"] * (16 if c["masked"] else 12) + c["n"] * 24, "flops": 12 * c["tokens"]}
    if c["kind"] == "i8":
        size = 4 if c["dtype"] == "f32" else 2
        out = 4 if c["out"] == "f32" else 2
        return {"bytes": c["m"] * c["k"] * size + c["n"] * (c["k"] + 4) + c["m"] * c["n"] * out, "flops": 2 * c["m"] * c["n"] * c["k"]}
    m, n = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
    # The two symmetric products by half, the third whole.
    return {"bytes": c["batch"] * m * n * ((4 if c["dtype"] == "f32" else 2) + 2), "flops": c["batch"] * STEPS * (3 * m * m * n + m * m * m)}


# ---- the definitions in 64 bits -------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"logprob": _exact_logprob, "loss": _exact_loss, "i8": _exact_i8, "ortho": _exact_ortho}[case["kind"]](s)


def _exact_logprob(s):
    c = s["case"]
    z = s["logits"].double() / c["temperature"]
    lse = torch.logsumexp(z, 1, keepdim=True)
    lp = z - lse
    p = torch.exp(lp)
    plogp = torch.where(p > 0, p * lp, 0.0)
    h = -plogp.sum(1)
    live, t = s["ids"] >= 0, s["ids"].clamp(min=0).long()
    out = {"logp": torch.where(live, lp.gather(1, t[:, None])[:, 0], 0.0), "entropy": torch.where(live, h, 0.0)}
    if c["top"]:
        out["top_ids"] = None
        out["top_logp"] = torch.where(live[:, None], lp.sort(1, descending=True).values[:, :c["top"]], -math.inf)
    if c["grad"]:
        one = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
        grad = s["g"].double()[:, None] * (one - p)
        if s["gh"] is not None:
            grad = grad - s["gh"].double()[:, None] * (plogp + p * h[:, None])
        out["grad"] = torch.where(live[:, None], grad / c["temperature"], 0.0)
    return out


def _exact_loss(s):
    c = s["case"]
    off = s["off"]
    L = off[1:] - off[:-1]
    d = (s["lp_n"] - s["lp_b"]).double()                   # the log ratio is a binary32 number by definition
    live = torch.ones(c["tokens"], dtype=torch.bool, device=DEV) if s["tags"] is None else s["tags"] != -1
    each = s["adv"].double() * (1.0 if s["weight"] is None else s["weight"].double()) / c["tokens"]
    g = torch.repeat_interleave(each, L, output_size=c["tokens"])
    r = torch.exp(d)
    bounded = torch.minimum(torch.maximum(r, torch.tensor(1 - CLIP_LOW, device=DEV).double()), torch.tensor(DUAL_CLIP, device=DEV).double())
    loss = torch.where(g > 0, -g * r.clamp(max=1 + CLIP_HIGH), -g * bounded)
    free = torch.where(g > 0, r <= 1 + CLIP_HIGH, (r >= 1 - CLIP_LOW) & (r <= DUAL_CLIP))
    grad = torch.where(free & live, -g * r, 0.0)
    kl = torch.expm1(d) - d

    def sums(v):
        run = torch.zeros(c["tokens"] + 1, dtype=torch.float64, device=DEV)
        torch.cumsum(torch.where(live, v, 0.0), 0, out=run[1:])
        return run[off[1:]] - run[off[:-1]]

    return {"grad": grad, "loss": sums(loss), "kl": sums(kl), "clipped": None}


def _exact_i8(s):
    x = s["x"].double()
    most = x.abs().amax(1, keepdim=True)
    q = torch.round(x * (127.0 / most))
    scale = most / 127.0
    return {"out": (q @ s["w"].double().t()) * scale * s["w_scale"].double()[None, :], "scale": scale[:, 0]}


def _exact_ortho(s):
    x = s["update"].double()
    if x.shape[1] > x.shape[2]:
        return {"out": _exact_wide(x.transpose(1, 2)).transpose(1, 2)}
    return {"out": _exact_wide(x)}


def _exact_wide(x):
    """The steps as one polynomial of the Gram matrix, which commutes with its own polynomials."""
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + EPS)
    gram = x @ x.transpose(1, 2)
    one = torch.eye(gram.shape[1], dtype=torch.float64, device=DEV).expand_as(gram)
    whole = one
    for _ in range(STEPS):
        step = COEFS[0] * one + COEFS[1] * gram + COEFS[2] * (gram @ gram)
        whole = step @ whole
        gram = step @ gram @ step
    return whole @ x
