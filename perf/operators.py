"""The losses over a language model's logits that this framework's speed is
judged by, as a training program calls them.

A program holds the logits of a step (rows x vocabulary, the largest tensor of
it) and what its loss needs beside them: the next tokens, with -100 where a
prompt or padding is not trained on, and

  score       nothing else: the log-probabilities of given tokens (a reference
              model's, an old policy's, an evaluation's)
  logp        the weight of each token's log-probability in the loss (-1 / count
              is cross entropy): log-probabilities and the gradient
  preference  pairs of a chosen and a rejected sequence and the reference
              model's log-probabilities of both
  policy      the old policy's and a reference's log-probability of each token
              and its advantage: the clipped surrogate with a KL term
  distill     a teacher's top logits of each row, perhaps its log-sum-exp (the
              mass outside the list) and the hard label

and takes the loss with its gradient with respect to the logits.  Rows come
padded (batch x steps, the logits of all positions but the last against the
tokens of all but the first, so neither tensor is contiguous) or packed (the
sequences one behind the other).
"""
from __future__ import annotations

import math
import random

import torch

own = False

IGNORE = -100
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
REST_FLOOR = 2.0 ** -20     # mass outside the teacher's list below this is rounding: none


# ----------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------
def _case(name, op, seqs, steps, vocab, dtype, packed=False, masked=0.0, vocab_pad=0, lens_seed=1, full=False, **more):
    """seqs sequences of up to `steps` rows, `masked` of each one's rows a
    prompt; the last `vocab_pad` columns are padding of the vocabulary (-inf)."""
    c = {"op": op, "seqs": seqs, "steps": steps, "vocab": vocab, "dtype": dtype, "packed": packed,
         "masked": masked, "vocab_pad": vocab_pad, "lens_seed": lens_seed, "full": full, **more}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the next token of one sequence scored: launches and latency
        _case("score_1x32000", "score", 1, 1, 32000, "bf16", packed=True, full=True, temperature=1.0),
        # a reference model's pass over a large packed batch: 2.2e9 logits
        _case("score_17000x128000", "score", 17, 1000, 128000, "bf16", packed=True, full=True, temperature=1.0),
        # cross entropy of one pre-training batch in fp32, odd vocabulary
        _case("logp_2047x50265_fp32", "logp", 1, 2047, 50265, "fp32", full=True, temperature=1.0),
        # one pair of short answers
        _case("preference_2x48", "preference", 2, 48, 32000, "bf16", masked=0.3, kind="sigmoid", beta=0.1,
              smoothing=0.0, average=False, grad_scale=1.0),
        # eight pairs, padded to 512 tokens, prompts not trained on
        _case("preference_16x512", "preference", 16, 512, 32000, "bf16", masked=0.4, kind="sigmoid", beta=0.1,
              smoothing=0.1, average=False, grad_scale=1.0),
        # sixteen packed pairs over a large vocabulary in fp16, with loss scaling
        _case("preference_packed_128000_fp16", "preference", 32, 200, 128000, "fp16", packed=True, masked=0.25,
              kind="squared", beta=0.1, smoothing=0.0, average=True, grad_scale=4096.0),
        # one short sampled answer in fp32
        _case("policy_1x64_fp32", "policy", 1, 64, 32000, "fp32", full=True, kl=0.0, low=0.2, high=0.2,
              reduction="token", temperature=1.0),
        # a group of eight samples with a KL term, the padded vocabulary masked
        _case("policy_8x1024", "policy", 8, 1024, 50304, "bf16", masked=0.25, vocab_pad=39, kl=0.04, low=0.2,
              high=0.28, reduction="token", temperature=1.0),
        # packed samples of a large vocabulary, each sequence with the same weight
        _case("policy_packed_128000", "policy", 16, 400, 128000, "bf16", packed=True, masked=0.2, kl=0.01, low=0.2,
              high=0.2, reduction="sequence", temperature=0.8),
        # eight teacher entries a row, a short batch
        _case("distill_64x32000_k8", "distill", 1, 64, 32000, "bf16", packed=True, full=True, top=8,
              temperature=1.0, rest=False, hard=0.0, ragged=False),
        # odd vocabulary in fp32, the mass outside the list counted, lists of different lengths
        _case("distill_2048x50265_k64_rest_fp32", "distill", 4, 512, 50265, "fp32", packed=True, full=True, top=64,
              temperature=2.0, rest=True, hard=0.0, ragged=True),
        # the largest: teacher lists of 128 and hard labels
        _case("distill_4000x128000_k128_hard", "distill", 4, 1000, 128000, "bf16", packed=True, masked=0.1,
              full=True, top=128, temperature=2.0, rest=False, hard=0.3, ragged=False),
    ]


def draw(rng):
    """One call of the same ranges: vocabularies from 256 (bytes) to 131072,
    one row to as many as 5e8 logits (2.2e9 where only log-probabilities are
    asked for) hold, odd sizes as often as round ones, every type, masks from
    none to most of the rows."""
    op = rng.choice(["score", "logp", "preference", "policy", "distill"])
    vocab = int(round(math.exp(rng.uniform(math.log(256), math.log(131072)))))
    unit = rng.choice([1, 1, 8, 64])
    vocab = max(256, vocab // unit * unit)
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    most = (2.0e9 if op == "score" else 4.5e8) / (2 if dtype == "fp32" else 1)
    rows = math.exp(rng.uniform(0.0, math.log(min(most / vocab, 60000))))
    if op == "preference":
        seqs = 2 * int(round(math.exp(rng.uniform(0.0, math.log(min(32, max(1.0, rows / 2)))))))
    else:
        seqs = int(round(math.exp(rng.uniform(0.0, math.log(min(64, max(1.0, rows)))))))
    steps = max(1, int(rows / seqs))
    common = dict(packed=rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.25, 0.5, 0.8]),
                  vocab_pad=rng.choice([0, 0, rng.randint(1, 63)]), lens_seed=rng.randint(1, 1 << 20),
                  full=rng.random() < 0.3)
    if op == "score" or op == "logp":
        more = dict(temperature=rng.choice([1.0, 1.0, 0.7, 1.5]))
    elif op == "preference":
        kind = rng.choice(["sigmoid", "sigmoid", "hinge", "squared"])
        more = dict(kind=kind, beta=rng.choice([0.05, 0.1, 0.3]), average=kind == "squared",
                    smoothing=rng.choice([0.0, 0.1]) if kind == "sigmoid" else 0.0,
                    grad_scale=4096.0 if dtype == "fp16" else 1.0)
    elif op == "policy":
        more = dict(kl=rng.choice([0.0, 0.01, 0.1]), low=0.2, high=rng.choice([0.2, 0.28]),
                    reduction=rng.choice(["token", "sequence"]), temperature=rng.choice([1.0, 1.0, 0.8]))
    else:
        top = int(round(math.exp(rng.uniform(0.0, math.log(256)))))
        more = dict(top=min(top, vocab // 4), temperature=rng.choice([1.0, 2.0, 0.5]), rest=rng.random() < 0.4,
                    hard=rng.choice([0.0, 0.3]), ragged=rng.random() < 0.3)
    return _case(None, op, seqs, steps, vocab, dtype, **common, **more)


def _spans(case):
    """(first row, first trained row, end, rows held) of each sequence."""
    r = random.Random(case["lens_seed"])
    out, at = [], 0
    for i in range(case["seqs"]):
        n = case["steps"] if case["full"] or i == 0 else int(round(case["steps"] * r.uniform(0.1, 1.0)))
        held = n if case["packed"] else case["steps"]
        out.append((at, at + int(n * case["masked"]), at + n, held))
        at += held
    return out


def _rows(case):
    first, _, _, held = _spans(case)[-1]
    return first + held


def _trained(case):
    return sum(end - start for _, start, end, _ in _spans(case))


def work(case):
    """Bytes: the logits of the rows that are trained on once, the gradient of
    every row once, what each row has beside them.  Flops: difference, scale,
    exponential and sum of an element, three more for its gradient, twice the
    first where hard labels need a second sum."""
    rows, used, V = _rows(case), _trained(case), case["vocab"]
    es = 4 if case["dtype"] == "fp32" else 2
    nbytes, flops = float(used) * V * es + 12.0 * rows, 4.0 * used * V
    if case["op"] != "score":
        nbytes += float(rows) * V * es
        flops += 3.0 * used * V
    if case["op"] == "policy":
        nbytes += 12.0 * rows
    if case["op"] == "distill":
        nbytes += 8.0 * rows * case["top"]
        if case["hard"] and case["temperature"] != 1.0:
            flops += 7.0 * used * V
    return {"bytes": nbytes, "flops": flops}


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _fill(case, gen, y):
    """Logits of every row as a model gives them: a spread of a few units and
    a token that stands out, the row's own target in most rows."""
    rows, V, pad = y.numel(), case["vocab"], case["vocab_pad"]
    z = torch.empty(rows, V, device="cuda", dtype=DTYPES[case["dtype"]])
    step = max(1, (1 << 27) // V)
    for a in range(0, rows, step):
        b = min(rows, a + step)
        x = torch.randn(b - a, V, generator=gen, device="cuda").mul_(2.0)
        if pad:
            x[:, V - pad:] = -math.inf
        z[a:b] = x
    like = torch.rand(rows, generator=gen, device="cuda")
    peak = 7.0 + 3.0 * torch.randn(rows, generator=gen, device="cuda")
    other = torch.randint(0, V - pad, (rows,), generator=gen, device="cuda")
    z[torch.arange(rows, device="cuda"), torch.where(like < 0.7, y, other)] = peak.to(z.dtype)
    return z


def _logps32(z, y, temperature):
    """Log-probabilities of the rows' tokens, some rows at a time."""
    out = torch.empty(z.shape[0], device="cuda")
    step = max(1, (1 << 27) // z.shape[1])
    for a in range(0, z.shape[0], step):
        x = z[a:a + step].float() / temperature
        m = x.amax(1)
        picked = x.gather(1, y[a:a + step, None])[:, 0]
        out[a:a + step] = picked - m - (x - m[:, None]).exp().sum(1).log()
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows, V, B, S = _rows(case), case["vocab"], case["seqs"], case["steps"]
    spans, top = _spans(case), V - case["vocab_pad"]
    shifted = not case["packed"]
    # all positions: a padded sequence holds one more token than trained rows
    held = B * (S + 1) if shifted else rows
    y_all = torch.randint(0, top, (held,), generator=gen, device="cuda")
    z_all = _fill(case, gen, y_all)
    live = torch.zeros(rows, dtype=torch.bool)
    for _, start, end, _ in spans:
        live[start:end] = True
    live = live.cuda()
    state = {"case": case}
    if shifted:
        # position t predicts token t + 1
        tokens = torch.empty(B, S + 1, device="cuda", dtype=torch.int64)
        tokens[:, 1:] = torch.where(live.view(B, S), y_all.view(B, S + 1)[:, :-1], IGNORE)
        tokens[:, 0] = 0
        state["logits"] = z_all.view(B, S + 1, V)[:, :-1]
        state["targets"] = tokens[:, 1:]
        z, y = state["logits"].reshape(rows, V) if case["op"] == "policy" else None, y_all.view(B, S + 1)[:, :-1].reshape(-1)
    else:
        state["logits"] = z = z_all
        state["targets"] = torch.where(live, y_all, IGNORE)
        y = y_all
    shape = state["targets"].shape
    if case["packed"] and case["op"] in ("preference", "policy"):
        ends = [spans[0][0]] + [s[0] + s[3] for s in spans]
        state["cu_seqlens"] = torch.tensor(ends, device="cuda", dtype=torch.int32)
    else:
        state["cu_seqlens"] = None
    if case["op"] == "logp":
        state["weights"] = torch.full((rows,), -1.0 / max(1, _trained(case)), device="cuda").view(shape)
    elif case["op"] == "preference":
        # the reference model's: what the policy has now, but for its training
        n = torch.tensor([e - s for _, s, e, _ in spans], device="cuda")
        mean = -math.log(top) * 0.5
        noise = torch.randn(B, generator=gen, device="cuda")
        state["ref"] = (mean + 0.1 * noise if case["average"] else mean * n + noise).float()
    elif case["op"] == "policy":
        lp = _logps32(z, y, case["temperature"])
        d = 0.15 * torch.randn(rows, generator=gen, device="cuda")
        # no token on the very edge of the clipped range, where the gradient has no single value
        for edge in (math.log1p(-case["low"]), math.log1p(case["high"])):
            d = torch.where((d - edge).abs() < 1e-3, d + 4e-3, d)
        state["old"] = (lp - d).view(shape)
        state["ref"] = (lp + 0.2 * torch.randn(rows, generator=gen, device="cuda")).view(shape) if case["kl"] else None
        state["advantages"] = (torch.randn(rows, generator=gen, device="cuda") + 0.3).view(shape)
    elif case["op"] == "distill":
        K = case["top"]
        stride = torch.randint(1, max(2, top // K + 1), (rows, 1), generator=gen, device="cuda")
        k = torch.arange(K, device="cuda")
        ids = (y[:, None] + k * stride) % top               # distinct: K * stride <= top
        gaps = torch.rand(rows, K, generator=gen, device="cuda") * (6.0 / (1.0 + k))
        t = 9.0 - gaps.cumsum(1) + torch.randn(rows, 1, generator=gen, device="cuda")
        if case["ragged"]:
            n = torch.randint(0, K + 1, (rows, 1), generator=gen, device="cuda")
            ids = torch.where(k < n, ids, -1)
        state["ids"] = ids.to(torch.int32).view(*shape, K)
        # in the precision that the list was stored in
        state["teacher"] = t.to(DTYPES[case["dtype"]]).view(*shape, K)
        state["lse"] = None
        if case["rest"]:
            t = torch.where(ids >= 0, state["teacher"].view(rows, K).float() / case["temperature"], -math.inf)
            inside = 0.7 + 0.29 * torch.rand(rows, generator=gen, device="cuda")
            lse = t.logsumexp(1) - inside.log()
            state["lse"] = torch.where(lse.isfinite(), lse, 0.0).view(shape)
    return state


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def run(state):
    case = state["case"]
    return (_own if own else _plain)(case, state)


def _own(case, st):
    from paper_2507_08784_amd import losses

    op = case["op"]
    if op == "score":
        r = losses.token_logprobs(st["logits"], st["targets"], temperature=case["temperature"])
        return {"logps": r.logps}
    if op == "logp":
        r = losses.token_logprobs(st["logits"], st["targets"], weights=st["weights"], temperature=case["temperature"])
        return {"logps": r.logps, "dlogits": r.dlogits}
    if op == "preference":
        r = losses.preference_loss(st["logits"], st["targets"], st["ref"], beta=case["beta"], kind=case["kind"],
                                   label_smoothing=case["smoothing"], average=case["average"],
                                   cu_seqlens=st["cu_seqlens"], grad=True, grad_scale=case["grad_scale"])
        return {"loss": r.loss, "logps": r.logps, "rewards": r.rewards, "dlogits": r.dlogits}
    if op == "policy":
        r = losses.policy_loss(st["logits"], st["targets"], st["old"], st["advantages"], ref_logps=st["ref"],
                               clip_low=case["low"], clip_high=case["high"], kl_coef=case["kl"],
                               reduction=case["reduction"], cu_seqlens=st["cu_seqlens"],
                               temperature=case["temperature"], grad=True)
        return {"loss": r.loss, "logps": r.logps, "kl": r.kl, "clipped": r.clipped, "dlogits": r.dlogits}
    r = losses.distill_loss(st["logits"], st["ids"], st["teacher"], temperature=case["temperature"],
                            teacher_lse=st["lse"], targets=st["targets"], hard_weight=case["hard"], grad=True)
    return {"loss": r.loss, "losses": r.losses, "dlogits": r.dlogits}


def _softmax(logits, temperature):
    """Rows as fp32 x = z / temperature, their probabilities, and log sum exp
    in its two parts (the row's maximum and the logarithm above it)."""
    x = logits.float().reshape(-1, logits.shape[-1])
    if temperature != 1.0:
        x = x / temperature
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    s = e.sum(1, keepdim=True)
    return x, e / s, m, torch.log(s)


def _members(case, st, rows):
    """sequences x rows: which rows belong to which sequence."""
    r = torch.arange(rows, device="cuda")
    if st["cu_seqlens"] is not None:
        cu = st["cu_seqlens"][:, None]
        return (r >= cu[:-1]) & (r < cu[1:])
    return r // case["steps"] == torch.arange(case["seqs"], device="cuda")[:, None]


def _plain(case, st):
    """Elementary operations in fp32."""
    op, dtype, shape = case["op"], st["logits"].dtype, st["targets"].shape
    y = st["targets"].reshape(-1)
    live = y != IGNORE
    safe = torch.where(live, y, 0)[:, None]
    zero = torch.zeros((), device="cuda")
    if op == "distill":
        return _plain_distill(case, st, live, safe, dtype, shape)
    temperature = case.get("temperature", 1.0)
    x, p, m, logs = _softmax(st["logits"], temperature)
    lp = torch.where(live, (x.gather(1, safe) - m - logs)[:, 0], zero)
    out = {}
    if op == "score":
        return {"logps": lp.view(shape)}
    if op == "logp":
        out["logps"], coef = lp.view(shape), st["weights"].reshape(-1)
    elif op == "preference":
        member = _members(case, st, y.numel())
        n = (member & live).sum(1).clamp(min=1) if case["average"] else torch.ones(case["seqs"], device="cuda")
        seq = (member * lp).sum(1) / n
        half, beta, smooth = case["seqs"] // 2, case["beta"], case["smoothing"]
        ratio = seq - st["ref"]
        delta = ratio[:half] - ratio[half:]
        h = beta * delta
        if case["kind"] == "sigmoid":
            pos = torch.log1p(torch.exp(-h.abs()))
            loss = (1 - smooth) * (pos + (-h).clamp(min=0)) + smooth * (pos + h.clamp(min=0))
            slope = beta * (smooth - 1 / (1 + torch.exp(h)))
        elif case["kind"] == "hinge":
            loss, slope = (1 - h).clamp(min=0), torch.where(h < 1, -beta, 0.0)
        else:
            off = delta - 1 / (2 * beta)
            loss, slope = off * off, 2 * off
        slope = slope * (case["grad_scale"] / half)
        per = torch.cat([slope, -slope]) / n
        coef = (member * per[:, None]).sum(0)
        out.update(loss=loss.sum() / half, logps=seq, rewards=beta * ratio)
    else:
        if case["reduction"] == "token":
            w = live / live.sum().clamp(min=1)
        else:
            member = _members(case, st, y.numel())
            n = (member & live).sum(1).clamp(min=1) * case["seqs"]
            w = (member / n[:, None]).sum(0)
        A = st["advantages"].reshape(-1)
        r = torch.exp(lp - st["old"].reshape(-1))
        free, bound = r * A, r.clamp(1 - case["low"], 1 + case["high"]) * A
        term, slope = -torch.minimum(free, bound), torch.where(free <= bound, -free, zero)
        out["kl"] = zero
        if st["ref"] is not None:
            d = st["ref"].reshape(-1) - lp
            k = torch.expm1(d) - d
            out["kl"] = torch.where(live, w * k, zero).sum()
            term, slope = term + case["kl"] * k, slope - case["kl"] * torch.expm1(d)
        out["loss"] = torch.where(live, w * term, zero).sum()
        out["clipped"] = torch.where(live, w * (free > bound), zero).sum()
        out["logps"], coef = lp.view(shape), w * slope
    # d lp / d z = (onehot - p) / temperature
    coef = torch.where(live, coef / temperature, zero)[:, None]
    g = torch.where(live[:, None], -p * coef, zero)
    g.scatter_add_(1, safe, coef)
    out["dlogits"] = g.to(dtype).view(st["logits"].shape)
    return out


def _plain_distill(case, st, live, safe, dtype, shape):
    tau, hard, rows, K = case["temperature"], case["hard"], live.numel(), case["top"]
    ids = st["ids"].reshape(rows, K).long()
    t = st["teacher"].reshape(rows, K).float() / tau
    zero = torch.zeros((), device="cuda")
    there = (ids >= 0) & (t != -math.inf)
    at = torch.where(there, ids, 0)
    t = torch.where(there, t, -math.inf)
    x, q, m, logs = _softmax(st["logits"], tau)
    if case["rest"]:
        logp = t - st["lse"].reshape(-1, 1)
    else:
        high = t.amax(1, keepdim=True)
        high = torch.where(high == -math.inf, zero, high)
        logp = t - high - torch.log(torch.exp(t - high).sum(1, keepdim=True))
    p = torch.where(there, torch.exp(logp), zero)
    logq = x.gather(1, at) - m - logs
    kl = torch.where(there, p * (logp - logq), zero).sum(1)
    mass = p.sum(1, keepdim=True)
    lead = mass
    outside = torch.ones_like(q)
    outside.scatter_(1, at, torch.where(there, 0.0, outside.gather(1, at)))
    if case["rest"]:
        rest = 1 - mass
        rest = torch.where((rest < REST_FLOOR) | ~there.any(1, keepdim=True), zero, rest)
        qr = (q * outside).sum(1, keepdim=True)
        use = rest > 0
        kl = kl + torch.where(use, rest * (torch.log(rest) - torch.log(qr)), zero)[:, 0]
        lead = mass + rest
        g = q * lead - torch.where(use, rest / qr, zero) * (q * outside)
    else:
        g = q * lead
    g.scatter_add_(1, at, -p)
    row, g = (1 - hard) * tau * tau * kl, g * ((1 - hard) * tau)
    if hard:
        if tau != 1.0:
            x, q, m, logs = _softmax(st["logits"], 1.0)
        row = row - hard * (x.gather(1, safe) - m - logs)[:, 0]
        g = g + hard * q
        g.scatter_add_(1, safe, torch.full_like(safe, -hard, dtype=torch.float32))
    row = torch.where(live, row, zero)
    n = live.sum().clamp(min=1)
    g = torch.where(live[:, None], g / n, zero)
    return {"loss": row.sum() / n, "losses": row.view(shape), "dlogits": g.to(dtype).view(st["logits"].shape)}


# ----------------------------------------------------------------------------
# the same in 64 bits, by differentiating each loss as it is defined
# ----------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    z = st["logits"].reshape(-1, case["vocab"])
    y = st["targets"].reshape(-1)
    rows = y.numel()
    index = (y != IGNORE).nonzero()[:, 0]
    op = case["op"]
    grad = None if op == "score" else torch.zeros(rows, case["vocab"], device="cuda", dtype=torch.float64)
    out = {}
    if op == "distill":
        per = _exact_distill(case, st, z, y, index, grad)
        n = max(1, index.numel())
        out = {"loss": per.sum() / n, "losses": per.view(y.shape if case["packed"] else st["targets"].shape)}
        grad /= n
    else:
        tau = case.get("temperature", 1.0)
        lp = torch.zeros(rows, device="cuda", dtype=torch.float64)
        for part in _parts(index, case):
            lp[part] = _token(z[part].double(), y[part], tau)
        if op == "score":
            return {"logps": lp.view(st["targets"].shape)}
        leaf = lp.clone().requires_grad_(True)
        out, objective = _exact_objective(case, st, leaf, index)
        coef = torch.autograd.grad(objective, leaf)[0]
        for part in _parts(index, case):
            x = z[part].double().requires_grad_(True)
            grad[part] = torch.autograd.grad((_token(x, y[part], tau) * coef[part]).sum(), x)[0]
        if op == "preference":
            grad *= case["grad_scale"]
        out = {k: v.detach() for k, v in out.items()}
    out["dlogits"] = grad.view(st["logits"].shape)
    return out


def _parts(index, case):
    return index.split(max(1, (1 << 26) // case["vocab"]))


def _token(x, y, tau):
    return torch.log_softmax(x / tau, 1).gather(1, y[:, None])[:, 0]


def _exact_objective(case, st, lp, index):
    """(outputs, what is differentiated) as functions of the rows' log-probabilities."""
    spans = _spans(case)
    if case["op"] == "logp":
        return {"logps": lp.view(st["targets"].shape)}, (lp * st["weights"].reshape(-1).double()).sum()
    if case["op"] == "preference":
        seq = torch.stack([lp[s:e].sum() / (max(1, e - s) if case["average"] else 1) for _, s, e, _ in spans])
        half = len(spans) // 2
        ratio = seq - st["ref"].double()
        delta = ratio[:half] - ratio[half:]
        h = case["beta"] * delta
        ls = torch.nn.functional.logsigmoid
        if case["kind"] == "sigmoid":
            loss = -(1 - case["smoothing"]) * ls(h) - case["smoothing"] * ls(-h)
        elif case["kind"] == "hinge":
            loss = torch.relu(1 - h)
        else:
            loss = (delta - 0.5 / case["beta"]) ** 2
        loss = loss.mean()
        return {"loss": loss, "logps": seq, "rewards": case["beta"] * ratio}, loss
    A, old = st["advantages"].reshape(-1).double(), st["old"].reshape(-1).double()
    r = torch.exp(lp - old)
    inside = torch.clip(r, 1 - case["low"], 1 + case["high"])
    term = -torch.min(r * A, inside * A)
    cut = (r * A > inside * A).double()
    k = torch.zeros_like(lp)
    if st["ref"] is not None:
        d = st["ref"].reshape(-1).double() - lp
        k = torch.exp(d) - 1 - d
    w = torch.zeros_like(cut)
    if case["reduction"] == "token":
        w[index] = 1.0 / max(1, index.numel())
    else:
        for _, s, e, _ in spans:
            w[s:e] = 1.0 / (len(spans) * max(1, e - s))
    loss = (w * (term + case["kl"] * k)).sum()
    return {"loss": loss, "logps": lp.view(st["targets"].shape), "kl": (w * k).sum(), "clipped": (w * cut).sum()}, loss


def _exact_distill(case, st, z, y, index, grad):
    tau, K = case["temperature"], case["top"]
    ids, t = st["ids"].reshape(-1, K).long(), st["teacher"].reshape(-1, K).double() / tau
    lse = st["lse"].reshape(-1).double() if st["lse"] is not None else None
    per = torch.zeros(y.numel(), device="cuda", dtype=torch.float64)
    for part in _parts(index, case):
        x = z[part].double().requires_grad_(True)
        logq = torch.log_softmax(x / tau, 1)
        has = ids[part] >= 0
        some = has.any(1)
        a = t[part].masked_fill(~has, -math.inf)
        if lse is None:
            a = a.masked_fill(~some[:, None], 0.0)
            p = torch.softmax(a, 1) * some[:, None]
        else:
            p = torch.exp(a - lse[part][:, None])
        there = ids[part].clamp(min=0)
        kl = torch.special.xlogy(p, p).sum(1) - (p * torch.where(has, logq.gather(1, there), 0.0)).sum(1)
        if lse is not None:
            rest = 1 - p.sum(1)
            rest = torch.where((rest >= REST_FLOOR) & some, rest, 0.0)
            hidden = torch.zeros_like(x, dtype=torch.int8).scatter_add_(1, there, has.to(torch.int8)) > 0
            logr = torch.logsumexp(logq.masked_fill(hidden, -math.inf), 1)
            kl = kl + torch.special.xlogy(rest, rest) - rest * logr
        loss = (1 - case["hard"]) * tau * tau * kl
        if case["hard"]:
            loss = loss - case["hard"] * torch.log_softmax(x, 1).gather(1, y[part, None])[:, 0]
        grad[part] = torch.autograd.grad(loss.sum(), x)[0]
        per[part] = loss.detach()
    return per
