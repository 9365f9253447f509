"""The objectives of a language model's worker, and the sparse end of its gradient, as they are measured: the calls, over the range of sizes
they are made with.

  logprobs    log-probabilities of given tokens from rows of logits (forward), and the logits' gradient (backward)
  preference  the logistic loss of paired log ratios: loss, rewards, and the gradient of every token's log-probability
  policy      the clipped policy loss with a KL term: its terms, and the gradient of every token's log-probability
  balance     the balance loss of a router: loss, tokens per expert, mean probabilities, the gradient of the router's logits
  embedding   rows of a table by token, scaled (forward), and the table's gradient, added up by token (backward)
"""
import math

import torch

own = False

IGNORE = -100
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # scoring the next token of a few sequences: latency
        {"name": "logprobs_few", "op": "logprobs", "direction": "forward", "type": "bf16", "batch": 20, "length": 1, "vocab": 32768, "shift": False,
         "ignored": 0.0},
        # scoring whole sequences, an odd vocabulary, every position against the token behind it, a third of them prompt
        {"name": "logprobs_odd", "op": "logprobs", "direction": "forward", "type": "f16", "batch": 8, "length": 511, "vocab": 50257, "shift": True,
         "ignored": 0.33},
        # the backward pass of a training step with a large vocabulary
        {"name": "logprobs_grad", "op": "logprobs", "direction": "backward", "type": "bf16", "batch": 4, "length": 1024, "vocab": 131072, "shift": False,
         "ignored": 0.0},
        # four pairs of short answers: latency
        {"name": "preference_few", "op": "preference", "type": "f32", "pairs": 4, "length": 512, "masked": True, "smoothing": 0.0},
        # a large batch of long pairs, an odd length
        {"name": "preference_many", "op": "preference", "type": "f32", "pairs": 512, "length": 8191, "masked": True, "smoothing": 0.1},
        # one prompt's group of samples: latency
        {"name": "policy_few", "op": "policy", "type": "f32", "rows": 8, "length": 300, "masked": True, "reduction": "token", "kl": 0.05,
         "per_token": False},
        # a rollout's batch of long answers, every sequence of the same weight
        {"name": "policy_many", "op": "policy", "type": "f32", "rows": 1024, "length": 8192, "masked": True, "reduction": "sequence", "kl": 0.01,
         "per_token": True},
        # a router of eight experts over one short sequence: latency
        {"name": "balance_few", "op": "balance", "type": "f32", "rows": 512, "experts": 8, "chosen": 2, "masked": False},
        # many experts, a training batch with padding
        {"name": "balance_many", "op": "balance", "type": "bf16", "rows": 131072, "experts": 256, "chosen": 8, "masked": True},
        # first layer of a training batch
        {"name": "embedding_rows", "op": "embedding", "direction": "forward", "type": "bf16", "tokens": 16384, "vocab": 131072, "dim": 4096},
        # gradient of a small table from one sequence
        {"name": "embedding_grad_few", "op": "embedding", "direction": "backward", "type": "f32", "tokens": 1000, "vocab": 1024, "dim": 257},
        # gradient of a large table from a training batch; some tokens come thousands of times
        {"name": "embedding_grad_many", "op": "embedding", "direction": "backward", "type": "bf16", "tokens": 65536, "vocab": 50257, "dim": 2048},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "preference", "policy", "balance", "embedding", "embedding"])
    type_ = rng.choice(["f32", "bf16", "f16"])
    if op == "logprobs":
        vocab = _log_int(rng, 1000, 160000)
        most = max(1, (1 << 28) // vocab)
        batch = _log_int(rng, 1, min(64, most))
        return {"op": op, "direction": rng.choice(["forward", "backward"]), "type": type_, "batch": batch, "length": _log_int(rng, 1, max(1, min(2048, most // batch))),
                "vocab": vocab, "shift": rng.random() < 0.5, "ignored": rng.choice([0.0, 0.25, 0.5])}
    if op == "preference":
        return {"op": op, "type": type_, "pairs": _log_int(rng, 1, 512), "length": _log_int(rng, 1, 8192), "masked": rng.random() < 0.7,
                "smoothing": rng.choice([0.0, 0.1])}
    if op == "policy":
        return {"op": op, "type": type_, "rows": _log_int(rng, 1, 1024), "length": _log_int(rng, 1, 8192), "masked": rng.random() < 0.7,
                "reduction": rng.choice(["token", "sequence"]), "kl": rng.choice([0.0, 0.02]), "per_token": rng.random() < 0.5}
    if op == "balance":
        experts = _log_int(rng, 2, 512)
        return {"op": op, "type": type_, "rows": _log_int(rng, 1, min(131072, (1 << 25) // experts)), "experts": experts,
                "chosen": rng.randint(1, min(8, experts)), "masked": rng.random() < 0.5}
    dim = _log_int(rng, 8, 4096)
    return {"op": op, "direction": rng.choice(["forward", "backward"]), "type": type_, "tokens": _log_int(rng, 1, min(65536, (1 << 27) // dim)),
            "vocab": _log_int(rng, 100, min(131072, 100000000 // dim)), "dim": dim}


def _answers(g, rows, length, masked):
    """Which positions count: a prompt in front does not, neither does padding behind; the last of several rows has none left."""
    if not masked:
        return None
    at = torch.arange(length, device="cuda")
    begin = (torch.rand(rows, 1, device="cuda", generator=g) * 0.4 * length).long()
    end = (length * (0.5 + 0.5 * torch.rand(rows, 1, device="cuda", generator=g))).long() + 1
    if rows > 4:
        end[-1] = 0
    return (at >= begin) & (at < end)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = TYPES.get(case["type"])

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    s = {"case": case}
    op = case["op"]
    if op == "logprobs":
        b, n, v = case["batch"], case["length"], case["vocab"]
        whole = torch.randn(b, n + (1 if case["shift"] else 0), v, device="cuda", generator=g, dtype=t).mul_(2.5)
        s["logits"] = whole[:, :n]                     # with a shift: a view, the last position of each sequence has no token behind it
        s["targets"] = torch.randint(0, v, (b, n), device="cuda", generator=g)
        if case["ignored"]:
            s["targets"][torch.rand(b, n, device="cuda", generator=g) < case["ignored"]] = IGNORE
        s["scale"] = 0.8 if case["shift"] else 1.0     # one over a temperature
        if case["direction"] == "backward":
            weight = randn(b, n) / (b * n)
            s["grad"] = torch.where(torch.rand(b, n, device="cuda", generator=g) < 0.1, torch.zeros_like(weight), weight)
            # the forward pass leaves these; sums of many terms, a slab of rows at a time
            rows = s["logits"].reshape(b * n, v) if not case["shift"] else s["logits"].flatten(0, 1)
            lse = torch.cat([torch.logsumexp(r.float() * s["scale"], -1) for r in rows.split(512)]).view(b, n)
            s["lse"] = torch.where(s["targets"] == IGNORE, torch.zeros_like(lse), lse)
    elif op in ("preference", "policy"):
        rows, n = (2 * case["pairs"] if op == "preference" else case["rows"]), case["length"]
        lp = -torch.empty(rows, n, device="cuda").exponential_(1.0, generator=g)
        s["logps"] = lp.to(t)
        s["ref"] = (lp + 0.05 * randn(rows, n)).clamp_(max=0.0).to(t)
        s["mask"] = _answers(g, rows, n, case["masked"])
        if op == "policy":
            s["old"] = (lp + 0.15 * randn(rows, n)).clamp_(max=0.0).to(t)
            s["advantages"] = (randn(rows, n) if case["per_token"] else randn(rows)).to(t)
    elif op == "balance":
        rows, e = case["rows"], case["experts"]
        s["logits"] = (randn(rows, e) + 0.5 * randn(e)).to(t)
        s["experts"] = torch.topk(s["logits"].float(), case["chosen"], dim=-1).indices
        s["mask"] = torch.rand(rows, device="cuda", generator=g) < 0.85 if case["masked"] else None
    else:
        v, d, n = case["vocab"], case["dim"], case["tokens"]
        # ranks as words have them: the chance of rank r falls as 1 / r
        rank = (v ** torch.rand(n, device="cuda", generator=g, dtype=torch.float64)).long().clamp_(max=v) - 1
        s["tokens"] = rank * 7919 % v
        s["scale"] = math.sqrt(d)
        if case["direction"] == "forward":
            s["weight"] = torch.randn(v, d, device="cuda", generator=g, dtype=t).mul_(0.02)
        else:
            s["grad"] = torch.randn(n, d, device="cuda", generator=g, dtype=t).mul_(0.01)
    return s


BETA, LOW, HIGH, WEIGHT = 0.1, 0.2, 0.28, 0.01


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_2106_05203_b200 import binding as B
        if op == "logprobs":
            if case["direction"] == "forward":
                return tuple(B.token_logprobs(s["logits"], s["targets"], scale=s["scale"]))
            return B.token_logprobs_grad(s["logits"], s["targets"], s["lse"], s["grad"], scale=s["scale"])
        if op == "preference":
            return tuple(B.preference_loss(s["logps"], s["ref"], mask=s["mask"], beta=BETA, smoothing=case["smoothing"]))
        if op == "policy":
            return tuple(B.policy_loss(s["logps"], s["old"], s["advantages"], mask=s["mask"], ref_logps=s["ref"], clip_low=LOW, clip_high=HIGH,
                                       kl_weight=case["kl"], reduction=case["reduction"]))
        if op == "balance":
            return tuple(B.balance_loss(s["logits"], s["experts"], mask=s["mask"], weight=WEIGHT))
        if case["direction"] == "forward":
            return B.embedding(s["weight"], s["tokens"], scale=s["scale"])
        return B.embedding_grad(s["grad"], s["tokens"], case["vocab"], scale=s["scale"], dtype=torch.float32)
    if op == "logprobs":
        return _plain_logprobs(s) if case["direction"] == "forward" else _plain_logprobs_grad(s)
    if op == "preference":
        return _plain_preference(s)
    if op == "policy":
        return _plain_policy(s)
    if op == "balance":
        return _plain_balance(s)
    if case["direction"] == "forward":
        return (s["weight"][s["tokens"]].float() * s["scale"]).to(s["weight"].dtype)
    table = torch.zeros(case["vocab"], case["dim"], device="cuda")
    return table.index_add_(0, s["tokens"], s["grad"].float()) * s["scale"]


def _plain_logprobs(s):
    x = s["logits"].float() * s["scale"]
    top = x.amax(-1, keepdim=True)
    lse = torch.log(torch.exp(x - top).sum(-1)) + top[..., 0]
    skip = s["targets"] == IGNORE
    at = x.gather(-1, torch.where(skip, 0, s["targets"])[..., None])[..., 0]
    zero = torch.zeros_like(lse)
    return torch.where(skip, zero, at - lse), torch.where(skip, zero, lse)


def _plain_logprobs_grad(s):
    g = torch.where(s["targets"] == IGNORE, torch.zeros_like(s["grad"]), s["grad"]) * s["scale"]
    d = torch.exp(s["logits"].float() * s["scale"] - s["lse"][..., None])
    d.neg_()
    at = torch.where(s["targets"] == IGNORE, 0, s["targets"])[..., None]
    d.scatter_add_(-1, at, torch.ones_like(at, dtype=torch.float32))
    d.mul_(g[..., None])
    return torch.where(g[..., None] == 0, torch.zeros_like(d), d).to(s["logits"].dtype)


def _plain_preference(s):
    case = s["case"]
    pairs, eps = case["pairs"], case["smoothing"]
    ratio = s["logps"].float() - s["ref"].float()
    if s["mask"] is not None:
        ratio = torch.where(s["mask"], ratio, torch.zeros_like(ratio))
    total = ratio.sum(-1, dtype=torch.float64)               # a long sum of small terms of both signs
    z = BETA * (total[:pairs] - total[pairs:])
    minus_log_sigma = torch.log1p(torch.exp(-z.abs())) + torch.clamp(-z, min=0)          # of z; of -z it is larger by z
    loss = (minus_log_sigma + eps * z).mean()
    sigma = torch.exp(-(minus_log_sigma + z))                # of -z
    slope = BETA / pairs * (sigma - eps)
    slope = torch.cat([-slope, slope]).float()[:, None].expand_as(ratio)
    grad = slope if s["mask"] is None else torch.where(s["mask"], slope, torch.zeros_like(slope))
    return loss.float(), (BETA * total).float(), grad.to(s["logps"].dtype).contiguous()


def _plain_policy(s):
    case = s["case"]
    lp, old, ref, adv = (s[k].float() for k in ("logps", "old", "ref", "advantages"))
    if adv.dim() == 1:
        adv = adv[:, None].expand_as(lp)
    mask = torch.ones_like(lp) if s["mask"] is None else s["mask"].float()
    if case["reduction"] == "token":
        w = mask / mask.sum(dtype=torch.float64).clamp(min=1).float()
    else:
        tokens = mask.sum(-1, keepdim=True)
        w = mask / (tokens.clamp(min=1) * (tokens > 0).sum())
    # on which side of the clip's border: in 64 bits, the gradient jumps there
    d = lp.double() - old.double()
    clipped = ((adv > 0) & (d > math.log1p(HIGH))) | ((adv < 0) & (d < math.log1p(-LOW)))
    ratio = torch.exp(lp - old)
    pg = -torch.where(clipped, torch.where(adv > 0, 1.0 + HIGH, 1.0 - LOW), ratio) * adv
    delta = (ref - lp).double()                              # exp(delta) - 1 - delta of small ones: 64 bits
    kl = (torch.expm1(delta) - delta).float()
    grad = torch.where(clipped, torch.zeros_like(adv), -adv * ratio) - case["kl"] * torch.expm1(ref - lp)
    zero = torch.zeros_like(lp)
    keep = mask > 0
    pg, kl = torch.where(keep, pg, zero), torch.where(keep, kl, zero)
    terms = [(w * x).sum(dtype=torch.float64) for x in (pg, kl, clipped.float())]
    terms = torch.stack([terms[0] + case["kl"] * terms[1], *terms]).float()
    return terms, torch.where(keep, w * grad, zero).to(s["logps"].dtype)


def _plain_balance(s):
    case = s["case"]
    e, k = case["experts"], case["chosen"]
    x = s["logits"].float()
    keep = torch.ones(case["rows"], dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    chosen = torch.where(keep[:, None], s["experts"], e)
    counts = torch.zeros(e + 1, dtype=torch.int32, device="cuda").index_add_(0, chosen.reshape(-1), torch.ones_like(chosen, dtype=torch.int32).reshape(-1))[:e]
    n = keep.sum().clamp(min=1).double()
    mean = torch.where(keep[:, None], p, torch.zeros_like(p)).sum(0, dtype=torch.float64) / n
    share = counts.double() / (k * n)
    loss = WEIGHT * e * (share * mean).sum()
    apart = (share - 1.0 / e).float()                        # differences of shares that are alike: about their mean
    grad = (WEIGHT * e / n).float() * p * (apart - (p * apart).sum(-1, keepdim=True))
    grad = torch.where(keep[:, None], grad, torch.zeros_like(grad))
    return loss.float(), counts, mean.float(), grad.to(s["logits"].dtype)


def work(case):
    op, e = case["op"], BYTES[case["type"]]
    if op == "logprobs":
        rows, v = case["batch"] * case["length"], case["vocab"]
        read = rows * (1.0 - case["ignored"]) * v * e                    # rows that are ignored need not be read
        if case["direction"] == "forward":
            return {"bytes": read + rows * 16, "flops": 4.0 * rows * (1.0 - case["ignored"]) * v}
        return {"bytes": 0.9 * read + rows * v * e + rows * 16, "flops": 4.0 * 0.9 * rows * (1.0 - case["ignored"]) * v}
    if op == "preference":
        cells = 2 * case["pairs"] * case["length"]
        return {"bytes": cells * (3 * e + (1 if case["masked"] else 0)) + 8 * case["pairs"] + 4, "flops": 3.0 * cells}
    if op == "policy":
        cells = case["rows"] * case["length"]
        return {"bytes": cells * (4 * e + (1 if case["masked"] else 0)) + (cells if case["per_token"] else case["rows"]) * e + 16, "flops": 30.0 * cells}
    if op == "balance":
        rows, ex = case["rows"], case["experts"]
        return {"bytes": 2 * rows * ex * e + rows * (8 * case["chosen"] + (1 if case["masked"] else 0)) + 8 * ex + 4, "flops": 10.0 * rows * ex}
    n, d, v = case["tokens"], case["dim"], case["vocab"]
    if case["direction"] == "forward":
        return {"bytes": (n + min(n, _seen(n, v))) * d * e + 8 * n, "flops": 1.0 * n * d}
    return {"bytes": n * d * e + v * d * 4 + 8 * n, "flops": 1.0 * n * d}


def _seen(n, v):
    """About how many different ones of v tokens come up in n draws."""
    ln = math.log(v)
    step = max(1, v // 4096)
    return int(sum(step * (1.0 - (1.0 - math.log1p(1.0 / (r + 1)) / ln) ** n) for r in range(0, v, step)))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "logprobs":
        v = case["vocab"]
        targets = s["targets"].reshape(-1)
        rows = s["logits"].flatten(0, 1)
        if case["direction"] == "forward":
            out = [], []
            for x, t in zip(rows.split(256), targets.split(256)):
                x = x.double() * s["scale"]
                lse = torch.logsumexp(x, -1)
                named = t != IGNORE
                out[0].append((x[torch.arange(len(t), device="cuda"), t.clamp(min=0)] - lse) * named)
                out[1].append(lse * named)
            return tuple(torch.cat(o).view(s["targets"].shape) for o in out)
        grads = torch.empty(rows.shape, dtype=torch.float64 if rows.numel() <= 1 << 30 else torch.float32, device="cuda")
        scaled = (s["grad"].double() * s["scale"] * (s["targets"] != IGNORE)).reshape(-1)
        for at in range(0, len(rows), 256):
            x, t = rows[at:at + 256].double() * s["scale"], targets[at:at + 256]
            p = (x - s["lse"].reshape(-1)[at:at + 256, None].double()).exp()
            p = (torch.arange(v, device="cuda") == t[:, None]).double() - p
            p[scaled[at:at + 256] == 0] = 0.0
            grads[at:at + 256] = p * scaled[at:at + 256, None]
        return grads.view(s["logits"].shape)
    if op == "preference":
        m = torch.ones(s["logps"].shape, dtype=torch.float64, device="cuda") if s["mask"] is None else s["mask"].double()
        sums = ((s["logps"].double() - s["ref"].double()) * m).sum(1)
        half = case["pairs"]
        margin = BETA * (sums[:half] - sums[half:])
        eps = case["smoothing"]
        loss = -((1 - eps) * torch.nn.functional.logsigmoid(margin) + eps * torch.nn.functional.logsigmoid(-margin)).sum() / half
        by_margin = -((1 - eps) * torch.sigmoid(-margin) - eps * torch.sigmoid(margin)) / half
        return loss, BETA * sums, torch.cat([by_margin, -by_margin])[:, None] * BETA * m
    if op == "policy":
        lp = s["logps"].double().requires_grad_()
        adv = s["advantages"].double().reshape(case["rows"], -1)
        m = torch.ones_like(lp) if s["mask"] is None else s["mask"].double()
        per_row = m.sum(1, keepdim=True)
        w = m / m.sum().clamp(min=1) if case["reduction"] == "token" else m / per_row.clamp(min=1) / (per_row > 0).sum()
        r = (lp - s["old"].double()).exp()
        inside = r.clamp(1 - LOW, 1 + HIGH)
        gain = torch.minimum(r * adv, inside * adv)
        apart = s["ref"].double() - lp
        pg, kl = -(gain * w).sum(), ((apart.exp() - 1 - apart) * w).sum()
        loss = pg + case["kl"] * kl
        loss.backward()
        share = ((gain < r * adv).double() * w).sum()
        return torch.stack([loss, pg, kl, share]).detach(), lp.grad
    if op == "balance":
        e = case["experts"]
        x = s["logits"].double().requires_grad_()
        m = torch.ones(case["rows"], dtype=torch.float64, device="cuda") if s["mask"] is None else s["mask"].double()
        n = m.sum().clamp(min=1)
        counts = torch.bincount(s["experts"][m > 0].flatten(), minlength=e).to(torch.int32)
        mean = (x.softmax(-1) * m[:, None]).sum(0) / n
        loss = WEIGHT * e * (counts / (case["chosen"] * n) * mean).sum()
        loss.backward()
        return loss.detach(), counts, mean.detach(), x.grad
    if case["direction"] == "forward":
        return s["weight"].double().index_select(0, s["tokens"]) * s["scale"]
    order = torch.sort(s["tokens"], stable=True).indices
    sums = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device="cuda")
    for at in order.split(16384):
        sums.index_add_(0, s["tokens"][at], s["grad"][at].double())
    return sums * s["scale"]
