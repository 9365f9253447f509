"""Helpers of the tests of a language model's calls: plain forms in 64 bits, and comparison within a tolerance per element."""
import torch

EPS = 2.0 ** -24                                     # half a unit in the last place of fp32, relative
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def half_step(t):
    """What rounding to a type costs at most: (relative to the value, absolute where the type runs out of exponents)."""
    tiny = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}[t]
    return torch.finfo(t).eps / 2, tiny


def rounding(want, t):
    rel, tiny = half_step(t)
    return want.abs() * rel + tiny


def assert_within(got, want, tol, what=""):
    """|got - want| <= tol, element by element; NaN and infinities in the same places."""
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities"
    off = (got - want).abs()[fine]
    tol = torch.as_tensor(tol, dtype=torch.float64, device=got.device).expand(want.shape)[fine]
    bad = off > tol
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the tolerance, worst {float((off / tol.clamp(min=1e-300)).max()):.3g} times it"


def f32(x):
    """A Python float as fp32 holds it."""
    return float(torch.tensor(x, dtype=torch.float32))


# -- token log-probabilities ----------------------------------------------------------------------------------------------------------

def logprobs64(logits, targets, scale=1.0, ignore=-100):
    vocab = logits.shape[-1]
    x = logits.double() * f32(scale)
    lse = torch.logsumexp(x, -1)
    skip, inside = targets == ignore, (targets >= 0) & (targets < vocab)
    at = x.gather(-1, torch.where(inside, targets.long(), 0)[..., None])[..., 0]
    logp = torch.where(lse == -torch.inf, lse, at - lse)
    nan = torch.full_like(lse, torch.nan)
    logp, lse = torch.where(inside, logp, nan), torch.where(inside, lse, nan)
    return torch.where(skip, 0.0, logp), torch.where(skip, 0.0, lse)


def logprobs_tolerance(logits, lse, logp, scale=1.0):
    """An exponent (x - m) scale log2 e carries four roundings, of a number up to 2 A (A = max |scale x| log2 e), times ln 2: 6 A; 2^x is good to 2^-22 (4 EPS); the sum of
    a thread's 32 values per step and V / 8192 steps (one warp: V / 1024), then of 32 lanes, eight warps and eight blocks: up to 32 + V / 1024 + 11 additions, of the
    relative error of each EPS; the logarithm, the factor ln 2 and the last sums: a few EPS of the result."""
    x = torch.where(torch.isfinite(logits), logits.double() * scale, 0.0)
    A = x.abs().amax(-1) * 1.4427 if logits.shape[-1] else 0.0
    steps = 32 + logits.shape[-1] / 1024 + 11
    fin = lambda t: torch.where(torch.isfinite(t), t.abs(), 0.0)
    return EPS * (6 * A + 4 + steps + 4 * fin(lse) + 4 * fin(logp) + 4)


def logprobs_grad64(logits, targets, lse, grad, scale=1.0, ignore=-100):
    """(gradient, tolerance in fp32 without the last rounding).  p = 2^((scale x - lse) log2 e), the exponent with three roundings of at most
    |scale x| + |lse|, in base 2; 2^x to 4 EPS; two products and a sum: 3 EPS.  Below 2^-126 2^x is 0."""
    vocab = logits.shape[-1]
    s = f32(scale)
    x, l = logits.double() * s, lse.double()[..., None]
    p = torch.exp(x - l)
    inside = ((targets >= 0) & (targets < vocab))[..., None]
    hot = torch.arange(vocab, device=logits.device) == targets[..., None]
    a = grad.double()[..., None] * s
    want = torch.where(inside, a * (hot.double() - p), torch.nan)
    zero = ((targets == ignore) | (grad == 0) | (lse == -torch.inf))[..., None]
    want = torch.where(zero, 0.0, want)
    fin = lambda t: torch.where(torch.isfinite(t), t.abs(), 0.0)
    rel = EPS * (0.7 * 3 * 1.4427 * (fin(x) + fin(l)) + 4 + 4)
    tol = a.abs() * (fin(p) * rel + hot * 3 * EPS + 2.0 ** -126)
    return want, torch.where(zero, 0.0, tol)


# -- preference loss ------------------------------------------------------------------------------------------------------------------

def preference64(logps, ref, mask, beta, smoothing, norm=None):
    """((loss, rewards, grad), (their tolerances without the gradient's last rounding)).  A log ratio is rounded once, up to eight are added in fp32, the rest in
    fp64: 9 EPS of the sum of magnitudes.  The loss changes by at most the margin's error, its slope by a quarter of it."""
    pairs = logps.shape[0] // 2
    norm = pairs if norm is None else norm
    d = logps.double() - (0.0 if ref is None else ref.double())
    if mask is not None:
        d = torch.where(mask != 0, d, 0.0)
    s, off = d.sum(1), 9 * EPS * d.abs().sum(1)
    z, z_off = beta * (s[:pairs] - s[pairs:]), abs(beta) * (off[:pairs] + off[pairs:])
    ls = torch.nn.functional.logsigmoid
    each = -(1 - smoothing) * ls(z) - smoothing * ls(-z)
    slope = beta / norm * (torch.sigmoid(-z) - smoothing)
    m = torch.ones_like(d) if mask is None else (mask != 0).double()
    grad = torch.cat([-slope, slope])[:, None] * m
    slope_off = abs(beta) / norm * (z_off / 4 + 2 * EPS)
    loss = each.sum() / norm
    return (loss, beta * s, grad), (z_off.sum() / norm + 2 * EPS * loss.abs(), abs(beta) * off + 2 * EPS * (beta * s).abs(),
                                    torch.cat([slope_off, slope_off])[:, None] * m + 2 * EPS * grad.abs())


# -- policy loss ----------------------------------------------------------------------------------------------------------------------

def policy64(logps, old, adv, mask, ref, low, high, weight, reduction, norm=None):
    """((terms, grad), (their tolerances without the gradient's last rounding)).  d = lp - old is rounded once, so exp(d) is off by |d| EPS and 4 EPS of its own; three
    products: |A| r (|d| + 8) EPS.  delta likewise; exp(delta) - 1 - delta is off by EPS (8 k + 2 |delta| |exp(delta) - 1|), beyond |delta| = 1, where it is a plain
    difference, by EPS 4 (exp(delta) + |delta|) more; its slope k + delta by that and 2 EPS (|slope| + |delta|).  A term's sum: up to eight are added in fp32."""
    rows, length = logps.shape
    keep = torch.ones(rows, length, dtype=torch.bool, device=logps.device) if mask is None else mask != 0
    zero = torch.zeros((), dtype=torch.float64, device=logps.device)
    pick = lambda t: torch.where(keep, t.double(), zero)
    adv = adv.reshape(rows, 1).expand(rows, length) if adv.numel() == rows and adv.shape != logps.shape else adv
    lp, o, A = pick(logps), pick(old), pick(adv)
    tokens = keep.sum(1, keepdim=True).double()
    if reduction == "token":
        n = tokens.sum() if norm is None else norm
        w = keep.double() / (n if norm is not None else n.clamp(min=1))
    else:
        n = (tokens > 0).sum().clamp(min=1) if norm is None else norm
        w = keep.double() / (tokens.clamp(min=1) * n)
    d = lp - o
    r = torch.exp(d)
    clipped = ((A > 0) & (r > 1 + high)) | ((A < 0) & (r < 1 - low))
    edge = torch.where(A > 0, 1 + high, 1 - low)
    gain = torch.where(A == 0, 0.0, torch.where(clipped, edge, r) * A)
    grad = torch.where(clipped | (A == 0), 0.0, -A * r)
    grad_off = torch.where(clipped | (A == 0), 0.0, A.abs() * r * (d.abs() + 8) * EPS)
    gain_off = torch.where(clipped, gain.abs() * 4 * EPS, grad_off)
    kl = torch.zeros_like(lp)
    kl_off = torch.zeros_like(lp)
    if ref is not None:
        delta = pick(ref) - lp
        slope = torch.expm1(delta)
        kl = slope - delta
        kl_off = EPS * (8 * kl + 2 * delta.abs() * slope.abs() + torch.where(delta.abs() > 1, 4 * (slope.abs() + 1 + delta.abs()), zero))
        grad = grad - weight * slope
        grad_off = grad_off + abs(weight) * (kl_off + 2 * EPS * (slope.abs() + delta.abs())) + 3 * EPS * grad.abs()
    terms = [-(w * gain).sum(), (w * kl).sum(), (w * clipped).sum()]
    off = [(w * (gain_off + 12 * EPS * gain.abs())).sum(), (w * (kl_off + 12 * EPS * kl)).sum(), 12 * EPS * terms[2]]
    terms = torch.stack([terms[0] + weight * terms[1], *terms])
    off = torch.stack([off[0] + abs(weight) * off[1], *off])
    return (terms, w * grad), (off + 4 * EPS * terms.abs(), w * (grad_off + 6 * EPS * grad.abs()))


# -- balance loss ---------------------------------------------------------------------------------------------------------------------

def balance64(logits, choices, mask, weight):
    """((loss, counts, probs, grad), (tolerances of loss, probs and the gradient without its last rounding)).  p: the exponents with three roundings of up to 2 A
    (A = max |x| log2 e), 2^x to 4 EPS, a sum of E / 32 terms and five steps, a division and a product.  Column sums: up to `rows` additions."""
    rows, E = logits.shape
    keep = torch.ones(rows, dtype=torch.bool, device=logits.device) if mask is None else mask != 0
    x = torch.where(keep[:, None], logits.double(), 0.0)
    p = torch.where((x == -torch.inf).all(-1, keepdim=True), 0.0, torch.softmax(x, -1))
    p = torch.where(keep[:, None], p, 0.0)
    n = keep.sum().double()
    c = choices[keep].flatten()
    c = c[(c >= 0) & (c < E)].long()
    counts = torch.bincount(c, minlength=E).to(torch.int32)
    if n == 0:
        z = torch.zeros((), dtype=torch.float64, device=logits.device)
        return (z, counts, torch.zeros(E, dtype=torch.float64, device=logits.device), torch.zeros_like(x)), (0.0, 0.0, 0.0)
    share, mean = counts.double() / (choices.shape[1] * n), p.sum(0) / n
    loss = weight * E * (share * mean).sum()
    apart = share - 1.0 / E
    inner = (p * apart).sum(-1, keepdim=True)
    grad = weight * E / n * p * (apart - inner)
    A = torch.where(torch.isfinite(x), x.abs(), 0.0).amax() * 1.4427
    rel = EPS * (6 * A + 4 + E / 32 + 5 + 4)
    spread = (p * apart.abs()).sum(-1, keepdim=True)
    grad_off = abs(weight) * E / n * p * (rel * ((apart - inner).abs() + spread) + EPS * ((E / 32 + 8) * spread + 4 * apart.abs()))
    probs_off = mean * (rel + EPS * (min(rows, 2048) + 64))
    return (loss, counts, mean, grad), ((share * probs_off).sum() * abs(weight) * E + 2 * EPS * loss.abs(), probs_off + 2 * EPS * mean, grad_off + 4 * EPS * grad.abs())
