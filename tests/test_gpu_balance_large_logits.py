"""The balance loss on rows of large finite logits: masks by a large negative number, choices forced by a large positive one, rows that such a mask leaves nothing of."""
import pytest
import torch

from model_util import EPS, TYPES, assert_within, generator, rounding

pytestmark = pytest.mark.gpu

LEAST = 2.0 ** -120                                    # (exponentials below 2^-126 are 0)


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


def definition(x, choices, mask, weight):
    """((loss, counts, probs, grad), their tolerances without the gradient's last rounding).  Only the distance of a logit from its row's maximum enters: with d = x - max an
    exponent is d log2 e with a rounded difference and a rounded product, or one rounded product that adds the same to all of a row and cancels in p, and 2^x is good to
    4 EPS: relative 4 (|d| + 1) EPS, for d above -104 (below, 0).  A lane adds up to 16 pairs, then their two halves and up to five lanes: 22 additions.  p: the sum's error, a
    reciprocal of 4 EPS, a product.  The gradient: four products and a difference, its inner sum 22 additions more; f - 1/E is rounded once.  Column sums: up to `rows` additions."""
    rows, E = x.shape
    keep = torch.ones(rows, dtype=torch.bool, device=x.device) if mask is None else mask
    y = torch.where(keep[:, None], x.double(), 0.0)
    top = y.amax(-1, keepdim=True)
    d = torch.where(top == -torch.inf, -torch.inf, y - top)
    e = torch.exp(d) * keep[:, None]
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    n = keep.sum().double()
    counts = torch.bincount(choices[keep].flatten(), minlength=E).to(torch.int32)
    share = counts.double() / (choices.shape[1] * n)
    mean = p.sum(0) / n
    loss = weight * E * (share * mean).sum()
    apart = share - 1.0 / E
    inner = (p * apart).sum(-1, keepdim=True)
    grad = weight * E / n * p * (apart - inner)
    term = EPS * 4 * (d.clamp(min=-104.0).abs() + 1)
    of_total = (p * term).sum(-1, keepdim=True) + 22 * EPS
    rel = term + of_total + 5 * EPS
    spread = (p * apart.abs()).sum(-1, keepdim=True)
    inner_off = (p * term * apart.abs()).sum(-1, keepdim=True) + (of_total + 28 * EPS) * spread
    grad_off = abs(weight) * E / n * (p * ((rel + 8 * EPS) * (apart.abs() + spread) + inner_off) + LEAST)
    probs_off = (p * rel).sum(0) / n + EPS * (min(rows, 2048) + 64) * mean + LEAST
    loss_off = abs(weight) * E * (share * probs_off).sum() + 4 * EPS * loss.abs()
    return (loss, counts, mean, grad), (loss_off, probs_off, grad_off + 4 * EPS * grad.abs())


def check(B, x, choices, mask=None, weight=0.5):
    got = B.balance_loss(x, choices, mask=mask, weight=weight)
    (loss, counts, probs, grad), (t0, t1, t2) = definition(x, choices, mask, weight)
    assert torch.equal(got.counts, counts)
    assert_within(got.loss, loss, t0, "loss")
    assert_within(got.probs, probs, t1, "probs")
    assert_within(got.grad, grad, t2 + rounding(grad, x.dtype), "gradient")


def batch(rows, experts, dtype, seed):
    g = generator(seed)
    x = (torch.randn(rows, experts, device="cuda", generator=g) * 2).to(dtype)
    return x, torch.topk(x.float(), min(2, experts), dim=-1).indices, torch.rand(rows, device="cuda", generator=g) < 0.8


SIZES = [1e4, 6e4, 1e6, 1e8, 1.5e9, 1e10, 1e11, 1e12, 1e20, 1e30, 1e37, 1e38, 3e38]


@pytest.mark.parametrize("dtype,size", [(t, s) for t in TYPES for s in SIZES if s <= torch.finfo(t).max])
@pytest.mark.parametrize("experts", [2, 7, 64, 100, 160, 256, 512, 1000])
@pytest.mark.parametrize("rows", [24, 5000])
def test_rows_of_large_logits(B, dtype, experts, rows, size):
    """Rows that are all -size, or all +size; most of a row at -size; one or two experts at +size; size and its next neighbours in the type, apart from one another."""
    x, choices, mask = batch(rows, experts, dtype, rows + experts)
    v = torch.tensor(size, dtype=dtype, device="cuda")
    x[0::8] = -v
    x[1::8] = v
    x[2::8, 1:] = -v
    x[3::8, experts // 2] = v
    x[4::8, 0] = v; x[4::8, experts - 1] = v
    x[5::8, 1] = torch.nextafter(v, torch.zeros_like(v)); x[5::8, 0] = v
    mask[:8] = True
    check(B, x, choices, mask)
    check(B, x, choices)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts", [8, 70, 256])
@pytest.mark.parametrize("low", [-1e4, -6e4, "lowest", "-inf"])
def test_masked_experts(B, dtype, experts, low):
    """Experts that are switched off, in some rows nearly all of them; the others' probabilities are held to what their own logits allow."""
    low = {"lowest": torch.finfo(dtype).min, "-inf": -float("inf")}.get(low, low)
    x, choices, mask = batch(300, experts, dtype, experts)
    x[:, 1] = low
    x[::4, 2:] = low
    mask[:4] = True
    check(B, x, choices, mask)


def test_a_spread_of_every_size(B):
    """Logits 2^-20 to 2^20 times apart: from all alike to one that takes all."""
    for k in range(-20, 21):
        x, choices, mask = batch(50, 12, torch.float32, k + 20)
        check(B, x * 2.0 ** k, choices, mask)
        check(B, x * 2.0 ** k + 1e7, choices, mask)
