"""The policy loss on tokens whose log-probabilities are far from those that they are compared with: exponentials beyond 32 bits."""
import pytest
import torch

from model_util import EPS, TYPES, assert_within, generator, rounding

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


def fitted(want, dtype):
    """What a type holds of a 64-bit value."""
    return torch.where(want.abs() > torch.finfo(dtype).max, torch.sign(want) * INF, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", [1, 8, 19])
def test_ratios_beyond_all_types(B, dtype, length):
    """A < 0 is never clipped from above: the loss and the token's gradient are +inf, nothing is NaN, and the other tokens keep theirs."""
    for far in [100.0 + 0.5 * k for k in range(40)] + [150.0, 1e3, 12345.0, 6e4]:
        lp = torch.full((2, length), -1.0, device="cuda", dtype=dtype)
        old = lp.clone()
        adv = torch.full_like(lp, -1.0)
        old[0, length // 2] = -1.0 - far
        got = B.policy_loss(lp, old, adv)
        assert got.terms[0] == INF and got.terms[1] == INF and got.terms[2] == 0 and got.terms[3] == 0, far
        want = torch.full((2, length), 1.0 / (2 * length), dtype=torch.float64, device="cuda")
        want[0, length // 2] = INF
        assert_within(got.grad, want, rounding(want, dtype) + 8 * EPS * want, f"gradient at {far}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", [5, 24])
@pytest.mark.parametrize("reduction", ["token", "sequence"])
@pytest.mark.parametrize("masked", [False, True])
def test_a_reference_that_is_only_watched(B, dtype, length, reduction, masked):
    """kl_weight 0: the KL term is told, and has no part in the loss or its gradient, however far the reference is."""
    g = generator(length)
    lp = (-torch.rand(6, length, device="cuda", generator=g)).to(dtype)
    old = (lp + 0.1 * torch.randn(6, length, device="cuda", generator=g)).to(dtype)
    adv = torch.randn(6, length, device="cuda", generator=g).to(dtype)
    mask = torch.rand(6, length, device="cuda", generator=g) < 0.7 if masked else None
    if masked:
        mask[:, 2] = True
    alone = B.policy_loss(lp, old, adv, mask=mask, reduction=reduction)
    for far in (0.5, 89.0, 100.0, 3e4, INF, -3e4, -INF, NAN):
        ref = lp.clone()
        ref[::2, 2] = far
        got = B.policy_loss(lp, old, adv, mask=mask, ref_logps=ref, reduction=reduction)
        assert torch.equal(got.grad, alone.grad), far
        assert torch.equal(got.terms[:2], alone.terms[:2]) and torch.equal(got.terms[3:], alone.terms[3:]), far
    # a policy that rules the token out itself: its log-probability is the type's lowest value
    low = lp.clone(); low[::2, 2] = torch.finfo(dtype).min
    alone = B.policy_loss(low, low, adv, mask=mask, reduction=reduction)
    got = B.policy_loss(low, low, adv, mask=mask, ref_logps=lp, reduction=reduction)
    assert torch.equal(got.grad, alone.grad) and torch.equal(got.terms[:2], alone.terms[:2]) and bool(torch.isfinite(got.grad).all())


@pytest.mark.parametrize("rows,length", [(1, 64), (16, 24), (16, 27), (700, 41)])
@pytest.mark.parametrize("reduction", ["token", "sequence"])
@pytest.mark.parametrize("masked", [False, True])
def test_ratios_that_fit_once_they_are_weighted(B, rows, length, reduction, masked):
    """exp(d) is beyond fp32 from d = 88.73 on, exp(d) |A| over the number of tokens need not be.  d is rounded once (|d| EPS in the exponent); what is summed in 64 bits is
    rounded once more; the weight carries 4 EPS, ratios within 32 bits (|d| + 8) EPS and 12 EPS of additions as ever: (|d| + 24) EPS of the sum of magnitudes."""
    g = generator(rows + length)
    lp = -torch.rand(rows, length, device="cuda", generator=g)
    old = lp + 0.1 * torch.randn(rows, length, device="cuda", generator=g)
    old[0, 3] = lp[0, 3] - 89.25
    old[0, 11] = lp[0, 11] - 91.5
    old[rows - 1, length - 1] = lp[rows - 1, length - 1] - 90.125
    adv = -torch.rand(rows, length, device="cuda", generator=g) - 0.01
    adv[0, 11] = -1e-3
    mask = None
    if masked:
        mask = torch.rand(rows, length, device="cuda", generator=g) < 0.8
        mask[0, 3] = mask[0, 11] = True
        mask[rows - 1, length - 1] = False                                # (and what the mask leaves out may be as far as it likes)
    keep = torch.ones(rows, length, dtype=torch.bool, device="cuda") if mask is None else mask
    got = B.policy_loss(lp, old, adv, mask=mask, reduction=reduction, norm=None)
    tokens = keep.sum(1, keepdim=True).double()
    w = keep.double() / (tokens.sum() if reduction == "token" else tokens.clamp(min=1) * (tokens > 0).sum())
    d = (lp - old).double()                                               # (the rounded difference: what is left is the exponential's)
    r = torch.exp(d)
    grad = torch.where(r < 0.8, 0.0, -adv.double() * r) * w
    gain = torch.where(r < 0.8, 0.8, r) * adv.double() * w
    loss = -gain.sum()
    assert float(loss) < torch.finfo(torch.float32).max and float(grad.abs().max()) > 1e34
    off = gain.abs() * (d.abs() + 24) * EPS
    assert_within(got.terms[:2], torch.stack([loss, loss]), off.sum(), "terms")
    assert_within(got.grad, grad, off + rounding(grad, torch.float32), "gradient")


@pytest.mark.parametrize("rows,length", [(1, 64), (16, 24), (16, 27), (700, 41)])
@pytest.mark.parametrize("weight", [0.25, 1e-3])
def test_references_that_fit_once_they_are_weighted(B, rows, length, weight):
    """The same of exp(delta) in the KL term, its weight included: the loss and the gradient are finite where the term before its weight may not be.  Tolerances as above."""
    g = generator(rows)
    lp = -torch.rand(rows, length, device="cuda", generator=g)
    ref = lp + 0.1 * torch.randn(rows, length, device="cuda", generator=g)
    lp[0, 2] = ref[0, 2] - 89.5
    lp[0, 9] = ref[0, 9] - (94.0 if weight < 0.01 else 90.5)
    lp[rows - 1, length - 1] = ref[rows - 1, length - 1] - 89.0
    zero = torch.zeros_like(lp)
    got = B.policy_loss(lp, lp, zero, ref_logps=ref, kl_weight=weight)
    c = float(torch.tensor(weight, dtype=torch.float32))
    delta = (ref - lp).double()
    slope = torch.expm1(delta)
    k = slope - delta
    n = rows * length
    small = 8 * k + 2 * delta.abs() * slope.abs() + torch.where(delta.abs() > 1, 4 * (slope.abs() + 1 + delta.abs()), torch.zeros_like(k))
    k_off = EPS * (small + (delta.abs() + 24) * k)
    term = k.sum() / n
    want = torch.stack([c * term, fitted(term, torch.float32)])
    assert float(want[0]) < torch.finfo(torch.float32).max
    assert_within(got.terms[0], want[0], c * k_off.sum() / n + 4 * EPS * want[0], "loss")
    assert_within(got.terms[2], want[1], k_off.sum() / n + 4 * EPS * term, "KL term")
    grad = -c * slope / n
    assert_within(got.grad, grad, c / n * (k_off + EPS * (slope.abs() + delta.abs()) * (delta.abs() + 24)) + rounding(grad, torch.float32), "gradient")


def test_one_far_token_leaves_its_neighbours_alone(B):
    """Bit for bit: the gradients of the tokens beside one whose ratio is infinite."""
    g = generator(1)
    lp = -torch.rand(9, 400, device="cuda", generator=g)
    old, adv = lp + 0.1 * torch.randn(9, 400, device="cuda", generator=g), torch.randn(9, 400, device="cuda", generator=g)
    clean = B.policy_loss(lp, old, adv, ref_logps=old, kl_weight=0.1)
    at = torch.zeros(9, 400, dtype=torch.bool, device="cuda")
    at[::3, 5::97] = True
    got = B.policy_loss(lp, torch.where(at, lp - 500, old), torch.where(at, -1.0, adv), ref_logps=old, kl_weight=0.1)
    assert torch.equal(got.grad[~at], clean.grad[~at]) and bool((got.grad[at] == INF).all()) and got.terms[0] == INF
