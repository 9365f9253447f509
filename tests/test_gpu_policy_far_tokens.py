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
