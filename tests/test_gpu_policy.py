"""The clipped policy loss against the definition in 64 bits (tolerances: model_util)."""
import pytest
import torch

from model_util import EPS, TYPES, assert_within, generator, policy64, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


def inputs(rows, length, dtype, seed, masked=True, per_token=True):
    g = generator(seed)
    lp = -torch.empty(rows, length, device="cuda").exponential_(generator=g)
    near = lambda by: (lp + by * torch.randn(rows, length, device="cuda", generator=g)).to(dtype)
    adv = torch.randn(rows, length, device="cuda", generator=g) if per_token else torch.randn(rows, device="cuda", generator=g)
    if adv.numel():
        adv.view(-1)[0] = 0.0
    mask = torch.rand(rows, length, device="cuda", generator=g) < 0.6 if masked else None
    return lp.to(dtype), near(0.25), adv.to(dtype), mask, near(0.3)


def check(B, lp, old, adv, mask, ref, low=0.2, high=0.28, weight=0.04, reduction="token", norm=None):
    got = B.policy_loss(lp, old, adv, mask=mask, ref_logps=ref, clip_low=low, clip_high=high, kl_weight=weight, reduction=reduction, norm=norm)
    (terms, grad), (t0, t1) = policy64(lp, old, adv, mask, ref, low, high, weight, reduction, norm)
    assert got.terms.dtype == torch.float32 and got.grad.dtype == lp.dtype and got.grad.shape == lp.shape and got.grad.is_contiguous()
    assert_within(got.terms, terms, t0, "terms")
    assert_within(got.grad, grad, t1 + rounding(grad, lp.dtype), "gradient")
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,length", [(1, 1), (1, 7), (3, 1), (5, 3), (4, 8), (8, 300), (2, 1001), (700, 5), (9, 4096), (1, 30000), (150, 2047)])
@pytest.mark.parametrize("reduction", ["token", "sequence"])
@pytest.mark.parametrize("masked", [False, True])
def test_against_the_definition(B, dtype, rows, length, reduction, masked):
    for per_token in (False, True):
        lp, old, adv, mask, ref = inputs(rows, length, dtype, rows + length, masked, per_token)
        check(B, lp, old, adv, mask, ref, reduction=reduction)
    check(B, lp, old, adv, mask, None, weight=0.0, reduction=reduction, norm=17.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("reduction", ["token", "sequence"])
def test_views(B, dtype, reduction):
    lp, old, adv, mask, ref = inputs(10, 203, dtype, 5)
    pad = lambda t, by, at: torch.nn.functional.pad(t, (at, by - at))[:, at:at + t.shape[1]]
    for by, at in ((1, 1), (8, 0), (5, 3)):
        check(B, pad(lp, by, at), old, adv, mask, pad(ref, by, at), reduction=reduction)
        check(B, lp, pad(old, by, at), pad(adv, by, at), pad(mask.to(torch.uint8) * 200, by, at), ref, reduction=reduction)
    row = adv[:, 0].contiguous()
    want = check(B, lp, old, row, mask, ref, reduction=reduction)
    for same in (row[:, None], row[:, None].expand(10, 203), adv[:, 0], adv[:, :1]):        # one value per row, however it is laid out
        got = B.policy_loss(lp, old, same, mask=mask, ref_logps=ref, clip_high=0.28, kl_weight=0.04, reduction=reduction)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    check(B, lp, old[:1].expand(10, 203), adv, mask[:1].expand(10, 203), ref, reduction=reduction)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", [64, 67])
@pytest.mark.parametrize("reduction", ["token", "sequence"])
def test_what_the_mask_leaves_out(B, dtype, length, reduction):
    lp, old, adv, mask, ref = inputs(7, length, dtype, 3)
    mask[2] = False; mask[6] = False                                    # rows of nothing: not counted among the sequences
    clean = check(B, lp, old, adv, mask, ref, reduction=reduction)
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min):
        hole = lambda t: torch.where(mask, t, torch.tensor(bad, dtype=dtype, device="cuda"))
        got = B.policy_loss(hole(lp), hole(old), hole(adv), mask=mask, ref_logps=hole(ref), clip_high=0.28, kl_weight=0.04, reduction=reduction)
        assert all(torch.equal(a, b) for a, b in zip(got, clean))
    nothing = B.policy_loss(lp, old, adv, mask=torch.zeros_like(mask), ref_logps=ref, kl_weight=0.1, reduction=reduction)
    assert not bool(nothing.terms.any()) and not bool(nothing.grad.any())


@pytest.mark.parametrize("shape", [(0, 5), (3, 0)])
@pytest.mark.parametrize("reduction", ["token", "sequence"])
def test_no_tokens(B, shape, reduction):
    t = torch.zeros(shape, device="cuda")
    for mask in (None, torch.ones(shape, dtype=torch.bool, device="cuda")):
        got = B.policy_loss(t, t, t, mask=mask, reduction=reduction)
        assert got.grad.shape == shape and not bool(got.terms.any())


def test_borders_of_the_clip(B):
    """Ratios just inside and outside of the borders: the gradient is there, or 0 (the KL term aside); on the border of its own the choice does not matter to the loss."""
    inside, outside = [], []
    for border in (1.28, 0.8):
        d = torch.tensor(border, dtype=torch.float64).log()
        for step in (1e-6, 1e-5, 1e-3):
            (inside if border < 1 else outside).append(float(d + step)); (outside if border < 1 else inside).append(float(d - step))
    d = torch.tensor(inside + outside, dtype=torch.float32, device="cuda")[None]
    adv = torch.where(d > 0, 1.0, -1.0)                                 # the sign for which the border counts
    got = check(B, d, torch.zeros_like(d), adv, None, None, weight=0.0)
    n = len(inside)
    assert bool((got.grad[0, :n] != 0).all()) and not bool(got.grad[0, n:].any())
    free = B.policy_loss(d, torch.zeros_like(d), -adv, clip_high=0.28)  # the other sign is never clipped
    assert bool((free.grad != 0).all()) and free.terms[3] == 0


def test_small_and_large_differences(B):
    """exp(x) - 1 - x from 1e-12 to 1e9: small ones keep their digits."""
    delta = torch.tensor([0.0, 1e-6, -1e-6, 1e-3, -1e-3, 0.1, -0.1, 0.99, -0.99, 1.01, -1.01, 5.0, -5.0, 20.0, -80.0], device="cuda")
    for v in delta:
        lp = torch.zeros(1, 1, device="cuda")
        got = B.policy_loss(lp, lp, lp, ref_logps=v.view(1, 1), kl_weight=1.0)
        k = float(torch.expm1(v.double()) - v.double())
        assert abs(float(got.terms[2]) - k) <= EPS * (12 * k + (4 * (k + 2 * abs(float(v)) + 2) if abs(v) > 1 else 0.0)), float(v)
    far = torch.full((1, 4), -200.0, device="cuda")                     # exp overflows: what the clip takes is finite
    zero = torch.zeros(1, 4, device="cuda")
    got = B.policy_loss(zero, far, torch.tensor([[1.0, 2.0, 0.5, 0.0]], device="cuda"))
    assert abs(float(got.terms[0]) + 1.2 * 3.5 / 4) < 1e-6 and not bool(got.grad.any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", [16, 19])
def test_tokens_that_the_reference_rules_out(B, dtype, length):
    """delta far below 0, down to the type's lowest value and -inf: the KL term grows without bound, its slope is -1.  d = 0 and A = 0, so the gradient is the
    slope's alone, weight (1 - exp(delta)) / tokens: exact to the roundings of the weight, the product and the result."""
    lp = torch.full((2, length), -1.0, device="cuda", dtype=dtype)
    zero = torch.zeros_like(lp)
    for low in (-30.0, -3000.0, -65504.0, torch.finfo(dtype).min, -float("inf")):
        ref = torch.full_like(lp, -1.0)
        ref[0, 3] = low; ref[1, length - 1] = low
        got = B.policy_loss(lp, lp, zero, ref_logps=ref, kl_weight=0.5)
        want = torch.zeros(2, length, dtype=torch.float64, device="cuda")
        want[0, 3] = want[1, length - 1] = 0.5 * -torch.expm1(torch.tensor(low + 1.0, dtype=torch.float64)) / (2 * length)
        assert_within(got.grad, want, rounding(want, dtype) + 6 * EPS * want.abs(), f"gradient at {low}")


def test_gradient_against_differences(B):
    """Central differences of the 64-bit definition, h = 1e-5, at tokens away from the borders (no third derivative over 10 / 60 tokens): below 1e-10; the kernel 2^-18."""
    lp, old, adv, mask, ref = inputs(3, 20, torch.float32, 8)
    got = B.policy_loss(lp, old, adv, mask=mask, ref_logps=ref, kl_weight=0.5, reduction="sequence")
    d = (lp - old).double()
    away = (d.exp() - 1.2).abs().minimum((d.exp() - 0.8).abs()) > 1e-3
    for r, t in ((0, 1), (1, 5), (2, 19), (2, 0)):
        if not bool(away[r, t]):
            continue
        at = []
        for sign in (1, -1):
            x = lp.double(); x[r, t] += sign * 1e-5
            at.append(policy64(x, old, adv, mask, ref, 0.2, 0.2, 0.5, "sequence")[0][0][0])
        assert abs(float((at[0] - at[1]) / 2e-5 - got.grad[r, t].double())) < 1e-9 + 2.0 ** -18


def test_repeated_captured_and_on_another_stream(B):
    lp, old, adv, mask, ref = inputs(500, 1003, torch.float32, 6)
    call = lambda **k: B.policy_loss(lp, old, adv, mask=mask, ref_logps=ref, kl_weight=0.1, reduction="sequence", **k)
    want = call()
    assert all(torch.equal(a, b) for a, b in zip(call(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    with torch.cuda.graph(other):
        more = call()
    lp.mul_(0.9)
    want = call()
    for _ in range(2):
        graph.replay(); other.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(more, want))
