"""The preference loss against the definition in 64 bits (tolerances: model_util)."""
import pytest
import torch

from model_util import EPS, TYPES, assert_within, generator, preference64, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


def inputs(rows, length, dtype, seed, masked):
    g = generator(seed)
    lp = -torch.empty(rows, length, device="cuda").exponential_(generator=g)
    ref = lp + 0.2 * torch.randn(rows, length, device="cuda", generator=g)
    mask = torch.rand(rows, length, device="cuda", generator=g) < 0.6 if masked else None
    return lp.to(dtype), ref.to(dtype), mask


def check(B, lp, ref, mask, beta=0.1, smoothing=0.0, norm=None):
    got = B.preference_loss(lp, ref, mask=mask, beta=beta, smoothing=smoothing, norm=norm)
    (loss, rewards, grad), (t0, t1, t2) = preference64(lp, ref, mask, beta, smoothing, norm)
    assert got.loss.dtype == got.rewards.dtype == torch.float32 and got.grad.dtype == lp.dtype and got.grad.is_contiguous()
    assert_within(got.loss, loss, t0, "loss")
    assert_within(got.rewards, rewards, t1, "rewards")
    assert_within(got.grad, grad, t2 + rounding(grad, lp.dtype), "gradient")
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairs,length", [(1, 0), (1, 1), (2, 3), (3, 8), (5, 17), (1, 4097), (33, 255), (7, 1000), (1300, 5), (40, 2051), (300, 64)])
@pytest.mark.parametrize("masked", [False, True])
def test_against_the_definition(B, dtype, pairs, length, masked):
    lp, ref, mask = inputs(2 * pairs, length, dtype, pairs + length, masked)
    check(B, lp, ref, mask, beta=0.1 + 0.01 * length, smoothing=0.1 if pairs % 2 else 0.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_views(B, dtype):
    lp, ref, mask = inputs(12, 301, dtype, 9, True)
    want = check(B, lp, ref, mask)
    pad = lambda t, by, at: torch.nn.functional.pad(t, (at, by - at))[:, at:at + t.shape[1]]
    for by, at in ((1, 1), (8, 0), (16, 8), (3, 2), (11, 8)):           # pitches and beginnings, of the same phase and others
        got = B.preference_loss(pad(lp, by, at), pad(ref, by, at), mask=pad(mask, by, at))
        for a, b in zip(got, want):
            assert torch.allclose(a.float(), b.float(), rtol=1e-5, atol=1e-8)
        check(B, pad(lp, by, at), ref, pad(mask.to(torch.uint8) * 3, by, at))
    check(B, lp, None, mask)
    check(B, lp, ref[:1].expand(12, 301), mask[:1].expand(12, 301))     # one row for all
    check(B, lp, ref, mask, norm=1000.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", [40, 41])
def test_what_the_mask_leaves_out(B, dtype, length):
    lp, ref, mask = inputs(8, length, dtype, 4, True)
    mask[1] = False; mask[5] = False                                    # a pair of nothing: log 2
    mask[2] = False                                                     # one side of nothing
    clean = B.preference_loss(lp, ref, mask=mask)
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min):
        got = B.preference_loss(torch.where(mask, lp, torch.tensor(bad, dtype=dtype, device="cuda")), torch.where(mask, ref, torch.tensor(bad, dtype=dtype, device="cuda")), mask=mask)
        assert all(torch.equal(a, b) for a, b in zip(got, clean))
    check(B, lp, ref, mask)
    assert clean.rewards[1] == 0 and clean.rewards[2] == 0


def test_far_margins(B):
    """Margins at which exp overflows: the loss is linear on one side, 0 on the other."""
    lp = torch.zeros(6, 10, device="cuda"); lp[0] = 5000.0; lp[4] = 9000.0; lp[2] = 0.01
    for smoothing in (0.0, 0.3):
        check(B, lp, torch.zeros_like(lp), None, beta=1.0, smoothing=smoothing)
    lp[3] = float("nan")
    got = B.preference_loss(lp, torch.zeros_like(lp))
    assert torch.isnan(got.loss) and torch.isnan(got.grad[0]).all() and not torch.isnan(got.grad[1]).any()


def test_gradient_against_differences(B):
    """Central differences of the 64-bit definition (h = 1e-4, |slope'''| < 0.2 beta^3): below 1e-9; the kernel: 2^-20 of the slope."""
    lp, ref, mask = inputs(6, 30, torch.float32, 2, True)
    got = B.preference_loss(lp, ref, mask=mask, beta=0.5, smoothing=0.1)
    for r, t in ((0, 0), (2, 7), (4, 29), (5, 13)):
        at = []
        for sign in (1, -1):
            x = lp.double(); x[r, t] += sign * 1e-4
            at.append(preference64(x, ref, mask, 0.5, 0.1)[0][0])
        assert abs(float((at[0] - at[1]) / 2e-4 - got.grad[r, t].double())) < 1e-9 + 0.5 * 2.0 ** -20


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", [12, 300, 2051])
def test_tokens_that_are_ruled_out(B, dtype, length):
    """Log-probabilities of the type's lowest value and of -inf, in one vector and in several: the loss is the formula's (a margin of -+inf: infinite where its term has a
    weight, 0 where not), the slope beta / P times 1 - eps or -eps, exact to its roundings, as the sigma is 0 or 1."""
    pairs, beta, least = 3, 0.1, torch.finfo(dtype).min
    for low in (least, -float("inf")):
        for side, eps in ((0, 0.0), (0, 0.1), (1, 0.0), (1, 0.1), (0, 1.0), (1, 1.0)):
            lp = torch.full((2 * pairs, length), -1.0, device="cuda", dtype=dtype)
            lp[side * pairs, 8:12] = low
            got = B.preference_loss(lp, beta=beta, smoothing=eps)
            d = lp.double().sum(1)
            z = beta * (d[:pairs] - d[pairs:])
            term = lambda weight, v: weight * torch.nn.functional.softplus(v) if weight else torch.zeros_like(v)
            each = term(1 - eps, -z) + term(eps, z)
            # sums of magnitudes: those of at most `length` ones, and up to eight added in 32 bits
            off = 12 * EPS * (each[torch.isfinite(each)].abs().sum() + beta * length)
            assert_within(got.loss, each.sum() / pairs, off, "loss")
            assert_within(got.rewards, beta * d, 12 * EPS * (beta * d).abs(), "rewards")
            slope = beta / pairs * (torch.sigmoid(-z) - eps)
            want = torch.cat([-slope, slope])[:, None].expand(2 * pairs, length)
            tol = rounding(want, dtype) + 4 * EPS * want.abs()
            assert_within(got.grad, want, tol, "gradient")


def test_repeated_captured_and_on_another_stream(B):
    lp, ref, mask = inputs(600, 900, torch.float32, 7, True)
    want = B.preference_loss(lp, ref, mask=mask)
    assert all(torch.equal(a, b) for a, b in zip(B.preference_loss(lp, ref, mask=mask), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.preference_loss(lp, ref, mask=mask, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):                                                  # two graphs, replayed in turn: a workspace each
        graphs.append((torch.cuda.CUDAGraph(), []))
        with torch.cuda.graph(graphs[-1][0]):
            graphs[-1][1].extend(B.preference_loss(lp, ref, mask=mask))
    lp.mul_(0.5)
    want = B.preference_loss(lp, ref, mask=mask)
    for graph, got in graphs + graphs:
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
