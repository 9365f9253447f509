"""The balance loss of a router against the definition in 64 bits (tolerances: model_util)."""
import pytest
import torch

from model_util import EPS, TYPES, assert_within, balance64, generator, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


def inputs(rows, experts, chosen, dtype, seed, masked=True):
    g = generator(seed)
    x = (torch.randn(rows, experts, device="cuda", generator=g) + torch.randn(experts, device="cuda", generator=g)).to(dtype)
    choices = torch.topk(x.float(), chosen, dim=-1).indices
    mask = torch.rand(rows, device="cuda", generator=g) < 0.7 if masked else None
    return x, choices, mask


def check(B, x, choices, mask, weight=0.01):
    got = B.balance_loss(x, choices, mask=mask, weight=weight)
    (loss, counts, probs, grad), (t0, t1, t2) = balance64(x, choices, mask, weight)
    assert got.counts.dtype == torch.int32 and torch.equal(got.counts, counts)
    assert got.grad.dtype == x.dtype and got.grad.shape == x.shape and got.grad.is_contiguous()
    assert_within(got.loss, loss, t0, "loss")
    assert_within(got.probs, probs, t1, "probs")
    assert_within(got.grad, grad, t2 + rounding(grad, x.dtype), "gradient")
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,chosen", [(1, 1, 1), (1, 2, 2), (5, 3, 1), (100, 8, 2), (513, 7, 3), (64, 33, 4), (1000, 64, 6), (77, 100, 5), (300, 128, 8), (4099, 160, 6), (50, 256, 8),
                                                 (33, 257, 2), (20, 512, 10), (9, 1000, 1), (40, 1024, 16), (30000, 16, 1)])
@pytest.mark.parametrize("masked", [False, True])
def test_against_the_definition(B, dtype, rows, experts, chosen, masked):
    check(B, *inputs(rows, experts, chosen, dtype, rows + experts, masked))


@pytest.mark.parametrize("experts", [6, 64, 96])
def test_views_and_choices(B, experts):
    x, choices, mask = inputs(200, experts, 4, torch.bfloat16, 3)
    want = check(B, x, choices, mask)
    wide = torch.nn.functional.pad(x, (3, 4))[:, 3:-4]
    more = torch.nn.functional.pad(choices, (0, 3))[:, :4].to(torch.int32)
    every = mask.to(torch.uint8).mul_(7)
    spread = torch.zeros(400, dtype=torch.uint8, device="cuda"); spread[::2] = every
    for a in (x, wide):
        for c in (choices, choices.int(), more):
            got = B.balance_loss(a, c, mask=every, weight=0.01)
            assert torch.equal(got.counts, want.counts) and torch.equal(got.grad, want.grad) and torch.equal(got.loss, want.loss)
    choices[::3, 1] = -1                                                # dropped, and the same expert twice
    choices[1::3, 2] = experts
    choices[2::3, 3] = choices[2::3, 0]
    check(B, x, choices, mask)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts", [8, 70])
def test_masked_rows_and_logits(B, dtype, experts):
    x, choices, mask = inputs(60, experts, 2, dtype, 8)
    x[:, 1] = -float("inf")                                             # an expert that is switched off
    x[::4, 2] = torch.finfo(dtype).min
    mask[:4] = True
    x[0] = -float("inf")                                                # no expert left
    x[1] = torch.finfo(dtype).min                                       # all alike
    clean = check(B, x, choices, mask)
    assert not bool(clean.grad[0].any())
    for bad in (float("nan"), float("inf")):
        y = torch.where(mask[:, None], x, torch.tensor(bad, dtype=dtype, device="cuda"))
        c = torch.where(mask[:, None], choices, 1 << 40)
        got = B.balance_loss(y, c, mask=mask, weight=0.01)
        assert all(torch.equal(a, b) for a, b in zip(got, clean))
    nothing = B.balance_loss(x, choices, mask=torch.zeros_like(mask))
    assert not any(bool(t.any()) for t in nothing)
    empty = B.balance_loss(x[:0], choices[:0])
    assert empty.grad.shape == (0, experts) and empty.loss == 0 and not bool(empty.counts.any()) and not bool(empty.probs.any())
    x[3, 0] = float("nan")
    assert torch.isnan(B.balance_loss(x, choices, mask=mask).loss)


def test_a_balanced_router_has_no_gradient(B):
    """Every expert the same number of tokens: the shares' differences are exact zeros, and the loss is the weight."""
    x = torch.randn(96, 12, device="cuda")
    choices = (torch.arange(96, device="cuda")[:, None] + torch.arange(3, device="cuda")) % 12
    got = B.balance_loss(x, choices, weight=0.5)
    assert not bool(got.grad.any()) and abs(float(got.loss) - 0.5) < 1e-6 and bool((got.counts == 24).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts", [7, 64, 512])
def test_choices_forced_by_the_largest_value(B, dtype, experts):
    """Logits of the type's largest value: the probabilities are 1, 1/2 and 0.  Tolerance: a share's rounding, the row's sums, the reciprocal (2 units), three products:
    below 16 EPS of twice the largest share apart from the mean."""
    x = torch.zeros(40, experts, device="cuda", dtype=dtype)
    x[:, 3] = torch.finfo(dtype).max
    x[20:, 5] = torch.finfo(dtype).max
    choices = torch.full((40, 1), 3, device="cuda")
    choices[30:] = 5
    got = B.balance_loss(x, choices, weight=1.0)
    p = torch.softmax(x.double(), -1)
    share = torch.bincount(choices.flatten(), minlength=experts).double() / 40
    apart = share - 1.0 / experts
    grad = experts / 40 * p * (apart - (p * apart).sum(-1, keepdim=True))
    assert_within(got.grad, grad, experts / 40 * p * 32 * EPS * apart.abs().max() + rounding(grad, dtype), "gradient")
    assert_within(got.probs, p.mean(0), 48 * EPS * p.mean(0), "probs")            # (40 additions at most, and the probabilities' own four)
    loss = experts * (share * p.mean(0)).sum()
    assert_within(got.loss, loss, 50 * EPS * loss, "loss")


def test_gradient_against_differences(B):
    """Central differences of the loss in 64 bits (h = 1e-4): below 1e-8; the kernel: 2^-18 of E weight / N."""
    x, choices, mask = inputs(20, 9, 2, torch.float32, 4)
    got = B.balance_loss(x, choices, mask=mask, weight=1.0)
    for r, e in ((0, 0), (3, 8), (11, 4), (19, 2)):
        at = []
        for sign in (1, -1):
            y = x.double(); y[r, e] += sign * 1e-4
            at.append(balance64(y, choices, mask, 1.0)[0][0])
        assert abs(float((at[0] - at[1]) / 2e-4 - got.grad[r, e].double())) < 1e-8 + 2.0 ** -18


def test_repeated_captured_and_on_another_stream(B):
    x, choices, mask = inputs(20000, 48, 4, torch.bfloat16, 6)
    call = lambda **k: B.balance_loss(x, choices, mask=mask, **k)
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
    x.neg_()
    want = call()
    for _ in range(2):
        graph.replay(); other.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(more, want))
