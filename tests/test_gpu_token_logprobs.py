"""Log-probabilities of tokens and the logits' gradient, against the definition in 64 bits (tolerances: model_util)."""
import pytest
import torch

from model_util import TYPES, assert_within, generator, logprobs64, logprobs_grad64, logprobs_tolerance, rounding

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


def check(B, logits, targets, scale=1.0, ignore=-100, seed=5):
    logp, lse = B.token_logprobs(logits, targets, scale=scale, ignore=ignore)
    want_logp, want_lse = logprobs64(logits, targets, scale, ignore)
    tol = logprobs_tolerance(logits, want_lse, want_logp, scale)
    assert logp.shape == lse.shape == targets.shape and logp.dtype == lse.dtype == torch.float32
    assert_within(lse, want_lse, tol, "lse")
    assert_within(logp, want_logp, tol, "logp")
    grad = torch.randn(targets.shape, device="cuda", generator=generator(seed))
    grad[torch.rand(targets.shape, device="cuda", generator=generator(seed + 1)) < 0.2] = 0.0
    dx = B.token_logprobs_grad(logits, targets, lse, grad, scale=scale, ignore=ignore)
    want, tol = logprobs_grad64(logits, targets, lse, grad, scale, ignore)
    assert dx.shape == logits.shape and dx.dtype == logits.dtype
    assert_within(dx, want, tol * 1.01 + rounding(want, logits.dtype), "gradient")
    return logp, lse, grad, dx


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 2), (3, 7), (9, 31), (5, 257), (17, 2047), (2, 2048), (1, 2049), (4, 4099), (1, 16384), (3, 32768), (700, 4097), (2, 131073), (300, 5000)])
def test_against_the_definition(B, dtype, rows, vocab):
    g = generator(rows * 1000 + vocab)
    logits = torch.randn(rows, vocab, device="cuda", generator=g).mul_(3).to(dtype)
    targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    if rows > 2:
        targets[1] = -100
    check(B, logits, targets, scale=1.0 if vocab % 2 else 0.7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,length,vocab", [(3, 5, 4097), (2, 1, 33), (4, 9, 2500), (1, 12, 50257), (40, 9, 4099), (3, 100, 9001)])
def test_views_of_a_batch(B, dtype, batch, length, vocab):
    """Every position against the token behind it: no row of the last position is touched; gradients into a view of a table of their own."""
    g = generator(vocab)
    whole = torch.randn(batch, length + 1, vocab, device="cuda", generator=g).mul_(2).to(dtype)
    tokens = torch.randint(0, vocab, (batch, length + 1), device="cuda", generator=g, dtype=torch.int32)
    _, lse, grad, dx = check(B, whole[:, :-1], tokens[:, 1:], scale=1.3)
    full = torch.full_like(whole, 7.0)
    got = B.token_logprobs_grad(whole[:, :-1], tokens[:, 1:], lse, grad, scale=1.3, out=full[:, :-1])
    assert got.data_ptr() == full.data_ptr() and torch.equal(full[:, :-1], dx) and bool((full[:, -1] == 7.0).all())
    own = whole.clone()                                               # in place, rows behind the last one as they were
    B.token_logprobs_grad(own[:, :-1], tokens[:, 1:], lse, grad, scale=1.3, out=own[:, :-1])
    assert torch.equal(own[:, :-1], dx) and torch.equal(own[:, -1], whole[:, -1])
    padded = torch.zeros(batch * length, vocab + 5, device="cuda", dtype=dtype)          # another pitch
    padded[:, 2:vocab + 2] = whole[:, :-1].reshape(-1, vocab)
    again, _ = B.token_logprobs(padded[:, 2:vocab + 2], tokens[:, 1:].reshape(-1), scale=1.3)
    want, want_lse = logprobs64(whole[:, :-1].reshape(-1, vocab), tokens[:, 1:].reshape(-1), 1.3)
    assert_within(again, want, logprobs_tolerance(padded[:, 2:vocab + 2], want_lse, want, 1.3))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [50, 9001])
def test_masked_and_non_finite_logits(B, dtype, vocab):
    g = generator(vocab + 1)
    logits = torch.randn(10, vocab, device="cuda", generator=g).mul_(2).to(dtype)
    targets = torch.randint(0, vocab, (10,), device="cuda", generator=g)
    low = torch.finfo(dtype).min
    logits[0] = -INF                                                   # nothing left
    logits[1, : vocab // 2] = -INF; targets[1] = vocab - 1             # half of the vocabulary
    logits[2, 3] = INF
    logits[3, 4] = float("nan")
    logits[4] = -INF; logits[4, 7] = 1.5; targets[4] = 7               # one left: probability 1
    logits[5, 5] = -INF; targets[5] = 5                                # a target that cannot be
    logits[6, : vocab - 2] = low; targets[6] = vocab - 1               # the type's lowest value as a mask
    logits[7] = float("nan"); targets[7] = -100                        # ignored: not read
    logits[8] = low                                                    # all of them: the same value
    targets[9] = vocab                                                 # no such token
    logp, lse = B.token_logprobs(logits, targets)
    want, want_lse = logprobs64(logits, targets)
    want[2:4] = torch.nan; want_lse[2:4] = torch.nan                   # +inf and NaN: no distribution
    tol = logprobs_tolerance(logits, want_lse, want)
    assert_within(logp, want, tol); assert_within(lse, want_lse, tol)
    assert logp[4] == 0.0 and logp[0] == -INF and logp[7] == 0.0 and lse[7] == 0.0
    grad = torch.ones(10, device="cuda")
    dx = B.token_logprobs_grad(logits, targets, lse, grad)
    wdx, tol = logprobs_grad64(logits, targets, lse, grad)
    assert_within(dx, wdx, tol * 1.01 + rounding(wdx, dtype))
    assert not bool(dx[0].any()) and not bool(dx[7].any()) and bool(torch.isnan(dx[9]).all())
    assert not bool(B.token_logprobs_grad(logits, targets, lse, torch.zeros(10, device="cuda")).any())      # NaN in rows without a gradient


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(3, 77), (2, 30000), (300, 4100)])
def test_a_target_that_a_mask_took(B, dtype, rows, vocab):
    """Of the type's lowest value: its log-probability is that value (times the scale), less the row's lse -- a finite number."""
    logits = torch.randn(rows, vocab, device="cuda", generator=generator(vocab)).to(dtype)
    logits[:, ::2] = torch.finfo(dtype).min
    targets = torch.arange(rows, device="cuda") % (vocab // 2) * 2
    for scale in (1.0, 0.5):
        logp, lse, grad, dx = check(B, logits, targets, scale=scale)
        assert bool(torch.isfinite(logp).all()) and bool((logp < scale * 0.99 * torch.finfo(dtype).min).all())


def test_large_logits_and_int32(B):
    logits = torch.full((3, 3000), 30000.0, device="cuda"); logits[1] = -30000.0; logits[2, 1700] = 30100.0
    targets = torch.tensor([5, 2999, 1700], device="cuda", dtype=torch.int32)
    check(B, logits, targets)
    check(B, logits.half(), targets)
    a, b = B.token_logprobs(logits, targets), B.token_logprobs(logits, targets.long())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_gradient_against_differences(B):
    """d logp / d x by central differences of the definition in 64 bits: their own error is below h^2 / 6 + 2^-49 / h < 1e-8; the
    kernel's, with |x| and lse below 6 and lse itself rounded, below 60 * 2^-24 < 4e-6."""
    g = generator(3)
    logits = torch.randn(4, 90, device="cuda", generator=g)
    targets = torch.randint(0, 90, (4,), device="cuda", generator=g)
    _, lse = B.token_logprobs(logits, targets, scale=0.5)
    dx = B.token_logprobs_grad(logits, targets, lse, torch.ones(4, device="cuda"), scale=0.5).double()
    h = 1e-4
    for j in (0, 17, 89, int(targets[0])):
        at = []
        for sign in (1, -1):
            x = logits.double(); x[:, j] += sign * h
            at.append((x * 0.5).gather(1, targets[:, None])[:, 0] - torch.logsumexp(x * 0.5, 1))
        assert float(((at[0] - at[1]) / (2 * h) - dx[:, j]).abs().max()) < 1e-8 + 4e-6


def test_empty_and_repeated(B):
    for shape in ((0, 5), (2, 0, 7)):
        logits = torch.zeros(shape, device="cuda")
        logp, lse = B.token_logprobs(logits, torch.zeros(shape[:-1], dtype=torch.int64, device="cuda"))
        assert logp.shape == shape[:-1]
        assert B.token_logprobs_grad(logits, torch.zeros(shape[:-1], dtype=torch.int64, device="cuda"), lse, logp).shape == shape
    logits = torch.randn(50, 40001, device="cuda", dtype=torch.bfloat16)
    targets = torch.randint(0, 40001, (50,), device="cuda")
    first = B.token_logprobs(logits, targets)
    for _ in range(3):
        again = B.token_logprobs(logits, targets)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_offsets_beyond_32_bits(B):
    """A row that starts more than 2^32 bytes, and more than 2^31 elements, behind the first one."""
    vocab, rows = 140001, 16000
    logits = torch.zeros(rows, vocab, device="cuda", dtype=torch.bfloat16)            # 4.5 GB
    logits[-1].copy_(torch.randn(vocab, device="cuda"))
    targets = torch.full((rows,), -100, device="cuda"); targets[-1] = vocab - 1
    logp, lse = B.token_logprobs(logits, targets)
    want, want_lse = logprobs64(logits[-1:], targets[-1:])
    assert_within(logp[-1:], want, logprobs_tolerance(logits[-1:], want_lse, want))
    assert not bool(logp[:-1].any())
    grad = torch.ones(rows, device="cuda")
    want, tol = logprobs_grad64(logits[-1:], targets[-1:], lse[-1:], grad[-1:])
    B.token_logprobs_grad(logits, targets, lse, grad, out=logits)
    assert_within(logits[-1:], want, tol * 1.01 + rounding(want, torch.bfloat16))
    assert not bool(logits[-2].any())


def test_captured_and_on_another_stream(B):
    logits = torch.randn(6, 9000, device="cuda")
    targets = torch.randint(0, 9000, (6,), device="cuda")
    want = B.token_logprobs(logits, targets)
    grad = torch.randn(6, device="cuda")
    want_dx = B.token_logprobs_grad(logits, targets, want[1], grad)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = B.token_logprobs(logits, targets, stream=side)
    side.synchronize()
    assert torch.equal(other[0], want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.token_logprobs(logits, targets)
        dx = B.token_logprobs_grad(logits, targets, got[1], grad)
    logits.normal_(); grad.normal_()
    graph.replay()
    want = B.token_logprobs(logits, targets)
    want_dx = B.token_logprobs_grad(logits, targets, want[1], grad)
    assert torch.equal(got[0], want[0]) and torch.equal(dx, want_dx)
