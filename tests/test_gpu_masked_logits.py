"""Log-probabilities of rows that a mask of large negative numbers leaves little of, and of rows far from 0: held to what the distance of a logit from its row's maximum allows,
however large the masked logits are."""
import pytest
import torch

from model_util import EPS, TYPES, assert_within, f32, generator, logprobs64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


def tolerance(logits, targets, scale, logp, lse):
    """With d = scale (x - max): an exponent carries a rounded difference, the rounded factor scale log2 e and a rounded product, 3 |d| EPS, whatever rescalings it goes through on
    the way (their distances add up to d); below d = -104 it is 0.  2^x and the factor of a rescaling are good to 4 EPS, an addition to 1: a thread takes V / 1024 steps (a warp
    alone, fp32) of 32 additions and a rescaling, then follow 24 merges of lanes, warps, blocks or units.  That is the error of the sum, and of its logarithm the absolute one.
    logp = d_target - log sum: a rounded difference and product, the logarithm's 2 EPS and the factor ln 2, a last rounding; lse the same with scale max, which is rounded as lse is."""
    s = f32(scale)
    x = logits.double()
    top = x.amax(-1, keepdim=True)
    d = torch.where(torch.isfinite(top), (x - top) * s, 0.0)
    p = torch.softmax(torch.where(torch.isfinite(top), x * s, 0.0), -1)
    steps = logits.shape[-1] / 1024 + 1
    of_sum = EPS * (3 * (p * d.clamp(min=-104.0).abs()).sum(-1) + 4 + 37 * steps + 6 * 24)
    log_sum = -torch.log(p.amax(-1))
    at = d.gather(-1, targets.clamp(min=0)[..., None])[..., 0].abs()
    fin = lambda t: torch.where(torch.isfinite(t), t.abs(), 0.0)
    return of_sum + EPS * (3 * fin(at) + 4 * log_sum + 2 * fin(logp)), of_sum + EPS * (4 * log_sum + 2 * fin(lse))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(40, 100), (40, 1999), (24, 5001), (8, 50257), (320, 4099), (400, 30000)])
@pytest.mark.parametrize("low", [-30.0, -1e4, -6e4, -1e30, "lowest", "-inf"])
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_rows_with_little_left(B, dtype, rows, vocab, low, scale):
    """Two of three logits masked; all but five; all but one; none, but 100 above or below the others' range.  Targets of both kinds."""
    low = {"lowest": torch.finfo(dtype).min, "-inf": -float("inf")}.get(low, low)
    if low == -1e30 and dtype == torch.float16:
        low = -65000.0
    g = generator(rows + vocab)
    x = (torch.randn(rows, vocab, device="cuda", generator=g) * 3).to(dtype)
    at = torch.rand(rows, vocab, device="cuda", generator=g)
    kind = torch.arange(rows, device="cuda")[:, None] % 4
    x[(kind == 0) & (at < 0.67)] = low
    x[(kind == 1) & (at > at.topk(5, dim=-1, largest=False).values[:, -1:])] = low
    x[(kind == 2) & (at > at.amin(-1, keepdim=True))] = low
    x = torch.where(kind == 3, x + 100 * (2 * (torch.arange(rows, device="cuda")[:, None] // 4 % 2) - 1).to(dtype), x)
    targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    targets[::2] = x.argmax(-1)[::2]
    got = B.token_logprobs(x, targets, scale=scale)
    want = logprobs64(x, targets, scale)
    t0, t1 = tolerance(x, targets, scale, *want)
    beyond = torch.finfo(torch.float32).max
    logp = torch.where(want[0] < -beyond, -torch.inf, want[0])
    assert_within(got[0], logp, t0, "logp")
    assert_within(got[1], want[1], t1, "lse")
