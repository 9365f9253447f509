"""The preference loss where two finite log-probabilities differ by more than fp32 holds: whole vectors, the elements around them and single elements alike."""
import pytest
import torch

from model_util import TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", [t for t in TYPES if t != torch.float16])
@pytest.mark.parametrize("length", [16, 19, 300, 303])
@pytest.mark.parametrize("shifted", [False, True])
def test_differences_beyond_fp32(B, dtype, length, shifted):
    """lp - ref = -2 max in the chosen row, the same in the rejected row at another place: the margin is 0 and the gradient beta / 2.  An infinite sum on either side would
    make it NaN.  The sums are exact in 64 bits: they hold nothing else."""
    big = torch.finfo(dtype).max
    lp, ref = (torch.zeros(2, length + shifted, device="cuda", dtype=dtype)[:, shifted:] for _ in range(2))
    for here, there in ((0, length - 1), (length - 1, 0), (length // 2, length - 1), (1, length // 2)):
        lp.zero_(); ref.zero_()
        lp[0, here] = -big; ref[0, here] = big
        lp[1, there] = -big; ref[1, there] = big
        got = B.preference_loss(lp, ref, beta=0.5)
        assert abs(float(got.loss) - 0.6931471805599453) < 2.0 ** -23
        assert bool((got.grad[0] == -0.25).all()) and bool((got.grad[1] == 0.25).all())
        got = B.preference_loss(lp, ref, beta=2.0 ** -100)
        want = -2.0 * float(big) * 2.0 ** -100
        assert bool((got.rewards.double() - want).abs().max() <= abs(want) * 2.0 ** -24)
