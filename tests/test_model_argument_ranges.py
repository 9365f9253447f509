"""Numbers and addresses that the entries of a language model's worker refuse because the kernels could not work with them; on a machine without a GPU: an entry returns before it
touches a device."""
import pytest
import torch

from paper_2106_05203_b200 import binding as B

INVALID = 1
L = B._lib
P = 4096                                             # an address that is looked at, never followed

LOGPROBS = dict(logits=P, dtype=1, batch=2, length=3, vocab=10, bs=30, rs=10, targets=P, index=1, ts=3, scale=1.0, ignore=-100, logps=P, lse=P, ws=None, n=0, stream=None)
LOGPROBS_GRAD = dict(logits=P, dtype=1, batch=2, length=3, vocab=10, bs=30, rs=10, targets=P, index=1, ts=3, lse=P, grad=P, scale=1.0, ignore=-100, out=None, obs=30, ors=10, stream=None)
PREFERENCE = dict(logps=P, ref=P, mask=P, dtype=0, pairs=4, length=100, ls=100, rs=100, ms=100, beta=0.1, smoothing=0.0, norm=4.0, loss=P, rewards=P, grad=P, ws=None, n=0, stream=None)
POLICY = dict(logps=P, old=P, ref=P, adv=P, mask=P, dtype=0, rows=4, length=100, a=100, b=100, c=100, d=100, e=100, per_token=1, low=0.2, high=0.2, kl=0.1, reduction=0, norm=0.0, terms=P, grad=P,
              ws=None, n=0, stream=None)
BALANCE = dict(logits=P, dtype=0, rows=4, experts=8, ls=8, choices=P, index=1, chosen=2, cs=2, mask=P, weight=0.1, loss=P, counts=P, probs=P, grad=P, ws=None, n=0, stream=None)
EMBEDDING = dict(weight=P, dtype=1, vocab=10, dim=8, stride=8, tokens=P, index=1, count=5, scale=1.0, out=None, stream=None)
EMBEDDING_GRAD = dict(grad=P, dtype=1, count=5, dim=8, stride=8, tokens=P, index=1, vocab=10, padding=-1, scale=1.0, out=P, out_dtype=1, out_stride=8, accumulate=0, ws=None, n=0, stream=None)


def status(entry, good, **bad):
    """No call gets as far as a launch: each lacks its workspace, or its output."""
    return getattr(L, entry)(*{**good, **bad}.values())


def fine(entry, good, **more):
    """Whether the arguments are taken, up to the workspace that is not there (3), or with no row at all (0)."""
    return status(entry, good, **more) in (0, 3)


@pytest.mark.parametrize("entry,good,rows", [("ef21_token_logprobs", LOGPROBS, {}), ("ef21_token_logprobs_grad", LOGPROBS_GRAD, {"length": 0})])
def test_scales_whose_product_with_log2_e_is_infinite(entry, good, rows):
    """One over a temperature: times log2 e it has to be a number of 32 bits, or every exponent is 0 times infinity."""
    for scale in (2.4e38, 3e38, 3.4e38):
        assert status(entry, good, scale=scale, **rows) == INVALID
    for scale in (1e-30, 1.0, 1e30, 2.3e38):
        assert fine(entry, good, scale=scale, **rows)


def test_weights_beyond_fp32():
    """They are held in 32 bits beside the logits or log-probabilities."""
    for kl in (1e39, -1e39, 1e300):
        assert status("ef21_policy_loss", POLICY, kl=kl) == INVALID
    assert fine("ef21_policy_loss", POLICY, kl=1e38) and fine("ef21_policy_loss", POLICY, kl=-0.5)
    for norm in (1e-39, 1e-300):
        assert status("ef21_policy_loss", POLICY, norm=norm) == INVALID
    assert fine("ef21_policy_loss", POLICY, norm=1e-30) and fine("ef21_policy_loss", POLICY, norm=1e30)
    for weight in (1e38, 1e39, -1e300):
        assert status("ef21_balance_loss", BALANCE, weight=weight) == INVALID          # (times eight experts)
    assert fine("ef21_balance_loss", BALANCE, weight=1e37) and fine("ef21_balance_loss", BALANCE, weight=-1.0)


@pytest.mark.parametrize("entry,good,fields,rows", [
    ("ef21_token_logprobs", LOGPROBS, [("targets", 4), ("logps", 2), ("lse", 2)], {}),
    ("ef21_token_logprobs_grad", LOGPROBS_GRAD, [("targets", 4), ("lse", 2), ("grad", 2)], {"out": P, "length": 1}),
    ("ef21_preference_loss", PREFERENCE, [("loss", 2), ("rewards", 2)], {}),
    ("ef21_policy_loss", POLICY, [("terms", 2)], {}),
    ("ef21_balance_loss", BALANCE, [("choices", 4), ("loss", 2), ("counts", 2), ("probs", 2)], {}),
    ("ef21_embedding", EMBEDDING, [("tokens", 4)], {"out": P}),
    ("ef21_embedding_grad", EMBEDDING_GRAD, [("tokens", 4)], {}),
])
def test_addresses_between_two_elements(entry, good, fields, rows):
    """Indices and fp32 arrays as well as the tensors: a load from there would be a fault of the device.  (Refused before anything else; with a device at hand it is not
    tried out what became of a call that is not.)"""
    if torch.cuda.is_available():
        pytest.skip("entries by themselves, without a device")
    for field, off in fields:
        assert status(entry, good, **rows, **{field: P + off}) == INVALID, field
        if field in ("targets", "choices", "tokens"):
            assert status(entry, good, **rows, **{field: P + 2, "index": 0}) == INVALID, field


LAZY = [
    ("token_logprobs", lambda B, t, n: B.token_logprobs(n(2, 8), t.zeros(2, dtype=torch.int64))),
    ("token_logprobs_grad", lambda B, t, n: B.token_logprobs_grad(t.ones(2, 8), t.zeros(2, dtype=torch.int64), t.ones(2), n(2))),
    ("preference_loss", lambda B, t, n: B.preference_loss(n(4, 5))),
    ("preference_loss, reference", lambda B, t, n: B.preference_loss(t.ones(4, 5), n(4, 5))),
    ("policy_loss", lambda B, t, n: B.policy_loss(t.ones(4, 5), t.ones(4, 5), n(4))),
    ("balance_loss", lambda B, t, n: B.balance_loss(n(4, 5), t.zeros(4, 1, dtype=torch.int64))),
    ("embedding", lambda B, t, n: B.embedding(n(4, 5), t.zeros(3, dtype=torch.int64))),
    ("embedding_grad", lambda B, t, n: B.embedding_grad(n(3, 5), t.zeros(3, dtype=torch.int64), 4)),
]


class On:
    """torch's constructors on a device."""

    def __init__(self, device):
        self.zeros = lambda *s, **k: torch.zeros(*s, device=device, **k)
        self.ones = lambda *s, **k: torch.ones(*s, device=device, **k)


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
@pytest.mark.parametrize("call", [c for _, c in LAZY], ids=[n for n, _ in LAZY])
def test_negatives_that_are_not_taken_yet(device, call):
    """What x.conj().imag of a complex x is: the negative is taken when a value is read, the memory holds the opposite."""
    with pytest.raises(TypeError, match="negative"):
        call(B, On(device), lambda *s: torch._neg_view(torch.ones(*s, device=device)))
