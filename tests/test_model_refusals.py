"""Arguments that the calls of a language model's worker refuse, on a machine without a GPU: the C entries return before they touch a device, the binding
looks at shapes and types before devices."""
import ctypes

import pytest
import torch

from paper_2106_05203_b200 import binding as B

INVALID, WORKSPACE, UNSUPPORTED = 1, 3, 7
L = B._lib
P = 4096                                             # an address that is looked at, never followed
NAN, INF = float("nan"), float("inf")


def test_token_logprobs_entry():
    good = dict(logits=P, dtype=1, batch=2, length=3, vocab=10, bs=30, rs=10, targets=P, index=1, ts=3, scale=1.0, ignore=-100, logps=P, lse=P, ws=P, n=1 << 20, stream=None)
    for bad in (dict(dtype=3), dict(dtype=-1), dict(batch=-1), dict(length=-1), dict(vocab=0), dict(vocab=1 << 31), dict(batch=1 << 31), dict(batch=1 << 20, length=1 << 20), dict(index=2),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(logits=None), dict(logits=P + 1), dict(targets=None), dict(logps=None), dict(lse=None)):
        assert L.ef21_token_logprobs(*{**good, **bad}.values()) == INVALID, bad
    assert L.ef21_token_logprobs(*{**good, "batch": 0, "logits": None}.values()) == 0
    size = L.ef21_token_logprobs_workspace_bytes
    assert size(0, 2, 3, 10) > 0 and size(1, 64, 1000, 50000) > 64000 * 8 and size(3, 2, 3, 10) == 0 and size(0, -1, 3, 10) == 0 and size(0, 2, 3, 0) == 0
    for bad in (dict(ws=None), dict(ws=P + 1), dict(n=8)):
        assert L.ef21_token_logprobs(*{**good, **bad}.values()) == WORKSPACE, bad
    good = dict(logits=P, dtype=1, batch=2, length=3, vocab=10, bs=30, rs=10, targets=P, index=1, ts=3, lse=P, grad=P, scale=1.0, ignore=-100, out=P, obs=30, ors=10, stream=None)
    for bad in (dict(dtype=3), dict(vocab=0), dict(scale=NAN), dict(lse=None), dict(grad=None), dict(out=None), dict(out=P + 1), dict(index=-1)):
        assert L.ef21_token_logprobs_grad(*{**good, **bad}.values()) == INVALID, bad
    assert L.ef21_token_logprobs_grad(*{**good, "length": 0}.values()) == 0


def test_preference_entry():
    size = L.ef21_preference_loss_workspace_bytes
    assert size(4, 100) > 0 and size(0, 100) == 0 and size(-1, 5) == 0 and size(4, -1) == 0 and size(1 << 31, 1) == 0 and size(4, 1 << 31) == 0
    good = dict(logps=P, ref=P, mask=P, dtype=0, pairs=4, length=100, ls=100, rs=100, ms=100, beta=0.1, smoothing=0.0, norm=4.0, loss=P, rewards=P, grad=P, ws=P, n=1 << 20, stream=None)
    for bad in (dict(dtype=9), dict(pairs=0), dict(length=-1), dict(beta=NAN), dict(beta=INF), dict(smoothing=-0.1), dict(smoothing=1.1), dict(smoothing=NAN), dict(norm=0.0), dict(norm=-1.0),
                dict(norm=INF), dict(norm=NAN), dict(logps=None), dict(loss=None), dict(rewards=None), dict(grad=None), dict(logps=P + 2), dict(ref=P + 2), dict(grad=P + 2)):
        assert L.ef21_preference_loss(*{**good, **bad}.values()) == INVALID, bad
    for bad in (dict(ws=None), dict(ws=P + 64), dict(n=8)):
        assert L.ef21_preference_loss(*{**good, **bad}.values()) == WORKSPACE, bad


def test_policy_entry():
    size = L.ef21_policy_loss_workspace_bytes
    assert size(4, 100) > 0 and size(0, 100) > 0 and size(-1, 5) == 0 and size(4, -1) == 0 and size(1 << 31, 1) == 0
    good = dict(logps=P, old=P, ref=P, adv=P, mask=P, dtype=0, rows=4, length=100, a=100, b=100, c=100, d=100, e=100, per_token=1, low=0.2, high=0.2, kl=0.1, reduction=0, norm=0.0, terms=P,
                grad=P, ws=P, n=1 << 24, stream=None)
    for bad in (dict(dtype=5), dict(rows=-1), dict(length=-1), dict(low=1.0), dict(low=-0.1), dict(low=NAN), dict(high=-0.1), dict(high=INF), dict(high=NAN), dict(kl=NAN), dict(kl=INF), dict(ref=None),
                dict(reduction=2), dict(reduction=-1), dict(norm=-1.0), dict(norm=NAN), dict(norm=INF), dict(terms=None), dict(logps=None), dict(old=None), dict(adv=None), dict(grad=None),
                dict(old=P + 1), dict(adv=P + 2)):
        assert L.ef21_policy_loss(*{**good, **bad}.values()) == INVALID, bad
    for bad in (dict(ws=None), dict(ws=P + 1), dict(n=64)):
        assert L.ef21_policy_loss(*{**good, **bad}.values()) == WORKSPACE, bad


def test_balance_entry():
    size = L.ef21_balance_loss_workspace_bytes
    assert size(4, 8) > 0 and size(0, 1024) > 0 and size(4, 1025) == 0 and size(4, 0) == 0 and size(-1, 8) == 0 and size(1 << 31, 8) == 0
    good = dict(logits=P, dtype=0, rows=4, experts=8, ls=8, choices=P, index=1, chosen=2, cs=2, mask=P, weight=0.1, loss=P, counts=P, probs=P, grad=P, ws=P, n=1 << 24, stream=None)
    for bad in (dict(dtype=5), dict(rows=-1), dict(experts=0), dict(experts=2000), dict(chosen=0), dict(chosen=9), dict(index=3), dict(rows=1 << 30, chosen=8), dict(weight=NAN), dict(weight=INF),
                dict(loss=None), dict(counts=None), dict(probs=None), dict(grad=None), dict(logits=None), dict(choices=None), dict(logits=P + 2)):
        assert L.ef21_balance_loss(*{**good, **bad}.values()) == INVALID, bad
    for bad in (dict(ws=None), dict(ws=P + 1), dict(n=64)):
        assert L.ef21_balance_loss(*{**good, **bad}.values()) == WORKSPACE, bad


def test_embedding_entries():
    good = dict(weight=P, dtype=1, vocab=10, dim=8, stride=8, tokens=P, index=1, count=5, scale=1.0, out=P, stream=None)
    for bad in (dict(dtype=5), dict(vocab=0), dict(vocab=1 << 31), dict(dim=0), dict(dim=1 << 31), dict(count=-1), dict(count=1 << 31), dict(index=2), dict(scale=NAN), dict(scale=INF), dict(weight=None),
                dict(tokens=None), dict(out=None), dict(weight=P + 1), dict(out=P + 1)):
        assert L.ef21_embedding(*{**good, **bad}.values()) == INVALID, bad
    assert L.ef21_embedding(*{**good, "count": 0}.values()) == 0
    size = L.ef21_embedding_grad_workspace_bytes
    assert size(5, 10, 8) > 0 and size(0, 10, 8) > 0 and size(-1, 10, 8) == 0 and size(5, 0, 8) == 0 and size(5, 10, 0) == 0 and size(1 << 31, 10, 8) == 0
    good = dict(grad=P, dtype=1, count=5, dim=8, stride=8, tokens=P, index=1, vocab=10, padding=-1, scale=1.0, out=P, out_dtype=1, out_stride=8, accumulate=0, ws=P, n=1 << 24, stream=None)
    for bad in (dict(dtype=5), dict(out_dtype=2), dict(out_dtype=7), dict(count=-1), dict(dim=0), dict(vocab=0), dict(index=2), dict(scale=NAN), dict(out=None), dict(grad=None), dict(tokens=None),
                dict(grad=P + 1), dict(out=P + 1)):
        assert L.ef21_embedding_grad(*{**good, **bad}.values()) == INVALID, bad
    for bad in (dict(ws=None), dict(ws=P + 1), dict(n=64)):
        assert L.ef21_embedding_grad(*{**good, **bad}.values()) == WORKSPACE, bad


def f(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def i(*shape, dtype=torch.int64):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("error,call", [
    (TypeError, lambda: B.token_logprobs(f(2, 3, dtype=torch.float64), i(2))),
    (TypeError, lambda: B.token_logprobs(f(2, 3), i(2, dtype=torch.int16))),
    (TypeError, lambda: B.token_logprobs(f(3, 2).t(), i(2))),
    (ValueError, lambda: B.token_logprobs(f(2, 3), i(3))),
    (ValueError, lambda: B.token_logprobs(f(3), i())),
    (ValueError, lambda: B.token_logprobs(f(2, 2, 2, 3), i(2, 2, 2))),
    (TypeError, lambda: B.token_logprobs_grad(f(2, 3), i(2), f(2, dtype=torch.float64), f(2))),
    (ValueError, lambda: B.token_logprobs_grad(f(2, 3), i(2), f(3), f(2))),
    (ValueError, lambda: B.token_logprobs_grad(f(2, 3), i(2), f(2), f(2), out=f(3, 3))),
    (ValueError, lambda: B.token_logprobs_grad(f(2, 3), i(2), f(2), f(2), out=f(1, 3).expand(2, 3))),
    (ValueError, lambda: (lambda x: B.token_logprobs_grad(x[:, :-1], i(4, 5), f(4, 5), f(4, 5), out=x[:, 1:]))(f(4, 6, 8))),
    (ValueError, lambda: (lambda x: B.token_logprobs_grad(x[:4], i(4), f(4), f(4), out=x[1:]))(f(5, 8))),
    (ValueError, lambda: B.token_logprobs_grad(f(2, 2, 8), i(2, 2), f(2, 2), f(2, 2), out=f(100).as_strided((2, 2, 8), (8, 8, 1)))),
    (ValueError, lambda: B.preference_loss(f(3, 4))),
    (ValueError, lambda: B.preference_loss(f(0, 4))),
    (ValueError, lambda: B.preference_loss(f(4))),
    (ValueError, lambda: B.preference_loss(f(4, 5), f(4, 6))),
    (TypeError, lambda: B.preference_loss(f(4, 5), f(4, 5, dtype=torch.float16))),
    (TypeError, lambda: B.preference_loss(f(4, 5), mask=f(4, 5))),
    (ValueError, lambda: B.preference_loss(f(4, 5), mask=i(4, 4, dtype=torch.bool))),
    (TypeError, lambda: B.preference_loss(f(5, 4).t())),
    (ValueError, lambda: B.policy_loss(f(4), f(4), f(4))),
    (ValueError, lambda: B.policy_loss(f(4, 5), f(4, 6), f(4))),
    (ValueError, lambda: B.policy_loss(f(4, 5), f(4, 5), f(5))),
    (TypeError, lambda: B.policy_loss(f(4, 5), f(4, 5), f(4, dtype=torch.bfloat16))),
    (ValueError, lambda: B.policy_loss(f(4, 5), f(4, 5), f(4), kl_weight=0.1)),
    (ValueError, lambda: B.policy_loss(f(4, 5), f(4, 5), f(4), reduction="mean")),
    (ValueError, lambda: B.policy_loss(f(4, 5), f(4, 5), f(4), norm=0)),
    (ValueError, lambda: B.balance_loss(f(4), i(4, 1))),
    (ValueError, lambda: B.balance_loss(f(4, 8), i(3, 1))),
    (TypeError, lambda: B.balance_loss(f(4, 8), f(4, 1))),
    (ValueError, lambda: B.balance_loss(f(4, 8), i(4, 1), mask=i(4, 1, dtype=torch.bool))),
    (ValueError, lambda: B.balance_loss(f(4, 8), i(4, 1), mask=i(3, dtype=torch.bool))),
    (TypeError, lambda: B.balance_loss(f(4, 8), i(4, 1), mask=i(8, dtype=torch.bool)[::2])),
    (ValueError, lambda: B.embedding(f(4), i(2))),
    (TypeError, lambda: B.embedding(f(4, 3), f(2))),
    (ValueError, lambda: B.embedding_grad(f(4, 3), i(3), 10)),
    (TypeError, lambda: B.embedding_grad(f(4, 3, dtype=torch.bfloat16), i(4), 10, dtype=torch.float16)),
    (TypeError, lambda: B.embedding_grad(f(4, 3), i(4), 10, out=f(10, 3, dtype=torch.float16))),
    (ValueError, lambda: B.embedding_grad(f(4, 3), i(4), 10, out=f(9, 3))),
    (ValueError, lambda: B.embedding_grad(f(4, 3), i(4), 10, out=f(1, 3).expand(10, 3))),
    (ValueError, lambda: B.embedding_grad(f(4, 3), i(4), 10, accumulate=True)),
    (ValueError, lambda: (lambda x: B.embedding_grad(x[:4], i(4), 4, out=x[2:6]))(f(6, 3))),
    (TypeError, lambda: B.embedding_grad(f(2, 3, 8)[:, :2], i(2, 2), 10)),
], ids=lambda v: "" if not isinstance(v, type) else v.__name__)
def test_the_binding_refuses(error, call):
    with pytest.raises(error):
        call()


@pytest.mark.parametrize("call", [lambda: B.token_logprobs(f(2, 3), i(2)), lambda: B.token_logprobs_grad(f(2, 3), i(2), f(2), f(2)), lambda: B.preference_loss(f(4, 5)),
                                  lambda: B.policy_loss(f(4, 5), f(4, 5), f(4)), lambda: B.balance_loss(f(4, 8), i(4, 1)), lambda: B.embedding(f(4, 3), i(2)),
                                  lambda: B.embedding_grad(f(4, 3), i(4), 10)])
def test_there_is_no_cpu_path(call):
    with pytest.raises(TypeError, match="CUDA"):
        call()


def test_outputs_on_what_is_still_read():
    """An output that lies on the other inputs of its call: rows would be looked up in what has been overwritten."""
    lse, grad = torch.zeros(4), torch.zeros(4)
    for shared in (lse, grad):
        with pytest.raises(ValueError, match="apart"):
            B.token_logprobs_grad(torch.zeros(4, 1), torch.zeros(4, dtype=torch.int64), lse, grad, out=shared.view(4, 1))
    store = torch.zeros(16)
    with pytest.raises(ValueError, match="apart"):
        B.embedding_grad(torch.zeros(4, 3), store[:4].view(torch.int32), 5, out=store[:15].view(5, 3))
