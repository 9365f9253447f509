"""The calls of a language model's worker by their native form and by the general one: the same results and the same refusals."""
import threading

import pytest
import torch

from model_util import generator

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    assert type(binding._model_calls) is not binding._GeneralCalls
    return binding


def calls(B, dtype=torch.float32, seed=0):
    """name -> (call, its arguments)"""
    g = generator(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g).to(dtype)
    i = lambda high, *s: torch.randint(0, high, s, device="cuda", generator=g)
    mask = i(2, 6, 40).bool()
    lse = torch.logsumexp(r(4, 9, 50).float(), -1)
    return {
        "token_logprobs": (B.token_logprobs, (r(4, 10, 50)[:, :-1], i(50, 4, 10)[:, 1:], 0.5, 3)),
        "token_logprobs_grad": (B.token_logprobs_grad, (r(4, 9, 50), i(50, 4, 9), lse, torch.randn(4, 9, device="cuda", generator=g), 1, -100)),
        "preference_loss": (B.preference_loss, (r(6, 40), r(6, 40), mask, 0.2, 0.1, 5)),
        "preference_loss, many": (B.preference_loss, (r(200, 400),)),
        "policy_loss": (B.policy_loss, (r(6, 40), r(6, 40), r(6), mask, r(6, 40), 0.1, 0.3, 0.05, "sequence", 4.0)),
        "policy_loss, many": (B.policy_loss, (r(60, 4000), r(60, 4000), r(60, 4000))),
        "balance_loss": (B.balance_loss, (r(30, 12), i(12, 30, 2), i(2, 30).bool(), 0.5)),
        "balance_loss, many": (B.balance_loss, (r(9000, 12), i(12, 9000, 2).int())),
        "embedding": (B.embedding, (r(20, 24), i(20, 3, 5), 2)),
        "embedding_grad": (B.embedding_grad, (r(3, 5, 24), i(20, 3, 5), 20, 2.0, 4, torch.float32)),
        "embedding_grad, many": (B.embedding_grad, (r(9001, 8), i(300, 9001), 300)),
    }


def flat(result):
    return list(result) if isinstance(result, tuple) else [result]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_same_results(B, dtype, monkeypatch):
    for name, (call, args) in calls(B, dtype).items():
        native = call(*args)
        general = call(*args, stream=torch.cuda.current_stream())
        with monkeypatch.context() as m:
            m.setattr(B, "_model_calls", B._GeneralCalls())
            plain = call(*args)
        assert type(native) is type(general) is type(plain), name
        for a, b, c in zip(flat(native), flat(general), flat(plain)):
            assert a.dtype == b.dtype == c.dtype and a.shape == b.shape == c.shape and a.stride() == b.stride(), name
            assert torch.equal(a.float().nan_to_num(), b.float().nan_to_num()) and torch.equal(a.float().nan_to_num(), c.float().nan_to_num()), name


def test_the_current_stream_is_taken(B):
    for name, (call, args) in calls(B).items():
        want = flat(call(*args))
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            got = flat(call(*args))
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
        with pytest.raises(TypeError):
            call(*args, stream=0)


def test_parameters_and_gradients(B):
    """A subclass takes the general call; results are constants of autograd either way."""
    for name, (call, args) in calls(B).items():
        want = flat(call(args[0].detach().clone(), *args[1:]))         # (in the clones' layout: a row's sums are in an order that goes by its alignment)
        leaf = args[0].detach().clone().requires_grad_()
        for first in (torch.nn.Parameter(args[0].detach().clone()), leaf):
            got = flat(call(first, *args[1:]))
            assert all(torch.equal(a, b) and not a.requires_grad for a, b in zip(got, want)), name


def test_refusals(B):
    for name, (call, args) in calls(B).items():
        for k, t in enumerate(args):
            if not isinstance(t, torch.Tensor):
                continue
            bad = [t.cpu(), t.to(torch.complex64), t.unsqueeze(0).unsqueeze(0)]
            if not (name.startswith("embedding") and k == 1):          # (tokens may have any shape)
                bad.append(t[:0] if t.dim() > 1 and "grad" not in name and name != "embedding" else t.unsqueeze(0).unsqueeze(0))
            if name.startswith("embedding"):
                bad = bad[:2]
            for b in bad:
                if b.numel() == 0 and k == 0:                          # (an empty first argument may be a call of its own, with others that fit)
                    continue
                with pytest.raises((TypeError, ValueError, B.Ef21Error)):
                    call(*args[:k], b, *args[k + 1:])
    x, t = torch.zeros(2, 8, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(B.Ef21Error):
            B.token_logprobs(x, t, scale=scale)
    with pytest.raises(B.Ef21Error):
        B.preference_loss(x, smoothing=2.0)
    with pytest.raises(B.Ef21Error):
        B.policy_loss(x, x, x, clip_low=1.0)
    with pytest.raises(ValueError):
        B.policy_loss(x, x, x, reduction="mean")
    with pytest.raises(ValueError):
        B.policy_loss(x, x, x, norm=-1.0)
    with pytest.raises(B.Ef21Error):
        B.balance_loss(torch.zeros(4, 1025, device="cuda"), torch.zeros(4, 1, dtype=torch.int64, device="cuda"))
    with pytest.raises(B.Ef21Error):
        B.balance_loss(x, torch.zeros(2, 9, dtype=torch.int64, device="cuda"))
    with pytest.raises(B.Ef21Error):
        B.embedding(x, t, scale=float("nan"))
    with pytest.raises(B.Ef21Error):
        B.embedding_grad(x, t, 0)


def test_calls_from_several_threads(B):
    """Two at once, each on a stream of its own: no workspace is shared."""
    want = {name: flat(call(*args)) for name, (call, args) in calls(B).items()}
    torch.cuda.synchronize()
    wrong = []

    def work(seed):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            mine = calls(B)
            for _ in range(20):
                for name, (call, args) in mine.items():
                    got = flat(call(*args))
                    stream.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[name])):
                        wrong.append((seed, name))
    threads = [threading.Thread(target=work, args=(k,)) for k in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == []
