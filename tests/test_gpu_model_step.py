"""The calls together, as a language model's workers use them: embedding -> (torch: one layer and a router) -> logits -> log-probabilities -> loss, and
back; the workers' gradients go into EF21 rounds."""
import numpy as np
import pytest
import torch

from model_util import generator

pytestmark = pytest.mark.gpu
V, D, E, K, PAIRS, T, N = 300, 32, 6, 2, 3, 21, 4
BETA, WEIGHT = 0.5, 0.1


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


def weights(seed):
    g = generator(seed)
    return [0.3 * torch.randn(s, device="cuda", generator=g) for s in ((V, D), (D, V), (D, E))]


def batch(seed):
    g = generator(seed)
    tokens = torch.randint(0, V, (2 * PAIRS, T), device="cuda", generator=g)
    mask = torch.rand(2 * PAIRS, T - 1, device="cuda", generator=g) < 0.7
    mask[1] = False
    ref = -6 + torch.randn(2 * PAIRS, T - 1, device="cuda", generator=g)
    return tokens, mask, ref


def local_gradient(B, table, unembed, router, tokens, mask, ref, kind):
    """Loss and gradient (one flat vector) of one worker by the framework's calls."""
    h = B.embedding(table, tokens[:, :-1], scale=D ** 0.5)
    flat = h.view(-1, D)
    logits = h @ unembed
    logps, lse = B.token_logprobs(logits, tokens[:, 1:])
    if kind == "preference":
        loss, _, dlogps = B.preference_loss(logps, ref, mask=mask, beta=BETA)
    else:
        terms, dlogps = B.policy_loss(logps, ref, ref[:, 0].contiguous(), mask=mask, ref_logps=ref, kl_weight=0.1, reduction="sequence", clip_high=4.0, clip_low=0.9)
        loss = terms[0]
    scores = flat @ router
    choices = torch.topk(scores, K).indices
    balance = B.balance_loss(scores, choices, mask=mask.flatten(), weight=WEIGHT)
    dlogits = B.token_logprobs_grad(logits, tokens[:, 1:], lse, dlogps, out=logits)
    dh = dlogits.view(-1, V) @ unembed.t() + balance.grad @ router.t()
    dtable = B.embedding_grad(dh, tokens[:, :-1].reshape(-1), V, scale=D ** 0.5)
    return loss + balance.loss, torch.cat([dtable.flatten(), (flat.t() @ dlogits.view(-1, V)).flatten(), (flat.t() @ balance.grad).flatten()])


def local_gradient64(table, unembed, router, tokens, mask, ref, kind):
    """The same by autograd, in 64 bits."""
    W = [t.double().requires_grad_() for t in (table, unembed, router)]
    h = W[0][tokens[:, :-1]] * D ** 0.5
    logp = torch.log_softmax(h @ W[1], -1).gather(-1, tokens[:, 1:, None])[..., 0]
    m, r = mask.double(), ref.double()
    if kind == "preference":
        s = ((logp - r) * m).sum(1)
        loss = -torch.nn.functional.logsigmoid(BETA * (s[:PAIRS] - s[PAIRS:])).mean()
    else:
        n = m.sum(1, keepdim=True)
        w = m / n.clamp(min=1) / (n > 0).sum()
        ratio, A = torch.exp(logp - r), r[:, :1]
        pg = torch.minimum(ratio * A, ratio.clamp(0.1, 5.0) * A)
        loss = (w * (-pg + 0.1 * (torch.exp(r - logp) - (r - logp) - 1))).sum()
    scores = h.view(-1, D) @ W[2]
    choices = torch.topk(scores, K).indices
    keep = mask.flatten()
    f = torch.bincount(choices[keep].flatten(), minlength=E).double() / (K * keep.sum())
    loss = loss + WEIGHT * E * (f * scores.softmax(-1)[keep].mean(0)).sum()
    loss.backward()
    return loss.detach(), torch.cat([w.grad.flatten() for w in W])


@pytest.mark.parametrize("kind", ["preference", "policy"])
def test_gradients_of_the_whole(B, kind):
    """Norm-wise 1e-5, the bar of the framework's local gradients: fp32 products of 32 and 300 terms (300 * 2^-24 = 1.8e-5 at most, a tenth of it as a rule of
    signs that do not agree), the calls an order below."""
    for seed in range(3):
        args = (*weights(seed), *batch(seed + 10), kind)
        loss, grad = local_gradient(B, *args)
        want_loss, want = local_gradient64(*args)
        assert abs(float(loss) - float(want_loss)) <= 1e-5 * max(1.0, abs(float(want_loss)))
        assert float((grad.double() - want).norm()) <= 1e-5 * float(want.norm())


@pytest.mark.parametrize("kind", ["preference", "policy"])
def test_the_step_in_a_graph(B, kind):
    """A whole local step is captured once and replayed on other weights and tokens: bit for bit the eager one."""
    w, b = weights(1), batch(2)
    local_gradient(B, *w, *b, kind)                                     # torch's own products set themselves up outside of the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grad = local_gradient(B, *w, *b, kind)
    for seed in (3, 4):
        for old, new in zip((*w, *b), (*weights(seed), *batch(seed))):
            old.copy_(new)
        graph.replay()
        want_loss, want = local_gradient(B, *w, *b, kind)
        assert torch.equal(loss, want_loss) and torch.equal(grad, want)


def test_rounds_on_the_workers_gradients(B, oracle32):
    """EF21 rounds (Top-k of every worker's gradient) on these gradients: given them, the state is the oracle's, bit for bit."""
    import oracle
    w = weights(5)
    d, k, gamma = sum(t.numel() for t in w), 200, 0.05
    data = [batch(20 + i) for i in range(N)]
    h = B.EF21(N, d, k, gamma)
    st = oracle.State(oracle32, N, d, k, gamma)
    x0 = torch.cat([t.flatten() for t in w])
    h.set_x(x0)
    h.init_grads(None, B.INIT_ZERO)
    st.init(1)
    st.x[:] = x0.cpu().numpy()
    for _ in range(3):
        x = h.get_state()[0]
        parts = [p.view(s.shape) for p, s in zip(x.split([t.numel() for t in w]), w)]
        grads = torch.stack([local_gradient(B, *parts, *b, "preference")[1] for b in data])
        h.step_grads(grads, 1)
        st.step_grads(grads.cpu().numpy(), 1)
        x, g, gi, li, lv = h.get_state_host()
        assert np.array_equal(li, st.idx) and np.array_equal(lv, st.val) and np.array_equal(gi, st.gi) and np.array_equal(g, st.g) and np.array_equal(x, st.x)
    assert h.poll() == 0
