"""Rows of a table by token, and the table's gradient, against plain forms (a sum of k terms in fp32: k steps of 2^-24 of the sum of magnitudes)."""
import pytest
import torch

from model_util import EPS, TYPES, assert_within, generator, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2106_05203_b200 import binding
    return binding


def grad64(grad, tokens, vocab, scale, padding=-1):
    """(sums, sums of magnitudes, terms of every row)"""
    t, g = tokens.reshape(-1).long(), grad.reshape(-1, grad.shape[-1]).double()
    keep = (t >= 0) & (t < vocab) & (t != padding)
    t, g = t[keep], g[keep]
    z = lambda: torch.zeros(vocab, grad.shape[-1], dtype=torch.float64, device="cuda")
    n = torch.bincount(t, minlength=vocab).double()[:, None]
    return z().index_add_(0, t, g) * scale, z().index_add_(0, t, g.abs()) * abs(scale), n


def check_grad(B, grad, tokens, vocab, scale=1.0, padding=-1, dtype=None):
    got = B.embedding_grad(grad, tokens, vocab, scale=scale, padding=padding, dtype=dtype)
    want, size, n = grad64(grad, tokens, vocab, scale, padding)
    assert got.shape == want.shape and got.dtype == (dtype or grad.dtype)
    assert_within(got, want, (n + 2) * EPS * size + rounding(want, got.dtype), "gradient")
    assert not bool(got[n[:, 0] == 0].any())
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count,vocab,dim", [(1, 1, 1), (3, 5, 7), (100, 50, 8), (1000, 3000, 257), (33, 100, 4096), (5000, 777, 64), (2, 9, 12000)])
def test_rows(B, dtype, count, vocab, dim):
    g = generator(count)
    weight = torch.randn(vocab, dim, device="cuda", generator=g).to(dtype)
    tokens = torch.randint(0, vocab, (count,), device="cuda", generator=g)
    if count > 2:
        tokens[1] = -1; tokens[2] = vocab
    inside = ((tokens >= 0) & (tokens < vocab))[:, None]
    want = torch.where(inside, (weight[tokens.clamp(0, vocab - 1)].float() * 1.7).to(dtype), torch.zeros((), dtype=dtype, device="cuda"))
    assert torch.equal(B.embedding(weight, tokens, scale=1.7), want)
    assert torch.equal(B.embedding(weight, tokens.int(), scale=1.7), want)
    wide = torch.nn.functional.pad(weight, (1, 2))[:, 1:-2]
    assert torch.equal(B.embedding(wide, tokens.view(count, 1), scale=1.7), want[:, None])
    weight[0] = float("nan"); weight[-1] = float("inf")
    if count > 2:
        assert not bool(B.embedding(weight, tokens[1:3], scale=float(2 ** 100)).any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count,vocab,dim", [(1, 1, 1), (3, 5, 7), (32, 1, 8), (33, 1, 8), (100, 50, 24), (1000, 3000, 257), (64, 100, 2050), (8192, 40, 16), (8193, 40, 16), (5000, 70000, 8), (20000, 511, 33),
                                             (40000, 512, 8), (70001, 300000, 8), (100000, 5, 40), (9000, 262144, 16)])
def test_gradient(B, dtype, count, vocab, dim):
    g = generator(count + vocab)
    grad = torch.randn(count, dim, device="cuda", generator=g).to(dtype)
    uniform = torch.randint(0, vocab, (count,), device="cuda", generator=g)
    skewed = (vocab ** torch.rand(count, device="cuda", generator=g, dtype=torch.float64)).long().clamp_(max=vocab) - 1
    for tokens in (uniform, skewed):
        check_grad(B, grad, tokens, vocab, scale=1.5)
        check_grad(B, grad, tokens.int(), vocab, scale=-0.25, dtype=torch.float32)
    tokens = skewed.clone()
    tokens[::5] = -1; tokens[1::7] = vocab; tokens[2::11] = 1 << 40
    check_grad(B, grad, tokens, vocab, padding=0)


@pytest.mark.parametrize("count", [1000, 33000])
@pytest.mark.parametrize("kind", ["one token", "two tokens", "runs at chunk borders", "outside", "descending"])
def test_special_orders(B, count, kind):
    grad = torch.randn(count, 40, device="cuda", generator=generator(count))
    at = torch.arange(count, device="cuda")
    tokens = {"one token": torch.full_like(at, 7), "two tokens": at % 2 * 9, "runs at chunk borders": at // 32, "outside": torch.full_like(at, -3), "descending": count - 1 - at}[kind]
    check_grad(B, grad, tokens, max(10, count), scale=2.0)
    if kind == "runs at chunk borders":
        for shift in (1, 16, 31):                                       # runs of 33 and 65 positions about the chunks' borders
            check_grad(B, grad, (at + shift) // 33, count)
            check_grad(B, grad, (at + shift) // 65, count)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 65])
def test_adding_to_a_gradient(B, dtype, dim):
    g = generator(dim)
    grad = torch.randn(3, 700, dim, device="cuda", generator=g).to(dtype)
    tokens = torch.randint(0, 90, (3, 700), device="cuda", generator=g)
    tokens[:, ::3] = 4
    for out_dtype in {dtype, torch.float32}:
        table = torch.randn(120, dim + 3, device="cuda", generator=g).to(out_dtype)
        before = table.clone()
        got = B.embedding_grad(grad, tokens, 120, scale=0.5, out=table[:, :dim], accumulate=True)
        want, size, n = grad64(grad, tokens, 120, 0.5)
        old = before[:, :dim].double()
        assert got.data_ptr() == table.data_ptr()
        assert_within(got, want + old, (n + 2) * EPS * size + 2 * EPS * old.abs() + rounding(want + old, out_dtype))
        assert torch.equal(table[:, dim:], before[:, dim:])                             # what is between the rows
        assert torch.equal(table[90:], before[90:])                                    # rows that no token names
        B.embedding_grad(grad, tokens, 120, scale=0.5, out=table[:, :dim])
        assert torch.equal(table[:, :dim], B.embedding_grad(grad, tokens, 120, scale=0.5, dtype=out_dtype)) and torch.equal(table[:, dim:], before[:, dim:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count,vocab,dim", [(4, 98621, 61), (3000, 70000, 64), (900, 20000, 333), (70000, 300000, 16), (40000, 12000, 1001), (1, 5, 2000003)])
def test_large_tables(B, dtype, count, vocab, dim):
    """Tables that are cleared first, and rows formed four to a team; with and without gaps between the rows, which stay as they are."""
    g = generator(count)
    grad = torch.randn(count, dim, device="cuda", generator=g).to(dtype)
    tokens = (vocab ** torch.rand(count, device="cuda", generator=g, dtype=torch.float64)).long().clamp_(max=vocab) - 1
    if count > 1:
        tokens[::9] = vocab
        tokens[1::50] = vocab - 1
    want = check_grad(B, grad, tokens, vocab, scale=0.5, dtype=torch.float32)
    table = torch.full((vocab, dim + 3), 7.0, device="cuda")
    B.embedding_grad(grad, tokens, vocab, scale=0.5, out=table[:, 1:dim + 1])
    assert torch.equal(table[:, 1:dim + 1], want) and bool((table[:, 0] == 7).all()) and bool((table[:, dim + 1:] == 7).all())
    check_grad(B, grad, tokens, vocab)


def test_views_and_empty(B):
    grad = torch.randn(50, 24, device="cuda", dtype=torch.bfloat16)
    tokens = torch.randint(0, 9, (50,), device="cuda")
    want = B.embedding_grad(grad, tokens, 9)
    for by, at in ((8, 0), (8, 8), (3, 1)):
        view = torch.nn.functional.pad(grad, (at, by - at))[:, at:at + 24]
        assert torch.equal(B.embedding_grad(view, tokens, 9), want)
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert B.embedding(grad, none).shape == (0, 24)
    assert not bool(B.embedding_grad(grad[:0], none, 9).any())
    table = torch.ones(9, 24, device="cuda")
    assert bool((B.embedding_grad(grad[:0], none, 9, out=table, accumulate=True) == 1).all())


def test_gradient_against_differences(B):
    """The lookup is linear: for any direction, <grad, embedding(D)> = <embedding_grad(grad), D>, up to 2^-24 of the sum of magnitudes per term."""
    g = generator(1)
    grad = torch.randn(300, 20, device="cuda", generator=g)
    tokens = torch.randint(0, 11, (300,), device="cuda", generator=g)
    D = torch.randn(11, 20, device="cuda", generator=g)
    a = (grad.double() * B.embedding(D, tokens, scale=3.0).double()).sum()
    b = (B.embedding_grad(grad, tokens, 11, scale=3.0).double() * D.double()).sum()
    size = (grad.abs().double() * D[tokens].abs().double()).sum() * 3
    assert abs(float(a - b)) <= 60 * EPS * float(size)


def test_offsets_beyond_32_bits(B):
    vocab, dim = 600000, 4096                                           # 2.4e9 elements, 4.9 GB
    weight = torch.zeros(vocab, dim, device="cuda", dtype=torch.bfloat16)
    weight[-1] = torch.arange(dim, device="cuda")
    tokens = torch.tensor([vocab - 1, 3, vocab - 1], device="cuda")
    out = B.embedding(weight, tokens)
    assert torch.equal(out[0], weight[-1]) and not bool(out[1].any()) and torch.equal(out[2], weight[-1])
    B.embedding_grad(out, tokens, vocab, out=weight)
    assert torch.equal(weight[-1], out[0] * 2) and not bool(weight[3].any()) and not bool(weight[-2].any())
    many = torch.zeros(600000, 4096, device="cuda", dtype=torch.bfloat16)
    many[-1] = 1.0
    tokens = torch.arange(600000, device="cuda") // 64
    got = B.embedding_grad(many, tokens, 600000 // 64, out=weight[:600000 // 64])
    assert bool((got[-1] == 1).all()) and not bool(got[:-1].any())


def test_repeated_captured_and_on_another_stream(B):
    g = generator(2)
    for count in (2000, 30000):
        grad = torch.randn(count, 96, device="cuda", generator=g)
        tokens = (5000 ** torch.rand(count, device="cuda", generator=g)).long()
        call = lambda **k: B.embedding_grad(grad, tokens, 5001, **k)
        want = call()
        assert torch.equal(call(), want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        with torch.cuda.graph(other):
            more = call()
        tokens.copy_(tokens.flip(0)); grad.mul_(2.0)
        want = call()
        for _ in range(2):
            graph.replay(); other.replay()
        assert torch.equal(got, want) and torch.equal(more, want)
