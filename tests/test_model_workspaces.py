"""Workspaces of a language model's calls.  A size query that answers 256 (EF21_NO_WORKSPACE) says that the call keeps nothing there, and then any aligned address is
handed over, an output's among them; whatever a call writes or reads there needs memory of its own, and more than 256 bytes say so."""
import pytest
import torch

from paper_2106_05203_b200 import binding as B

UNUSED = 256


@pytest.mark.parametrize("pairs,length", [(1, 1), (4, 512), (64, 256), (1, 8191), (2, 4096), (8, 300)])
def test_preference_by_one_cluster_keeps_nothing(pairs, length):
    assert B._lib.ef21_preference_loss_workspace_bytes(pairs, length) == UNUSED


@pytest.mark.parametrize("pairs,length", [(65, 256), (256, 100), (9, 300), (16, 2048), (32, 8191), (4, 8192), (8, 2048), (5, 5000), (33, 400)])
def test_preference_by_several_clusters_keeps_the_pairs_losses(pairs, length):
    """Eight bytes a pair, or per block of eight pairs: 16 to 264 of them, written by one kernel and read by the next."""
    assert B._lib.ef21_preference_loss_workspace_bytes(pairs, length) > UNUSED


@pytest.mark.parametrize("vocab,dim", [(1, 1), (16, 8), (32, 1), (32, 4096), (33, 8)])
def test_a_table_s_gradient_reads_its_runs_without_a_token_too(vocab, dim):
    assert B._lib.ef21_embedding_grad_workspace_bytes(0, vocab, dim) > UNUSED


@pytest.mark.parametrize("count,vocab,dim", [(1, 1, 1), (1, 32, 8), (31, 1, 3)])
def test_a_small_table_s_gradient(count, vocab, dim):
    assert B._lib.ef21_embedding_grad_workspace_bytes(count, vocab, dim) > UNUSED


def test_the_others():
    assert B._lib.ef21_policy_loss_workspace_bytes(0, 0) > UNUSED and B._lib.ef21_balance_loss_workspace_bytes(0, 1) > UNUSED
    assert B._lib.ef21_token_logprobs_workspace_bytes(0, 1, 1, 32768) == UNUSED                     # (one block or cluster a row)
    assert B._lib.ef21_token_logprobs_workspace_bytes(0, 1, 296, 2049) > UNUSED                     # (units of a warp, joined by a second kernel)


def allocations(call):
    call()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    result = call()
    return torch.cuda.memory_stats()["allocation.all.allocated"] - before, result


@pytest.mark.gpu
@pytest.mark.parametrize("pairs,length,own", [(4, 512, False), (16, 2048, True), (256, 100, True), (4, 8192, True)])
def test_the_native_call_hands_over_memory_of_its_own(pairs, length, own):
    """Loss, rewards and gradient, and a workspace where the call uses one."""
    x = torch.randn(2 * pairs, length, device="cuda")
    assert type(B._model_calls) is not B._GeneralCalls
    count, got = allocations(lambda: B._model_calls.preference_loss(x, None, None, 0.1, 0.0, None))
    assert count == 3 + own
    general = B.preference_loss(x, stream=torch.cuda.current_stream())
    assert all(torch.equal(a, b) for a, b in zip(got, general))


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,dim", [(1, 1), (16, 8), (32, 3)])
def test_no_token_at_all(vocab, dim):
    grad, tokens = torch.zeros(0, dim, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda")
    count, got = allocations(lambda: B._model_calls.embedding_grad(grad, tokens, vocab, 1.0, -1, None))
    assert count == 2 and got.shape == (vocab, dim) and not bool(got.any())
