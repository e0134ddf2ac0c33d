"""Sessions and models used for fewer positions, or more sentences, than they were made for."""
import ctypes as C

import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import layers as L

BF16 = torch.bfloat16


@pytest.mark.parametrize("vocab, width", [(10, 8), (300, 264), (32000, 1024), (85000, 500), ((1 << 20) + 1, 1), (50, 2100)])
def test_embedding_workspace_is_for_up_to_so_many_positions(vocab, width):
    """A session has one workspace for every number of positions up to its own: more positions never ask for less."""
    lib, most = L.load_library(), 0
    for tokens in (0, 1, 7, 16, 17, 500, 3385, 4000, 5225, 8191, 8192, 8193, 9000, 10000, 16000, 16384, 22336, 27232, 32768, 131072):
        size = C.c_size_t(0)
        assert lib.gd_embedding_workspace_bytes(tokens, vocab, width, C.byref(size)) == B.GD_OK
        assert size.value >= most, tokens
        most = size.value


@pytest.mark.gpu
@pytest.mark.parametrize("vocab, width", [(32000, 1024), (300, 264)])
def test_embedding_gradient_of_fewer_positions_than_the_session_is_for(cuda_device, vocab, width):
    """On either side of the switch between the two sorts: the bits of a session of just that size."""
    gen = torch.Generator(device=cuda_device).manual_seed(width)
    dy = torch.randn(16384, width, generator=gen, device=cuda_device).to(BF16)
    ids = (torch.rand(16384, generator=gen, device=cuda_device) ** 3 * vocab).long()
    ids[::11] = -100
    for most in (16384, 9000, 8193):
        s = L.EmbeddingSession(vocab, width, most, device=cuda_device)
        for n in (most, 8192, 4000, 5225, 17, 1):
            got, want = (torch.full((vocab, width), float("nan"), device=cuda_device) for _ in range(2))
            s.backward(dy[:n], ids[:n], got)
            L.EmbeddingSession(vocab, width, n, device=cuda_device).backward(dy[:n], ids[:n], want)
            assert torch.equal(got, want), (most, n)


@pytest.mark.gpu
@pytest.mark.parametrize("gradient", [False, True])
def test_lookup_of_any_number_of_ids(cuda_device, gradient):
    """max_tokens is the workspace's, which a lookup does not take; the gradient of more positions is refused."""
    s = L.EmbeddingSession(10, 8, 4, device=cuda_device, gradient=gradient)
    table, ids = torch.randn(10, 8, device=cuda_device), torch.arange(5000, device=cuda_device) % 10
    assert torch.equal(s.forward(table, ids), table[ids])
    with pytest.raises(ValueError):
        s.backward(table[ids], ids, torch.empty_like(table))


@pytest.mark.gpu
def test_answers_to_more_sentences_than_a_batch_has(cuda_device):
    """One more token of 20 sentences, by a model made for batches of nine sentences in 300 positions: each as if it were alone, but for sums in
    another order."""
    from paper_1704_05021_b200 import train_lm as M
    model = M.Lm(vocab=64, width=64, hidden=64, blocks=2, rows=300, sentences=9, device=cuda_device)
    tokens = torch.randint(64, (20,), generator=torch.Generator(device=cuda_device).manual_seed(1), device=cuda_device)
    state = model.new_state(20)
    got = [model.answer(tokens, state).clone() for _ in range(2)]
    assert all(bool(torch.isfinite(t).all()) for t in got)
    few = model.new_state(9)
    for n in range(2):
        want = model.answer(tokens[:9], few)
        assert float((got[n][:9].float() - want.float()).abs().max()) <= 10 * 2.0 ** -8 * float(want.float().abs().max())
