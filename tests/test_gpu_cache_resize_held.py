"""Resizes whose `columns` count fewer columns than are held: the held ones are named all the same, so that none of
them is replaced by a page of the pool. Oracle and comparison are those of the other resizes, with the
columns that are there."""
import pytest
import torch

from test_gpu_cache_resize import DEV, I32, Both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs", [1, 5, 64, 1024, 1500], ids=lambda n: f"{n} sequences")
@pytest.mark.parametrize("said", [0, 1, -7, 2])
def test_held_columns_are_never_taken(seqs, said):
    """Every sequence begins with a held prefix of three columns alone; one launch and two."""
    held = [3 if i % 3 else 0 for i in range(seqs)]
    b = Both(31, [0] * seqs, 16, 9, 6 * seqs, held=held)
    b.columns.copy_(torch.tensor([min(h, said) for h in held], dtype=I32))
    shared = b.cache.pages[:, :3].clone()
    taken = set(b.host.free)
    b.step([(17 * i) % 100 for i in range(seqs)])
    mine = torch.tensor(held, device=DEV) > 0
    assert torch.equal(b.cache.pages[mine][:, :3], shared[mine]) and not taken & set(shared[mine].flatten().tolist())
    b.columns.copy_(torch.minimum(b.columns, torch.where((b.columns == 3) & mine, said, 99)).to(I32))
    b.step([0] * seqs)
    b.columns.copy_(torch.where(mine, min(said, 3), b.columns).to(I32))
    b.step([48] * seqs)


def test_who_gets_no_page_keeps_the_held_ones():
    b = Both(32, [0, 0, 0, 0], 16, 9, 2, held=[4, 0, 4, 2])
    b.columns.copy_(torch.tensor([0, 0, 3, 1], dtype=I32))
    assert b.step([200, 16, 64, 40]) == [0, 0, 1, 0]
