"""Draws and verifications of more rows than one launch takes: the same bits as by calls of fewer rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


def logits(rows, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(rows, 8, generator=g, device=DEV).to(torch.bfloat16), torch.rand(rows, generator=g, device=DEV)


def test_a_draw_of_more_rows_than_one_launch_takes():
    import paper_2604_02945_amd as msao
    rows, some = (1 << 22) + 5, 1 << 20
    x, u = logits(rows, 1)
    top_k = torch.arange(rows, device=DEV, dtype=torch.int32) % 7
    got = msao.msao_sample(x, u, top_k=top_k, vocab=7)
    for at in range(0, rows, some):
        want = msao.msao_sample(x[at:at + some], u[at:at + some], top_k=top_k[at:at + some], vocab=7)
        for k in ("token", "logprob", "kept"):
            assert torch.equal(got[k][at:at + some], want[k])
    assert int(got["token"].min()) >= 0


@pytest.mark.parametrize("seqs,new", [((1 << 20) + 1, 2), ((1 << 21) + 3, 2)])
@pytest.mark.parametrize("drawn", [False, True], ids=["certain", "drawn"])
def test_a_verification_of_more_rows_than_one_launch_takes(seqs, new, drawn):
    """Row 2 s and 2 s + 1 of sequence s; of the last launch some."""
    import paper_2604_02945_amd as msao
    rows, some = seqs * new, 1 << 18
    x, u = logits(rows, 2)
    y, ua = logits(rows, 3)
    y = y if drawn else None
    tokens = torch.randint(7, (rows,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(4)).to(torch.int32)
    start = torch.arange(0, rows + 1, new, device=DEV, dtype=torch.int32)
    length = torch.full((seqs,), 100, device=DEV, dtype=torch.int32)
    got = msao.msao_verify(start, new, tokens, x, ua, u, vocab=7, draft_logits=y, length=length)
    for at in range(0, seqs, some):
        n = min(some, seqs - at)
        r = slice(at * new, (at + n) * new)
        want = msao.msao_verify(start[:n + 1], new, tokens[r], x[r], ua[r], u[r], vocab=7, draft_logits=None if y is None else y[r],
                                length=length[:n])
        for k in ("next", "logprob"):
            assert torch.equal(torch.nan_to_num(got[k][r].float(), nan=9e9), torch.nan_to_num(want[k].float(), nan=9e9))
        for k in ("accepted", "length"):
            assert torch.equal(got[k][at:at + n], want[k])
    assert 0 < int(got["accepted"].sum()) < seqs
