"""The order of card_beam_select's candidates where scores are equal."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _row(vocab, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(vocab, generator=g) * 2).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab,beams,out_beams", [(3001, 8, 8), (3002, 8, 5), (20011, 8, 8), (128257, 4, 12), (5003, 32, 20)])
def test_beams_with_the_same_logits(vocab, beams, out_beams, dtype):
    """Equal scores go by beam, then by token, also where rows begin at different places of the memory's units of 16 bytes."""
    import paper_2508_04462_amd as card

    for seed in range(4):
        row = _row(vocab, dtype, seed)
        best = row.double().sort(descending=True, stable=True).indices[:out_beams]
        want = sorted((-float(row[t]), b, int(t)) for t in best for b in range(beams))[:out_beams]
        got = card.beam_select(row.repeat(beams, 1).cuda(), torch.full((1, beams), -3.5).cuda(), out_beams)
        assert got["parents"][0].tolist() == [b for _, b, _ in want], seed
        assert got["tokens"][0].tolist() == [t for _, _, t in want], seed


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 5, 63, 1000, 30011, 128256])
def test_the_same_logits_at_other_addresses(vocab, dtype):
    """The same bits of the scores, and so the same beams, wherever the logits lie."""
    import paper_2508_04462_amd as card

    x = torch.stack([_row(vocab, dtype, seed) for seed in range(6)])
    scores = -torch.rand((2, 3), generator=torch.Generator().manual_seed(1)).cuda()
    want = card.beam_select(x.cuda(), scores, 4)
    for first in range(8):
        for stride in (vocab + 8, (vocab + 15) // 16 * 16):
            if stride < first + vocab:
                continue
            wide = torch.full((6, stride), 100.0, dtype=dtype)
            wide[:, first:first + vocab] = x
            got = card.beam_select(wide.cuda()[:, first:first + vocab], scores, 4)
            for name in want:
                assert torch.equal(got[name], want[name]), (first, stride, name)


def test_zero_and_minus_zero_are_equal_scores():
    import paper_2508_04462_amd as card

    x = torch.full((2, 300), -float("inf"))
    x[:, 200] = 5.0  # probability 1
    for scores, done in (([-0.0, 0.0], [1, 0]), ([0.0, -0.0], [0, 1])):
        got = card.beam_select(x.cuda(), torch.tensor([scores]).cuda(), 2, done=torch.tensor([done], dtype=torch.int32).cuda(), eos=4)
        assert got["parents"][0].tolist() == [0, 1], scores
        # (more candidates: they are taken one by one)
        got = card.beam_select(x.repeat(16, 1).cuda(), torch.tensor([scores * 16]).cuda(), 32, done=torch.tensor([done * 16], dtype=torch.int32).cuda(), eos=4)
        assert got["parents"][0].tolist() == list(range(32)), scores
