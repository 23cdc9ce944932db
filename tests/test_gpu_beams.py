"""card_beam_select on the GPU against its definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def reference(logits, scores, out_beams, done=None, eos=-1, temperature=1.0, history=None, lengths=None):
    """Candidate by candidate, in lists."""
    groups, beams = scores.shape
    vocab = logits.shape[1]
    # (the library's reciprocal is of the fp32 temperature)
    x = logits.double().view(groups, beams, vocab)
    temperature = float(torch.tensor(temperature, dtype=F32))
    res = {"scores": torch.full((groups, out_beams), -math.inf, dtype=torch.float64), "tokens": torch.full((groups, out_beams), -1),
           "parents": torch.zeros((groups, out_beams), dtype=torch.int64), "done": torch.ones((groups, out_beams), dtype=torch.int64)}
    if history is not None:
        res["history"] = torch.zeros((groups, out_beams, history.shape[2]), dtype=torch.int32)
    gap = math.inf  # between neighbours of different beams, among those that are chosen and the first that is not
    for g in range(groups):
        found = []
        for b in range(beams):
            held = float(scores[g, b])
            if not math.isfinite(held):
                continue
            if done is not None and int(done[g, b]):
                found.append((-held, b, eos))
                continue
            row = x[g, b]
            if bool(row.isnan().any()) or bool((row == math.inf).any()) or bool((row == -math.inf).all()):
                continue
            d = (row - row.max()) / temperature
            p = held + (d - d.exp().sum().log())
            best = torch.sort(p, descending=True, stable=True).indices[:out_beams + 1]
            found += [(-float(p[t]), b, int(t)) for t in best if p[t] > -math.inf]
        found.sort()
        for k, (s, b, t) in enumerate(found[:out_beams]):
            res["scores"][g, k], res["tokens"][g, k], res["parents"][g, k] = -s, t, b
            res["done"][g, k] = int(t == eos and eos >= 0 or done is not None and int(done[g, b]) != 0)
            if history is not None:
                n = min(max(int(lengths[g]), 0), history.shape[2])
                res["history"][g, k, :n] = history[g, b, :n]
                if n < history.shape[2]:
                    res["history"][g, k, n] = t
        for (s, b, _), (s2, b2, _) in zip(found[:out_beams], found[1:]):
            if b != b2 and s != s2:
                gap = min(gap, s2 - s)
    return res, gap


def check(logits, scores, out_beams, exact_ties=False, **more):
    import paper_2508_04462_amd as card

    want, gap = reference(logits, scores, out_beams, **more)
    on = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in more.items()}
    got = card.beam_select(logits.cuda(), scores.cuda(), out_beams, **on)
    torch.cuda.synchronize()
    # (Sums of exponentials in fp32 make ln s uncertain by about 1e-6: which of two candidates is better is sure beyond that.)
    assert gap > 4e-6, "the inputs decide nothing"
    for name in ("tokens", "parents", "done", "history"):
        if name in want:
            assert torch.equal(got[name].cpu().long(), want[name].long()), name
    s, w = got["scores"].cpu().double(), want["scores"]
    assert torch.equal(s == -math.inf, w == -math.inf)
    fine = w > -math.inf
    assert ((s - w).abs()[fine] <= w.abs()[fine] * 2.0 ** -24 + 2e-6).all()
    return got


def _logits(rows, vocab, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, vocab), generator=g) * spread
    at = torch.randint(0, vocab, (rows, 5), generator=g)
    return x.scatter_add_(1, at, torch.rand((rows, 5), generator=g) * 10).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("groups,beams,out_beams,vocab", [(1, 1, 1, 2), (1, 1, 4, 1024), (3, 3, 3, 1000), (2, 4, 4, 128256), (1, 32, 32, 5000), (9, 5, 8, 20003),
                                                          (300, 3, 3, 4097), (2, 12, 20, 37), (1, 1, 32, 70000)], ids=lambda v: str(v))
def test_beams(groups, beams, out_beams, vocab, dtype):
    g = torch.Generator().manual_seed(vocab)
    scores = -torch.rand((groups, beams), generator=g) * 4 - 100
    done = (torch.rand((groups, beams), generator=g) < 0.2).int()
    lengths = torch.randint(0, 41, (groups,), generator=g).int()
    history = torch.randint(0, vocab, (groups, beams, 40), generator=g).int()
    logits = _logits(groups * beams, vocab, dtype, vocab)
    check(logits, scores, out_beams, eos=1, done=done, history=history, lengths=lengths)
    check(logits, scores, out_beams, temperature=0.7)


def test_beams_without_candidates():
    """Fewer candidates than beams: -inf logits, beams that are none, void rows, ended ones."""
    inf = math.inf
    x = torch.full((4, 50), -inf)
    x[0, [3, 7]] = torch.tensor([1.0, 2.0])
    x[1, 5] = 0.5
    x[2] = 1.0
    x[2, 9] = math.nan
    x[3] = 2.0
    x[3, 11] = inf
    scores = torch.tensor([[-1.0, -2.0, -0.1, -0.2]])
    got = check(x, scores, 6, eos=5, history=torch.zeros((1, 4, 3), dtype=torch.int32) + 4, lengths=torch.tensor([2], dtype=torch.int32))
    assert got["tokens"][0].tolist()[3:] == [-1] * 3 and got["done"][0].tolist()[3:] == [1] * 3
    assert (got["history"][0, 3:] == 0).all()
    for bad in (-inf, inf, math.nan):
        check(x, torch.tensor([[bad, -2.0, -0.1, -0.2]]), 3)
    check(x, torch.tensor([[-1.0, -2.0, -0.1, -0.2]]), 4, done=torch.tensor([[0, 0, 1, 7]], dtype=torch.int32), eos=5)
    check(x, torch.tensor([[-inf, -inf, -0.1, -inf]]), 2, done=torch.tensor([[0, 1, 1, 0]], dtype=torch.int32))  # ended, without a token for it
    check(torch.full((2, 9), -inf), torch.zeros(1, 2), 2)


def test_equal_scores():
    """By beam, then by token: beams with the same logits and scores, equal logits in a row, an ended beam beside a candidate of its score."""
    x = torch.zeros(3, 4096 * 5 + 3)
    x[:, [17, 4096 * 3 + 1, 20000]] = 3.0
    got = check(x, torch.full((1, 3), -7.0), 8)
    assert got["parents"][0].tolist() == [0, 0, 0, 1, 1, 1, 2, 2]
    assert got["tokens"][0].tolist() == [17, 4096 * 3 + 1, 20000] * 2 + [17, 4096 * 3 + 1]
    x = torch.full((2, 300), -math.inf)
    x[:, 200] = 5.0  # probability 1
    got = check(x, torch.full((1, 2), -3.0), 2, done=torch.tensor([[0, 1]], dtype=torch.int32), eos=4)
    assert got["parents"][0].tolist() == [0, 1] and got["tokens"][0].tolist() == [200, 4]


def test_equal_logits_of_a_row():
    """Logits in coarse steps, so that the best of a row are equal by twos and more, in rows of several parts whose sums are any numbers."""
    for seed in range(6):
        g = torch.Generator().manual_seed(seed)
        for groups, beams, vocab in ((1, 1, 30011), (20, 6, 20011), (60, 5, 9001)):
            x = (torch.randn((groups * beams, vocab), generator=g) * 3).round() * 0.25
            x[:, ::7] += torch.rand((groups * beams, 1), generator=g).bfloat16().float() * 0.125
            scores = -torch.rand((groups, beams), generator=g) * 20 - 600
            want, _ = reference(x.bfloat16(), scores, beams + 2)
            import paper_2508_04462_amd as card

            got = card.beam_select(x.bfloat16().cuda(), scores.cuda(), beams + 2)
            for a in range(groups):  # (of different beams, candidates may be as near as their scores are certain)
                far = all(p == q or abs(s - t) > 4e-6 for p, q, s, t in zip(want["parents"][a], want["parents"][a][1:], want["scores"][a], want["scores"][a][1:]))
                if far:
                    assert torch.equal(got["parents"][a].cpu().long(), want["parents"][a]), (seed, groups, a)
                    assert torch.equal(got["tokens"][a].cpu().long(), want["tokens"][a]), (seed, groups, a)


def test_scores_of_long_texts_are_compared_in_64_bits():
    """Sums of thousands, between which fp32 has no room for the candidates' differences."""
    x = torch.full((4, 1000), -20.0)
    for b in range(4):
        x[b, b] = 10.0
        x[b, 100 + b] = 10.0 - 2.0 ** -12 * (b + 1)
    scores = torch.full((1, 4), -20000.0)
    check(x, scores, 6)
    want, _ = reference(x, scores, 6)
    assert len(set(want["scores"][0].float().tolist())) < 6 == len(set(want["scores"][0].tolist()))


def test_rows_as_they_lie():
    """Rows further apart than they are long, from any place."""
    g = torch.Generator().manual_seed(1)
    wide = torch.randn((6, 5200), generator=g)
    import paper_2508_04462_amd as card

    for first, vocab in ((0, 5001), (3, 4999), (7, 5111)):
        for dtype in (BF16, F32):
            x = wide.to(dtype).cuda()[:, first:first + vocab]
            scores = -torch.rand((2, 3), generator=g)
            got = card.beam_select(x, scores.cuda(), 3)
            want, _ = reference(x.cpu(), scores, 3)
            assert torch.equal(got["tokens"].cpu().long(), want["tokens"]) and torch.equal(got["parents"].cpu().long(), want["parents"])
