"""What card_beam_select and SequencePool.reorder refuse, and the bookkeeping of reorder; no GPU: nothing gets as far as a launch."""
import math
import types

import pytest
import torch

import paper_2508_04462_amd as card
from test_serving_host import PlayedPool

A = 0x10000  # an address: nothing is read or written


def _beams(**more):
    d = dict(groups=2, beams=3, out_beams=3, eos_token=-1, scores_dev=A, done_dev=A, history_dev=A, lengths_dev=A, history_len=10, out_scores_dev=A,
             out_tokens_dev=A, out_parents_dev=A, out_done_dev=A, out_history_dev=A)
    return card.CardBeams(*dict(d, **more).values())


def _select(beams=None, logits=A, type=card.CARD_F32, vocab=1000, stride=1000, temperature=1.0, ws=A):
    return card.lib.card_beam_select(logits, type, vocab, stride, beams, temperature, ws, None)


def test_beam_select_refusals():
    assert _select(_beams(groups=0)) == card.CARD_OK
    assert _select(None) == _select(_beams(), type=2) == _select(_beams(), vocab=0) == _select(_beams(), stride=999) == card.CARD_EINVAL
    for t in (0.0, -1.0, math.nan, math.inf, 1e-31):
        assert _select(_beams(), temperature=t) == card.CARD_EINVAL
    assert _select(_beams(groups=-1)) == _select(_beams(history_len=-1)) == card.CARD_EINVAL
    for bad in (dict(beams=0), dict(beams=33), dict(out_beams=0), dict(out_beams=33), dict(eos_token=-2), dict(eos_token=1000), dict(groups=(1 << 24) // 3 + 1)):
        assert _select(_beams(**bad)) == card.CARD_ERANGE, bad
    assert _select(_beams(), vocab=1 << 30, stride=1 << 30) == card.CARD_ERANGE
    for gone in ("scores_dev", "out_scores_dev", "out_tokens_dev", "out_parents_dev", "lengths_dev", "out_history_dev"):
        assert _select(_beams(**{gone: None})) == card.CARD_EINVAL, gone
    assert _select(_beams(), logits=None) == _select(_beams(), ws=None) == _select(_beams(), ws=A + 8) == card.CARD_EINVAL


def test_beam_select_workspace():
    need = card.card_beam_select_workspace_bytes
    assert need(0, 1, 1, 10) == need(1, 0, 1, 10) == need(1, 33, 1, 10) == need(1, 1, 0, 10) == need(1, 1, 33, 10) == need(1, 1, 1, 0) == 0
    assert need(1 << 24, 1, 1, 10) == 0
    assert need(1, 1, 1, 10) >= 24
    for vocab in (1000, 128256):
        sizes = [need(n, 4, 4, vocab) for n in range(1, 400)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))  # enough for fewer groups


def test_wrapper_refuses_before_the_library():
    logits, scores = torch.zeros(6, 20), torch.zeros(2, 3)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    for bad in (dict(logits=torch.zeros(5, 20)), dict(scores=torch.zeros(2, 3, dtype=torch.float64)), dict(scores=torch.zeros(3, 2).T), dict(done=i32(2, 2)),
                dict(done=torch.zeros(2, 3)), dict(history=i32(2, 3, 4)), dict(lengths=i32(2)), dict(history=i32(2, 3, 4), lengths=i32(3)),
                dict(history=i32(2, 2, 4), lengths=i32(2))):
        with pytest.raises(ValueError):
            card.beam_select(**dict(dict(logits=logits, scores=scores), **bad))
    assert card.card_beam_select(logits, _beams(groups=3), 1.0, A) == card.CARD_EINVAL


def _sequence(pool, values):
    seq = pool.new()
    pool.extend(seq, len(values))
    pool.write(seq, 0, values)
    return seq


def test_reorder_against_lists(monkeypatch):
    """Beams over many steps: each text is what lists say, pages are shared while they are full, and none is lost."""
    g = torch.Generator().manual_seed(3)
    pool = PlayedPool(monkeypatch, 200, 512)
    prompt = list(range(37))
    seqs, texts = [_sequence(pool, prompt)], [list(prompt)]
    other = _sequence(pool, [7] * 20)
    for step in range(60):
        n = int(torch.randint(1, 7, (1,), generator=g))
        parents = torch.randint(0, len(seqs), (n,), generator=g).tolist()
        seqs = pool.reorder(seqs, parents)
        texts = [list(texts[p]) for p in parents]
        assert len(set(seqs)) == n
        for i, seq in enumerate(seqs):
            pool.extend(seq, 1)
            texts[i].append(1000 * step + i)
            pool.write(seq, len(texts[i]) - 1, texts[i][-1:])
        for seq, text in zip(seqs, texts):
            assert pool.text(seq) == text and pool.length(seq) == len(text)
        held = {p for s in pool._seqs.values() for p in s.pages}
        assert len(held) + pool.free_pages == 200
        users = [sum(p in s.pages for s in pool._seqs.values()) for p in range(200)]
        assert users == pool._users
    assert pool.text(other) == [7] * 20
    for seq in seqs + [other]:
        pool.free(seq)
    assert pool.free_pages == 200


def test_reorder_refuses(monkeypatch):
    pool = PlayedPool(monkeypatch, 4, 512)
    a, b = _sequence(pool, [1] * 20), _sequence(pool, [2] * 20)
    before = [list(pool._seqs[s].pages) for s in (a, b)]
    for bad in (([a, a], [0]), ([a, b], [2]), ([a, b], [-1])):
        with pytest.raises(ValueError):
            pool.reorder(*bad)
    with pytest.raises(KeyError):
        pool.reorder([a, 99], [0])
    with pytest.raises(card.CardError) as e:
        pool.reorder([a, b], [0, 1, 1])  # no page for the copy of the last one
    assert e.value.status == card.CARD_ECAPACITY
    assert [list(pool._seqs[s].pages) for s in (a, b)] == before and pool.free_pages == 0
    # a beam that is given up leaves its pages to those that go on
    c = pool.reorder([a, b], [1, 1])
    assert [pool.text(s) for s in c] == [[2] * 20] * 2 and c[0] == b
    assert pool.free_pages == 1
    assert pool.reorder(c, []) == [] and pool.free_pages == 4


def test_reorder_ends_plans(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=0))
    pool = PlayedPool(monkeypatch, 40, 512)
    a, b = _sequence(pool, [1] * 20), _sequence(pool, [2] * 20)
    plan = pool.plan([a, b], [1, 1])
    pool.reorder([a, b], [0, 0])
    with pytest.raises(card.CardError) as e:
        pool._still_holds(plan, False, "attend")
    assert e.value.status == card.CARD_ESTALE
