"""SequencePool of 4 bits on the CPU."""
import pytest
import torch

import card_inputs as ci
import paper_2508_04462_amd as card

TINY = ci.SHAPES["tiny"]


def _pool(bits):
    pool = card.SequencePool.__new__(card.SequencePool)
    pool._setup(card.make_cfg(TINY, 160), 8, torch.device("cpu"), bits)
    seq = pool.new()
    pool.extend(seq, 20)
    return pool, seq


def test_a_pool_of_4_bits_has_no_cache_for_steps_and_prompts():
    """They, and card_kv_gather, would read its pages as pages of 16 bits, far behind the pool's end."""
    pool, seq = _pool(16)
    assert pool.kv(seq).n_pages == 8
    pool, seq = _pool(4)
    with pytest.raises(ValueError):
        pool.kv(seq)


def test_compaction_in_4_bits(monkeypatch):
    from paper_2508_04462_amd import binding

    pool, seq = _pool(4)
    calls = []
    monkeypatch.setattr(binding, "card_kv4_move_slots", lambda cfg, kv, src, dst, stream: calls.append((kv.k_pages, kv.n_pages, src, dst)) or card.CARD_OK)
    monkeypatch.setattr(card.SequencePool, "_stream", lambda self: 0)
    pages = list(pool._seqs[seq].pages)
    pool.compact(seq, 3, [5, 17])
    assert calls == [(pool.k_pages.data_ptr(), 8, [pages[0] * 16 + 5, pages[1] * 16 + 1], [pages[0] * 16 + 3, pages[0] * 16 + 4])] and pool.length(seq) == 5
