"""What card_kv_copy_pages, card_kv_move_slots, card_kv_attend and card_logprobs refuse, and the bookkeeping of SequencePool; no GPU:
nothing gets as far as a launch."""
import pytest
import torch

import card_inputs as ci
import paper_2508_04462_amd as card
from serving_common import Batch

TINY = ci.SHAPES["tiny"]
A = 0x10000  # an address: nothing is read or written


def _kv(n_pages=16, k=A, v=A):
    return card.CardKV(k, v, None, n_pages, -1)


def test_page_lists_are_checked_on_the_host():
    cfg = card.make_cfg(TINY, 256)
    copy = lambda src, dst, kv=_kv(): card.card_kv_copy_pages(cfg, kv, src, dst)  # noqa: E731
    assert copy([], []) == card.CARD_OK
    for bad in (-1, 16, 2 ** 31 - 1, -2 ** 31):
        assert copy([bad], [3]) == copy([3], [bad]) == card.CARD_ERANGE
    assert copy([0, 1], [5, 5]) == card.CARD_EINVAL  # written twice
    assert copy([0, 5], [5, 6]) == copy([5, 0], [6, 5]) == copy([4], [4]) == card.CARD_EINVAL  # read and written
    assert copy([0], [1, 2]) == card.CARD_EINVAL
    assert copy([0], [1], _kv(k=None)) == copy([0], [1], _kv(v=None)) == copy([0], [1], _kv(0)) == card.CARD_EINVAL
    assert copy([0], [1], _kv(k=A + 8)) == card.CARD_EINVAL
    bad_cfg = card.make_cfg(TINY, 256)
    bad_cfg.head_dim = 96
    assert card.card_kv_copy_pages(bad_cfg, _kv(), [0], [1]) == card.CARD_EINVAL
    assert card.lib.card_kv_copy_pages(cfg, _kv(), 1, None, None, None) == card.CARD_EINVAL
    assert card.lib.card_kv_copy_pages(cfg, _kv(), -1, None, None, None) == card.CARD_EINVAL


def test_slot_lists_are_checked_on_the_host():
    cfg = card.make_cfg(TINY, 256)
    move = lambda src, dst, kv=_kv(): card.card_kv_move_slots(cfg, kv, src, dst)  # noqa: E731
    assert move([], []) == card.CARD_OK
    for bad in (-1, 256, 2 ** 31 - 1):
        assert move([bad], [3]) == move([3], [bad]) == card.CARD_ERANGE
    assert move([1, 2], [9, 9]) == card.CARD_EINVAL  # written twice
    assert move([1, 9], [9, 10]) == card.CARD_EINVAL  # read after it was written
    many = list(range(100, 200))
    assert move(many, [m + 1 for m in many]) == card.CARD_EINVAL  # (a gap opened from the front)
    assert move([1], [2], _kv(v=None)) == move([1], [2, 3]) == card.CARD_EINVAL


def _rows(type=card.CARD_BF16, row=512, head=64, data=A):
    return card.CardRows(data, type, row, head)


def test_attend_refuses_what_it_cannot_run():
    cfg = card.make_cfg(TINY, 256)

    def batch(**change):
        b = card.CardKVBatch(A, A, 16, 2, A, 4, 8, A, A, 4, 64)
        for name, value in change.items():
            setattr(b, name, value)
        return b

    def call(b=None, layer=0, q=_rows(), k=_rows(), v=_rows(), out=_rows(), mask=None, cfg_=cfg, ws=A):
        return card.card_kv_attend(cfg_, b or batch(), layer, q, k, v, out, mask, ws)

    assert call(batch(n_rows=0)) == card.CARD_OK  # nothing to do
    for change in ({"k_pages": None}, {"v_pages": None}, {"block_tables": None}, {"ctx_lens": None}, {"row_starts": None}, {"n_pages": 0},
                   {"n_seqs": 0}, {"table_pages": 0}, {"n_rows": -1}, {"max_new": -1}, {"max_len": -1}, {"k_pages": A + 4}):
        assert call(batch(**change)) == card.CARD_EINVAL, change
    assert call(layer=-1) == call(layer=2) == card.CARD_ERANGE
    assert call(batch(n_rows=1 << 30)) == card.CARD_ERANGE
    assert call(k=None) == call(v=None) == card.CARD_EINVAL  # one without the other
    for name in ("q", "k", "v", "out"):
        assert call(**{name: _rows(card.CARD_F32)}) == card.CARD_EINVAL  # types differ
        assert call(**{name: _rows(7)}) == call(**{name: _rows(data=None)}) == card.CARD_EINVAL
        assert call(**{name: _rows(data=A + 2)}) == call(**{name: _rows(row=511)}) == call(**{name: _rows(head=60)}) == card.CARD_EINVAL
        assert call(**{name: _rows(row=-512)}) == card.CARD_EINVAL
    assert call(out=_rows(row=0)) == call(out=_rows(head=0)) == card.CARD_EINVAL  # rows of the output over each other
    for mask in (card.CardRowMask(None, A, 1), card.CardRowMask(A, None, 1), card.CardRowMask(A, A, 0)):
        assert call(mask=mask) == card.CARD_EINVAL
    bad = card.make_cfg(TINY, 256)
    bad.n_kv_heads = 3
    assert call(cfg_=bad) == card.CARD_EINVAL and card.card_kv_attend_workspace_bytes(bad, batch()) == 0
    with pytest.raises(ValueError):
        card.card_rows(torch.zeros(4, 64, 4).transpose(1, 2))
    assert card.card_rows(torch.zeros(4, 2, 64, dtype=torch.float16)).type == -1


def test_logprobs_refuses_what_it_cannot_run():
    logits = torch.zeros(4, 100)
    call = lambda x=logits, tok=A, t=1.0, top=2, lp=A, en=A, tt=A, tl=A, ws=A: card.card_logprobs(x, tok, t, top, lp, en, tt, tl, ws)  # noqa: E731
    assert call(torch.zeros(0, 100)) == card.CARD_OK
    assert call(top=-1) == call(top=33) == card.CARD_ERANGE
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        assert call(t=t) == card.CARD_EINVAL, t
    assert call(tok=None) == call(lp=None) == call(tt=None) == call(tl=None) == card.CARD_EINVAL
    assert call(tok=None, lp=None, en=None, top=0) == card.CARD_EINVAL  # nothing asked for
    assert call(torch.zeros(4, 100, dtype=torch.float16)) == call(torch.zeros(4, 100).expand(4, 100)[:, :0]) == card.CARD_EINVAL
    assert call(torch.zeros(1, 100).expand(4, 100)) == card.CARD_EINVAL  # rows over each other
    with pytest.raises(ValueError):
        call(torch.zeros(100, 4).T)


def test_reference_sees_what_its_pools_hold():
    """The reference's own layout: what it stores comes back from the pool where an independent reading of the page order finds it."""
    b = Batch((4, 2, 64), [(5, 3), (16, 1)], torch.bfloat16, fill=0.0)
    _, _, _, kp, vp = b.reference()
    for s, (c, n) in enumerate(b.lens):
        for pos in (0, c - 1, c, c + n - 1):
            page, t = int(b.tables[s, pos // 16]), pos % 16
            want_k = b.keys[s][pos] if pos < c else b.k[int(b.starts[s]) + pos - c]
            want_v = b.values[s][pos] if pos < c else b.v[int(b.starts[s]) + pos - c]
            for head in range(2):
                k = kp[1, page, head].view(8, 16, 8)[:, t].reshape(64)
                v = vp[1, page, head].view(2, 4, 16, 2, 4)[:, t // 4, :, :, t % 4].transpose(1, 2).reshape(64)
                assert torch.equal(k, want_k[head]) and torch.equal(v, want_v[head])
