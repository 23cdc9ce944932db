"""What card_kv_append and the functions of the cache of 4 bits refuse; no GPU: nothing gets as far as a launch."""
import math

import pytest
import torch

import card_inputs as ci
import paper_2508_04462_amd as card
from cache4_common import model_freqs, quantised, values
from serving_common import Batch

TINY = ci.SHAPES["tiny"]
A = 0x10000  # an address: nothing is read or written


def _batch(**more):
    d = dict(k_pages=A, v_pages=A, n_pages=16, n_seqs=2, block_tables=A, table_pages=8, n_rows=3, ctx_lens=A, row_starts=A, max_new=3, max_len=100)
    return card.CardKVBatch(*dict(d, **more).values())


def _rows(data=A, type=card.CARD_BF16, row=512, head=64):
    return card.CardRows(data, type, row, head)


def _append(name, batch=None, layer=0, rotation="model", q="rows", q_out="rows", k="rows", v="rows", cfg=None):
    row = lambda x: _rows() if x == "rows" else x  # noqa: E731
    return getattr(card, name)(cfg or card.make_cfg(TINY, 256), batch or _batch(n_rows=0 if batch is None else 3), layer,
                               card.card_rotation() if rotation == "model" else rotation, row(q), row(q_out), row(k), row(v))


@pytest.mark.parametrize("name", ["card_kv_append", "card_kv4_append"])
def test_append_refusals(name):
    call = lambda **more: _append(name, **dict(dict(batch=_batch()), **more))  # noqa: E731
    assert _append(name) == card.CARD_OK  # no rows
    for bad in (dict(k_pages=None), dict(v_pages=None), dict(k_pages=A + 8), dict(block_tables=None), dict(ctx_lens=None), dict(row_starts=None),
                dict(n_pages=0), dict(n_seqs=0), dict(table_pages=0), dict(table_pages=1 << 27), dict(n_rows=-1), dict(max_new=-1), dict(max_len=-1)):
        assert call(batch=_batch(**bad)) == card.CARD_EINVAL, bad
    assert call(layer=-1) == call(layer=2) == card.CARD_ERANGE
    assert call(batch=_batch(n_rows=2 ** 31 - 1)) == card.CARD_ERANGE
    assert call(k=None) == call(v=None) == card.CARD_EINVAL
    assert call(q=None) == call(q_out=None) == call(rotation=None) == card.CARD_EINVAL  # q without q_out, and the other way; q that is not rotated
    for bad in (_rows(None), _rows(A + 8), _rows(row=516), _rows(head=68), _rows(type=2), _rows(type=card.CARD_F32), _rows(row=-512)):
        for which in ("q", "q_out", "k", "v"):
            assert call(**{which: bad}) == card.CARD_EINVAL, which
    assert call(q_out=_rows(head=0)) == call(q_out=_rows(row=32)) == card.CARD_EINVAL
    for bad in (math.nan, math.inf, -math.inf):
        assert call(rotation=card.card_rotation([bad] + model_freqs(1e4, 64)[1:])) == card.CARD_EINVAL
    assert call(rotation=card.card_rotation(model_freqs(1e4, 128))) == card.CARD_EINVAL  # of another head size
    assert call(rotation=card.card_rotation([])) == card.CARD_EINVAL  # (a table of none would be read behind its end)
    cfg = card.make_cfg(TINY, 256)
    cfg.head_dim = 96
    assert call(cfg=cfg) == card.CARD_EINVAL


def test_attend4_and_read_refusals():
    cfg = card.make_cfg(TINY, 256)
    call = lambda batch=None, layer=0, q=_rows(), k=None, v=None, out=_rows(), mask=None, ws=A: card.card_kv4_attend(  # noqa: E731
        cfg, batch or _batch(), layer, q, k, v, out, mask, ws)
    assert call(_batch(n_rows=0)) == card.CARD_OK
    assert call(_batch(k_pages=None)) == call(_batch(v_pages=A + 4)) == call(q=None) == call(out=None) == card.CARD_EINVAL
    assert call(layer=2) == call(_batch(n_rows=2 ** 31 - 1)) == card.CARD_ERANGE
    assert call(k=_rows()) == call(v=_rows()) == call(k=_rows(), v=_rows(type=card.CARD_F32)) == card.CARD_EINVAL
    assert call(q=_rows(type=card.CARD_F32)) == call(out=_rows(head=32)) == call(q=_rows(type=7), out=_rows(type=7)) == card.CARD_EINVAL
    for bad in (card.CardRowMask(None, A, 1), card.CardRowMask(A, None, 1), card.CardRowMask(A, A, 0), card.CardRowMask(A, A, (1 << 25) + 1)):
        assert call(mask=bad) == card.CARD_EINVAL
    cut = _batch(table_pages=4096, max_len=65536)
    assert card.card_kv4_attend_workspace_bytes(cfg, cut) > 0
    assert call(cut, ws=None) == call(cut, ws=A + 4) == card.CARD_EINVAL
    assert card.card_kv4_attend_workspace_bytes(cfg, _batch(n_rows=0)) == card.card_kv4_attend_workspace_bytes(cfg, _batch(n_seqs=0)) == 0
    read = lambda batch=None, layer=0, k=_rows(), v=_rows(): card.card_kv4_read(cfg, batch or _batch(), layer, k, v)  # noqa: E731
    assert read(_batch(n_rows=0)) == card.CARD_OK
    assert read(k=None) == read(v=None) == read(k=_rows(head=0)) == read(v=_rows(row=32)) == read(k=_rows(type=card.CARD_F32)) == card.CARD_EINVAL
    assert read(layer=-1) == card.CARD_ERANGE and read(_batch(k_pages=None)) == card.CARD_EINVAL


def test_page_and_slot_lists_of_4_bits():
    cfg = card.make_cfg(TINY, 256)
    kv = lambda n_pages=16, k=A, v=A: card.CardKV(k, v, None, n_pages, -1)  # noqa: E731
    copy = lambda src, dst, kv=kv(): card.card_kv4_copy_pages(cfg, kv, src, dst)  # noqa: E731
    move = lambda src, dst, kv=kv(): card.card_kv4_move_slots(cfg, kv, src, dst)  # noqa: E731
    for call, most in ((copy, 16), (move, 256)):
        assert call([], []) == card.CARD_OK
        for bad in (-1, most, 2 ** 31 - 1):
            assert call([bad], [3]) == call([3], [bad]) == card.CARD_ERANGE
        assert call([1, 2], [9, 9]) == call([1, 9], [9, 10]) == card.CARD_EINVAL  # written twice; read after it was written
        assert call([0], [1], kv(k=None)) == call([0], [1], kv(v=None)) == call([0], [1], kv(v=A + 8)) == call([0], [1], kv(0)) == card.CARD_EINVAL
        assert call([1], [2, 3]) == card.CARD_EINVAL
    assert copy([0, 5], [5, 6]) == copy([5, 0], [6, 5]) == copy([4], [4]) == card.CARD_EINVAL  # read and written
    for name in ("card_kv4_copy_pages", "card_kv4_move_slots"):
        assert getattr(card.lib, name)(cfg, kv(), 1, None, None, None) == getattr(card.lib, name)(cfg, kv(), -1, None, None, None) == card.CARD_EINVAL


def test_pool_bytes():
    cfg = card.make_cfg(TINY, 256)
    assert card.card_kv4_pool_bytes(cfg, 10) == 2 * 10 * 2 * 16 * (32 + 4)  # of a token of a head: 64 nibbles and a word
    assert card.card_kv4_pool_bytes(card.make_cfg(ci.SHAPES["llama70b"], 256), 10 ** 6) == 80 * 10 ** 6 * 8 * 1152
    assert card.card_kv4_pool_bytes(cfg, 0) == card.card_kv4_pool_bytes(cfg, -1) == 0


def test_workspaces_hold_for_either_type_and_fewer_rows():
    cfg = card.make_cfg(ci.SHAPES["llama8b"], 256)
    for rows, seqs in ((1, 1), (8, 8), (48, 48), (500, 1), (2000, 3)):
        need = card.card_kv4_attend_workspace_bytes(cfg, _batch(n_rows=rows, n_seqs=seqs, max_new=0, table_pages=2048, max_len=30000))
        assert need < 1 << 31


def test_definition_of_4_bits():
    """What the tests take for it: values are at most half a scale off, 16 levels for values of either sign and size, equal values, zeros."""
    g = torch.Generator().manual_seed(0)
    for x in (torch.randn(50, 2, 128, generator=g), torch.randn(50, 2, 128, generator=g) * 1e-20, torch.rand(50, 2, 128, generator=g) + 100,
              torch.full((3, 1, 64), -2.5), torch.zeros(3, 1, 64)):
        codes, words = quantised(x)
        scale = (words << 16).view(torch.float32).double().repeat_interleave(64, -1)
        assert codes.min() >= 0 and codes.max() <= 15
        assert ((values(codes, words) - x.double()).abs() <= scale * (0.5 + 2.0 ** -16)).all()
    b = Batch((4, 2, 64), [(3, 2)], torch.float32)
    assert b.n_rows == 2


def test_longest_tables():
    """Places are counted in 32 bits: of a table and of all new tokens that a launch has room for behind it."""
    cfg = card.make_cfg(TINY, 256)
    limit = (1 << 27) - (1 << 24)
    calls = [lambda b, name=name: _append(name, batch=b) for name in ("card_kv_append", "card_kv4_append")]
    calls += [lambda b, name=name: getattr(card, name)(cfg, b, 0, _rows(), None, None, _rows(), None, A) for name in ("card_kv_attend", "card_kv4_attend")]
    calls += [lambda b: card.card_kv4_read(cfg, b, 0, _rows(), _rows())]
    for call in calls:
        assert call(_batch(table_pages=limit, n_rows=0)) == call(_batch(table_pages=limit)) == card.CARD_EINVAL
        assert call(_batch(table_pages=limit - 1, n_rows=0)) == card.CARD_OK
    # page and place of the last unit of the largest launch, and the end of all its new tokens
    assert ((limit - 1) + (1 << 24)) * 16 + 15 < 1 << 31 and (limit - 1) * 16 + (1 << 28) < 1 << 31
