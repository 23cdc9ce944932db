"""What card_kv_copy_pages, card_kv_move_slots, card_kv_attend and card_logprobs refuse, and the bookkeeping of SequencePool; no GPU:
nothing gets as far as a launch."""
import types

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
    # launches of 2^24 workgroups
    q_heads, kv_heads = cfg.n_q_heads, cfg.n_kv_heads
    for big in (batch(n_rows=(1 << 28) // q_heads), batch(n_seqs=(1 << 23) // kv_heads), batch(n_rows=2 ** 31 - 1, n_seqs=2 ** 31 - 1)):
        assert call(big) == card.CARD_ERANGE and card.card_kv_attend_workspace_bytes(cfg, big) == 0
    assert card.card_kv_attend_workspace_bytes(cfg, batch(n_rows=(1 << 27) // q_heads, max_len=1)) == 0  # (one cut: none needed)
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
    raw = lambda rows, vocab: card.lib.card_logprobs(A, card.CARD_F32, rows, vocab, vocab, A, 1.0, 0, A, None, None, None, A, None)  # noqa: E731
    assert raw(1 << 24, 100) == raw(1, 1 << 30) == card.CARD_ERANGE
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


# ---- SequencePool's bookkeeping, its device calls played on the CPU -----------------------------------


class PlayedPool(card.SequencePool):
    """Pages hold one number per slot: what write() put there."""

    def __init__(self, monkeypatch, n_pages, max_ctx):
        from paper_2508_04462_amd import binding

        monkeypatch.setattr(binding, "card_kv_copy_pages", self._copy)
        monkeypatch.setattr(binding, "card_kv_move_slots", self._move)
        self._setup(card.make_cfg(TINY, max_ctx), n_pages, torch.device("cpu"))
        self.slots = [-1] * (n_pages * 16)

    def _stream(self):
        return 0

    def _copy(self, cfg, kv, src, dst, stream):
        assert not set(src) & set(dst) and len(set(dst)) == len(dst)
        for s, d in zip(src, dst):
            self.slots[d * 16:d * 16 + 16] = self.slots[s * 16:s * 16 + 16]
        return card.CARD_OK

    def _move(self, cfg, kv, src, dst, stream):
        assert all(s not in dst[:i] for i, s in enumerate(src))
        for s, d in zip(src, dst):
            self.slots[d] = self.slots[s]
        return card.CARD_OK

    def write(self, seq, first, values):
        assert self.writable(seq, first, first + len(values))
        for i, v in enumerate(values):
            p = first + i
            self.slots[self._seqs[seq].pages[p // 16] * 16 + p % 16] = v

    def text(self, seq):
        s = self._seqs[seq]
        assert len(s.pages) == (s.length + 15) // 16 and s.table[:len(s.pages)].tolist() == s.pages
        return [self.slots[s.pages[p // 16] * 16 + p % 16] for p in range(s.length)]

    def check(self):
        users = [0] * self.n_pages
        for s in self._seqs.values():
            for p in s.pages:
                users[p] += 1
        assert users == self._users and sorted(self._free) == [p for p in range(self.n_pages) if users[p] == 0]


def test_pool_against_lists(monkeypatch):
    """Random forks, extensions, cuts, compactions and ends of sequences, against plain lists."""
    import random

    rng = random.Random(5)
    pool = PlayedPool(monkeypatch, 40, 160)
    texts, value = {}, 0
    refused = 0
    for _ in range(3000):
        what = rng.choice(["new", "extend", "extend", "extend", "fork", "truncate", "compact", "free"])
        try:
            if what == "new":
                texts[pool.new()] = []
            elif texts:
                seq = rng.choice(list(texts))
                text = texts[seq]
                if what == "extend":
                    n = rng.choice([0, 1, 1, 5, 16, 40])
                    pool.extend(seq, n)
                    new = list(range(value, value + n))
                    value += n
                    pool.write(seq, len(text), new)
                    texts[seq] = text + new
                elif what == "fork":
                    texts[pool.fork(seq)] = list(text)
                elif what == "truncate":
                    keep = rng.randint(0, len(text))
                    pool.truncate(seq, keep)
                    texts[seq] = text[:keep]
                elif what == "compact":
                    first = rng.randint(0, len(text))
                    kept = sorted(rng.sample(range(first, len(text)), rng.randint(0, len(text) - first)))
                    pool.compact(seq, first, kept)
                    texts[seq] = text[:first] + [text[p] for p in kept]
                elif what == "free" and rng.random() < 0.5:
                    pool.free(seq)
                    del texts[seq]
        except card.CardError as e:
            assert e.status == card.CARD_ECAPACITY
            refused += 1
        pool.check()
        for seq, text in texts.items():
            assert pool.text(seq) == text and pool.length(seq) == len(text)
    assert 10 < refused < 2000


def test_pool_refuses(monkeypatch):
    pool = PlayedPool(monkeypatch, 4, 64)
    a = pool.new()
    pool.extend(a, 40)
    for bad in (lambda: pool.extend(a, -1), lambda: pool.truncate(a, 41), lambda: pool.truncate(a, -1), lambda: pool.compact(a, 41, []),
                lambda: pool.compact(a, 10, [9]), lambda: pool.compact(a, 10, [12, 12]), lambda: pool.compact(a, 10, [13, 12]),
                lambda: pool.compact(a, 10, [40])):
        with pytest.raises(card.CardError) as e:
            bad()
        assert e.value.status == card.CARD_ERANGE
    with pytest.raises(card.CardError) as e:
        pool.extend(a, 25)  # beyond max_ctx
    assert e.value.status == card.CARD_ECAPACITY
    b = pool.fork(a)
    with pytest.raises(card.CardError):
        pool.fork(b)  # no page for a copy of the last one
    assert pool.free_pages == 0 and pool.length(b) == 40
    assert pool.writable(b, 32, 40) and not pool.writable(b, 31, 40) and not pool.writable(b, 32, 41)
    with pytest.raises(card.CardError) as e:
        pool.plan([a], [9])  # rows on a page that the fork holds, too
    assert e.value.status == card.CARD_EINVAL
    with pytest.raises(ValueError):
        pool.plan([], [])
    with pytest.raises(ValueError):
        pool.plan([b, b], [2, 1])  # two rows would be one token
    # a mask in other memory than the pools
    plan = types.SimpleNamespace(n_rows=2, n_seqs=1)
    q, kv = torch.zeros(2, TINY.n_q_heads, TINY.head_dim), torch.zeros(2, TINY.n_kv_heads, TINY.head_dim)
    for mask_dev, base_dev in (("meta", "cpu"), ("cpu", "meta")):
        with pytest.raises(ValueError):
            pool.attend(plan, 0, q, kv, kv, mask=torch.zeros(2, 1, dtype=torch.int32, device=mask_dev),
                        mask_base=torch.zeros(1, dtype=torch.int32, device=base_dev))
    pool.free(a)
    with pytest.raises(KeyError):
        pool.length(a)
    assert pool.writable(b, 0, 40)
