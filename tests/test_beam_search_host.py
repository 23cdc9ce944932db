"""Target.beam_search on the CPU: what its sequences hold of the pool, and what a failed call leaves; the model, the cache and the selection are played."""
import types

import pytest
import torch

import paper_2508_04462_amd as card
from test_gpu_beams import reference
from test_serving_host import PlayedPool

VOCAB = 50


class PlayedTarget:
    """A model whose logits depend on the text that its sequence holds; logits_of(text) may say others."""

    beam_search = card.Target.beam_search
    attach = lambda self, pool, seq: setattr(self, "_attached", (pool, seq))  # noqa: E731

    def __init__(self, monkeypatch, logits_of=None, vocab=VOCAB):
        from paper_2508_04462_amd import sequences

        monkeypatch.setattr(sequences, "beam_select", self._select)
        self.cfg, self.device, self._attached = types.SimpleNamespace(vocab=vocab), torch.device("cpu"), None
        self.out = torch.zeros(4, dtype=torch.int32)
        self.logits_of = logits_of or self.drawn

    @staticmethod
    def drawn(text):
        g = torch.Generator().manual_seed(sum((i + 1) * 1009 * (t + 1) for i, t in enumerate(text)))
        return torch.randn(VOCAB, generator=g) * 2

    @staticmethod
    def _select(logits, scores, out_beams, done, eos, temperature, history, lengths):
        got, _ = reference(logits, scores, out_beams, done, eos, temperature, history, lengths)
        return dict(got, scores=got["scores"].float(), **{name: got[name].int() for name in ("tokens", "parents", "done")})

    def prefill(self, tokens):
        self._attached[0].write(self._attached[1], 0, list(tokens))

    def enqueue_verify(self, ctx_len, pending, r, logits, cand):
        pool, seq = self._attached
        pool.write(seq, ctx_len, cand.tolist())
        assert pool.length(seq) == ctx_len + 1
        logits[0] = self.logits_of(pool.text(seq))
        return card.CARD_OK


def search_on_lists(target, prompt, beams, n_tokens, eos):
    found = [(0.0, [])]
    for _ in range(n_tokens):
        more = []
        for score, text in found:
            if text and text[-1] == eos:
                more.append((score, text))
                continue
            p = torch.log_softmax(target.logits_of(prompt + text).double(), 0)
            more += [(score + float(p[t]), text + [t]) for t in range(VOCAB) if p[t] > -float("inf")]
        found = sorted(more, key=lambda x: -x[0])[:beams]
    return found


@pytest.mark.parametrize("beams,n_tokens,eos", [(1, 5, -1), (4, 9, -1), (3, 12, 7), (6, 20, 3)])
def test_search_against_lists(monkeypatch, beams, n_tokens, eos):
    target, pool = PlayedTarget(monkeypatch), PlayedPool(monkeypatch, 60, 512)
    prompt = list(range(20))
    got = target.beam_search(pool, prompt, beams, n_tokens, eos)
    want = search_on_lists(target, prompt, beams, n_tokens, eos)
    assert got["tokens"] == [t for _, t in want]
    assert all(abs(a - b) < 1e-4 for a, (b, _) in zip(got["scores"], want))
    assert pool.free_pages == 60 and not pool._seqs and target._attached is None


def test_beams_that_are_not_forwarded_hold_no_pages(monkeypatch):
    """Pools that just hold the texts that are: after the last step, and behind an end, no beam needs a sequence."""
    prompt = list(range(20))  # two pages, the second one in part

    target, pool = PlayedTarget(monkeypatch), PlayedPool(monkeypatch, 2, 512)
    got = target.beam_search(pool, prompt, 4, 1)
    assert got["tokens"] == [t for _, t in search_on_lists(target, prompt, 4, 1, -1)] and pool.free_pages == 2

    def ends(text):  # 3 ends it, 4 goes on: of two beams one ends at once, the other one at the third step
        x = torch.full((VOCAB,), -float("inf"))
        x[3], x[4] = (1.0, 0.9) if len(text) < 22 else (9.0, 0.0)
        return x

    target = PlayedTarget(monkeypatch, ends)
    got = target.beam_search(pool, prompt, 2, 8, eos=3)
    assert got["tokens"] == [t for _, t in search_on_lists(target, prompt, 2, 8, 3)] and pool.free_pages == 2
    assert [3] in got["tokens"] and len(got["tokens"]) == 2 and got["tokens"] != [[3], [3]]

    def only(text):  # one candidate: the other beams are none
        x = torch.full((VOCAB,), -float("inf"))
        x[len(text) % 5] = 1.0
        return x

    target = PlayedTarget(monkeypatch, only)
    got = target.beam_search(pool, prompt, 5, 6)
    assert got == {"tokens": [[0, 1, 2, 3, 4, 0]], "scores": [0.0]} and pool.free_pages == 2


def test_search_without_room(monkeypatch):
    target, pool = PlayedTarget(monkeypatch), PlayedPool(monkeypatch, 3, 512)
    with pytest.raises(card.CardError) as e:
        target.beam_search(pool, list(range(20)), 4, 2)
    assert e.value.status == card.CARD_ECAPACITY and pool.free_pages == 3 and not pool._seqs and target._attached is None


def test_search_whose_buffers_find_no_room(monkeypatch):
    """Nothing of the call stays in the caller's pool."""
    target, pool = PlayedTarget(monkeypatch, vocab=1 << 60), PlayedPool(monkeypatch, 3, 512)
    with pytest.raises(RuntimeError):
        target.beam_search(pool, list(range(20)), 4, 2)
    assert not pool._seqs and pool.free_pages == 3
