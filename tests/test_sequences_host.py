"""SequencePool and AttendPlan on the CPU: which plans attend() still takes after the pool has changed."""
import types

import pytest
import torch

import card_inputs as ci
import paper_2508_04462_amd as card
from test_serving_host import PlayedPool

TINY = ci.SHAPES["tiny"]


class AttendingPool(PlayedPool):
    """attend() gets as far as the library's call, which counts instead."""

    def __init__(self, monkeypatch, n_pages=40, max_ctx=160):
        from paper_2508_04462_amd import binding

        super().__init__(monkeypatch, n_pages, max_ctx)
        self.calls = 0
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=0))
        monkeypatch.setattr(binding, "card_kv_attend", self._attended)

    def _attended(self, *args):
        self.calls += 1
        return card.CARD_OK

    def run(self, plan, store=True):
        """Whether attend takes the plan; a plan that it does not take gets CARD_ESTALE, and no call."""
        q = torch.zeros(plan.n_rows, TINY.n_q_heads, TINY.head_dim, dtype=torch.bfloat16)
        kv = torch.zeros(plan.n_rows, TINY.n_kv_heads, TINY.head_dim, dtype=torch.bfloat16) if store else None
        before = self.calls
        try:
            self.attend(plan, 0, q, kv, kv)
        except card.CardError as e:
            assert e.status == card.CARD_ESTALE and self.calls == before
            return False
        assert self.calls == before + 1
        return True


@pytest.fixture
def pool(monkeypatch):
    return AttendingPool(monkeypatch)


def _sequence(pool, n):
    seq = pool.new()
    pool.extend(seq, n)
    return seq


def test_fork_between_plan_and_attend(pool):
    """The fork shares a page that the plan's rows would write."""
    a = _sequence(pool, 10)
    pool.extend(a, 20)
    plan = pool.plan([a], [20])
    assert pool.run(plan)
    b = pool.fork(a)
    assert not pool.run(plan)
    assert pool.run(plan, store=False)  # what the cache holds may still be read
    pool.free(b)
    assert pool.run(plan)


def test_fork_that_copies_all_that_is_written(pool):
    a = _sequence(pool, 16)
    pool.extend(a, 3)
    plan = pool.plan([a], [3])
    pool.fork(a)  # the rows' page is copied, not shared
    assert pool.run(plan) and pool.run(plan, store=False)


@pytest.mark.parametrize("end", ["truncate", "free", "compact"])
def test_pages_that_went_to_another_sequence(pool, end):
    a = _sequence(pool, 40)
    pool.extend(a, 8)
    plan = pool.plan([a], [8])
    assert pool.run(plan)
    if end == "truncate":
        pool.truncate(a, 5)
    elif end == "compact":
        pool.compact(a, 5, [9, 11])
    else:
        pool.free(a)
    assert not pool.run(plan) and not pool.run(plan, store=False)
    _sequence(pool, 60)
    assert not pool.run(plan) and not pool.run(plan, store=False)
    if end != "free":  # long enough again, on other pages
        pool.extend(a, 48 - pool.length(a))
        assert not pool.run(plan) and not pool.run(plan, store=False)


def test_tokens_given_up_inside_the_last_page(pool):
    a = _sequence(pool, 20)
    pool.extend(a, 8)
    plan = pool.plan([a], [8])
    pool.truncate(a, 25)
    assert not pool.run(plan)
    pool.extend(a, 3)  # the same places on the same page
    assert pool.run(plan)


def test_a_shared_page_that_gets_a_copy(pool):
    a = _sequence(pool, 32)
    b = pool.fork(a)
    plan = pool.plan([a], [0])
    pool.extend(b, 4)
    rows = pool.plan([b], [4])
    assert pool.run(rows)
    pool.truncate(a, 20)
    pool.extend(a, 2)  # writes to a page that the fork holds: gets a copy
    assert pool._seqs[a].pages[1] != pool._seqs[b].pages[1]
    late = pool.plan([a, b], [2, 4])
    assert pool.run(late) and pool.run(rows) and plan.n_rows == 0


def test_plan_of_another_pool(pool, monkeypatch):
    """Its pages are others, whatever its rows look like."""
    other = AttendingPool(monkeypatch)
    plans = []
    for p in (pool, other):
        a = _sequence(p, 20)
        plans.append(p.plan([a], [4]))
    for p, plan in ((pool, plans[1]), (other, plans[0])):
        with pytest.raises(ValueError):
            p.run(plan)
    assert other.run(plans[1]) and other.calls == 1


def test_changes_elsewhere_do_not_matter(pool):
    a, b = _sequence(pool, 10), _sequence(pool, 40)
    pool.extend(a, 2)
    plan = pool.plan([a], [2])
    pool.fork(b)
    pool.truncate(b, 3)
    c = _sequence(pool, 60)
    pool.free(b)
    pool.compact(c, 3, [7, 8])
    assert pool.run(plan)
    pool.extend(a, 30)  # longer: the plan's places stay where they are
    assert pool.run(plan) and pool.run(plan, store=False)


def test_plans_against_what_sequences_hold(pool):
    """Random changes: a plan is taken as long as its sequences have its tokens on its pages, and its rows' pages to themselves."""
    import random

    rng = random.Random(9)
    plans, taken, refused = [], 0, 0
    for step in range(1500):
        what = rng.choice(["new", "extend", "extend", "fork", "truncate", "compact", "free", "plan", "plan"])
        seqs = list(pool._seqs)
        try:
            if what == "new":
                pool.new()
            elif seqs:
                s = rng.choice(seqs)
                n = pool.length(s)
                if what == "extend":
                    pool.extend(s, rng.choice([1, 3, 16, 40]))
                elif what == "fork":
                    pool.fork(s)
                elif what == "truncate":
                    pool.truncate(s, rng.randint(n // 2, n))
                elif what == "compact":
                    first = rng.randint(0, n)
                    pool.compact(s, first, sorted(rng.sample(range(first, n), rng.randint(0, n - first))))
                elif what == "free" and rng.random() < 0.3:
                    pool.free(s)
                elif what == "plan":
                    group = rng.sample(seqs, rng.randint(1, min(3, len(seqs))))
                    new = [rng.randint(0, min(5, pool.length(g))) for g in group]
                    plan = pool.plan(group, new)
                    if plan.n_rows:
                        where = [(g, pool.length(g) - k, pool.length(g), list(pool._seqs[g].pages)) for g, k in zip(group, new)]
                        plans = plans[-12:] + [(plan, where)]
        except card.CardError as e:
            assert e.status in (card.CARD_ECAPACITY, card.CARD_EINVAL)
        for plan, where in plans:
            there = all(g in pool._seqs and pool.length(g) >= end and pool._seqs[g].pages[:len(pages)] == pages for g, _, end, pages in where)
            own = there and all(pool.writable(g, first, end) for g, first, end, _ in where)
            assert pool.run(plan) == own and pool.run(plan, store=False) == there
            taken, refused = taken + own, refused + (not own)
    assert taken > 500 and refused > 500


def test_pages_of_an_ended_text_are_cleared_for_the_next(monkeypatch):
    """Steps multiply the values behind a text's end with weights of zero: what its last owner left there, NaN perhaps, must not be in a page that is
    taken from the free ones.  Pages that a sequence holds, copies among them, keep what they have."""
    pool = PlayedPool(monkeypatch, 12, 160)
    values = pool.v_pages.view(torch.bfloat16).view(pool.cfg.n_layers, 12, -1)
    a, b = _sequence(pool, 40), _sequence(pool, 20)
    old = list(pool._seqs[a].pages)
    values[:, old + pool._seqs[b].pages] = float("nan")
    kept = list(pool._seqs[b].pages)
    pool.free(a)
    c = _sequence(pool, 10)
    pool.extend(c, 100)
    mine = pool._seqs[c].pages
    assert set(old) <= set(mine) and (values[:, mine] == 0).all()
    assert values[:, kept].isnan().all()
    # truncated pages, too; a copy of a shared page is a copy
    values[:, mine] = 1.0
    pool.truncate(c, 50)
    d = pool.fork(c)
    assert pool._seqs[d].pages[:3] == mine[:3]
    pool.extend(b, 30)
    assert (values[:, pool._seqs[b].pages[2:]] == 0).all() and values[:, kept].isnan().all() and (values[:, mine[:4]] == 1.0).all()
