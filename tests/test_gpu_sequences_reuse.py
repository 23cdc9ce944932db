"""Pages of a SequencePool that pass from one text to another."""
import pytest
import torch

from test_gpu_sequences import SHAPE, _step, _tokens, target  # noqa: F401

pytestmark = pytest.mark.gpu


def _store(pool, seq, n, seed, values=None):
    """The next n tokens of a sequence, in all layers, through attend()."""
    pool.extend(seq, n)
    plan = pool.plan([seq], [n])
    g = torch.Generator().manual_seed(seed)
    for layer in range(SHAPE.n_layers):
        q, k, v = (torch.randn((n, heads, SHAPE.head_dim), generator=g).bfloat16().cuda() for heads in (8, 2, 2))
        pool.attend(plan, layer, q, k, v if values is None else torch.full_like(v, values))


def test_a_step_behind_tokens_on_another_texts_pages(target):  # noqa: F811
    """The text before left NaN and infinities; a step in the middle of a page that attend() opened is what it is on a new pool."""
    import paper_2508_04462_amd as card

    got = []
    try:
        for before in (None, float("nan"), float("inf")):
            pool = card.SequencePool(SHAPE, 6, 512)
            if before is not None:
                a = pool.new()
                _store(pool, a, 90, 1, before)
                pool.free(a)
            b = pool.new()
            _store(pool, b, 20, 2)
            target.attach(pool, b)
            pool.extend(b, 4)
            got.append(_step(target, 20, _tokens(40, 4)))
            pool.extend(b, 30)
            got.append(_step(target, 24, _tokens(41, 8)))
    finally:
        target.attach()
    assert all(torch.isfinite(x).all() for x in got)
    assert torch.equal(got[2], got[0]) and torch.equal(got[4], got[0]) and torch.equal(got[3], got[1]) and torch.equal(got[5], got[1])


def test_pool_and_target_on_the_current_device(target):  # noqa: F811
    """"cuda" is the device that is current when pool or Target are made: the same memory, whatever it is called."""
    import paper_2508_04462_amd as card

    pool = card.SequencePool(SHAPE, 6, 512, device="cuda")
    assert pool.device == torch.device("cuda", torch.cuda.current_device())
    a = pool.new()
    pool.extend(a, 20)
    other = card.Target(SHAPE, 512, device="cuda")
    other.packed = target.packed
    try:
        target.attach(pool, a)
        token = target.prefill(_tokens(42, 20))
        pool.truncate(a, 0)
        pool.extend(a, 20)
        other.attach(pool, a)
        assert other.prefill(_tokens(42, 20)) == token
        here = card.SequencePool(SHAPE, 6, 512)
        other.attach(here, here.new())
    finally:
        target.attach()
