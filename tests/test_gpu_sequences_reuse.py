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


def test_plans_in_captured_graphs():
    """attend() of two plans captured into a graph each, one on a side stream, replayed with the program's own work and other calls between; each replay is
    what the eager calls give."""
    import paper_2508_04462_amd as card

    pool = card.SequencePool(SHAPE, 60, 512)
    seqs = [pool.new() for _ in range(3)]
    for i, s in enumerate(seqs):
        _store(pool, s, 90 + 40 * i, 50 + i)
    pool.extend(seqs[0], 3)
    pool.extend(seqs[2], 20)
    plans = [pool.plan([seqs[0]], [3]), pool.plan([seqs[2], seqs[1]], [20, 0])]
    g = torch.Generator().manual_seed(60)
    rows, graphs = [], []
    for plan in plans:
        q, k, v = (torch.randn((plan.n_rows, heads, SHAPE.head_dim), generator=g).bfloat16().cuda() for heads in (8, 2, 2))
        rows.append((q, k, v, torch.empty_like(q)))
        pool.attend(plan, 1, q, k, v)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            pool.attend(plan, 1, *rows[-1])
    other = torch.cuda.Stream()
    for turn in range(4):
        want = []
        for plan, (q, k, v, out) in zip(plans, rows):
            for t in (q, k, v):
                t.mul_(-0.9)
            want.append(pool.attend(plan, 1, q, k, v).clone())
            out.fill_(7.0)
        cache = pool.v_pages.clone()
        other.wait_stream(torch.cuda.current_stream())
        graphs[0].replay()
        with torch.cuda.stream(other):
            graphs[1].replay()
        torch.cuda.current_stream().wait_stream(other)
        torch.cuda.synchronize()
        for (_, _, _, out), w in zip(rows, want):
            assert torch.equal(out, w)
        assert torch.equal(pool.v_pages, cache)


def test_attend_of_rows_that_all_heads_and_tokens_share():
    """Keys, values and queries that are expanded: strides of zero."""
    import paper_2508_04462_amd as card

    pool = card.SequencePool(SHAPE, 60, 512)
    for n in (3, 70, 150):
        a = pool.new()
        _store(pool, a, 40, 70)
        pool.extend(a, n)
        plan = pool.plan([a], [n])
        g = torch.Generator().manual_seed(71)
        q, k, v = (torch.randn((1, 1, SHAPE.head_dim), generator=g).bfloat16().cuda().expand(n, heads, -1) for heads in (8, 2, 2))
        got = pool.attend(plan, 0, q, k, v, torch.empty((n, 8, SHAPE.head_dim), dtype=torch.bfloat16, device="cuda"))
        assert torch.equal(got, pool.attend(plan, 0, q.contiguous(), k.contiguous(), v.contiguous()))
        out = pool.attend(plan, 0, q, k, v)
        assert torch.equal(out, got) and out.is_contiguous()
        pool.free(a)
