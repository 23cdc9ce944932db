"""Several sequences on one pool: steps, prompts, drafts, attention, compaction and scores together, as a serving program uses them."""
import math

import pytest
import torch

import card_inputs as ci

pytestmark = pytest.mark.gpu

SHAPE = ci.ModelShape("mid", 3, 512, 8, 2, 128, 1048, 3001, ctx=200, r=8)


@pytest.fixture(scope="module")
def target():
    import paper_2508_04462_amd as card
    from paper_2508_04462_amd.synthetic import load_synthetic_weights

    tgt = card.Target(SHAPE, 512)
    load_synthetic_weights(tgt, SHAPE, 3, 0.2)
    return tgt


def _tokens(stream, n):
    return ci.uniform_tokens(11, "ctx_tokens", stream, n, SHAPE.vocab).tolist()


def _step(tgt, ctx, cand):
    res = tgt.verify(ctx, -1, cand, want_logits=True)
    assert res["accepted_len"] >= 0
    return res["logits"]


def test_forks_share_a_prompt_and_go_on_apart(target):
    """Three texts with one prompt: every step's logits are those, bit for bit, of a model that has a text to itself."""
    import paper_2508_04462_amd as card

    prompt, ends = _tokens(0, 150), [_tokens(s, 24) for s in (1, 2, 3)]
    want = []
    target.attach()
    for end in ends:
        target.prefill(prompt)
        want.append([_step(target, 150 + 8 * i, end[8 * i:8 * i + 8]) for i in range(3)])
    pool = card.SequencePool(SHAPE, 24, 512)
    a = pool.new()
    pool.extend(a, 150)
    target.attach(pool, a)
    try:
        target.prefill(prompt)
        used = 24 - pool.free_pages
        seqs = [a, pool.fork(a), pool.fork(a)]
        assert 24 - pool.free_pages == used + 2  # a copy of the last page each
        for i in range(3):
            for seq, end, logits in zip(seqs, ends, want):
                pool.extend(seq, 8)
                target.attach(pool, seq)
                assert torch.equal(_step(target, 150 + 8 * i, end[8 * i:8 * i + 8]), logits[i])
        with pytest.raises(card.CardError) as e:
            _step(target, 174, ends[2][:1])  # not extended to it
        assert e.value.status == card.CARD_ECAPACITY
        with pytest.raises(card.CardError):
            target.prefill(prompt)  # over pages that the forks hold
        with pytest.raises(ValueError):
            target.attach(card.SequencePool(ci.SHAPES["tiny"], 2, 64), 0)
    finally:
        target.attach()


def test_attach_refuses_shorter_tables(target):
    """A pool whose block tables end before the model's max_ctx."""
    import paper_2508_04462_amd as card

    pool = card.SequencePool(SHAPE, 8, 496)
    with pytest.raises(ValueError):
        target.attach(pool, pool.new())
    with pytest.raises(KeyError):
        target.attach(card.SequencePool(SHAPE, 8, 528), 0)
    target.attach()


def _cache(tgt, positions):
    got = [tgt.kv_gather(l, 0, max(positions) + 1) for l in range(SHAPE.n_layers)]
    return [(k[positions], v[positions]) for k, v in got]


def test_accepted_nodes_of_a_tree_become_text(target):
    """Two levels of a draft's tree; the accepted nodes' keys and values move behind the text, beside a fork that keeps the tree, and the next step
    sees them as if they had been forwarded there."""
    import paper_2508_04462_amd as card

    ctx, prompt = 100, _tokens(4, 100)
    pool = card.SequencePool(SHAPE, 40, 512)
    a = pool.new()
    pool.extend(a, ctx)
    target.attach(pool, a)
    try:
        target.prefill(prompt)
        base, words = ctx // 16 * 16, 2
        level1, level2 = _tokens(5, 5), _tokens(6, 9)
        parents = [0, 0, 1, 1, 2, 3, 3, 4, 4]
        pool.extend(a, 14)
        _, rows1 = card.card_tree_mask_level(None, [-1] * 5, ctx, ctx, base, words)
        target.draft_level(ctx, level1, [ctx] * 5, ctx, rows1, base, 4)
        _, rows2 = card.card_tree_mask_level(rows1, parents, ctx + 5, ctx, base, words)
        target.draft_level(ctx, level2, [ctx + 1] * 9, ctx + 5, rows2, base, 4)
        tree = pool.fork(a)
        node1, node2 = 3, 6  # the second a child of the first
        before = _cache(target, list(range(ctx)) + [ctx + node1, ctx + 5 + node2])
        whole = _cache(target, list(range(ctx + 14)))
        pool.compact(a, ctx, [ctx + node1, ctx + 5 + node2])
        assert pool.length(a) == ctx + 2
        after = _cache(target, list(range(ctx + 2)))
        for (k0, v0), (k1, v1) in zip(before, after):
            assert torch.equal(k0, k1) and torch.equal(v0, v1)
        target.attach(pool, tree)  # the fork has the tree as it was
        for (k0, v0), (k1, v1) in zip(whole, _cache(target, list(range(ctx + 14)))):
            assert torch.equal(k0, k1) and torch.equal(v0, v1)
        target.attach(pool, a)
        pool.extend(a, 4)
        got = _step(target, ctx + 2, _tokens(7, 4))
        target.attach()
        target.prefill(prompt)
        _step(target, ctx, [level1[node1], level2[node2]])
        want = _step(target, ctx + 2, _tokens(7, 4))
        # (the nodes were forwarded by other kernels: sums in another order, two of them rounded to bf16 in the cache)
        assert float((got - want).abs().max() / want.abs().max()) <= 2e-2
    finally:
        target.attach()


def test_attention_over_what_steps_have_stored(target):
    """pool.attend reads pages that prompts and steps wrote, and stores tokens that steps then read."""
    import paper_2508_04462_amd as card

    pool = card.SequencePool(SHAPE, 40, 512)
    lens, new = [150, 33], [5, 2]
    seqs = []
    try:
        for s, n in enumerate(lens):
            seqs.append(pool.new())
            pool.extend(seqs[-1], n)
            target.attach(pool, seqs[-1])
            target.prefill(_tokens(20 + s, n))
        for seq, n in zip(seqs, new):
            pool.extend(seq, n)
        plan = pool.plan(seqs, new)
        g = torch.Generator().manual_seed(1)
        q, k, v = (torch.randn((7, heads, 128), generator=g).bfloat16().cuda() for heads in (8, 2, 2))
        layer = 1
        out = pool.attend(plan, layer, q, k, v)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            again = pool.attend(pool.plan(seqs, new), layer, q, None, None)
        torch.cuda.current_stream().wait_stream(other)
        torch.cuda.synchronize()
        assert torch.equal(out, again)
        row = 0
        for seq, n0, n1 in zip(seqs, lens, new):
            target.attach(pool, seq)
            kk, vv = target.kv_gather(layer, 0, n0 + n1)
            assert torch.equal(kk[n0:], k[row:row + n1].float().cpu()) and torch.equal(vv[n0:], v[row:row + n1].float().cpu())
            for head in range(8):
                score = q[row:row + n1, head].double().cpu() @ kk[:, head // 4].double().T / math.sqrt(128)
                score = score.masked_fill(torch.arange(n0 + n1)[None, :] > n0 + torch.arange(n1)[:, None], -math.inf)
                p = score.softmax(-1)
                want, mean_abs = p @ vv[:, head // 4].double(), p @ vv[:, head // 4].double().abs()
                # weights and output are rounded to bf16 once each
                assert ((out[row:row + n1, head].double().cpu() - want).abs() <= (mean_abs + want.abs()) * 2.0 ** -8 * 1.01 + 1e-4 * mean_abs).all()
            row += n1
        with pytest.raises(ValueError):
            pool.attend(plan, layer, q[:6], k, v)
        with pytest.raises(ValueError):
            pool.attend(plan, layer, q, k, v, mask=torch.zeros((7, 1), dtype=torch.int32, device="cuda"))
        with pytest.raises(card.CardError):
            pool.attend(plan, 3, q, k, v)
    finally:
        target.attach()


@pytest.mark.parametrize("n,top,temperature", [(1, 0, 1.0), (45, 5, 0.7), (32, 1, 1.0)])
def test_score_of_a_text(target, n, top, temperature):
    """Log probabilities of a text against a softmax in 64 bits of the logits that verification gives."""
    import paper_2508_04462_amd as card

    ctx, text = 20, _tokens(30, 20 + n)
    target.attach()
    target.prefill(text[:ctx])
    got = target.score(text[ctx:], ctx, top, temperature)
    target.prefill(text[:ctx])
    logits = torch.cat([_step(target, ctx + s, text[ctx + s:ctx + min(n, s + 32)]) for s in range(0, n, 32)])
    p = torch.log_softmax(logits.double() / temperature, -1)
    entropy = -(p.exp() * p).sum(-1)
    # a dozen roundings of values below 2^4 or so, and the sum of 3001 terms
    tol = 2.0 ** -24 * (16 * p.abs().max() + 3001 / 64 + 64)
    assert got["logprob"].shape == (n - 1,) and ("top_tokens" in got) == (top > 0)
    want = p[torch.arange(n - 1), torch.tensor(text[ctx + 1:], dtype=torch.long)]
    assert ((got["logprob"].cpu().double() - want).abs() <= tol).all()
    assert ((got["entropy"].cpu().double() - entropy).abs() <= 4 * tol).all()
    if top:
        best = logits.sort(dim=-1, descending=True, stable=True)
        assert torch.equal(got["top_tokens"].cpu().long(), best.indices[:, :top])
        assert ((got["top_logprobs"].cpu().double() - p.gather(1, best.indices[:, :top])).abs() <= tol).all()
    one = card.token_logprobs(logits.cuda(), torch.tensor(text[ctx + 1:] + [-1], dtype=torch.int32, device="cuda"), top, temperature)
    assert torch.equal(one["entropy"], got["entropy"]) and torch.equal(one["logprob"][:n - 1], got["logprob"])


def test_score_refuses(target):
    import paper_2508_04462_amd as card

    target.attach()
    for bad in (lambda: target.score([]), lambda: target.score([1, SHAPE.vocab]), lambda: target.score([1, 2], 511), lambda: target.score([1, 2], top=33)):
        with pytest.raises(card.CardError):
            bad()
    with pytest.raises(ValueError):
        card.token_logprobs(torch.zeros((2, 10), device="cuda"), torch.zeros(2, device="cuda"))
