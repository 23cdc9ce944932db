"""The operators of a serving program together, as it uses them: rotation with storing, attention over 4 bits, forks, compaction, selection of beams and
sequences that follow it; a model's own beam search."""
import math

import pytest
import torch

import card_inputs as ci
from cache4_common import model_freqs, quantised, rotated, values
from test_gpu_beams import _logits as beam_logits

pytestmark = pytest.mark.gpu

SHAPE = ci.ModelShape("mid", 3, 512, 8, 2, 128, 1048, 3001, ctx=200, r=8)
TOY = ci.ModelShape("toy", 2, 256, 6, 2, 64, 256, 997)


@pytest.fixture(scope="module")
def target():
    import paper_2508_04462_amd as card
    from paper_2508_04462_amd.synthetic import load_synthetic_weights

    tgt = card.Target(SHAPE, 256)
    load_synthetic_weights(tgt, SHAPE, 3, 0.2)
    return tgt


def _tokens(stream, n):
    return ci.uniform_tokens(11, "ctx_tokens", stream, n, SHAPE.vocab).tolist()


def _last_logits(tgt, text):
    """Logits of what follows a text, on the Target's own pages."""
    tgt.attach()
    if len(text) > 1:
        tgt.prefill(text[:-1])
    return tgt.verify(len(text) - 1, -1, text[-1:], want_logits=True)["logits"][0].double()


@pytest.mark.parametrize("beams,eos,temperature", [(4, -1, 1.0), (3, 7, 0.7), (1, -1, 1.0)])
def test_beam_search_of_a_target(target, beams, eos, temperature):
    """Against a search that forwards every text from its beginning."""
    import paper_2508_04462_amd as card

    prompt, steps = _tokens(1, 45), 7
    found = [(0.0, [])]
    for step in range(steps):
        more = []
        for score, text in found:
            if text and text[-1] == eos:
                more.append((score, text))
                continue
            p = torch.log_softmax(_last_logits(target, prompt + text) / temperature, 0)
            if eos >= 0 and step == 1:  # (an end among the beams)
                assert p[eos] < p.max()
            best = p.topk(beams + 1)
            more += [(score + float(v), text + [int(t)]) for v, t in zip(*best)]
        more.sort(key=lambda x: -x[0])
        assert all(a[0] - b[0] > 1e-4 for a, b in zip(more[:beams], more[1:])), "the inputs decide nothing"
        found = more[:beams]
    pool = card.SequencePool(SHAPE, 40, 256)
    held = pool.new()
    pool.extend(held, 5)
    target.attach(pool, held)
    try:
        got = target.beam_search(pool, prompt, beams, steps, eos, temperature)
        assert target._attached == (pool, held)
    finally:
        target.attach()
    assert got["tokens"] == [t for _, t in found]
    # (the same positions, forwarded in one go or token by token: sums in another order)
    assert all(abs(a - b) < 2e-3 for a, (b, _) in zip(got["scores"], found))
    assert pool.free_pages == 39


def test_beam_search_that_ends(target):
    """With the most probable token as the end: the first beam ends at once and stays."""
    import paper_2508_04462_amd as card

    prompt = _tokens(2, 20)
    first = int(_last_logits(target, prompt).argmax())
    pool = card.SequencePool(SHAPE, 40, 256)
    got = target.beam_search(pool, prompt, 3, 5, eos=first)
    assert got["tokens"][0] == [first] and pool.free_pages == 40
    assert target.beam_search(pool, prompt, 1, 5, eos=first)["tokens"] == [[first]]
    with pytest.raises(card.CardError) as e:
        target.beam_search(card.SequencePool(SHAPE, 2, 256), prompt, 3, 30)
    assert e.value.status == card.CARD_ECAPACITY and target._attached is None
    with pytest.raises(card.CardError):
        target.beam_search(pool, [], 3, 5)
    with pytest.raises(card.CardError):
        target.beam_search(pool, prompt[:3] + [10 ** 6], 2, 2)
    assert pool.free_pages == 40


def test_pools_of_4_bits_are_not_for_targets(target):
    import paper_2508_04462_amd as card

    pool = card.SequencePool(SHAPE, 8, 256, bits=4)
    with pytest.raises(ValueError):
        target.attach(pool, pool.new())
    with pytest.raises(ValueError):
        card.SequencePool(SHAPE, 8, 256, bits=8)
    with pytest.raises(ValueError):
        card.SequencePool(SHAPE, 8, 256).read(0, 0)


class Layers:
    """A program with layers of its own, in plain torch around the library's operators, and the same on lists in 64 bits."""

    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)
        d, h = TOY.d_model, TOY.head_dim
        self.embed = torch.randn(TOY.vocab, d, generator=g)
        self.head = torch.randn(TOY.vocab, d, generator=g) / d ** 0.5 * 2
        self.qkv = [torch.randn((TOY.n_q_heads + 2 * TOY.n_kv_heads) * h, d, generator=g) / d ** 0.5 for _ in range(TOY.n_layers)]
        self.out = [torch.randn(d, TOY.n_q_heads * h, generator=g) / (TOY.n_q_heads * h) ** 0.5 for _ in range(TOY.n_layers)]

    def split(self, x, layer, w):
        y = (x @ w[layer].T).view(len(x), -1, TOY.head_dim)
        return y.split([TOY.n_q_heads, TOY.n_kv_heads, TOY.n_kv_heads], 1)

    def on_pool(self, pool, plan, tokens, dtype=torch.float32):
        qkv, out = ([w.cuda() for w in ws] for ws in (self.qkv, self.out))
        x = self.embed.cuda()[tokens]
        for layer in range(TOY.n_layers):
            q, k, v = (t.to(dtype) for t in self.split(x, layer, qkv))
            q = pool.append(plan, layer, q, k, v)
            x = x + pool.attend(plan, layer, q, None, None).float().flatten(1) @ out[layer].T
        return x @ self.head.cuda().T

    def on_list(self, text):
        """Logits of what follows every token, the cache as its 4 bits have it (the inputs of a layer come from the layer below on both sides)."""
        x = self.embed[text].double()
        n, h = len(text), TOY.head_dim
        seen = torch.ones(n, n).tril().bool()
        for layer in range(TOY.n_layers):
            q, k, v = self.split(x, layer, [w.double() for w in self.qkv])
            at = torch.arange(n)
            q, k = rotated(q, at, model_freqs(1e4, h))[0], rotated(k, at, model_freqs(1e4, h))[0]
            k, v = values(*quantised(k.float())), values(*quantised(v.float()))
            group = TOY.n_q_heads // TOY.n_kv_heads
            a = [torch.softmax((q[:, i] @ k[:, i // group].T / h ** 0.5).masked_fill(~seen, -math.inf), -1) @ v[:, i // group] for i in range(TOY.n_q_heads)]
            x = x + torch.cat(a, -1) @ self.out[layer].double().T
        return x @ self.head.double().T


def test_beams_on_a_pool_of_4_bits():
    """Two searches at once on one pool: prompts, steps, selection, sequences that follow it; at the end every beam's logits are those of its text."""
    import paper_2508_04462_amd as card

    net, g = Layers(), torch.Generator().manual_seed(5)
    pool = card.SequencePool(TOY, 60, 128, bits=4)
    prompts = [torch.randint(0, TOY.vocab, (n,), generator=g).tolist() for n in (37, 18)]
    seqs = [pool.new() for _ in prompts]
    for s, p in zip(seqs, prompts):
        pool.extend(s, len(p))
    logits = net.on_pool(pool, pool.plan(seqs, [len(p) for p in prompts]), torch.tensor(sum(prompts, [])).cuda())
    logits = logits[torch.tensor([36, 36 + 18]).cuda()]
    scores, groups = torch.zeros(2, 1).cuda(), [[s] for s in seqs]
    texts = [[list(p)] for p in prompts]
    for step in range(12):
        beams = 3
        got = card.beam_select(logits, scores, beams)
        scores = got["scores"]
        parents, tokens = got["parents"].tolist(), got["tokens"].tolist()
        for i in range(2):
            groups[i] = pool.reorder(groups[i], parents[i])
            texts[i] = [texts[i][p] + [t] for p, t in zip(parents[i], tokens[i])]
        flat = groups[0] + groups[1]
        for s in flat:
            pool.extend(s, 1)
        logits = net.on_pool(pool, pool.plan(flat, [1] * 6), got["tokens"].flatten().long())
    assert all(pool.length(s) == len(t) for s, t in zip(groups[0] + groups[1], texts[0] + texts[1]))
    for i, (text, row) in enumerate(zip(texts[0] + texts[1], logits.cpu().double())):
        want = net.on_list(text)[-1]
        # (a code that falls the other way moves a logit by much more than a rounding does, and few do)
        off = (row - want).norm() / want.norm()
        assert off < 2e-2, (i, float(off))
    first = [t[0] for t in texts]
    assert [len(set(map(tuple, t))) for t in texts] == [3, 3] and first[0][:37] == prompts[0]


@pytest.mark.parametrize("bits", [16, 4])
def test_append_then_attend_is_attend_of_rotated_rows(bits):
    """Tokens in two portions, with a fork between them and gaps closed after them, beside the same tokens stored by attend()."""
    import paper_2508_04462_amd as card

    g = torch.Generator().manual_seed(3)
    n, h = 61, TOY.head_dim
    q, k, v = (torch.randn(n, heads, h, generator=g).cuda() for heads in (TOY.n_q_heads, TOY.n_kv_heads, TOY.n_kv_heads))
    pool = card.SequencePool(TOY, 40, 128, bits=bits)
    a, b = pool.new(), pool.new()
    pool.extend(b, n)
    turned = [rotated(x.cpu(), torch.arange(n), model_freqs(1e4, h))[0].float().cuda() for x in (q, k)]
    plan = pool.plan([b], [n])
    want = pool.attend(plan, 1, turned[0], turned[1], v)
    outs = []
    for first, end in ((0, 37), (37, n)):
        pool.extend(a, end - first)
        plan_a = pool.plan([a], [end - first])
        qr = pool.append(plan_a, 1, q[first:end].contiguous(), k[first:end].contiguous(), v[first:end].contiguous())
        outs.append(pool.attend(plan_a, 1, qr, None, None))
        fork = pool.fork(a)
    # cosines and sines in fp32 or 64 bits: 2^-24 of a key's size, which may also take a code or a bf16 across a border
    off = (torch.cat(outs) - want).norm() / want.norm()
    assert off < (1e-3 if bits == 16 else 1e-2), float(off)
    assert torch.equal(pool.append(pool.plan([fork], [0]), 0, q[:0], k[:0], v[:0]), q[:0])
    pool.compact(fork, 5, [9, 20, 33, 34, 60])
    if bits == 4:
        whole, some = pool.read(a, 1), pool.read(fork, 1)
        at = torch.tensor([0, 1, 2, 3, 4, 9, 20, 33, 34, 60]).cuda()
        for x, y in zip(whole, some):
            assert torch.equal(x[at], y)


def test_append_refuses(monkeypatch):
    import paper_2508_04462_amd as card

    pool = card.SequencePool(TOY, 20, 128, bits=4)
    a = pool.new()
    pool.extend(a, 20)
    plan = pool.plan([a], [20])
    q, k = (torch.zeros(20, heads, 64, device="cuda") for heads in (TOY.n_q_heads, TOY.n_kv_heads))
    for bad in (dict(q=k), dict(k=q), dict(k=k[:5]), dict(q=None, out=q), dict(positions=torch.zeros(20, device="cuda")),
                dict(positions=torch.zeros(19, dtype=torch.int32, device="cuda")), dict(positions=torch.zeros(20, dtype=torch.int32))):
        with pytest.raises(ValueError):
            pool.append(plan, 0, **dict(dict(q=q, k=k, v=k), **bad))
    with pytest.raises(card.CardError) as e:
        pool.append(plan, 0, q.bfloat16(), k, k)
    assert e.value.status == card.CARD_EINVAL
    with pytest.raises(card.CardError):
        pool.append(plan, 2, q, k, k)
    with pytest.raises(card.CardError):
        pool.append(plan, 0, q, k, k, freqs=[1.0])
    assert pool.append(plan, 0, None, k, k) is None
    b = pool.fork(a)
    with pytest.raises(card.CardError) as e:
        pool.append(plan, 0, q, k, k)  # to a page that the fork holds
    assert e.value.status == card.CARD_ESTALE
    pool.free(b)
    pool.append(plan, 0, q, k, k)
    pool.truncate(a, 3)
    for first, end in ((0, 4), (-1, 2), (3, 2)):
        with pytest.raises(card.CardError):
            pool.read(a, 0, first, end)
    assert pool.read(a, 0, 3)[0].shape == (0, TOY.n_kv_heads, 64)


def test_operators_in_a_captured_graph():
    """A decoding step of two layers with everything in a graph; between replays other contents, lengths and positions come into its buffers, and eager work runs."""
    import paper_2508_04462_amd as card
    from paper_2508_04462_amd.runtime import _lane_streams

    g = torch.Generator(device="cuda").manual_seed(1)
    pool = card.SequencePool(TOY, 80, 256, bits=4)
    seqs = [pool.new() for _ in range(3)]
    for s, n in zip(seqs, (200, 33, 16)):
        pool.extend(s, n)
    plan = pool.plan(seqs, [200, 33, 16])
    new = lambda n, heads: torch.randn((n, heads, 64), device="cuda", generator=g)  # noqa: E731
    for layer in range(2):
        pool.append(plan, layer, new(249, TOY.n_q_heads), new(249, TOY.n_kv_heads), new(249, TOY.n_kv_heads))
    for s in seqs:
        pool.extend(s, 4)
    plan = pool.plan(seqs, [4, 4, 4])
    q, k, v = new(12, TOY.n_q_heads), new(12, TOY.n_kv_heads), new(12, TOY.n_kv_heads)
    held = [torch.zeros_like(k) for _ in range(2)]
    positions = torch.arange(12, dtype=torch.int32, device="cuda")

    def step():
        outs = []
        for layer in range(2):
            qr = pool.append(plan, layer, q, k, v, positions)
            outs.append(pool.attend(plan, layer, qr, None, None))
        st = card.card_kv4_read(pool.cfg, plan.batch, 1, card.card_rows(held[0]), card.card_rows(held[1]), torch.cuda.current_stream().cuda_stream)
        assert st == card.CARD_OK
        return outs, [t.clone() for t in held]

    side = _lane_streams(torch.device("cuda:0"), 2)[0]  # (of the library's own: with more streams, two of a loop may share a hardware queue)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    full = plan.ctx_lens.clone()
    for i in range(4):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))
        positions.add_(1000 * i)
        plan.ctx_lens.copy_(full - 3 * i)
        pools = [p.clone() for p in (pool.k_pages, pool.v_pages)]
        graph.replay()
        torch.cuda.synchronize()
        after = [p.clone() for p in (pool.k_pages, pool.v_pages)]
        pool.k_pages.copy_(pools[0])
        pool.v_pages.copy_(pools[1])
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got[0] + list(got[1]), want[0] + list(want[1])):
            assert torch.equal(a, b), i
        assert torch.equal(after[0], pool.k_pages) and torch.equal(after[1], pool.v_pages)


def test_beams_in_a_captured_graph():
    """Replays with other logits, scores and lengths in the same buffers, each against the eager call."""
    import paper_2508_04462_amd as card
    from paper_2508_04462_amd.runtime import _lane_streams

    g = torch.Generator().manual_seed(2)
    groups, beams, vocab, most = 4, 5, 30011, 64
    logits, scores = beam_logits(groups * beams, vocab, torch.float32, 1).cuda(), torch.zeros(groups, beams).cuda()
    done, history, lengths = (torch.zeros(s, dtype=torch.int32).cuda() for s in ((groups, beams), (groups, beams, most), (groups,)))
    args = dict(done=done, eos=3, history=history, lengths=lengths)
    side = _lane_streams(torch.device("cuda:0"), 2)[0]  # (of the library's own: with more streams, two of a loop may share a hardware queue)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        card.beam_select(logits, scores, **args)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = card.beam_select(logits, scores, **args)
    for i in range(4):
        logits.copy_(beam_logits(groups * beams, vocab, torch.float32, 10 + i))
        scores.copy_(-torch.rand((groups, beams), generator=g))
        done.copy_((torch.rand((groups, beams), generator=g) < 0.3).int())
        lengths.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        want = card.beam_select(logits, scores, **args)
        torch.cuda.synchronize()
        for name in ("scores", "tokens", "parents", "done"):
            assert torch.equal(out[name], want[name]), (i, name)
        assert torch.equal(out["history"][:, :, :i + 1], want["history"][:, :, :i + 1])


def test_calls_on_another_stream():
    """A plan that is dropped while another stream still works on it; results as on its own stream."""
    import paper_2508_04462_amd as card
    from paper_2508_04462_amd.runtime import _lane_streams

    g = torch.Generator(device="cuda").manual_seed(4)
    pool = card.SequencePool(TOY, 80, 1024, bits=4)
    a = pool.new()
    pool.extend(a, 900)
    new = lambda heads: torch.randn((900, heads, 64), device="cuda", generator=g)  # noqa: E731
    q, k, v = new(TOY.n_q_heads), new(TOY.n_kv_heads), new(TOY.n_kv_heads)
    plan = pool.plan([a], [900])
    want = pool.attend(plan, 0, pool.append(plan, 0, q, k, v), None, None)
    torch.cuda.synchronize()
    side = _lane_streams(torch.device("cuda:0"), 2)[0]
    for _ in range(3):
        plan = pool.plan([a], [900])
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(5):
                qr = pool.append(plan, 0, q, k, v)
                got = pool.attend(plan, 0, qr, None, None)
        del plan
        junk = [torch.full((2 ** 16,), 2 ** 30, dtype=torch.int32, device="cuda") for _ in range(20)]
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        del junk


def test_pages_beyond_4_gib():
    """A layer of a pool of more than 4 GiB, whose last page a text is on, and a pool whose second layer begins behind them."""
    import paper_2508_04462_amd as card

    shape = ci.ModelShape("wide", 2, 256, 64, 64, 128, 256, 64)
    cfg = card.make_cfg(shape, 64)
    n_pages = (1 << 32) // (64 * 1152) + 7
    assert card.card_kv4_pool_bytes(cfg, n_pages) > 2 << 32
    pool = card.SequencePool(shape, n_pages, 64, bits=4)
    a = pool.new()
    pool._free = list(range(n_pages))  # (the last page is taken first)
    pool.extend(a, 16)
    assert pool._seqs[a].pages == [n_pages - 1]
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn((16, 64, 128), device="cuda", generator=g) for _ in range(3))
    small = card.SequencePool(shape, 4, 64, bits=4)
    b = small.new()
    small.extend(b, 16)
    for layer in range(2):
        outs = []
        for p, s in ((pool, a), (small, b)):
            plan = p.plan([s], [16])
            outs.append((p.attend(plan, layer, p.append(plan, layer, q, k, v), None, None), *p.read(s, layer)))
        for x, y in zip(*outs):
            assert torch.equal(x, y)
    c = pool.fork(a)
    pool.extend(c, 3)
    pool.compact(c, 2, [5, 9, 16])
    assert pool._seqs[c].pages == [n_pages - 3]
    for got, want in zip(pool.read(c, 1), pool.read(a, 1)):
        assert torch.equal(got[:4], want[[0, 1, 5, 9]])
