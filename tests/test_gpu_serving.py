"""card_kv_attend, card_kv_copy_pages, card_kv_move_slots and card_logprobs on the GPU against their definitions in 64 bits."""
import math

import pytest
import torch

import card_inputs as ci
from serving_common import PAGE, Batch, k_places, logprob_reference, v_places

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _cfg(heads, layers=2):
    import paper_2508_04462_amd as card

    q_heads, kv_heads, h = heads
    return card.make_cfg(ci.ModelShape("heads", layers, 256, q_heads, kv_heads, h, 256, 64), 4096)


class Call:
    """One batch on the GPU, its buffers and its arguments."""

    def __init__(self, b, max_new=None, max_len=None, out_fill=7.0, stored=False):
        import paper_2508_04462_amd as card

        self.b, self.cfg = b, _cfg((b.q_heads, b.kv_heads, b.h), b.k_pool.shape[0])
        self.k_pool, self.v_pool, self.tables = b.k_pool.cuda(), b.v_pool.cuda(), b.tables.cuda()
        self.ctx, self.starts = b.ctx.cuda(), b.starts.cuda()
        self.q, self.k, self.v = (self._like(t) for t in (b.q, b.k, b.v))
        self.out = torch.full((b.n_rows, b.q_heads, b.h), out_fill, dtype=b.dtype, device="cuda")
        most_new = max(n for _, n in b.lens) if max_new is None else max_new
        most = max(c + n for c, n in b.lens) if max_len is None else max_len
        self.batch = card.CardKVBatch(self.k_pool.data_ptr(), self.v_pool.data_ptr(), b.n_pages, len(b.lens), self.tables.data_ptr(), b.width,
                                      b.n_rows, self.ctx.data_ptr(), self.starts.data_ptr(), most_new, most)
        self.mask = None
        if b.mask is not None:
            self.mask_dev, self.base_dev = b.mask.cuda(), b.mask_base.cuda()
            self.mask = card.CardRowMask(self.mask_dev.data_ptr(), self.base_dev.data_ptr(), b.mask.shape[1])
        self.stored = stored
        self.ws = torch.full((card.card_kv_attend_workspace_bytes(self.cfg, self.batch),), 0xA5, dtype=torch.uint8, device="cuda")

    @staticmethod
    def _like(t):
        """On the GPU with the same strides."""
        span = 1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
        flat = torch.as_strided(t, (span,), (1,)).cuda()
        return torch.as_strided(flat, t.shape, t.stride())

    def run(self):
        import paper_2508_04462_amd as card

        k, v = (None, None) if self.stored else (card.card_rows(self.k), card.card_rows(self.v))
        st = card.card_kv_attend(self.cfg, self.batch, self.b.layer, card.card_rows(self.q), k, v, card.card_rows(self.out), self.mask, self.ws,
                                 torch.cuda.current_stream().cuda_stream)
        assert st == card.CARD_OK, card.card_strerror(st)
        return self

    def check(self, ref=None):
        torch.cuda.synchronize()
        out, mean_abs, score_abs, kp, vp = ref or self.b.reference()
        got, rows = self.out.cpu(), int(self.b.starts[-1])
        err = (got.double() - out).abs()[:rows]
        tol = self.b.tolerance(out, mean_abs, score_abs)[:rows]
        assert torch.isfinite(got[:rows].double()).all()
        worst = float((err / tol.clamp(min=1e-30)).max()) if rows else 0.0
        assert worst <= 1.0, worst
        assert (got[rows:] == 7.0).all()
        if not self.stored:
            for g, w in ((self.k_pool, kp), (self.v_pool, vp)):
                assert torch.equal(g.cpu().view(torch.int16), w.view(torch.int16))
        return worst


HEADS = [(4, 2, 64), (10, 2, 128), (7, 1, 128), (8, 8, 64), (34, 2, 64), (28, 4, 128), (48, 1, 128)]
LENS = [
    [(0, 1)],
    [(15, 1), (16, 1), (17, 1), (0, 1)],
    [(0, 33), (100, 5), (7, 0), (31, 17), (0, 0), (1, 1)],
    [(2047, 3)],
    [(5, 130), (300, 1)],
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens", LENS, ids=lambda v: "+".join("%d_%d" % x for x in v))
@pytest.mark.parametrize("heads", HEADS, ids=lambda v: "%dx%dx%d" % v)
def test_attend_causal(heads, lens, dtype):
    b = Batch(heads, lens, dtype, seed=len(lens))
    ref = b.reference()
    first = Call(b).run()
    first.check(ref)
    # the same rows again, now that the cache holds their keys and values
    again = Call(b, stored=True)
    again.k_pool, again.v_pool = first.k_pool, first.v_pool
    again.batch.k_pages, again.batch.v_pages = first.k_pool.data_ptr(), first.v_pool.data_ptr()
    again.run().check(ref)


@pytest.mark.parametrize("order", ["fused", "heads"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_attend_reads_rows_as_they_lie(order, dtype):
    Call(Batch((10, 2, 128), [(40, 20), (3, 1)], dtype, order=order, extra_rows=5)).run().check()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128)], ids=lambda v: "%dx%dx%d" % v)
def test_attend_under_tree_masks(heads, dtype):
    lens = [(70, 40), (16, 9), (0, 3), (129, 1)]
    Call(Batch(heads, lens, dtype, fill=0.0).tree_mask(density=0.3)).run().check()
    # a mask that ends before the sequence does, one from slot 0 on, and rows that see nothing
    Call(Batch(heads, lens, dtype, fill=0.0).tree_mask(words=1, bases=[64, 0, 0, 128])).run().check()
    c = Call(Batch(heads, lens, dtype, fill=0.0).tree_mask(empty=True)).run()
    c.check()
    assert (c.out[::2] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128), (40, 2, 64), (7, 1, 128)], ids=lambda v: "%dx%dx%d" % v)
def test_attend_of_few_rows_under_tree_masks(heads, dtype):
    lens = [(70, 3), (16, 1), (0, 2), (530, 3)]
    Call(Batch(heads, lens, dtype).tree_mask(density=0.5)).run().check()
    Call(Batch(heads, lens, dtype).tree_mask(words=2, bases=[16, 0, 0, 512])).run().check()
    c = Call(Batch(heads, lens, dtype).tree_mask(empty=True)).run()
    c.check()
    assert (c.out[::2] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,new", [((8, 8, 64), (16, 17, 64, 65)), ((4, 2, 64), (8, 9, 63, 64, 65, 128, 129)), ((4, 1, 128), (4, 5, 64, 65, 80)),
                                       ((8, 1, 64), (2, 3, 32, 33))], ids=lambda v: "_".join("%d" % x for x in v))
def test_attend_at_the_ends_of_its_variants(heads, new, dtype):
    """As many rows x heads as one kind of workgroup takes, and one token more, behind texts of several lengths."""
    for n in new:
        lens = [(19, 1), (419, n), (0, n), (3, 0)]
        Call(Batch(heads, lens, dtype, seed=n)).run().check()
        masked = Batch(heads, lens, dtype, seed=n).tree_mask(density=0.4)
        ref = masked.reference()
        first = Call(masked).run()
        first.check(ref)
        again = Call(masked, stored=True)
        again.k_pool.copy_(first.k_pool)
        again.v_pool.copy_(first.v_pool)
        again.run().check(ref)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,new", [((4, 2, 64), (1, 9, 64, 129)), ((4, 1, 128), (2, 20, 65)), ((20, 2, 128), (1, 3, 30))],
                         ids=lambda v: "_".join("%d" % x for x in v))
def test_attend_of_texts_in_cuts(heads, new, dtype):
    """Texts of which the longest is cut, some ending in its first cuts."""
    for n in new:
        lens = [(0, n), (1711, n), (130, 1), (900, 0), (701, n // 2 + 1)]
        Call(Batch(heads, lens, dtype, seed=n)).run().check()
        masked = Batch(heads, lens, dtype, seed=n).tree_mask(density=0.4)
        ref = masked.reference()
        first = Call(masked).run()
        first.check(ref)
        again = Call(masked, stored=True)
        again.k_pool.copy_(first.k_pool)
        again.v_pool.copy_(first.v_pool)
        again.run().check(ref)
        blind = Call(Batch(heads, lens, dtype, seed=n).tree_mask(empty=True)).run()
        blind.check()
        assert (blind.out[::2] == 0).all()


def test_one_graph_of_the_operators():
    """Page copies, moves, attention and log probabilities captured together; the lists stay with the graph.  Replayed with the program's own
    work between, every replay is the eager calls' result."""
    import paper_2508_04462_amd as card

    heads, layers = (10, 2, 128), 2
    cfg = _cfg(heads, layers)
    b = Batch(heads, [(100, 3), (700, 1), (40, 2)], BF16, layers=layers, seed=8, fill=0.0, spare=4)
    pages = [p for p in range(b.n_pages) if p not in set(b.tables[b.tables < 2 ** 30].tolist())]
    first = int(b.tables[0, 0])
    call = Call(b)
    logits = (torch.randn((9, 5000), generator=torch.Generator().manual_seed(1)) * 3).cuda()
    tokens = torch.arange(9, dtype=torch.int32, device="cuda")
    got = [torch.empty(9, device="cuda"), torch.empty(9, device="cuda"), torch.empty((9, 4), dtype=torch.int32, device="cuda"), torch.empty((9, 4), device="cuda")]
    ws = torch.empty(card.card_logprobs_workspace_bytes(9, 5000, 4), dtype=torch.uint8, device="cuda")

    def all_of_them():
        stream = torch.cuda.current_stream().cuda_stream
        kv = card.CardKV(call.k_pool.data_ptr(), call.v_pool.data_ptr(), None, b.n_pages, -1)
        src, dst = [first], [pages[0]]
        assert card.card_kv_copy_pages(cfg, kv, src, dst, stream) == card.CARD_OK
        src[0] = dst[0] = -1  # read during the call only
        slots = [first * PAGE + 2, first * PAGE + 5], [first * PAGE, first * PAGE + 1]
        assert card.card_kv_move_slots(cfg, kv, *slots, stream) == card.CARD_OK
        call.run()
        assert card.card_logprobs(logits, tokens, 1.0, 4, *got, ws, stream) == card.CARD_OK

    def state():
        torch.cuda.synchronize()
        return [t.clone() for t in (call.out, call.k_pool, call.v_pool, *got)]

    def reset(turn):
        call.k_pool.copy_(b.k_pool)
        call.v_pool.copy_(b.v_pool)
        call.out.fill_(7.0)
        logits.mul_(1.0 + 0.1 * turn)
        for t in got:
            t.zero_()

    graph = torch.cuda.CUDAGraph()
    all_of_them()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        all_of_them()
    for turn in range(4):
        kept = logits.clone()
        reset(turn)
        all_of_them()
        want = state()
        logits.copy_(kept)
        reset(turn)
        graph.replay()
        for w, g in zip(want, state()):
            assert torch.equal(w, g)
        assert int(got[2].min()) >= 0 and not torch.equal(call.k_pool.cpu(), b.k_pool)


def test_attend_over_what_the_cache_holds_already():
    b = Batch((10, 2, 128), [(40, 20), (3, 1)], BF16)
    first = Call(b).run()
    first.check()
    again = Call(b, stored=True)
    again.k_pool.copy_(first.k_pool)
    again.v_pool.copy_(first.v_pool)
    again.run().check()
    assert torch.equal(first.out, again.out)


@pytest.mark.parametrize("hints", [(0, 0), (1, 16), (500, 60000)])
def test_attend_is_right_whatever_the_bounds_say(hints):
    Call(Batch((8, 2, 128), [(700, 40), (33, 1), (0, 3)], BF16, slack=3), max_new=hints[0], max_len=hints[1]).run().check()
    Call(Batch((4, 2, 64), [(30, 100), (0, 0), (5, 70)], F32), max_new=hints[0], max_len=hints[1]).run().check()
    Call(Batch((10, 2, 128), [(130, 100), (0, 65)], BF16).tree_mask(), max_new=hints[0], max_len=hints[1]).run().check()


def test_attend_of_many_sequences():
    """More than the 64 that one look at the row starts takes in; lengths of zero among them."""
    g = torch.Generator().manual_seed(4)
    lens = [(int(c), int(n)) for c, n in zip(torch.randint(0, 90, (150,), generator=g), torch.randint(0, 4, (150,), generator=g))]
    Call(Batch((4, 2, 64), lens, BF16)).run().check()
    Call(Batch((8, 2, 64), [(c, 1) for c, _ in lens[:70]] + [(2000, 1)], F32)).run().check()


def test_attend_of_thousands_of_sequences():
    lens = [(i % 5, 1 if i % 7 else 0) for i in range(4200)]
    Call(Batch((2, 1, 64), lens, BF16)).run().check()


def test_attend_far_apart_scores():
    """Scores that differ by hundreds: weights that vanish, a maximum that moves late."""
    b = Batch((4, 2, 64), [(200, 20)], F32)
    b.q = b.q * 60.0
    ref = b.reference()
    Call(b).run().check(ref)


@pytest.mark.parametrize("heads,lens", [((8, 2, 128), [(700, 3)]), ((8, 2, 64), [(700, 3)]), ((8, 2, 128), [(300, 150), (2000, 20)])],
                         ids=["few_128", "few_64", "many"])
def test_attend_keeps_the_bits_of_fp32(heads, lens):
    """The mean error, where roundings add as squares.  q and k are N(0, 1): a score and its partial sums have magnitude 1 or less, so the 3 h additions
    of three-part products leave sqrt(3 h) 2^-24 / sqrt(3); so does a weight, relative to itself, with a handful more from exp2; partial sums of the
    output are no larger than itself, and n keys leave sqrt(n) 2^-24 / sqrt(3).  q in two parts alone would leave 2^-17 / sqrt(3) = 4.4e-6, beyond the bound."""
    b = Batch(heads, lens, F32, seed=3)
    out, mean_abs, score_abs, _, _ = ref = b.reference()
    c = Call(b).run()
    c.check(ref)
    err = c.out.cpu().double() - out
    n = max(c + m for c, m in lens)
    bound = 2.0 ** -24 * (math.sqrt(heads[2] + 8) + math.sqrt(n / 3))
    assert bound < 2.0 ** -17 / math.sqrt(3)
    assert float(err.square().mean().sqrt()) <= bound * float(out.square().mean().sqrt())


def test_attend_with_pages_that_are_not_there():
    """A page id outside the pool, and a text longer than its table: such tokens are not stored and not seen."""
    b = Batch((4, 2, 64), [(40, 6), (20, 2)], BF16, fill=0.0)
    c = Call(b)
    c.tables[0, 1] = b.n_pages
    c.tables[1, 1] = -5
    before = c.k_pool.clone()
    c.run()
    torch.cuda.synchronize()
    # the same with the missing slots masked away
    bases, words = [0, 0], 2
    m = Batch((4, 2, 64), [(40, 6), (20, 2)], BF16, fill=0.0).tree_mask(words=words, bases=bases)
    m.bits[:] = False
    for r in range(6):
        m.bits[r, :16], m.bits[r, 32:40 + r + 1] = True, True
    m.bits[6:, :16] = True
    out, mean_abs, score_abs, _, _ = m.reference()
    err = (c.out.cpu().double() - out).abs()
    assert (err <= m.tolerance(out, mean_abs, score_abs)).all()
    changed = (c.k_pool != before).flatten(2).any(-1)
    assert changed[1].nonzero().flatten().tolist() == [int(b.tables[0, 2])] and not changed[0].any()


def test_attend_beyond_four_gib():
    """Pages whose offset in the layer passes 32 bits."""
    heads, lens = (8, 8, 128), [(35, 2)]
    b = Batch(heads, lens, BF16, layers=1, layer=0)
    c = Call(b)
    far = (1 << 32) // (8 * 16 * 128 * 2) + 1000
    k_pool = torch.empty((1, far + b.n_pages, 8, PAGE * 128), dtype=BF16, device="cuda")
    v_pool = torch.empty_like(k_pool)
    k_pool[0, far:], v_pool[0, far:] = c.k_pool[0], c.v_pool[0]
    c.tables += far
    c.batch.k_pages, c.batch.v_pages, c.batch.n_pages = k_pool.data_ptr(), v_pool.data_ptr(), far + b.n_pages
    c.run()
    c.k_pool, c.v_pool = k_pool[:, far:], v_pool[:, far:]
    c.check()


def test_attend_in_a_graph_with_other_lengths():
    """A captured call reads its lengths when it is replayed; every replay is compared with the eager call."""
    lens = [[(50, 3), (0, 9), (600, 1)], [(90, 1), (17, 12), (3, 0)], [(0, 5), (640, 7), (15, 1)]]
    calls = [Call(Batch((10, 2, 128), x, BF16, seed=i, fill=0.0)) for i, x in enumerate(lens)]
    pages, rows = max(c.b.n_pages for c in calls), max(c.b.n_rows for c in calls)
    width = max(c.b.width for c in calls)
    box = Batch((10, 2, 128), [(0, 0)] * 3, BF16, spare=pages, extra_rows=rows, slack=width - 1, fill=0.0)
    g = Call(box, max_new=12, max_len=650)
    g.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.run()
    for c in calls + calls[:1]:
        ref = c.b.reference()
        g.k_pool[:, :c.b.n_pages], g.v_pool[:, :c.b.n_pages] = c.b.k_pool.cuda(), c.b.v_pool.cuda()
        g.tables[:, :c.b.width], g.ctx[:], g.starts[:] = c.b.tables.cuda(), c.b.ctx.cuda(), c.b.starts.cuda()
        for name in ("q", "k", "v"):
            getattr(g, name)[:c.b.n_rows] = getattr(c, name)
        g.out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        out, mean_abs, score_abs, kp, vp = ref
        err = (g.out[:c.b.n_rows].cpu().double() - out).abs()
        assert (err <= c.b.tolerance(out, mean_abs, score_abs)).all()
        assert (g.out[c.b.n_rows:] == 7.0).all()
        assert torch.equal(g.k_pool[:, :c.b.n_pages].cpu(), kp) and torch.equal(g.v_pool[:, :c.b.n_pages].cpu(), vp)


# ---- pages and slots ----------------------------------------------------------------------------------


def _pools(layers, pages, kv_heads, h, seed=0):
    """Every bit pattern, NaN ones included: copies are of bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (layers, pages, kv_heads, PAGE * h)
    return [torch.randint(-32768, 32767, shape, dtype=torch.int16, device="cuda", generator=g) for _ in range(2)]


def _copy(cfg, pools, src, dst, call="card_kv_copy_pages"):
    import paper_2508_04462_amd as card

    kv = card.CardKV(pools[0].data_ptr(), pools[1].data_ptr(), None, pools[0].shape[1], -1)
    st = getattr(card, call)(cfg, kv, src, dst, torch.cuda.current_stream().cuda_stream)
    assert st == card.CARD_OK, card.card_strerror(st)
    torch.cuda.synchronize()


@pytest.mark.parametrize("heads,layers,n", [((4, 2, 64), 2, 1), ((7, 1, 64), 1, 5), ((6, 3, 128), 5, 40), ((8, 8, 128), 3, 700)])
def test_copy_pages(heads, layers, n):
    pools = _pools(layers, 2 * n + 3, heads[1], heads[2])
    order = torch.randperm(2 * n + 3, generator=torch.Generator().manual_seed(n)).tolist()
    src, dst = order[:n], order[n:2 * n]
    src[-1] = src[0]  # one page to two places
    want = [p.clone() for p in pools]
    for p in want:
        p[:, dst] = p[:, src]
    _copy(_cfg(heads, layers), pools, src, dst)
    assert all(torch.equal(p, w) for p, w in zip(pools, want))


def _move_reference(pools, h, src, dst):
    """One move after the other."""
    want = [p.cpu() for p in pools]
    for s, d in zip(src, dst):
        for p, places in zip(want, (k_places, v_places)):
            i, o = places(torch.tensor([s % PAGE]), h)[0], places(torch.tensor([d % PAGE]), h)[0]
            p[:, d // PAGE, :, o] = p[:, s // PAGE, :, i]
    return want


def _move_lists(kind, pages, seed):
    g = torch.Generator().manual_seed(seed)
    slots = pages * PAGE
    if kind == "one":
        return [slots - 1], [0]
    if kind == "itself":
        return [3, 40], [3, 41]
    if kind == "scattered":  # from one half of the slots to the other
        order = torch.randperm(slots, generator=g).tolist()
        n = slots // 2
        return order[:n], order[n:2 * n]
    if kind == "same source":
        return [7] * 40, list(range(32, 72))
    drop = {"gaps": 0.3, "one gap": 0.0, "half": 0.5}[kind]
    kept = (torch.rand(slots, generator=g) >= drop).nonzero().flatten().tolist()
    kept = [k for k in kept if k >= 6]  # (at least a shift of one: the front goes)
    return kept, [5 + i for i in range(len(kept))]


@pytest.mark.parametrize("kind", ["one", "itself", "scattered", "same source", "gaps", "one gap", "half"])
@pytest.mark.parametrize("heads,layers,pages", [((4, 2, 64), 2, 12), ((3, 3, 128), 3, 9), ((2, 1, 128), 1, 70)])
def test_move_slots(heads, layers, pages, kind):
    src, dst = _move_lists(kind, pages, pages)
    pools = _pools(layers, pages, heads[1], heads[2], seed=pages)
    want = _move_reference(pools, heads[2], src, dst)
    _copy(_cfg(heads, layers), pools, src, dst, "card_kv_move_slots")
    assert all(torch.equal(p.cpu(), w) for p, w in zip(pools, want))


@pytest.mark.parametrize("at", [0, 3])
def test_move_slots_in_lists_of_every_length(at):
    """Lengths about those of a round and of a launch, the tokens closing up from place `at` of a page on."""
    heads, pages = (2, 1, 64), 64
    for n in (2, 31, 32, 33, 95, 96, 97, 191, 192, 193, 221, 224, 225, 288, 289, 477, 480, 481, 673):
        g = torch.Generator().manual_seed(n)
        src = sorted(torch.randperm(pages * PAGE - at - 1, generator=g)[:n].add(at + 1).tolist())
        dst = [at + i for i in range(n)]
        pools = _pools(1, pages, heads[1], heads[2], seed=n)
        want = _move_reference(pools, heads[2], src, dst)
        _copy(_cfg(heads, 1), pools, src, dst, "card_kv_move_slots")
        assert all(torch.equal(p.cpu(), w) for p, w in zip(pools, want)), n


def test_copies_and_moves_beyond_four_gib():
    heads, pages = (8, 8, 128), (1 << 32) // (8 * 16 * 128 * 2) + 50
    pools = [torch.zeros((2, pages, 8, PAGE * 128), dtype=torch.int16, device="cuda") for _ in range(2)]
    for i, p in enumerate(pools):
        p[:, pages - 2] = torch.arange(8 * PAGE * 128, device="cuda").view(8, -1).to(torch.int16) + i
    _copy(_cfg(heads, 2), pools, [pages - 2], [pages - 1])
    assert all(torch.equal(p[:, pages - 1], p[:, pages - 2]) for p in pools)
    _copy(_cfg(heads, 2), pools, [pages * PAGE - 20], [3], "card_kv_move_slots")
    t = torch.tensor([12, 3])
    for p, places in zip(pools, (k_places, v_places)):
        at = places(t, 128).cuda()
        assert torch.equal(p[:, 0][:, :, at[1]], p[:, pages - 2][:, :, at[0]])


# ---- log probabilities --------------------------------------------------------------------------------


def _logprobs(logits, tokens, temperature, top):
    import paper_2508_04462_amd as card

    rows, vocab = logits.shape
    dev = dict(device="cuda")
    lp, en = torch.full((rows,), 9.0, **dev), torch.full((rows,), 9.0, **dev)
    tt, tl = torch.full((rows, top), 9, dtype=torch.int32, **dev), torch.full((rows, top), 9.0, **dev)
    ws = torch.full((card.card_logprobs_workspace_bytes(rows, vocab, top),), 0xA5, dtype=torch.uint8, **dev)
    tok = None if tokens is None else tokens.to(torch.int32).cuda()
    st = card.card_logprobs(logits, tok, temperature, top, None if tokens is None else lp, en, tt, tl, ws, torch.cuda.current_stream().cuda_stream)
    assert st == card.CARD_OK, card.card_strerror(st)
    torch.cuda.synchronize()
    return lp.cpu(), en.cpu(), tt.cpu(), tl.cpu()


def _check_logprobs(logits, tokens, temperature, top):
    """logits: on the CPU, any strides.  A difference d = (x - max) / T carries three roundings, its exponential those and 2 ulp more; the sum is
    taken in at most vocab / 64 + 64 steps; the entropy weighs |d| with the probabilities, one more rounding each."""
    span = 1 + sum((n - 1) * s for n, s in zip(logits.shape, logits.stride()))
    on_gpu = torch.as_strided(torch.as_strided(logits, (span,), (1,)).cuda(), logits.shape, logits.stride())
    lp, en, tt, tl = _logprobs(on_gpu, tokens, temperature, top)
    want_lp, want_en, want_tt, want_tl = logprob_reference(logits, tokens, temperature, top)
    assert torch.equal(tt.long(), want_tt)
    ulp = 2.0 ** -24
    x = logits.double()
    peak = torch.where(torch.isfinite(x), x, -1e30).max(-1).values
    d = ((x - peak[:, None]) / temperature).clamp(min=-104.0)
    d = torch.where(torch.isfinite(d), d, -104.0)
    p = torch.softmax(d, -1)
    lse_tol = ulp * (3 * (p * d.abs()).sum(-1) + 4 + logits.shape[1] / 64 + 64)
    en_tol = lse_tol * 2 + ulp * (p * d.abs() * (6 * d.abs() + 8 + logits.shape[1] / 64 + 64)).sum(-1)

    def close(got, want, tol):
        # (-6.8e38 = (-3.4e38 - -5) / 0.5 is beyond the largest fp32, 3.403e38: rounded to fp32 it is -inf)
        want = torch.where(want.abs() > 3.4028236e38, want.float().double(), want)
        both = torch.isfinite(want)
        assert torch.equal(both, torch.isfinite(got))
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~both & ~torch.isnan(want)].double(), want[~both & ~torch.isnan(want)])
        err = (got.double() - want).abs()
        assert (err[both] <= (tol.expand_as(want) + 4 * ulp * want.abs())[both]).all(), float((err / (tol.expand_as(want) + 1e-30))[both].max())

    if tokens is not None:
        close(lp, want_lp, lse_tol)
    close(en, want_en, en_tol)
    if top:
        close(tl, want_tl, lse_tol[:, None])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,top,temperature", [
    (1, 1, 1, 1.0), (3, 2, 5, 1.0), (5, 63, 32, 0.7), (2, 1000, 0, 1.0), (7, 1024, 20, 1.3), (1, 3001, 5, 1.0), (33, 3001, 8, 0.3),
    (1, 128256, 32, 1.0), (8, 152064, 5, 1.0), (40, 16387, 1, 2.0), (300, 4099, 4, 1.0)])
def test_logprobs(rows, vocab, top, temperature, dtype):
    g = torch.Generator().manual_seed(rows * 7 + vocab)
    logits = (torch.randn((rows, vocab), generator=g) * 3).to(dtype)
    tokens = torch.randint(0, vocab, (rows,), generator=g)
    tokens[::3] = logits[::3].float().argmax(-1)
    _check_logprobs(logits, tokens, temperature, top)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_logprobs_of_unusual_rows(dtype):
    vocab = 5003
    g = torch.Generator().manual_seed(2)
    x = torch.randn((16, vocab), generator=g) * 2
    lowest = torch.finfo(dtype).min
    x[0] = 0.0  # all equal: the lowest ids
    x[1] = -math.inf
    x[2] = -math.inf
    x[2, 4000] = 3.0  # one token left
    x[3] = lowest  # masked by the type's lowest value
    x[4] = lowest
    x[4, 17] = -5.0
    x[5, 1234] = math.nan
    x[6, 77] = math.inf
    x[7, :5000] = -math.inf  # three left, of 8 asked for
    x[8] = torch.arange(vocab).float() / 64  # ascending
    x[9] = -torch.arange(vocab).float() / 64
    x[10] = torch.arange(vocab) % 7
    x[11] += 1e4  # far from zero
    x[12] -= 1e4
    x[13, ::2], x[13, 1::2] = 0.0, -0.0  # zeros of both signs are equal
    x[14] = -300.0
    x[14, 4999] = 100.0
    x[15, :40] = 90.0  # the most probable ones all at the front
    tokens = torch.randint(0, vocab, (16,), generator=g)
    tokens[0], tokens[1], tokens[2], tokens[4], tokens[7], tokens[14] = 0, 5, 4000, 18, 3, 0
    tokens[9], tokens[10], tokens[11] = -1, vocab, -2 ** 31
    _check_logprobs(x.to(dtype), tokens, 1.0, 8)
    _check_logprobs(x.to(dtype), None, 0.5, 32)


def test_logprobs_of_rows_beyond_four_gib():
    far = (1 << 31) + 24
    store = torch.empty(far + 1000, dtype=BF16, device="cuda")
    g = torch.Generator().manual_seed(6)
    rows = (torch.randn((2, 1000), generator=g) * 3).bfloat16()
    logits = store.as_strided((2, 1000), (far, 1))
    logits.copy_(rows)
    tokens = torch.tensor([5, 999], dtype=torch.int32)
    got, want = _logprobs(logits, tokens, 1.0, 5), _logprobs(rows.cuda(), tokens, 1.0, 5)
    assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_logprobs_of_a_slice():
    """Rows longer than the vocabulary, a first logit off any boundary, an odd stride."""
    g = torch.Generator().manual_seed(3)
    for dtype in (F32, BF16):
        wide = (torch.randn((6, 4111), generator=g) * 3).to(dtype)
        wide[:, :3], wide[:, 4000:] = 50.0, math.nan
        _check_logprobs(wide[:, 3:4000], torch.randint(0, 3997, (6,), generator=g), 1.0, 5)
        _check_logprobs(wide[::2, 3:4000], torch.randint(0, 3997, (3,), generator=g), 1.0, 5)
