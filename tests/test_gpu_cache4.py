"""card_kv_append, and the cache of 4 bits (card_kv4_*), on the GPU against their definitions in 64 bits."""
import math

import pytest
import torch

from cache4_common import Batch4, k_nibbles, model_freqs, put_tokens, quantised, rotated, v_nibbles, values
from serving_common import PAGE, Batch
from test_gpu_serving import Call, _cfg

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


class Call4(Call):
    """One batch on pools of 4 bits."""

    def __init__(self, b, **more):
        import paper_2508_04462_amd as card

        super().__init__(b, **more)
        self.ws = torch.full((card.card_kv4_attend_workspace_bytes(self.cfg, self.batch),), 0xA5, dtype=torch.uint8, device="cuda")

    def run(self):
        import paper_2508_04462_amd as card

        k, v = (None, None) if self.stored else (card.card_rows(self.k), card.card_rows(self.v))
        st = card.card_kv4_attend(self.cfg, self.batch, self.b.layer, card.card_rows(self.q), k, v, card.card_rows(self.out), self.mask, self.ws,
                                  torch.cuda.current_stream().cuda_stream)
        assert st == card.CARD_OK, card.card_strerror(st)
        return self

    def check(self, ref=None):
        torch.cuda.synchronize()
        out, tol, kp, vp = ref or self.b.reference()
        got, rows = self.out.cpu(), int(self.b.starts[-1])
        assert torch.isfinite(got[:rows].double()).all()
        worst = float(((got.double() - out).abs()[:rows] / tol[:rows].clamp(min=1e-30)).max()) if rows else 0.0
        assert worst <= 1.0, worst
        assert (got[rows:] == 7.0).all()
        if not self.stored:
            assert torch.equal(self.k_pool.cpu(), kp) and torch.equal(self.v_pool.cpu(), vp)
        return worst


class Append:
    """card_kv_append or card_kv4_append of a batch."""

    def __init__(self, b, freqs=None, positions=None, in_place=False, rotate=True, with_q=True):
        import paper_2508_04462_amd as card

        self.b, self.bits, self.rotate, self.with_q = b, 4 if isinstance(b, Batch4) else 16, rotate, with_q
        self.cfg = _cfg((b.q_heads, b.kv_heads, b.h), b.k_pool.shape[0])
        self.c = (Call4 if self.bits == 4 else Call)(b)
        self.freqs = freqs or model_freqs(float(self.cfg.rope_theta), b.h)
        self.positions = positions
        self.q_in = self.c.q.clone()
        self.q_out = self.c.q if in_place else self.c.out
        self.pos_dev = None if positions is None else positions.cuda()
        self.rotation = card.card_rotation(freqs, self.pos_dev) if rotate else None
        call = card.card_kv4_append if self.bits == 4 else card.card_kv_append
        q, q_out = (card.card_rows(self.c.q), card.card_rows(self.q_out)) if rotate and with_q else (None, None)
        st = call(self.cfg, self.c.batch, b.layer, self.rotation, q, q_out, card.card_rows(self.c.k), card.card_rows(self.c.v),
                  torch.cuda.current_stream().cuda_stream)
        assert st == card.CARD_OK, card.card_strerror(st)
        torch.cuda.synchronize()

    def rows_positions(self):
        b = self.b
        if self.positions is not None:
            return self.positions
        pos = torch.zeros(b.n_rows, dtype=torch.int64)
        for s, (c, n) in enumerate(b.lens):
            pos[int(b.starts[s]):int(b.starts[s + 1])] = c + torch.arange(n)
        return pos

    def check(self):
        b, rows = self.b, int(self.b.starts[-1])
        half = 2.0 ** -8 if b.dtype == BF16 else 2.0 ** -24
        if self.rotate and self.with_q:
            want, size = rotated(b.q, self.rows_positions(), self.freqs)
            # cosines and sines are rounded to fp32 once, from angles that are off by 2^-52 of themselves; the sum once
            angle = 2.0 ** -52 * float(self.rows_positions().abs().max() + 1) * max(self.freqs)
            err = (self.q_out.cpu().double() - want).abs()
            assert (err <= size * (2.0 ** -24 * 1.01 + 2 * angle) + want.abs() * half * 1.01)[:rows].all()
        if not (self.rotate and self.with_q and self.q_out is self.c.q):
            assert torch.equal(self.q_in, self.c.q)
            assert (self.c.out.cpu()[rows if self.rotate and self.with_q else 0:] == 7.0).all()
        k_want, k_size = (rotated(b.k, self.rows_positions(), self.freqs)) if self.rotate else (b.k.double(), b.k.double().abs())
        k_pool, v_pool = b.k_pool.clone(), b.v_pool.clone()
        got_k, got_v = self.c.k_pool.cpu(), self.c.v_pool.cpu()
        if self.bits == 16:
            for s, (c, n) in enumerate(b.lens):
                r = slice(int(b.starts[s]), int(b.starts[s + 1]))
                b.put(k_pool, v_pool, s, torch.arange(c, c + n), k_want[r].float().bfloat16(), b.v[r].bfloat16())
            same = (got_k.double() - k_pool.double()).abs() <= 2.0 ** -7 * k_pool.double().abs() + 1e-6  # (a value next to a border of bf16 may lie beyond it)
            assert (same | (got_k.isnan() & k_pool.isnan())).all()
            assert torch.equal(got_k.isnan(), k_pool.isnan())
            assert (got_k.view(torch.int16) != k_pool.view(torch.int16)).double().mean() <= 1e-3
            assert torch.equal(got_v.view(torch.int16), v_pool.view(torch.int16))
            return self
        for s, (c, n) in enumerate(b.lens):
            r = slice(int(b.starts[s]), int(b.starts[s + 1]))
            b.put4(k_pool, v_pool, s, c, quantised(k_want[r].float()), quantised(b.v[r]))
        assert torch.equal(got_v, v_pool)
        if not self.rotate:
            assert torch.equal(got_k, k_pool)
        # a rotated key whose last bit differs may have another code or scale than the exact one: the bytes differ nowhere but there
        assert (got_k != k_pool).double().mean() <= 1e-4
        k, v = self.read()
        scale = (quantised(k_want.float())[1] << 16).view(torch.float32).double().repeat_interleave(64, -1)
        out = k.cpu().double()
        # half a scale (which may be rounded the other way: 2^-7 of it), the rotation's rounding and that of the row's type
        assert ((out - k_want).abs() <= scale * (0.5 + 2.0 ** -16 + 2.0 ** -7) + k_size * 2.0 ** -23 + out.abs() * half)[:rows].all()
        want_v = values(*quantised(b.v))
        assert ((v.cpu().double() - want_v).abs() <= want_v.abs() * half * 1.01 + 2.0 ** -22 * scale.max())[:rows].all()
        assert (k.cpu()[rows:] == 5).all() and (v.cpu()[rows:] == 5).all()
        return self

    def read(self):
        import paper_2508_04462_amd as card

        b = self.b
        k, v = (torch.full((b.n_rows, b.kv_heads, b.h), 5.0, dtype=b.dtype, device="cuda") for _ in range(2))
        st = card.card_kv4_read(self.cfg, self.c.batch, b.layer, card.card_rows(k), card.card_rows(v), torch.cuda.current_stream().cuda_stream)
        assert st == card.CARD_OK
        torch.cuda.synchronize()
        return k, v


HEADS = [(4, 2, 64), (10, 2, 128), (7, 1, 128), (8, 8, 64), (34, 2, 64), (28, 4, 128), (48, 1, 128)]
LENS = [
    [(0, 1)],
    [(15, 1), (16, 1), (17, 1), (0, 1)],
    [(0, 33), (100, 5), (7, 0), (31, 17), (0, 0), (1, 1)],
    [(2047, 3)],
    [(5, 130), (300, 1)],
]
ids_of = lambda v: "+".join("%d_%d" % x for x in v)  # noqa: E731
heads_of = lambda v: "%dx%dx%d" % v  # noqa: E731


@TYPES
@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16", "4"])
@pytest.mark.parametrize("lens", LENS, ids=ids_of)
@pytest.mark.parametrize("heads", HEADS, ids=heads_of)
def test_append(heads, lens, kind, dtype):
    Append(kind(heads, lens, dtype, seed=len(lens))).check()


@TYPES
@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16", "4"])
@pytest.mark.parametrize("order", ["fused", "heads"])
def test_append_of_rows_as_they_lie(order, kind, dtype):
    lens = [(40, 20), (3, 1)]
    Append(kind((10, 2, 128), lens, dtype, order=order, extra_rows=5)).check()
    Append(kind((10, 2, 128), lens, dtype, order=order, extra_rows=5), in_place=True).check()
    Append(kind((8, 8, 64), lens, dtype, order=order, extra_rows=5), rotate=False).check()
    Append(kind((8, 8, 64), lens, dtype, order=order, extra_rows=5), with_q=False).check()


@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16", "4"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (10, 2, 128)], ids=heads_of)
def test_append_at_positions_and_frequencies(heads, kind):
    """A tree's nodes, far and negative positions; stretched and zero frequencies."""
    lens = [(40, 20), (3, 1), (0, 40)]
    n = sum(x for _, x in lens)
    h = heads[2]
    freqs = [f / 8 for f in model_freqs(5e5, h)]
    freqs[3] = 0.0
    for positions in (torch.randint(0, 60, (n,)), torch.arange(n) * 20011 + 10 ** 6, -torch.arange(n) * 1001):
        b = kind(heads, lens, F32, seed=3)
        Append(b, positions=positions.to(torch.int32)).check()
        Append(b, positions=positions.to(torch.int32), freqs=freqs).check()


def test_quantising_extremes():
    """Groups of one value, of zeros, of tiny, huge and far apart values, of values next to a binade's end, with one that is not finite."""
    h, n = 128, 16
    b = Batch4((2, 2, h), [(0, n)], F32, seed=5)
    rows = torch.zeros(n, 2, h)
    g = torch.Generator().manual_seed(1)
    rows[0] = 0.0
    rows[1] = 3.14159
    rows[2] = -0.001
    rows[3] = torch.randn(2, h, generator=g) * 1e-3 + 100.0
    rows[4] = torch.randn(2, h, generator=g) * 2.0 ** -90
    rows[5] = torch.randn(2, h, generator=g) * 2.0 ** 95
    rows[6, :, ::7] = 40.0
    rows[7, :, 5] = -1.0
    rows[8] = torch.linspace(-1, 1, h)
    rows[9] = torch.linspace(4.0, 8.0, h)
    rows[10] = torch.linspace(-8.0, -7.9, h)
    rows[11:] = torch.randn(5, 2, h, generator=g)
    rows[12, 0, 3], rows[12, 1, 70], rows[13, 0, 100] = math.nan, math.inf, -math.inf
    b.k, b.v = rows.clone(), rows.flip(-1).contiguous().clone()
    a = Append(b, rotate=False)
    k, v = (x.cpu().double() for x in a.read())
    for got, x in ((k, b.k.double()), (v, b.v.double())):
        group = x.unflatten(-1, (2, 64))
        whole = torch.isfinite(group).all(-1, keepdim=True).expand_as(group).flatten(-2)
        assert torch.equal(torch.isnan(got), ~whole)
        scale = (quantised(x.float().nan_to_num(0, 0, 0))[1] << 16).view(torch.float32).double().repeat_interleave(64, -1)
        assert ((got - x).abs() <= scale * (0.5 + 2.0 ** -16) + got.abs() * 2.0 ** -24)[whole].all()
        most = group.abs().amax(-1, keepdim=True).expand_as(group).flatten(-2)
        assert (scale <= most * (2 * 17 / 256 + 1 / 1024) * (1 + 2.0 ** -8))[whole].all()
    k_pool, v_pool = b.k_pool.clone(), b.v_pool.clone()
    whole = [t for t in range(n) if t not in (12, 13)]
    put_tokens(k_pool[b.layer], int(b.tables[0, 0]), torch.tensor(whole), *(x[whole] for x in quantised(b.k)), k_nibbles)
    put_tokens(v_pool[b.layer], int(b.tables[0, 0]), torch.tensor(whole), *(x[whole] for x in quantised(b.v)), v_nibbles)
    for got, want, nibbles in ((a.c.k_pool, k_pool, k_nibbles), (a.c.v_pool, v_pool, v_nibbles)):
        got = got.cpu()[b.layer, int(b.tables[0, 0])]
        want = want[b.layer, int(b.tables[0, 0])]
        at = nibbles(torch.tensor(whole), h)
        for head in range(2):
            code = lambda p: torch.stack((p & 15, p >> 4), -1).flatten()[at]  # noqa: E731
            assert torch.equal(code(got[head]), code(want[head]))
            word = lambda p: p.view(torch.int32)[2 * h:].view(2, PAGE)[:, whole]  # noqa: E731
            assert torch.equal(word(got[head]), word(want[head]))


@TYPES
@pytest.mark.parametrize("lens", LENS, ids=ids_of)
@pytest.mark.parametrize("heads", HEADS, ids=heads_of)
def test_attend4_causal(heads, lens, dtype):
    b = Batch4(heads, lens, dtype, seed=len(lens))
    ref = b.reference()
    first = Call4(b).run()
    first.check(ref)
    # the same rows again, now that the cache holds their keys and values
    again = Call4(b, stored=True)
    again.k_pool, again.v_pool = first.k_pool, first.v_pool
    again.batch.k_pages, again.batch.v_pages = first.k_pool.data_ptr(), first.v_pool.data_ptr()
    again.run().check(ref)


@TYPES
@pytest.mark.parametrize("order", ["fused", "heads"])
def test_attend4_reads_rows_as_they_lie(order, dtype):
    Call4(Batch4((10, 2, 128), [(40, 20), (3, 1)], dtype, order=order, extra_rows=5)).run().check()


@TYPES
@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128), (7, 1, 128)], ids=heads_of)
def test_attend4_under_masks(heads, dtype):
    for lens in ([(70, 40), (16, 9), (0, 3), (129, 1)], [(70, 3), (16, 1), (0, 2), (530, 3)]):
        bases = [64, 0, 0, 128] if lens[0][1] == 40 else [16, 0, 0, 512]
        Call4(Batch4(heads, lens, dtype).tree_mask(density=0.3)).run().check()
        Call4(Batch4(heads, lens, dtype).tree_mask(words=1, bases=bases)).run().check()
        c = Call4(Batch4(heads, lens, dtype).tree_mask(empty=True)).run()
        c.check()
        assert (c.out[::2] == 0).all()


@TYPES
@pytest.mark.parametrize("heads,new", [((8, 8, 64), (16, 17, 64, 65)), ((4, 2, 64), (8, 9, 63, 64, 65, 128, 129, 257)), ((4, 1, 128), (4, 5, 64, 65, 80, 129)),
                                       ((8, 1, 64), (2, 3, 32, 33, 65))], ids=lambda v: "_".join("%d" % x for x in v))
def test_attend4_at_the_ends_of_its_variants(heads, new, dtype):
    for n in new:
        lens = [(19, 1), (419, n), (0, n), (3, 0)]
        Call4(Batch4(heads, lens, dtype, seed=n)).run().check()
        masked = Batch4(heads, lens, dtype, seed=n).tree_mask(density=0.4)
        Call4(masked).run().check()


@TYPES
@pytest.mark.parametrize("heads,lens", [((4, 2, 64), [(3000, 2), (40, 1)]), ((8, 1, 128), [(5003, 1)]), ((8, 1, 128), [(2500, 40)]), ((4, 4, 64), [(1800, 150), (700, 3)])],
                         ids=lambda v: heads_of(v) if isinstance(v, tuple) else ids_of(v))
def test_attend4_of_long_texts_in_cuts(heads, lens, dtype):
    b = Batch4(heads, lens, dtype, seed=9)
    ref = b.reference()
    c = Call4(b)
    assert c.ws.numel() > 0
    c.run().check(ref)
    first = c.out.clone()
    assert torch.equal(c.run().out, first)  # the same call, the same bits
    # whatever the sizes say that the work is cut by
    for max_new, max_len in ((0, 0), (1, 17), (10 ** 6, 10 ** 6)):
        Call4(b, max_new=max_new, max_len=max_len).run().check(ref)


@TYPES
def test_attend4_does_not_multiply_what_is_hidden(dtype):
    """NaN in keys and values that a row does not see; whoever sees them is NaN."""
    heads, lens = (4, 2, 128), [(70, 8), (20, 40)]
    b = Batch4(heads, lens, dtype, seed=2)
    clean = Call4(b).run()
    clean.check()
    hidden = [5, 8 + 21]  # rows whose keys and values are NaN
    b.k, b.v = b.k.clone(), b.v.clone()
    b.k[hidden[0]] = math.nan
    b.v[hidden[1]] = math.nan
    c = Call4(b).run()
    torch.cuda.synchronize()
    got, want = c.out.cpu(), clean.out.cpu()
    sees = [r for r in range(48) if (5 <= r < 8) or r >= 29]
    fine = [r for r in range(48) if r not in sees]
    assert torch.equal(got[fine], want[fine])
    assert got[sees].isnan().all()


def test_attend4_of_tables_out_of_range():
    """Tokens whose page is outside the pool or the table are not stored and not seen, and nothing is read for them."""
    import paper_2508_04462_amd as card

    heads = (4, 2, 64)
    b = Batch4(heads, [(100, 3), (10, 2)], BF16, seed=4)
    b.tables[0, 2] = -1
    b.tables[0, 4] = b.n_pages
    c = Call4(b).run()
    torch.cuda.synchronize()
    k = torch.cat([values(*b.keys[0]), values(*b.new_tokens(0)[0])])
    v = torch.cat([values(*b.values[0]), values(*b.new_tokens(0)[1])])
    j = torch.arange(103)
    for r in range(3):
        seen = (j <= 100 + r) & (j // 16 != 2) & (j // 16 != 4)
        for head in range(4):
            p = (k[:, head // 2] @ b.q[r, head].double() / 8).masked_fill(~seen, -math.inf).softmax(0)
            want = p @ v[:, head // 2]
            assert (c.out[r, head].cpu().double() - want).abs().max() <= 2.0 ** -7 * v.abs().max()
    # a text longer than its table: what has no place is not stored
    b = Batch4(heads, [(30, 10)], BF16, seed=4)
    b.width, b.tables = 2, b.tables[:, :2].contiguous()
    before = b.k_pool.clone()
    a = Append.__new__(Append)
    a.b, a.cfg, a.c = b, _cfg(heads), Call4(b)
    q_out = torch.zeros_like(a.c.q)
    st = card.card_kv4_append(a.cfg, a.c.batch, b.layer, card.card_rotation(), card.card_rows(a.c.q), card.card_rows(q_out), card.card_rows(a.c.k),
                              card.card_rows(a.c.v), torch.cuda.current_stream().cuda_stream)
    assert st == card.CARD_OK
    torch.cuda.synchronize()
    want, size = rotated(b.q, 30 + torch.arange(10), model_freqs(1e4, 64))
    assert ((q_out.cpu().double() - want).abs() <= size * 2.0 ** -23 + want.abs() * 2.0 ** -8 * 1.01).all()
    changed = (a.c.k_pool.cpu() != before).flatten(2).any(-1)
    assert changed.nonzero().tolist() == [[b.layer, int(b.tables[0, 1])]]


@TYPES
def test_attend4_precision(dtype):
    """Against 64 bits, relative to the output in the 2-norm: fp32 rows keep 24 bits of queries and weights, with bf16 rows the output's rounding (2^-8 at
    most, evenly spread: 1.65e-3) is what the error consists of."""
    for heads, lens in (((28, 4, 128), [(900, 1), (3000, 2), (50, 1)]), ((8, 1, 64), [(700, 90)])):
        b = Batch4(heads, lens, dtype, seed=8)
        out, _, _, _ = b.reference()
        c = Call4(b).run()
        torch.cuda.synchronize()
        off = float((c.out.cpu().double() - out).norm() / out.norm())
        assert off <= (1.75e-3 if dtype == BF16 else 2e-6), off


def _pools4(pages, heads, h, layers=3, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(0, 256, (layers, pages, heads, 9 * h), generator=g, dtype=torch.uint8) for _ in range(2)]


def _token(pool, values_, slot, h):
    """The nibbles and words of a slot, [layers][heads][..]."""
    page = pool[:, slot // PAGE]
    nibbles = torch.stack((page & 15, page >> 4), -1).flatten(-2)[..., (k_nibbles if values_ == "k" else v_nibbles)(torch.tensor([slot % PAGE]), h)[0]]
    words = page.contiguous().view(torch.int32)[..., 2 * h + torch.arange(h // 64) * PAGE + slot % PAGE]
    return nibbles.clone(), words.clone()


def _put_token(pool, values_, slot, h, token):
    for layer in range(pool.shape[0]):
        put_tokens(pool[layer], slot // PAGE, torch.tensor([slot % PAGE]), token[0][layer][None].long(), token[1][layer][None],
                   k_nibbles if values_ == "k" else v_nibbles)


@pytest.mark.parametrize("h,heads", [(64, 2), (128, 3)])
def test_copy_pages_and_move_slots_of_4_bits(h, heads):
    import paper_2508_04462_amd as card

    cfg, n_pages = _cfg((heads, heads, h), 3), 300
    g = torch.Generator().manual_seed(1)
    lists = [([3, 4, 9], [1, 2, 5]), ([299], [0]), (list(range(0, 300, 2))[:150], list(range(1, 300, 2))[:150])]
    for src, dst in lists:
        k, v = _pools4(n_pages, heads, h)
        kd, vd = k.cuda(), v.cuda()
        assert card.card_kv4_copy_pages(cfg, card.CardKV(kd.data_ptr(), vd.data_ptr(), None, n_pages, -1), src, dst, None) == card.CARD_OK
        torch.cuda.synchronize()
        for got, want in ((kd, k), (vd, v)):
            want[:, dst] = want[:, src]
            assert torch.equal(got.cpu(), want)
    closing = sorted(torch.randperm(900, generator=g)[:600].tolist())  # gaps that close: in order
    apart = torch.randperm(n_pages * 16, generator=g)[:140].tolist()
    moves = [([5], [7]), ([17, 33, 20], [3, 4, 31]), (apart[:70], apart[70:]), ([s + 5 for s in closing], list(range(5, 605))), (apart[:33], apart[100:133])]
    for src, dst in moves:
        src, dst = zip(*[(s, d) for s, d in zip(src, dst) if s != d])
        k, v = _pools4(n_pages, heads, h, seed=2)
        kd, vd = k.cuda(), v.cuda()
        assert card.card_kv4_move_slots(cfg, card.CardKV(kd.data_ptr(), vd.data_ptr(), None, n_pages, -1), src, dst, None) == card.CARD_OK
        torch.cuda.synchronize()
        for s, d in zip(src, dst):
            _put_token(k, "k", d, h, _token(k, "k", s, h))
            _put_token(v, "v", d, h, _token(v, "v", s, h))
        assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)
