"""card_kv_attend where its device data is short or wrong: tables that end before their texts, pages that are not there, masks that begin inside a page, lengths and
row starts out of range, pages beyond 4 GiB.  In every kind of workgroup, with guards around the pools and the output."""
import math

import pytest
import torch

from serving_common import PAGE, Batch
from test_gpu_serving import Call

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

# heads, new tokens of the longest text, type: new tokens stored on the way, or by a kernel in front; one tile, two, many
VARIANTS = {
    "one": ((8, 2, 128), 3, BF16),
    "two": ((8, 2, 64), 20, BF16),
    "two_in_front": ((2, 2, 128), 100, BF16),
    "few_in_front": ((8, 2, 64), 100, BF16),
    "many_64": ((8, 2, 64), 140, BF16),
    "many_128": ((8, 2, 128), 140, BF16),
    "f32": ((8, 2, 64), 9, F32),
    "f32_in_front": ((4, 2, 128), 140, F32),
}
CTX = {"whole": 90, "cut": 2500}
GUARD = 1 << 14  # elements before and behind


class Guarded(Call):
    """A call whose pools and output lie between values that nothing may change."""

    def __init__(self, b, table_pages=None, **kw):
        super().__init__(b, **kw)
        self.stores = []
        self.k_pool, self.v_pool, self.out = (self._guarded(t) for t in (self.k_pool, self.v_pool, self.out))
        self.batch.k_pages, self.batch.v_pages = self.k_pool.data_ptr(), self.v_pool.data_ptr()
        if table_pages is not None:
            self.tables = self.tables[:, :table_pages].contiguous()
            self.batch.block_tables, self.batch.table_pages = self.tables.data_ptr(), table_pages

    def _guarded(self, t):
        flat = torch.full((t.numel() + 2 * GUARD,), math.nan, dtype=t.dtype, device="cuda")
        for part in (flat[:GUARD], flat[-GUARD:]):
            part.view(torch.int16).copy_((torch.arange(part.numel() * t.element_size() // 2, device="cuda") % 30011).to(torch.int16))
        self.stores.append((flat, flat[:GUARD].view(torch.int16).clone(), flat[-GUARD:].view(torch.int16).clone()))
        view = flat[GUARD:-GUARD].view(t.shape)
        view.copy_(t)
        return view

    def guards_hold(self):
        torch.cuda.synchronize()
        for flat, front, back in self.stores:
            assert torch.equal(flat[:GUARD].view(torch.int16), front) and torch.equal(flat[-GUARD:].view(torch.int16), back)


def _reference(b, there):
    """As Batch.reference, over the slots that are there (bool, one per token of each sequence): the others are neither stored nor seen."""
    out = torch.full((b.n_rows, b.q_heads, b.h), math.nan, dtype=torch.float64)
    mean_abs, score_abs = torch.zeros_like(out), 0.0
    k_pool, v_pool = b.k_pool.clone(), b.v_pool.clone()
    for s, (c, n) in enumerate(b.lens):
        if n == 0:
            continue
        r0 = int(b.starts[s])
        k_new, v_new = b.k[r0:r0 + n].bfloat16(), b.v[r0:r0 + n].bfloat16()
        stored = there[s][c:]
        if stored.any():
            b.put(k_pool, v_pool, s, torch.arange(c, c + n)[stored], k_new[stored], v_new[stored])
        k, v = torch.cat([b.keys[s], k_new]).double(), torch.cat([b.values[s], v_new]).double()
        j = torch.arange(c + n)
        if b.mask is None:
            seen = j[None, :] <= c + torch.arange(n)[:, None]
        else:
            bit, bits = j - int(b.mask_base[s]), b.bits[r0:r0 + n]
            seen = (bit < 0)[None, :] | (bits[:, bit.clamp(0, bits.shape[1] - 1)] & ((bit >= 0) & (bit < bits.shape[1]))[None, :])
        seen = seen & there[s][None, :]
        for head in range(b.q_heads):
            q, kv = b.q[r0:r0 + n, head].double(), head // (b.q_heads // b.kv_heads)
            score = (q @ k[:, kv].T / math.sqrt(b.h)).masked_fill(~seen, -math.inf)
            score_abs = max(score_abs, float((q.abs() @ k[:, kv].abs().T / math.sqrt(b.h)).max()))
            top = score.max(-1, keepdim=True).values
            weight = (score - torch.where(top == -math.inf, 0.0, top)).exp()
            total = weight.sum(-1, keepdim=True)
            p = torch.where(total > 0, weight / total, 0.0)
            out[r0:r0 + n, head], mean_abs[r0:r0 + n, head] = p @ v[:, kv], p @ v[:, kv].abs()
    return out, mean_abs, score_abs, k_pool, v_pool


def _whole(b):
    return [torch.ones(c + n, dtype=torch.bool) for c, n in b.lens]


@pytest.mark.parametrize("masked", [False, True], ids=["causal", "masked"])
@pytest.mark.parametrize("ctx", CTX)
@pytest.mark.parametrize("variant", VARIANTS)
def test_attend_of_texts_longer_than_their_table(variant, ctx, masked):
    """The table ends among the first text's new tokens, in the middle of the second's cache, at the end of the third, behind the fourth."""
    heads, new, dtype = VARIANTS[variant]
    base = CTX[ctx]
    pages = (base + new) // PAGE  # (the first text's last token or more has no place)
    lens = [(base, new + PAGE), (pages * PAGE + 40, min(new, 5)), (pages * PAGE - 2, 2), (7, 1)]
    b = Batch(heads, lens, dtype, seed=31)
    if masked:
        b.tree_mask(density=0.5)
    there = [torch.arange(c + n) < pages * PAGE for c, n in lens]
    call = Guarded(b, table_pages=pages)
    call.run().check(_reference(b, there))
    call.guards_hold()
    again = Guarded(b, table_pages=pages, stored=True)  # over what is stored
    again.k_pool.copy_(call.k_pool)
    again.v_pool.copy_(call.v_pool)
    again.run().check(_reference(b, there))


@pytest.mark.parametrize("ctx", CTX)
@pytest.mark.parametrize("variant", VARIANTS)
def test_attend_with_pages_outside_the_pool(variant, ctx):
    """Page ids outside the pool: the first of a text, one in its middle, neighbours, one among the new tokens, all of a text."""
    heads, new, dtype = VARIANTS[variant]
    lens = [(CTX[ctx], new), (CTX[ctx] - 11, min(new, 5)), (20, 3), (5, 1)]
    for masked in (False, True):
        b = Batch(heads, lens, dtype, seed=32)
        if masked:
            b.tree_mask(density=0.5)
        call, there = Guarded(b), _whole(b)
        last = (lens[0][0] + new - 1) // PAGE
        for s, page, bad in ((0, 0, b.n_pages), (0, 2, -1), (0, 3, 2 ** 31 - 1), (0, last, -2 ** 31), (1, 1, b.n_pages + 7), (2, 0, -5), (2, 1, 2 ** 30)):
            call.tables[s, page] = bad
            there[s][page * PAGE:(page + 1) * PAGE] = False
        call.run().check(_reference(b, there))
        call.guards_hold()


@pytest.mark.parametrize("ctx", CTX)
@pytest.mark.parametrize("variant", VARIANTS)
def test_attend_under_masks_from_inside_a_page(variant, ctx):
    heads, new, dtype = VARIANTS[variant]
    lens = [(CTX[ctx], new), (37, 3), (0, 2), (60, 1)]
    for bases in ([CTX[ctx] - 9, 37, 0, 5], [37, 5, 1, 61], [CTX[ctx] + 1, 40, 5, 1000]):  # (beyond the text: all of it is seen)
        b = Batch(heads, lens, dtype, seed=33)
        words = (max(c + n - x for (c, n), x in zip(lens, bases)) + 31) // 32
        b.tree_mask(density=0.4, bases=bases, words=words)
        call = Guarded(b)
        call.run().check(_reference(b, _whole(b)))
        call.guards_hold()


@pytest.mark.parametrize("variant", VARIANTS)
def test_attend_with_lengths_and_starts_out_of_range(variant):
    """Nothing is written outside the output's rows and the pages of the tables; a right call behind it is right."""
    heads, new, dtype = VARIANTS[variant]
    lens = [(50, new), (33, 2), (0, 5)]
    far = 2 ** 31 - 1
    for masked in (False, True):
        b = Batch(heads, lens, dtype, seed=34, fill=0.0, spare=5)
        if masked:
            b.tree_mask(density=0.5)
        n = b.n_rows
        free = [p for p in range(b.n_pages) if p not in set(b.tables[b.tables < 2 ** 30].tolist())]
        for ctx in ([50, 33, 0], [-1, far, -far - 1], [far, far, far], [b.width * PAGE, b.width * PAGE - 1, 1]):
            for starts in (b.starts.tolist(), [0, n + 1000, far, far], [-5, 3, 2, n], [n, n // 2, 0, -far], [far, -1, far, n], [0, 0, 0, 0]):
                call = Guarded(b)
                call.ctx.copy_(torch.tensor(ctx, dtype=torch.int32))
                call.starts.copy_(torch.tensor(starts, dtype=torch.int32))
                call.run()
                call.guards_hold()
                for pool, was in ((call.k_pool, b.k_pool), (call.v_pool, b.v_pool)):
                    assert torch.equal(pool[0].cpu(), was[0]) and torch.equal(pool[1, free].cpu(), was[1, free])
        Call(b).run().check()


@pytest.mark.parametrize("heads,lens,dtype", [((8, 8, 128), [(35, 530), (40, 3)], BF16), ((16, 8, 128), [(35, 200), (40, 3)], BF16),
                                              ((8, 8, 128), [(35, 70), (2000, 3)], F32)], ids=["many", "few_in_front", "f32_cut"])
def test_attend_in_front_beyond_four_gib(heads, lens, dtype):
    """Pages whose offset in the layer passes 32 bits, where a kernel of its own stores the new tokens."""
    b = Batch(heads, lens, dtype, layers=1, layer=0)
    c = Call(b)
    far = (1 << 32) // (8 * PAGE * 128 * 2) + 1000
    k_pool = torch.empty((1, far + b.n_pages, 8, PAGE * 128), dtype=BF16, device="cuda")
    v_pool = torch.empty_like(k_pool)
    k_pool[0, far:], v_pool[0, far:] = c.k_pool[0], c.v_pool[0]
    c.tables += far
    c.batch.k_pages, c.batch.v_pages, c.batch.n_pages = k_pool.data_ptr(), v_pool.data_ptr(), far + b.n_pages
    c.run()
    c.k_pool, c.v_pool = k_pool[:, far:], v_pool[:, far:]
    c.check()
