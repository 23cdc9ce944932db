"""card_kv_attend where its device data is out of range: in every kind of workgroup, with guards around the pools and the output."""
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
