"""card_kv_append and the cache of 4 bits where lengths and tables do not fit each other."""
import pytest
import torch

from cache4_common import Batch4, model_freqs, rotated
from serving_common import Batch
from test_gpu_cache4 import Call4
from test_gpu_serving import Call, _cfg

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _append(b):
    """The pools before and after, and the rotated queries."""
    import paper_2508_04462_amd as card

    cfg, four = _cfg((b.q_heads, b.kv_heads, b.h)), isinstance(b, Batch4)
    c = (Call4 if four else Call)(b)
    q_out = torch.full_like(c.q, 9.0)
    before = [p.clone() for p in (c.k_pool, c.v_pool)]
    st = (card.card_kv4_append if four else card.card_kv_append)(cfg, c.batch, b.layer, card.card_rotation(), card.card_rows(c.q), card.card_rows(q_out),
                                                                card.card_rows(c.k), card.card_rows(c.v), torch.cuda.current_stream().cuda_stream)
    assert st == card.CARD_OK
    torch.cuda.synchronize()
    return before, (c.k_pool, c.v_pool), q_out.cpu()


def _check_rotation(q, q_out, positions, h):
    want, size = rotated(q, positions, model_freqs(1e4, h))
    half = 2.0 ** -8 if q.dtype == BF16 else 2.0 ** -24
    # cosines and sines in fp32, from angles off by 2^-50 of themselves (frequency, product and reduction in 64 bits); a sum rounded to fp32, then to its type
    off = 2.0 ** -24 * 1.01 + 2 * 2.0 ** -50 * float(positions.max())
    err = (q_out.double() - want).abs()
    assert (err <= size * (off + 2.0 ** -24) + want.abs() * half * 1.01).all(), float(err.max())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16", "4"])
def test_queries_of_texts_that_are_longer_than_their_tables(kind, dtype):
    """Their places are what the lengths say: tokens without a page are not stored, queries are rotated all the same."""
    heads, lens = (10, 2, 128), [(100, 10), (32, 20), (30, 7), (3, 1)]
    b = kind(heads, lens, dtype, seed=4)
    b.width, b.tables = 2, b.tables[:, :2].contiguous()  # 32 places each
    before, after, q_out = _append(b)
    positions = torch.cat([c + torch.arange(n) for c, n in lens])
    _check_rotation(b.q, q_out, positions, b.h)
    changed = {p for old, new in zip(before, after) for p in (old.view(torch.uint8) != new.view(torch.uint8)).flatten(2).any(-1).nonzero()[:, 1].tolist()}
    assert changed == {int(b.tables[2, 1]), int(b.tables[3, 0])}
