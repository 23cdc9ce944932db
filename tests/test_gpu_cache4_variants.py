"""Attention over 4 bits in every way that a call is run: tiles of rows, cuts of the pages, masks, together; and long histories of beams."""
import math

import pytest
import torch

from cache4_common import Batch4, values
from test_gpu_cache4 import F32, TYPES, Call4, heads_of, ids_of
from test_gpu_beams import _logits, check

pytestmark = pytest.mark.gpu


@TYPES
@pytest.mark.parametrize("heads,new", [((8, 8, 64), (1024, 1025)), ((8, 1, 128), (127, 128, 129, 132)), ((4, 2, 64), (512, 513))], ids=lambda v: "_".join("%d" % x for x in v))
def test_either_side_of_two_tiles(heads, new, dtype):
    """1024 rows x heads of a KV head, and more."""
    for n in new:
        lens = [(19, 1), (37, n), (0, 5)]
        Call4(Batch4(heads, lens, dtype, seed=n)).run().check()
        Call4(Batch4(heads, lens, dtype, seed=n).tree_mask(density=0.4)).run().check()
        c = Call4(Batch4(heads, lens, dtype, seed=n).tree_mask(empty=True)).run()
        c.check()
        assert (c.out[::2] == 0).all()


CUT = [((8, 1, 64), [(1700, 3), (40, 1)]), ((8, 1, 128), [(3100, 1)]), ((8, 1, 128), [(1500, 40), (1203, 2)]), ((8, 1, 128), [(1500, 133)]), ((16, 1, 64), [(1700, 70), (3, 1)])]


@TYPES
@pytest.mark.parametrize("heads,lens", CUT, ids=lambda v: heads_of(v) if isinstance(v, tuple) else ids_of(v))
def test_cuts_with_and_without_masks(heads, lens, dtype):
    """One tile and two; masks over all of the text, of which some rows see only one cut's keys or none."""
    for kind in ("causal", "mask", "words", "one cut", "empty"):
        b = Batch4(heads, lens, dtype, seed=len(kind))
        if kind == "mask":
            b.tree_mask(density=0.3, bases=[0] * len(lens))
        elif kind == "words":  # the last keys are behind the mask: nobody sees them
            b.tree_mask(words=9, bases=[800 // 16 * 16, 0][:len(lens)])
        elif kind == "one cut":
            b.tree_mask(density=1.0, bases=[0] * len(lens))
            b.bits[:] = False
            b.bits[::3, 600:700] = True
            b.bits[1::3, :16] = True
            value = (b.bits.view(b.n_rows, -1, 32).long() << torch.arange(32)).sum(-1)
            b.mask = torch.where(value >= 1 << 31, value - (1 << 32), value).to(torch.int32)
        elif kind == "empty":
            b.tree_mask(empty=True)
        c = Call4(b)
        need = c.ws.numel()
        assert need > 0
        guarded = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        c.ws = guarded[:need]
        c.run().check()
        assert (guarded[need:] == 0xA5).all()


def test_fp32_rows_are_as_exact_as_32_bits_are():
    """Against 64 bits in the 2-norm, and the same of a softmax in fp32 on the same values.  Both are made of roundings to 24 bits of products, scores, weights and sums, the kernel's in tiles
    (so of sums of fewer terms), its exp2 and queries and weights in three parts a few more: no more than half as much again.  With codes 16 .. 31 in place of centred
    ones, or weights in two parts (2^-17 each), the error would be 2 to 3 times and more."""
    for heads, lens in (((28, 4, 128), [(900, 1), (3000, 2), (50, 1)]), ((8, 1, 64), [(700, 90)])):
        b = Batch4(heads, lens, F32, seed=8)
        out, _, _, _ = b.reference()
        plain = torch.zeros_like(out, dtype=F32)
        for s, (c, n) in enumerate(lens):
            r, new = int(b.starts[s]), b.new_tokens(s)
            k, v = (values(*(torch.cat(x) for x in zip(old, fresh))).float() for old, fresh in zip((b.keys[s], b.values[s]), new))
            for head in range(heads[0]):
                a = head // (heads[0] // heads[1])
                score = (b.q[r:r + n, head] @ k[:, a].T / math.sqrt(heads[2])).masked_fill(~b.seen(s), -math.inf)
                plain[r:r + n, head] = score.softmax(-1) @ v[:, a]
        got = Call4(b).run().out.cpu()
        off, plain_off = (float((x.double() - out).norm() / out.norm()) for x in (got, plain))
        assert off <= 1.5 * plain_off, (off, plain_off)


@pytest.mark.parametrize("groups,beams,out_beams,most", [(2, 4, 8, 5000), (1, 1, 32, 3000), (3, 16, 16, 9000), (5, 3, 1, 2100)], ids=lambda v: str(v))
def test_long_histories(groups, beams, out_beams, most):
    """Of several workgroups a search, and several turns of a thread; full ones and empty ones."""
    g = torch.Generator().manual_seed(most)
    vocab = 1000
    scores = -torch.rand((groups, beams), generator=g) * 4 - 100
    done = (torch.rand((groups, beams), generator=g) < 0.2).int()
    history = torch.randint(0, vocab, (groups, beams, most), generator=g).int()
    logits = _logits(groups * beams, vocab, F32, most)
    for lengths in ([most - 1], [most, 0, 1023, 4096, 1], [1024, most + 7, -3, 2049, most // 2]):
        length = torch.tensor((lengths * groups)[:groups], dtype=torch.int32)
        check(logits, scores, out_beams, eos=1, done=done, history=history, lengths=length)
