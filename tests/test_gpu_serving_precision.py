"""What card_kv_attend keeps of the softmax weights of bf16 rows, and weights whose maximum moves late, in every kind of workgroup."""
import math

import pytest
import torch

from serving_common import Batch
from test_gpu_serving import Call

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16

# heads, texts: from a few rows x heads of a KV head (new tokens stored on the way, or in front) to many, then in cuts
VARIANTS = {
    "one_64": ((8, 2, 64), [(333, 3), (40, 1)]),
    "one_128": ((8, 2, 128), [(333, 3), (40, 1)]),
    "two_64": ((8, 2, 64), [(333, 20), (0, 9)]),
    "two_128": ((8, 2, 128), [(333, 20), (0, 9)]),
    "stored_64": ((2, 2, 64), [(333, 100), (16, 3)]),
    "stored_128": ((2, 2, 128), [(333, 100), (16, 3)]),
    "few_64": ((8, 2, 64), [(333, 90), (16, 3)]),
    "few_128": ((8, 2, 128), [(333, 90), (16, 3)]),
    "many_64": ((8, 2, 64), [(333, 150), (16, 3)]),
    "many_128": ((8, 2, 128), [(333, 150), (16, 3)]),
    "one_cut": ((8, 2, 128), [(3000, 3), (40, 1)]),
    "two_cut": ((8, 2, 64), [(3000, 20), (0, 9)]),
    "few_cut": ((8, 2, 128), [(3000, 90), (16, 3)]),
    "many_cut": ((8, 2, 128), [(3000, 150), (16, 3)]),
}


def _close_to_rounded(call, ref):
    """Weights go into the product as two bf16 parts: the first is off by 2^-8 of the weight at most, the second by 2^-8 of that, so 2^-16 is left, in the
    output's sum and at most once more in the sum of the weights; fp32 as in Batch.tolerance; then the output is rounded to bf16 once, by 2^-8 of itself."""
    torch.cuda.synchronize()
    b, (out, mean_abs, score_abs, _, _) = call.b, ref
    rows, n = int(b.starts[-1]), max(c + m for c, m in b.lens)
    ulp = 2.0 ** -24
    before = mean_abs * (2 * (3 * b.h + 4) * ulp * score_abs + 2 * (n + 32) * ulp + 2 * 2.0 ** -16)
    tol = (before + (out.abs() + before) * 2.0 ** -8)[:rows]
    err = (call.out.cpu().double() - out).abs()[:rows]
    worst = float((err / tol.clamp(min=1e-30)).max())
    assert worst <= 1.0, worst


@pytest.mark.parametrize("variant", VARIANTS)
def test_attend_rounds_the_output_alone(variant):
    heads, lens = VARIANTS[variant]
    b = Batch(heads, lens, BF16, seed=21)
    ref = b.reference()
    call = Call(b).run()
    _close_to_rounded(call, ref)
    call.check(ref)
    masked = Batch(heads, lens, BF16, seed=22).tree_mask(density=0.5)
    _close_to_rounded(Call(masked).run(), masked.reference())


@pytest.mark.parametrize("variant", VARIANTS)
def test_attend_with_a_maximum_that_moves_late(variant):
    """Keys that grow along the text, and queries of sixteen times the usual size: the largest score of a row passes the ones before it by far more than
    2^8 again and again, within a cut and from cut to cut; and the other way round, where what comes later vanishes."""
    heads, lens = VARIANTS[variant]
    for down in (False, True):
        b = Batch(heads, lens, BF16, seed=23)
        b.q = (b.q.float() * 16.0).to(BF16)
        for s, (c, _) in enumerate(lens):
            if c == 0:
                continue
            ramp = torch.linspace(0.05, 1.5, c)
            b.keys[s] = (b.keys[s].float() * (ramp.flip(0) if down else ramp)[:, None, None]).to(BF16)
            b.put(b.k_pool, b.v_pool, s, torch.arange(c), b.keys[s], b.values[s])
        ref = b.reference()
        # (the test's own claim: in log2 units, the largest score of the last tenth of the first text's keys against the first tenth's)
        c, n = lens[0]
        r = b.q[:n, 0].double() @ b.keys[0][:, 0].double().T / math.sqrt(b.h) * 1.4426950408889634
        step = r[:, -(c // 10):].max(-1).values - r[:, : c // 10].max(-1).values
        assert float((-step if down else step).min()) > 8.0
        call = Call(b).run()
        _close_to_rounded(call, ref)
        call.check(ref)
