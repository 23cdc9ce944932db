"""Log probabilities of logits at the ends of fp32's range."""
import pytest
import torch

from test_gpu_serving import F32, _check_logprobs, _logprobs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temperature", [1e30, 3e29, 7.0])
@pytest.mark.parametrize("vocab", [40, 9001])
def test_logits_further_apart_than_the_largest_fp32(vocab, temperature):
    """A difference of 6e38 is beyond fp32, 6e38 / 1e30 is not: the log probability of a finite logit is finite where it fits."""
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn((5, vocab), generator=g) * 1e30
    x[0, ::3], x[0, 1::3] = 3e38, -3e38
    x[1, :-1], x[1, -1] = -3.4028234e38, 3.4028234e38
    x[2, 7] = -3.4028234e38
    x[3] = x[3].sign() * 3e38
    x[3, 5] = 3.3e38
    x[4, 11], x[4, 12] = -float("inf"), 3e38
    tokens = torch.tensor([1, 0, 7, 6, 11])
    x[3, 6] = -3.3e38
    _check_logprobs(x, tokens, temperature, 30)
    if temperature == 1e30:
        lp, _, _, tl = _logprobs(x.cuda(), tokens, temperature, 30)
        assert torch.isfinite(lp[:4]).all() and lp[4] == -float("inf") and torch.isfinite(tl[1]).all()
