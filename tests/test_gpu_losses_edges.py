"""Where the losses could go wrong beside the cases of test_gpu_losses.py.  Definitions in float64; U as there."""
import math

import numpy as np
import pytest
import torch

from paper_2501_02379_amd import losses
from test_gpu_losses import DEV, TYPES, U, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temperature", [1.0, 0.7, 1.3])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("offset", [0.0, 3e6])
def test_rewards_have_no_error_of_one_sign(dtype, temperature, offset):
    """The mean error of a log ratio over 8192 tokens.  Roundings whose sign changes from row to row are below 4u each and leave
    less than u / 20 of it (4u / sqrt(8192)); a scale that is off by half an ulp moves every row the same way, by some 7 times that
    half ulp here (the tokens lie about 7 below the entries that make up the sum).  Bound: u / 4.  Rows far from zero take another path."""
    if offset and dtype != "f32":
        pytest.skip("a two-byte number has no fraction there")
    rows, vocab, parts = 8192, 3001, 4
    x, y = make(rows, vocab, dtype, seed=70)
    if offset:
        x += offset
        x = x.contiguous()
    shift = x.double().amax(1, keepdim=True)
    z = (x.double() - shift).div(float(np.float32(temperature)))
    logp = (z.gather(1, y[:, None])[:, 0] - torch.logsumexp(z, 1))
    ref = logp.float()
    start = torch.arange(parts + 1, device=DEV) * (rows // parts)
    r = losses.tgrad_preference_loss(x, y, torch.ones(rows, device=DEV), ref, start, beta=1.0, temperature=temperature, backward=False)
    want = (logp - ref.double()).view(parts, -1).sum(1)
    assert float((r.rewards.double() - want).abs().max()) / (rows // parts) <= U / 4 * math.sqrt(parts)
    assert abs(float((r.rewards.double() - want).sum())) / rows <= U / 4
