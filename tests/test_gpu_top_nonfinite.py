"""top_logits of rows that hold NaN and +inf: a NaN is no entry, +inf is the largest one, either
makes the row's log-sum-exp NaN, and no other row sees them.  Every way in which a row's members
are found: registers of a wavefront, lists of one and of four wavefronts, bit by bit."""
import math

import numpy as np
import pytest
import torch

import paper_2602_05774_amd as vsd
from oracle import losses as lo
from tests import loss_bars as bars
from tests.test_gpu_losses import _host, _rows

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("R,V,k", ((12, 300, 5), (12, 300, 64), (12, 900, 64), (1030, 1800, 40), (12, 1800, 40),
                                   (12, 3000, 9), (12, 9000, 12), (12, 9000, 50), (12, 70001, 30)))
@pytest.mark.parametrize("kind", ("bf16", "f32"))
@pytest.mark.parametrize("mapped", (False, True))
def test_nan_and_infinity(R, V, k, kind, mapped):
    _, Y = _rows(R, V, kind, 71)
    nan, inf = math.nan, math.inf
    Y[0, 3] = nan
    Y[1] = nan
    Y[2, V // 2:] = nan
    Y[3, [0, V - 1, V // 3]] = inf
    Y[4, :70] = inf                      # more of them than members
    Y[5] = inf
    Y[6, ::2], Y[6, 1::2] = nan, -inf
    Y[7, 7], Y[7, 8] = inf, nan
    Y[8] = torch.where(torch.arange(V, device=DEV) % 3 == 0, nan, 2.0).to(Y.dtype)  # NaN among equal logits
    d2t = torch.randperm(V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(72))[: V * 4 // 5].int() if mapped else None
    res = vsd.top_logits(Y, k, d2t=d2t)
    y = _host(Y)
    odd = np.isnan(y).any(1) | np.isposinf(y).any(1)
    with np.errstate(invalid="ignore"):
        idx, val, lse = lo.top(np.where(np.isnan(y), -np.inf, y), k, None if d2t is None else d2t.cpu().numpy())
    assert np.array_equal(res.idx.cpu().numpy(), idx)
    assert np.array_equal(_host(res.logits), val)
    got = _host(res.lse)
    assert np.isnan(got[odd]).all() and np.isfinite(got[~odd]).all()
    assert np.all(np.abs(got - lse)[~odd] <= bars.lse_bar(lse, y.max(1), V, 1.0)[~odd])
