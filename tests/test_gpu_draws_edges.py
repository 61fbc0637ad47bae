"""Draws from the whole softmax at the borders of its spans, against sums in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2602_05774_amd as vsd

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = math.inf
SPAN = 2048


@pytest.mark.parametrize("kind", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("seed", range(3))
def test_equal_spans_behind_masked_ones(kind, seed):
    """u Z at the border of a span of no entries: the token is an entry at that border."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    V, n = 1 << 18, 64
    x = torch.full((V // SPAN, SPAN), -INF, device=DEV, dtype=kind)
    x[1::2] = torch.randn(SPAN, generator=g, device=DEV).to(kind)
    x = x.view(V)
    u = torch.arange(n, device=DEV) / n
    res = vsd.sample_rows(x.expand(n, V).contiguous(), u)
    tok = res.tok.cpu().numpy()
    assert (tok >= 0).all() and (tok < V).all() and (tok // SPAN % 2 == 1).all() and int(res.device_error) == 0
    w = np.exp(x.double().cpu().numpy() - float(x.max()))
    c = np.cumsum(w.astype(np.longdouble))
    z, target = c[-1], u.cpu().numpy().astype(np.longdouble) * c[-1]
    # the border lies within the 1e-12 that the weights' sums are good to
    assert (c[tok] > target - 1e-12 * z).all() and (c[tok] - w[tok] <= target + 1e-12 * z).all()
    assert (res.kept == V // 2).all()
    want = (x.double().cpu().numpy()[tok] - float(x.max())) - float(np.log(z))
    assert np.all(np.abs(res.log_prob.double().cpu().numpy() - want) <= 2.0 ** -24 * np.abs(want) + 1e-12)
