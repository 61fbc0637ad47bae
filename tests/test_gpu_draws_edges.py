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


@pytest.mark.parametrize("V", (600, 5000, 40000, 262144))
@pytest.mark.parametrize("kind", (torch.bfloat16, torch.float32))
def test_no_weight_beside_an_infinite_logit(V, kind):
    """u = 0 and a +inf behind finite logits, in their span or in a later one: the first +inf."""
    x = torch.randn(3, (V + 7) // 8 * 8, device=DEV).to(kind)[:, :V]
    x[0, 300] = x[1, V - 1] = x[2, 1::2] = INF
    for u in (0.0, 2.0 ** -24):
        res = vsd.sample_rows(x, torch.full((3,), u, device=DEV))
        assert res.tok.tolist() == [300, V - 1, 1], u
        assert (res.kept == V).all() and res.log_prob.tolist()[:2] == [0.0, 0.0]
        n = V // 2
        assert abs(float(res.log_prob[2]) + math.log(n)) <= 2.0 ** -24 * math.log(n) + 1e-12


def test_weights_too_small_for_64_bits():
    """u = 0: an entry of weight 0 in 64 bits (here exp(-1e4) and below) is no token, one of
    weight exp(-600) is."""
    V = 30000
    x = torch.full((2, V), -1.0, device=DEV)
    x[0, V - 1], x[1, V - 1] = 0.0, 599.0
    res = vsd.sample_rows(x, torch.zeros(2, device=DEV), temp_target=torch.tensor([1e-4, 1.0], device=DEV))
    assert res.tok.tolist() == [V - 1, 0]
    assert res.log_prob.tolist() == [0.0, -600.0] and (res.kept == V).all()
