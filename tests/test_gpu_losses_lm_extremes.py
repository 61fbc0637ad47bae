"""The base losses through an LM head at small temperatures and in rows without a
finite logit, where an exponent formed other than from x - m leaves float32's
range: against the float64 oracle, for every way in which the head's gradient is
formed."""
import math

import numpy as np
import pytest
import torch

import paper_2602_05774_amd as vsd
from oracle import losses as lo
from tests import loss_bars as bars
from tests.test_gpu_losses import _host, _members
from tests.test_gpu_losses_lm import _check, _head

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
# products of 256 x 256 tiles (the logits formed again for the gradient), few rows and
# a small vocabulary (kept): 8 row tiles of 128 by 94 tiles of 64 columns are more than
# two for each of 256 CUs, as are 65 by 3 or any more than 8192 rows
AGAIN = [(900, 6000, 64), (8193, 130, 64)]
KEPT = [(20, 515, 192), (300, 2049, 256)]


def _one_hot(res, h, w, labels, weight, T, scale):
    """Rows whose largest logit is ahead by 200 T beyond both logits' rounding (H u sum |h w|
    each) have q = 1 there and exp(-200) at most elsewhere, so nothing of a logit's rounding is
    left in their gradient: the bars without it."""
    H = h.shape[1]
    mem = lo.label_members(labels)
    ref = lo.head(h, w, mem, weight, T, scale)
    hz = np.where(ref["live"][:, None], h, 0.0)
    x = hz @ w.T
    m = x.max(1)
    top = np.partition(x, -2, axis=1)
    sure = ref["live"] & (top[:, -1] - top[:, -2] > 2 * H * bars.U * np.max(np.abs(hz) @ np.abs(w).T, axis=1) + 200 * T)
    assert sure.sum() > ref["live"].sum() // 2
    k = np.abs(scale * np.where(ref["live"], weight, 0.0)) / T
    gb = bars.grad_bar(ref, x, mem[0], mem[1], m, w.shape[0], T, k, "bf16", 2 * math.ceil(w.shape[0] / 256))
    ga = np.abs(ref["grad"]) + gb
    bh = gb @ np.abs(w) + w.shape[0] * bars.U * (ga @ np.abs(w))
    bh += 2.0 ** -8 * (np.abs(ref["grad_hidden"]) + bh) + 1e-37
    off = np.abs(_host(res.grad.grad_hidden) - ref["grad_hidden"])
    assert np.all((off <= bh)[sure]), np.argwhere((off > bh) & sure[:, None])[:4]


@pytest.mark.parametrize("R,V,H", AGAIN + KEPT)
@pytest.mark.parametrize("T", (1e-6, 1e-9, 1e-30, 1e6))
def test_cross_entropy_at_any_temperature(R, V, H, T):
    h, w = _head(R, V, H, 51)
    g = torch.Generator(device=DEV).manual_seed(52)
    labels = torch.randint(0, V, (R,), device=DEV, dtype=torch.int32, generator=g)
    labels[::5] = -1
    weight = torch.rand(R, device=DEV, generator=g) + 0.5
    res = vsd.cross_entropy(vsd.LmHead(h, w), labels, weight, T, 1.5, grad=True, weight_grad=torch.float32)
    assert int(res.device_error) == 0
    for t in (res.loss_row, res.lse, res.loss_total, res.grad.grad_hidden, res.grad.grad_weight):
        assert torch.isfinite(t).all()
    _check(res, _host(h), _host(w), lo.label_members(labels.cpu().numpy()), weight, T, 1.5, V)
    if T < 1:
        _one_hot(res, _host(h), _host(w), labels.cpu().numpy(), weight.double().cpu().numpy(), T, 1.5)


@pytest.mark.parametrize("R,V,H", AGAIN + KEPT)
@pytest.mark.parametrize("loss", ("ce", "distill"))
@pytest.mark.parametrize("T", (1.0, 0.01, 3.0))
def test_rows_without_a_finite_logit(R, V, H, loss, T):
    """A row in play whose products all overflow to -inf: loss 0, lse -inf, gradient 0, and
    nothing of it in the weight's; then also one with a NaN, which makes its own results
    and the weight's gradient NaN and no other row's."""
    h, w = _head(R, V, H, 53)
    w[:, 0] = 4.0
    h[:, 0] = 0.0
    h[7, 0] = -3e38
    labels = torch.arange(R, device=DEV, dtype=torch.int32) % V
    mem, (idx, val, z) = _members(R, V, 5, 6, True, 1.0)
    idx[11] = torch.arange(5, device=DEV, dtype=torch.int32)
    idx[7] = idx[11]
    mem = [m.copy() for m in mem]
    if loss == "ce":
        mem = [m.copy() for m in lo.label_members(labels.cpu().numpy())]
    else:
        val[7], val[11], z[7], z[11] = val[3], val[3], z[3], z[3]
        val = torch.where(val != val, 1.0, val)
        mem = [m.copy() for m in lo.teacher_members(idx.cpu().numpy(), val.double().cpu().numpy(), z.double().cpu().numpy())]

    def call():
        head = vsd.LmHead(h, w)
        if loss == "ce":
            return vsd.cross_entropy(head, labels, None, T, grad=True, weight_grad=torch.float32)
        return vsd.distill_loss(head, idx, val, z, None, T, grad=True, weight_grad=torch.float32)

    def without(*rows):  # the oracle's members with those rows out of play
        idx_, p, plogp = [m.copy() for m in mem]
        for r in rows:
            idx_[r], p[r], plogp[r] = -1, 0.0, 0.0
        return idx_, p, plogp

    res = call()
    assert float(res.loss_row[7]) == 0 and float(res.lse[7]) == -math.inf
    assert torch.all(res.grad.grad_hidden[7] == 0) and torch.isfinite(res.grad.grad_weight).all()
    lse = res.lse.clone()
    lse[7] = 0.0
    _check(res._replace(lse=lse), _host(h), _host(w), without(7), None, T, 1.0, V)

    h[11, 3] = math.nan
    res = call()
    assert torch.isnan(res.loss_row[11]) and torch.isnan(res.lse[11]) and torch.isnan(res.loss_total).all()
    assert torch.isnan(res.grad.grad_hidden[11]).all() and torch.isnan(res.grad.grad_weight).any()
    assert float(res.loss_row[7]) == 0 and torch.all(res.grad.grad_hidden[7] == 0)
    row, lse, dh = res.loss_row.clone(), res.lse.clone(), res.grad.grad_hidden.clone()
    row[11], lse[7], lse[11], dh[11] = 0.0, 0.0, 0.0, 0.0
    rest = res._replace(loss_row=row, lse=lse, loss_total=row.double().sum(), grad=vsd.LmHeadGrad(dh, None, None))
    _check(rest, _host(h), _host(w), without(7, 11), None, T, 1.0, V)


@pytest.mark.parametrize("R,V", ((100, 700001), (20, 4000001)))  # (the total by a launch, by the last of the joins)
def test_few_rows_of_a_very_large_vocabulary_at_a_small_temperature(R, V):
    """More logits of few rows than are kept: the ones that give g are those whose maximum the
    row's sum refers to.  Against float64 on the device, rows with a clear largest logit (as in
    _one_hot) without any of the logits' rounding."""
    H, T = 64, 1e-9
    h, w = _head(R, V, H, 54)
    labels = torch.randint(0, V, (R,), device=DEV, dtype=torch.int32, generator=torch.Generator(device=DEV).manual_seed(55))
    res = vsd.cross_entropy(vsd.LmHead(h, w), labels, temp_draft=T, grad=True, weight_grad=torch.float32)
    for t in (res.loss_row, res.lse, res.loss_total, res.grad.grad_hidden, res.grad.grad_weight):
        assert torch.isfinite(t).all()
    total = res.loss_row.double().sum()
    assert abs(float(res.loss_total) - float(total)) <= 2 * bars.U * float(total)
    top, at = (h.double() @ w.double().t()).topk(2, dim=1)
    slack = 2 * H * bars.U * h.double().abs().sum(1) * w.double().abs().max()
    sure = top[:, 0] - top[:, 1] > slack + 200 * T
    assert sure.sum() > R // 2
    a, b = w[at[:, 0]].double(), w[labels.long()].double()
    dh = (a - b) / T
    # g's two elements and the result are rounded to bf16, 1 / T and the sum's scale to float32
    bar = (2.0 ** -8 * 1.01 * (a.abs() + b.abs()) / T + 2.0 ** -8 * dh.abs()) * 1.01
    off = (res.grad.grad_hidden.double() - dh).abs()
    assert torch.all((off <= bar)[sure]), (off / bar)[sure].amax(1)


@pytest.mark.parametrize("R,V,H", AGAIN + KEPT)
@pytest.mark.parametrize("T", (1e-4, 1e-6, 1e-9, 1e-30))
def test_members_are_never_above_the_largest_logit(R, V, H, T):
    """Labels and members at the rows' largest logits, whose own dot products may come out above
    the maximum: no log q is above 0 and no q above 1."""
    h, w = _head(R, V, H, 56)
    x = h.double() @ w.double().t()
    idx = x.topk(6, dim=1).indices.int()
    labels = idx[:, 0].contiguous()
    head = vsd.LmHead(h, w)
    ce = vsd.cross_entropy(head, labels, temp_draft=T, grad=True, weight_grad=torch.float32)
    assert torch.all(ce.loss_row >= 0)
    _check(ce, _host(h), _host(w), lo.label_members(labels.cpu().numpy()), None, T, 1.0, V)
    val = torch.randn(R, 6, device=DEV, generator=torch.Generator(device=DEV).manual_seed(57)).sort(dim=1, descending=True).values
    mem = lo.teacher_members(idx.cpu().numpy(), val.double().cpu().numpy())
    kd = vsd.distill_loss(head, idx, val, temp_draft=T, grad=True, weight_grad=torch.float32)
    # sum p log p >= -log 6, each term to a few roundings (bars.loss_bar: 140), and no log q above 0
    assert torch.all(kd.loss_row >= -math.log(6) - 1000 * bars.U)
    for t in (*ce[:3], *ce.grad[::2], *kd[:3], *kd.grad[::2]):
        assert torch.isfinite(t).all()
    _check(kd, _host(h), _host(w), mem, None, T, 1.0, V)
