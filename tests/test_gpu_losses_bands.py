"""The base losses in every length band and launch form against the float64 oracle
(bars: tests/loss_bars.py): the rows' gradients for each number of threads and columns
that a thread keeps, the LM head's joins by wavefronts and by workgroups, and as many rows as
make the widest launches fall back."""
import math

import pytest
import torch

import paper_2602_05774_amd as vsd
from oracle import losses as lo
from tests import loss_bars as bars
from tests.test_gpu_losses import SENTINEL, _check, _host, _members, _rows
from tests.test_gpu_losses_lm import _check as _check_head
from tests.test_gpu_losses_lm import _head

pytestmark = pytest.mark.gpu
DEV = "cuda"
# within each band of the rows' lengths and at both sides of its border
BANDS = (500, 2048, 2051, 4096, 4099, 8192, 8195, 12345, 16384, 16387, 32768, 32771, 50001, 65536, 65541, 100003,
         131072, 131075, 140001)


@pytest.mark.parametrize("V", BANDS)
@pytest.mark.parametrize("kind", ("bf16", "f32"))
def test_cross_entropy(V, kind):
    R = 5
    buf, X = _rows(R, V, kind, 61, pad=16 if V % 2 else 0)
    labels = torch.tensor([0, V - 1, -1, V // 2, V // 3], dtype=torch.int32, device=DEV)
    X[3, V // 4:] = -math.inf
    labels[3] = V // 8
    mem, x = lo.label_members(labels.cpu().numpy()), _host(X)
    w = torch.rand(R, device=DEV) + 0.5
    gbuf = torch.full_like(buf, SENTINEL)
    res = vsd.cross_entropy(X, labels, w, 0.7, 1.25, grad=gbuf[:, :V])
    assert int(res.device_error) == 0
    _check(res, x, mem, w, 0.7, 1.25, kind, gbuf)
    _check(vsd.cross_entropy(X, labels, w, 0.7, 1.25), x, mem, w, 0.7, 1.25, kind)
    same = vsd.cross_entropy(X, labels, w, 0.7, 1.25, grad=X)
    for a, b in zip(res[:4], same[:4]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("V", BANDS)
@pytest.mark.parametrize("kind", ("bf16", "f32"))
def test_distillation(V, kind):
    R, K = 5, 21
    buf, X = _rows(R, V, kind, 62, pad=16 if V % 2 else 0)
    mem, (idx, val, z) = _members(R, V, K, 7, V % 2 == 0, 1.25, dup=True)
    idx[4, 1] = idx[4, 0] = V - 1                       # the last column, named twice
    val[4, :2] = torch.tensor([5.0, 4.0], device=DEV)
    mem = lo.teacher_members(idx.cpu().numpy(), torch.nan_to_num(val, nan=0.0, neginf=-math.inf).double().cpu().numpy(),
                             None if z is None else z.double().cpu().numpy(), 1.25)
    x, w = _host(X), torch.rand(R, device=DEV) + 0.5
    gbuf = torch.full_like(buf, SENTINEL)
    res = vsd.distill_loss(X, idx, val, z, w, 0.8, 1.25, 0.75, grad=gbuf[:, :V])
    assert int(res.device_error) == 0
    _check(res, x, mem, w, 0.8, 0.75, kind, gbuf)
    _check(vsd.distill_loss(X, idx, val, z, w, 0.8, 1.25, 0.75), x, mem, w, 0.8, 0.75, kind)
    same = vsd.distill_loss(X, idx, val, z, w, 0.8, 1.25, 0.75, grad=X)
    for a, b in zip(res[:4], same[:4]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ("bf16", "f32"))
@pytest.mark.parametrize("R,V", ((200, 70001), (257, 70001), (65, 3000), (64, 3000)))
def test_loss_alone_of_few_long_rows(R, V, kind):
    """1024 threads up to 256 rows, 256 beyond; the total by the last of 64 rows, by a launch beyond."""
    _, X = _rows(R, V, kind, 63)
    labels = (torch.arange(R, device=DEV) * 997 % V).int()
    _check(vsd.cross_entropy(X, labels), _host(X), lo.label_members(labels.cpu().numpy()), None, 1.0, 1.0, kind)


@pytest.mark.parametrize("R,V,H,K", [(300, 16001, 64, 8), (140, 33000, 128, 64), (512, 9000, 64, 3),  # a workgroup a row
                                     (513, 9000, 64, 3), (600, 8200, 64, 64),                          # a wavefront a row
                                     (600, 8200, 2048, 64),                                            # long dot products
                                     (1025, 300, 64, 33), (1024, 300, 64, 33), (1024, 300, 64, 32), (513, 300, 64, 20)])
@pytest.mark.parametrize("grad", (True, None))
def test_distillation_through_the_head(R, V, H, K, grad):
    h, w = _head(R, V, H, 64)
    mem, (idx, val, z) = _members(R, V, K, 8, True, 1.0, dup=K == 33)
    h[2] = math.nan                                     # (a row without members)
    weight = torch.rand(R, device=DEV) + 0.5
    res = vsd.distill_loss(vsd.LmHead(h, w), idx, val, z, weight, 0.9, 1.0, 0.5, grad=grad,
                           weight_grad=torch.float32 if grad else False)
    assert int(res.device_error) == 0
    _check_head(res, _host(h), _host(w), mem, weight, 0.9, 0.5, V)


@pytest.mark.parametrize("R,V", ((8192, 28672), (8191, 30522), (8192, 30522), (8200, 28671)))
def test_distillation_of_many_rows(R, V):
    """Probabilities formed before the row is read and meanwhile, at both sides of the rule.  Every
    row against the first of its kind, those against the oracle."""
    kinds, K = 8, 13
    _, few = _rows(kinds, V, "bf16", 66)
    mem, (idx, val, z) = _members(kinds, V, K, 9, True, 1.25, dup=True)
    reps = -(-R // kinds)
    X = torch.full((R, (V + 7) // 8 * 8), math.nan, dtype=torch.bfloat16, device=DEV)[:, :V]
    X.copy_(few.repeat(reps, 1)[:R])
    many = [t.repeat(reps, *[1] * (t.dim() - 1))[:R].contiguous() for t in (idx, val, z)]
    res = vsd.distill_loss(X, *many, temp_draft=0.8, temp_target=1.25, loss_scale=0.5, grad=True)
    for r in range(0, R - R % kinds, 1024):
        part = res.grad[r:min(R - R % kinds, r + 1024)]
        assert torch.equal(part, res.grad[:kinds].repeat(len(part) // kinds, 1))
    assert torch.equal(res.loss_row, res.loss_row[:kinds].repeat(reps)[:R])
    ref = lo.losses(_host(few), *mem, None, 0.8, 0.5)
    first = vsd.LossResult(res.loss_row[:kinds], res.lse[:kinds], torch.tensor(ref["total"]), res.grad[:kinds], res.device_error)
    _check(first, _host(few), mem, None, 0.8, 0.5, "bf16")


def test_as_many_rows_as_leave_the_wide_launches():
    """2^22 rows of more than 4096 columns: 256 threads a row that read it twice, here into the
    logits' own place.  Every row against the first of its kind, those against the oracle."""
    V, kinds = 4104, 64
    R = 1 << 22
    free, _ = torch.cuda.mem_get_info()
    if free < 48 << 30:
        pytest.skip("needs 48 GB")
    _, few = _rows(kinds, V, "bf16", 65)
    labels = (torch.arange(kinds, device=DEV) * 61 % V).int()
    labels[5] = -1
    X = few.repeat(R // kinds, 1)
    x = _host(few)
    res = vsd.cross_entropy(X, labels.repeat(R // kinds), loss_scale=2.0 ** -10, grad=X)
    first = vsd.LossResult(res.loss_row[:kinds], res.lse[:kinds], None, res.grad[:kinds].clone(), res.device_error)
    for part in res.grad.view(R // kinds, kinds, V).split(1024):
        assert torch.equal(part, first.grad.expand_as(part))
    assert torch.equal(res.loss_row.view(-1, kinds), first.loss_row.expand(R // kinds, kinds))
    total = 2.0 ** -10 * first.loss_row.double().sum() * (R // kinds)
    assert abs(float(res.loss_total) - float(total)) <= 2 * bars.U * abs(float(total))
    mem = lo.label_members(labels.cpu().numpy())
    ref = lo.losses(x, *mem, None, 1.0, 2.0 ** -10)
    _check(first._replace(loss_total=torch.tensor(ref["total"])), x, mem, None, 1.0, 2.0 ** -10, "bf16")
