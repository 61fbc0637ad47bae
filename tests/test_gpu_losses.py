"""Cross entropy, distillation and top logits on materialised rows against the
float64 oracle (bars: tests/loss_bars.py)."""
import math

import numpy as np
import pytest
import torch

import paper_2602_05774_amd as vsd
from oracle import losses as lo
from tests import loss_bars as bars

pytestmark = pytest.mark.gpu
DEV = "cuda"
SENTINEL = -7.0
INF = math.inf


def _rows(R, V, kind, seed, spread=3.0, pad=0):
    """[R, V] view of a buffer with 16-byte rows whose padding holds NaN."""
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    per = 4 if kind == "f32" else 8
    ld = (V + per - 1) // per * per + pad
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    buf = torch.full((R, ld), math.nan, dtype=dt, device=DEV)
    buf[:, :V] = (torch.randn(R, V, generator=g, device=DEV) * spread).to(dt)
    return buf, buf[:, :V]


def _host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _members(R, V, K, seed, lse, tp, dtype=torch.float32, dup=False):
    rng = np.random.default_rng(seed)
    idx = np.stack([rng.integers(0, V, K) if dup or K > V else rng.permutation(V)[:K] for _ in range(R)]).astype(np.int32)
    t = torch.from_numpy(rng.normal(size=(R, K)) * 2 + 4).to(dtype)
    idx[rng.random((R, K)) < 0.1] = -1                    # members missing anywhere
    if R > 2:
        idx[2] = -1                                       # a row without members
    vals = t.clone()
    vals[torch.from_numpy(idx < 0)] = math.nan            # what a missing member holds is not used
    if K > 2 and R > 1:
        vals[1, 0] = -INF
        t[1, 0] = -INF
    zs = lo._lse(np.where(idx < 0, -np.inf, t.double().numpy() / tp))
    z = (np.where(np.isneginf(zs), 0.0, zs) + 0.25).astype(np.float32) if lse else None
    mem = lo.teacher_members(idx, t.double().numpy(), z, tp)
    dev = (torch.from_numpy(idx).to(DEV), vals.to(DEV), None if z is None else torch.from_numpy(z).to(DEV))
    return mem, dev


def _check(res, x, mem, w, T, scale, kind, gbuf=None):
    idx, p, plogp = mem
    wt = None if w is None else w.cpu().numpy()
    ref = lo.losses(x, idx, p, plogp, wt, T, scale)
    R, V = x.shape
    with np.errstate(invalid="ignore"):
        m = np.where(ref["live"], np.max(np.where(np.isnan(x), -np.inf, x), axis=1), 0.0)
    loss, lse = _host(res.loss_row), _host(res.lse)
    fin = np.isfinite(ref["loss"])
    safe = np.where(ref["live"][:, None], x, 0.0)
    bar = bars.loss_bar(ref, np.where(np.isfinite(safe), safe, 0.0), idx, p, m, V, T)
    assert np.array_equal(loss[~fin], ref["loss"][~fin])
    assert np.all(np.abs(loss[fin] - ref["loss"][fin]) <= bar[fin]), (loss, ref["loss"], bar)
    dead = ~ref["live"]
    assert np.array_equal(loss[dead], np.zeros(dead.sum()))
    assert np.array_equal(np.isneginf(lse), np.isneginf(ref["lse"]))
    ok = np.isfinite(ref["lse"])
    lbar = bars.lse_bar(ref["lse"], m, V, T)
    assert np.all(np.abs(lse[ok] - ref["lse"][ok]) <= lbar[ok])
    wv = np.ones(R) if wt is None else wt.astype(np.float64)
    if np.all(fin):
        tot = float(res.loss_total)
        used = np.where(ref["loss"] != 0, np.abs(wv), 0.0)
        assert abs(tot - ref["total"]) <= abs(scale) * np.sum(used * bar) + 2 * bars.U * abs(ref["total"]) + 1e-12
    if res.grad is None:
        return ref
    g = _host(res.grad)
    k = np.where(dead, 0.0, np.abs(scale * wv) / T)
    gb = bars.grad_bar(ref, np.where(np.isfinite(safe), safe, m[:, None] - 1e4), idx, p, m, V, T, k, kind)
    bad = np.abs(g - ref["grad"]) > gb
    assert not bad.any(), (np.argwhere(bad)[:4], g[bad][:4], ref["grad"][bad][:4], gb[bad][:4])
    assert np.all(g[dead] == 0)
    if gbuf is not None and gbuf.shape[1] > V:
        assert torch.all(gbuf[:, V:] == SENTINEL)
    return ref


SHAPES = [(1, 1, "f32"), (1, 8, "bf16"), (2, 7, "bf16"), (5, 9, "f32"), (33, 257, "bf16"), (192, 1000, "f32"),
          (70, 2049, "bf16"), (9, 5000, "bf16"), (6, 16385, "f32"), (7, 32003, "bf16"), (4, 65536, "bf16"),
          (3, 65541, "f32"), (5, 128256, "bf16"), (3, 131073, "bf16"), (2, 200003, "bf16"), (2, 150001, "f32")]


@pytest.mark.parametrize("R,V,kind", SHAPES)
def test_cross_entropy(R, V, kind):
    buf, X = _rows(R, V, kind, 11, pad=16 if V % 3 else 0)
    labels = torch.randint(0, V, (R,), device=DEV, dtype=torch.int32)
    w = torch.rand(R, device=DEV) + 0.5
    if R > 4:
        labels[1] = -1
        buf[1] = math.nan          # a row without a label may hold anything
        w[3] = 0.0
        buf[3, 0] = INF
        labels[4] = V - 1
    labels[0] = 0
    gbuf = torch.full_like(buf, SENTINEL)
    res = vsd.cross_entropy(X, labels, w, 0.7, 1.25, grad=gbuf[:, :V])
    assert int(res.device_error) == 0
    mem = lo.label_members(labels.cpu().numpy())
    _check(res, _host(X), mem, w, 0.7, 1.25, kind, gbuf)
    only = vsd.cross_entropy(X, labels, w, 0.7, 1.25)
    assert only.grad is None
    _check(only, _host(X), mem, w, 0.7, 1.25, kind)


@pytest.mark.parametrize("R,V,kind,K,lse,dtype", [
    (1, 1, "f32", 1, False, torch.float32), (4, 5, "bf16", 3, True, torch.float32), (5, 40, "f32", 64, False, torch.bfloat16),
    (33, 257, "bf16", 10, True, torch.bfloat16), (20, 5000, "bf16", 33, False, torch.float32),
    (9, 32003, "f32", 64, True, torch.float32), (6, 128256, "bf16", 16, False, torch.bfloat16),
    (3, 140000, "bf16", 7, True, torch.float32)])
def test_distillation(R, V, kind, K, lse, dtype):
    buf, X = _rows(R, V, kind, 12)
    mem, (idx, val, z) = _members(R, V, K, 3, lse, 1.25, dtype, dup=K > 8)
    if R > 2:
        buf[2] = math.nan
    w = torch.rand(R, device=DEV) + 0.5
    gbuf = torch.full_like(buf, SENTINEL)
    res = vsd.distill_loss(X, idx, val, z, w, 0.8, 1.25, 0.75, grad=gbuf[:, :V])
    assert int(res.device_error) == 0
    _check(res, _host(X), mem, w, 0.8, 0.75, kind, gbuf)
    only = vsd.distill_loss(X, idx, val, z, w, 0.8, 1.25, 0.75)
    _check(only, _host(X), mem, w, 0.8, 0.75, kind)


@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("V", (64, 4099, 33000))
def test_masked_logits(kind, V):
    """-inf columns, the type's lowest value, rows that leave nothing, a label at -inf."""
    buf, X = _rows(8, V, kind, 13)
    low = torch.finfo(buf.dtype).min
    X[0, 1:] = -INF                       # one logit
    X[1] = -INF                           # none
    X[2, V // 2:] = -INF
    X[3, : V // 2] = low
    X[4] = low                            # all equal, at the lowest value
    X[5, 3] = -INF                        # the label's
    X[6, 5:] = low
    X[6, :5] = 3e38
    X[7, : V - 1] = -INF
    labels = torch.tensor([0, 2, 1, V - 1, 7, 3, 4, V - 1], dtype=torch.int32, device=DEV)
    gbuf = torch.full_like(buf, SENTINEL)
    res = vsd.cross_entropy(X, labels, grad=gbuf[:, :V])
    _check(res, _host(X), lo.label_members(labels.cpu().numpy()), None, 1.0, 1.0, kind, gbuf)
    assert res.loss_row[5] == INF and res.loss_row[1] == 0 and res.lse[1] == -INF


def test_nan_in_a_live_row_shows_and_stays_there():
    buf, X = _rows(3, 3000, "bf16", 14)
    X[1, 77] = math.nan
    labels = torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV)
    res = vsd.cross_entropy(X, labels, grad=True)
    assert torch.isnan(res.loss_row[1]) and torch.isnan(res.lse[1]) and torch.isnan(res.grad[1]).all()
    assert torch.isfinite(res.loss_row[[0, 2]]).all() and torch.isfinite(res.grad[[0, 2]]).all()


@pytest.mark.parametrize("kind,V", [("bf16", 5001), ("f32", 5001), ("bf16", 32000), ("bf16", 140000), ("f32", 70000)])
def test_gradient_into_the_logits(kind, V):
    buf, X = _rows(6, V, kind, 15)
    mem, (idx, val, z) = _members(6, V, 9, 4, True, 1.0, dup=True)
    x = _host(X)
    out = vsd.distill_loss(X, idx, val, z, grad=True)
    keep = buf.clone()
    same = vsd.distill_loss(X, idx, val, z, grad=X)
    assert same.grad is X
    for a, b in zip(out[:4], same[:4]):
        assert torch.equal(a, b)
    _check(same, x, mem, None, 1.0, 1.0, kind)
    buf.copy_(keep)
    labels = torch.arange(6, device=DEV, dtype=torch.int32) * 800
    ref = vsd.cross_entropy(X, labels, grad=True)
    same = vsd.cross_entropy(X, labels, grad=X)
    for a, b in zip(ref[:4], same[:4]):
        assert torch.equal(a, b)


def test_bad_indices_are_reported_and_skipped():
    _, X = _rows(4, 100, "f32", 16)
    labels = torch.tensor([5, 100, -2, 7], dtype=torch.int32, device=DEV)
    res = vsd.cross_entropy(X, labels, grad=True)
    assert int(res.device_error) == 1 and res.loss_row[1] == 0 and res.loss_row[2] == 0
    assert torch.all(res.grad[1:3] == 0) and torch.all(res.grad[0] != 0)
    idx = torch.tensor([[3, 100], [1, -5], [2, 4], [-1, -1]], dtype=torch.int32, device=DEV)
    res = vsd.distill_loss(X, idx, torch.zeros(4, 2, device=DEV), grad=True)
    assert int(res.device_error) == 1 and torch.isfinite(res.loss_row).all()


def test_rows_far_past_32_bit_offsets():
    V, ld = 1003, 1 << 30
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GB")
    buf = torch.empty(2 * ld + 1008, dtype=torch.bfloat16, device=DEV)
    X = torch.as_strided(buf, (3, V), (ld, 1))
    X.copy_(torch.randn(3, V, device=DEV))
    gb = torch.empty(2 * ld + 1008, dtype=torch.bfloat16, device=DEV)
    g = torch.as_strided(gb, (3, V), (ld, 1))
    labels = torch.tensor([0, 1, 1002], dtype=torch.int32, device=DEV)
    res = vsd.cross_entropy(X, labels, grad=g)
    _check(res, _host(X), lo.label_members(labels.cpu().numpy()), None, 1.0, 1.0, "bf16")
    t = vsd.top_logits(X, 5)
    assert np.array_equal(t.idx.cpu().numpy(), lo.top(_host(X), 5)[0])


def test_other_stream_and_captured_calls():
    """On a stream of its own; captured once and replayed on new inputs, with
    eager work in between."""
    _, X = _rows(40, 9001, "bf16", 17)
    new = [_rows(40, 9001, "bf16", s)[1] for s in (18, 19, 20)]
    labels = torch.randint(-1, 9001, (40,), device=DEV, dtype=torch.int32)
    d2t = torch.randperm(9001, device=DEV)[:4000].int()

    def chain():
        t = vsd.top_logits(X, 12, d2t=d2t)
        d = vsd.distill_loss(X, torch.where(t.idx >= 0, d2t[t.idx.clamp(min=0).long()], -1), t.logits, t.lse, grad=True)
        c = vsd.cross_entropy(X, labels, grad=True)
        return [*t[:3], *d[:4], *c[:4]]

    side = torch.cuda.Stream()
    ref = chain()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(ref, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = chain()
    for x in new:
        X.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(chain(), outs):
            assert torch.equal(a, b)


# ------------------------------------------------------------- top logits ---
def _check_top(y, res, k, d2t=None, T=1.0):
    assert int(res.device_error) == 0
    idx, val, lse = lo.top(y, k, None if d2t is None else d2t.cpu().numpy(), T)
    assert np.array_equal(res.idx.cpu().numpy(), idx)
    assert np.array_equal(_host(res.logits), val)
    m = np.max(y, axis=1)
    got, fin = _host(res.lse), np.isfinite(lse)
    assert np.array_equal(got[~fin], lse[~fin])
    with np.errstate(invalid="ignore"):
        assert np.all((np.abs(got - lse) <= bars.lse_bar(lse, m, y.shape[1], T))[fin])


@pytest.mark.parametrize("R,V,kind", SHAPES)
@pytest.mark.parametrize("k", (1, 10, 64))
def test_top_logits(R, V, kind, k):
    _, Y = _rows(R, V, kind, 21)
    _check_top(_host(Y), vsd.top_logits(Y, k, temp_target=1.5), k, None, 1.5)


@pytest.mark.parametrize("V,vd,order", [(9, 4, "any"), (5000, 4999, "up"), (32003, 700, "any"), (128256, 32000, "up"),
                                        (128256, 32000, "any"), (300, 300, "any"), (140001, 50, "any")])
def test_top_logits_over_a_map(V, vd, order):
    _, Y = _rows(5, V, "bf16", 22)
    d2t = torch.randperm(V, device=DEV)[:vd].int()
    d2t = d2t.sort().values if order == "up" else d2t
    for k in (3, 16, 64):
        _check_top(_host(Y), vsd.top_logits(Y, k, d2t=d2t), k, d2t)


@pytest.mark.parametrize("V", (100, 20000, 128256, 150000))
@pytest.mark.parametrize("kind", ("bf16", "f32"))
@pytest.mark.parametrize("mapped", (False, True))
def test_top_logits_of_ties(V, kind, mapped):
    """Equal logits (more than a list holds), few logits above -inf, none, the lowest value, both zeros."""
    buf, Y = _rows(9, V, kind, 23)
    Y[0] = 1.5
    Y[1] = -INF
    Y[2] = -INF
    Y[2, [V - 1, 3, V // 2]] = torch.tensor([1.0, 2.0, 1.0], device=DEV).to(buf.dtype)
    Y[3] = Y[3].round()
    Y[4] = torch.finfo(buf.dtype).min
    Y[5] = 0.0
    Y[5, ::2] = -0.0
    Y[6] = (Y[6] > 0).to(buf.dtype)
    Y[7, : V - 1] = -INF
    Y[8] = 2.0
    Y[8, 7] = 3.0
    Y[8, V - 2] = 4.0
    d2t = torch.randperm(V, device=DEV)[: V * 9 // 10].int() if mapped else None
    for k in (1, 7, 64):
        _check_top(_host(Y), vsd.top_logits(Y, k, d2t=d2t), k, d2t)


@pytest.mark.parametrize("R,V", ((1030, 300), (1024, 700), (1025, 1025), (2000, 2048), (1023, 1900)))
@pytest.mark.parametrize("kind", ("bf16", "f32"))
@pytest.mark.parametrize("mapped", (False, True))
def test_top_logits_of_many_short_rows(R, V, kind, mapped):
    """Rows that stay in a wavefront: values of both signs, equal ones across the K-th place,
    fewer entries than K, none."""
    _, Y = _rows(R, V, kind, 33)
    g = torch.Generator(device=DEV).manual_seed(34)
    Y[: R // 2] = torch.randint(-3, 4, (R // 2, V), generator=g, device=DEV).to(Y.dtype)
    Y[0] = -7.0
    Y[1] = -math.inf
    Y[2, 30:] = -math.inf
    Y[3] = -torch.rand(V, generator=g, device=DEV).to(Y.dtype)
    Y[4] = torch.where(torch.arange(V, device=DEV) % 2 == 0, 0.0, -0.0).to(Y.dtype)
    d2t = torch.randperm(V, device=DEV, generator=g)[: V * 9 // 10].int() if mapped else None
    for k in (1, 33, 64):
        _check_top(_host(Y), vsd.top_logits(Y, k, d2t=d2t), k, d2t)


def test_top_logits_of_a_bad_map():
    _, Y = _rows(2, 64, "f32", 24)
    for bad, code in (([3, 3, 5, 1], 4), ([3, 64, 5, 1], 2), ([3, -1, 5, 1], 2)):
        res = vsd.top_logits(Y, 2, d2t=torch.tensor(bad, dtype=torch.int32, device=DEV))
        assert int(res.device_error) == code


def test_refusals_of_the_binding():
    _, X = _rows(4, 100, "f32", 25)
    lab = torch.zeros(4, dtype=torch.int32, device=DEV)
    bad = [lambda: vsd.cross_entropy(X, lab.long()), lambda: vsd.cross_entropy(X, lab[:3]),
           lambda: vsd.cross_entropy(X, lab.cpu()), lambda: vsd.cross_entropy(X.half(), lab),
           lambda: vsd.cross_entropy(X.t(), lab), lambda: vsd.cross_entropy(X[:0], lab[:0]),
           lambda: vsd.cross_entropy(X, lab, torch.ones(4, device=DEV, dtype=torch.float64)),
           lambda: vsd.cross_entropy(X, lab, grad=True, weight_grad=True),
           lambda: vsd.cross_entropy(X, lab, grad=X.bfloat16()), lambda: vsd.cross_entropy(X, lab, grad=X[:3]),
           lambda: vsd.cross_entropy(X, lab, device_error=torch.zeros(1, device=DEV)),
           lambda: vsd.distill_loss(X, lab, X[:, :1]), lambda: vsd.distill_loss(X, lab[:, None], X[:, :2]),
           lambda: vsd.distill_loss(X, torch.zeros(4, 65, dtype=torch.int32, device=DEV), X[:, :65].contiguous()),
           lambda: vsd.top_logits(X, 0), lambda: vsd.top_logits(X, 65), lambda: vsd.top_logits(X, 2, d2t=lab.long())]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: vsd.cross_entropy(X[:, 1:], lab), lambda: vsd.cross_entropy(X[:1].expand(4, 100), lab),
                 lambda: vsd.cross_entropy(X, lab, temp_draft=0.0), lambda: vsd.top_logits(X[:, 1:], 2),
                 lambda: vsd.top_logits(X, 2, d2t=torch.zeros(101, dtype=torch.int32, device=DEV))):
        with pytest.raises(vsd.VsdError):
            call()


def test_gradient_against_differences():
    """Central differences of loss_total in steps of 2^-5: the loss's float32 error over
    2^-4, and a sixth of its third derivative (at most 1/T^3) times the step squared."""
    R, V, T = 3, 40, 0.9
    _, X = _rows(R, V, "f32", 26, spread=1.0)
    _, (idx, val, z) = _members(R, V, 5, 7, True, 1.0)
    labels = torch.tensor([3, 39, 11], dtype=torch.int32, device=DEV)
    calls = [lambda x, **kw: vsd.cross_entropy(x, labels, temp_draft=T, **kw),
             lambda x, **kw: vsd.distill_loss(x, idx, val, z, temp_draft=T, **kw)]
    h = 2.0 ** -5
    for call in calls:
        g = call(X, grad=True).grad.clone()
        for r, v in [(0, 3), (0, 0), (1, 39), (1, 17), (2, 11), (2, 30)]:
            up, down = X.clone(), X.clone()
            up[r, v] += h
            down[r, v] -= h
            d = (float(call(up).loss_total) - float(call(down).loss_total)) / (2 * h)
            assert abs(d - float(g[r, v])) <= 2 * 3 * 8 * 4e-6 / (2 * h) + h * h / 6 / T ** 3
