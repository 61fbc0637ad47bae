"""Draws under the deployed rule against the float64 oracle: tokens and counts
exactly, log-probabilities to fp32's rounding."""
import math

import numpy as np
import pytest
import torch

import paper_2602_05774_amd as vsd
from oracle import draws as od

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = math.inf
LAST = 1 - 2.0 ** -24  # the largest u


def _rows(R, V, kind, seed, spread=3.0, pad=0):
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    per = 16 // dt.itemsize
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    buf = torch.full((R, (V + per - 1) // per * per + pad), math.nan, dtype=dt, device=DEV)
    buf[:, :V] = (torch.randn(R, V, generator=g, device=DEV) * spread).to(dt)
    return buf, buf[:, :V]


def _u(R, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    u = torch.rand(R, generator=g, device=DEV)
    if R > 3:
        u[0], u[1] = 0.0, LAST
    return u


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _check(res, X, u, settings, err=0):
    host = [s.cpu().numpy() if isinstance(s, torch.Tensor) else s for s in settings]
    tok, lp, kept = od.draws(_host(X), u.cpu().numpy(), *host)
    got = res.tok.cpu().numpy()
    bad = np.flatnonzero(got != tok)
    assert bad.size == 0, (bad[:5], got[bad[:5]], tok[bad[:5]])
    assert np.array_equal(res.kept.cpu().numpy(), kept), (res.kept, kept)
    # two roundings in 64 bits and one to fp32; the logit's part is exact in 64 bits
    # up to (x - max) / T times 2^-52
    have = _host(res.log_prob)
    nan = np.isnan(lp)
    assert np.array_equal(np.isnan(have), nan)
    assert np.all(np.abs(have - lp)[~nan] <= 2.0 ** -24 * np.abs(lp[~nan]) + 1e-12)
    assert int(res.device_error) == err


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (0.7, 5, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.3, 0, 1.0, 0.05),
            (0.8, 40, 0.95, 0.01), (1.0, 1, 1.0, 0.0), (1.0, 3000, 0.999, 0.0), (2.5, 0, 0.5, 1e-5), (1.0, 0, 1e-30, 0.0),
            (1.0, 0, 1.0, 1.0), (1e-30, 0, 0.9, 0.5), (1e30, 0, 1.0, 0.0)]


@pytest.mark.parametrize("R,V,kind", [(1, 1, "bf16"), (5, 7, "f32"), (9, 8, "bf16"), (6, 257, "f32"), (7, 2049, "bf16"),
                                      (5, 4097, "bf16"), (4, 8200, "f32"), (3, 32003, "bf16"), (2, 131073, "f32")])
@pytest.mark.parametrize("settings", SETTINGS)
def test_draws(R, V, kind, settings):
    _, X = _rows(R, V, kind, V + R, pad=16 if V % 3 else 0)
    u = _u(R, V)
    _check(vsd.sample_rows(X, u, *settings), X, u, settings)


@pytest.mark.parametrize("R,V,kind", [(40, 1000, "f32"), (64, 32000, "bf16")])
def test_settings_of_each_row(R, V, kind):
    _, X = _rows(R, V, kind, 3)
    u = _u(R, 4)
    pick = torch.arange(R) % len(SETTINGS)
    table = torch.tensor(SETTINGS, dtype=torch.float64)[pick]
    settings = [table[:, 0].float().to(DEV), table[:, 1].int().to(DEV), table[:, 2].float().to(DEV), table[:, 3].float().to(DEV)]
    res = vsd.sample_rows(X, u, *settings)
    _check(res, X, u, settings)
    mixed = [settings[0], 30, settings[2], 0.0]
    _check(vsd.sample_rows(X, u, *mixed), X, u, mixed)


@pytest.mark.parametrize("V", (9, 300, 5000, 40000))
@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("settings", [(1.0, 7, 1.0, 0.0), (1.0, 0, 0.6, 0.0), (0.5, 100, 0.7, 0.0), (1.0, 0, 1.0, 0.2),
                                      (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0)])
def test_equal_logits(V, kind, settings):
    """Few distinct values: the borders of top-k and top-p fall among equal logits, -0 and +0 among them."""
    buf, X = _rows(8, V, kind, 5)
    X.copy_(X.round().clamp(-2, 2))
    X[0] = 1.5                 # one value
    X[1] = 0.0
    X[1, ::3] = -0.0
    X[2, : V // 2] = -INF
    u = _u(8, V)
    _check(vsd.sample_rows(X, u, *settings), X, u, settings)


@pytest.mark.parametrize("V", (64, 4099, 33000))
@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("settings", SETTINGS[:7])
def test_masks(V, kind, settings):
    buf, X = _rows(8, V, kind, 6)
    low = torch.finfo(X.dtype).min
    X[0] = -INF                       # nothing left
    X[1, 1:] = -INF                   # one entry
    X[2, : V - 3] = -INF
    X[3, 5:] = low                    # masked by the type's lowest value
    X[4] = low                        # ... everywhere
    X[5, V // 2] = math.nan
    X[6, ::7] = INF                   # among themselves alike, all others 0
    u = _u(8, V)
    _check(vsd.sample_rows(X, u, *settings), X, u, settings)


def test_bad_settings_are_reported():
    _, X = _rows(12, 500, "f32", 7)
    u = _u(12, 8)
    ok = [torch.ones(12, device=DEV), torch.zeros(12, dtype=torch.int32, device=DEV), torch.ones(12, device=DEV),
          torch.zeros(12, device=DEV)]
    ok[0][2], ok[0][3], ok[0][4] = -1.0, math.nan, 1e-45
    ok[1][5] = -1
    ok[2][6], ok[2][7] = 0.0, 1.5
    ok[3][8], ok[3][9] = -0.1, 1.1
    u[10], u[11] = 1.0, math.nan
    res = vsd.sample_rows(X, u, *ok)
    _check(res, X, u, ok, err=5)
    assert (res.tok.cpu().numpy()[2:] == -1).all() and (res.tok.cpu().numpy()[:2] >= 0).all()


def test_flat_rows():
    """Thousands of entries kept, and the whole vocabulary."""
    _, X = _rows(4, 50001, "bf16", 9, spread=0.05)
    u = _u(4, 9)
    for s in [(1.0, 0, 0.99, 0.0), (1.0, 20000, 1.0, 0.0), (1.0, 20000, 0.9, 0.9), (1.0, 0, 1.0, 0.0)]:
        _check(vsd.sample_rows(X, u, *s), X, u, s)


@pytest.mark.parametrize("settings", [(1.0, 0, 1.0, 0.0), (0.8, 0, 0.3, 0.0), (1.0, 700, 1.0, 0.0), (0.7, 300, 0.9, 0.0),
                                      (1.2, 0, 1.0, 0.01), (1.0, 0, 0.5, 0.05), (0.0, 0, 1.0, 0.0)])
@pytest.mark.parametrize("V,kind", [(513, "f32"), (2048, "bf16"), (20000, "f32"), (65537, "bf16"), (262144, "bf16"),
                                    (262147, "bf16"), (300001, "f32")])
def test_lists_and_flat_rows_in_every_band(V, kind, settings):
    """Lists that fit and that do not, with the records' largest vocabulary and past it."""
    buf, X = _rows(5, V, kind, V)
    X[1] *= 0.1                # flat
    X[2] = X[2].round()        # long runs of equal logits
    X[3, V // 3] = 40.0        # one entry has it all
    X[4, ::2] = -INF
    u = _u(5, V + 1)
    _check(vsd.sample_rows(X, u, *settings), X, u, settings)


@pytest.mark.parametrize("kind", ("f32", "bf16"))
def test_borders_among_equal_logits_of_whole_rows(kind):
    """Equal weights sum exactly: p Z of V equal logits is the border itself."""
    for V in (500, 1000, 40000, 131072):
        _, X = _rows(3, V, kind, 1)
        X.fill_(2.5)
        X[1, ::2] = -INF
        u = _u(3, 2)
        for p in (0.5, 0.25, 0.125):
            _check(vsd.sample_rows(X, u, 0.7, 0, p, 0.0), X, u, (0.7, 0, p, 0.0))


def test_two_calls_at_once():
    """On two streams, each with its own workspace: the results of one after the other."""
    sets = []
    for seed, R, V in ((21, 600, 33000), (22, 300, 65000)):
        _, X = _rows(R, V, "bf16", seed)
        X[::7] *= 0.2
        u = _u(R, seed)
        sets.append((X, u, (0.9, 0, 0.9, 0.0), vsd.sample_rows(X, u, 0.9, 0, 0.9, 0.0)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        got = []
        for s, (X, u, st, _) in zip(streams, sets):
            with torch.cuda.stream(s):
                got.append(vsd.sample_rows(X, u, *st))
        torch.cuda.synchronize()
        for r, (_, _, _, want) in zip(got, sets):
            assert all(torch.equal(a, b) for a, b in zip(r[:3], want[:3]))


def test_a_row_alone_and_among_others():
    """The same results whatever the number of rows, their stride and the call."""
    buf, X = _rows(700, 3001, "bf16", 10)
    u = _u(700, 11)
    s = (0.9, 50, 0.95, 0.001)
    every = vsd.sample_rows(X, u, *s)
    again = vsd.sample_rows(buf.clone()[:, :3001], u, *s)
    odd = vsd.sample_rows(X[1::2], u[1::2].contiguous(), *s)
    one = vsd.sample_rows(X[699:], u[699:], *s)
    for a, b, c, d in zip(every[:3], again[:3], odd[:3], one[:3]):
        assert torch.equal(a, b) and torch.equal(a[1::2], c) and torch.equal(a[699:], d)
    _check(vsd.sample_rows(X[:5], u[:5], *s), X[:5], u[:5], s)


def test_column_range_of_a_wider_buffer():
    wide = torch.randn(6, 1024, device=DEV)
    X = wide[:, 256:256 + 301]
    u = _u(6, 12)
    _check(vsd.sample_rows(X, u, 1.0, 0, 0.8, 0.0), X, u, (1.0, 0, 0.8, 0.0))


def test_graph_and_stream():
    _, X = _rows(20, 9000, "bf16", 13)
    u = _u(20, 14)
    s = (0.8, 30, 0.9, 0.0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        vsd.sample_rows(X, u, *s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            res = vsd.sample_rows(X, u, *s)
    torch.cuda.synchronize()
    for k in range(3):
        X.copy_(torch.randn(20, 9000, device=DEV))
        u.copy_(torch.rand(20, device=DEV))
        graph.replay()
        eager = vsd.sample_rows(X, u, *s)
        torch.cuda.synchronize()
        for a, b in zip(res[:3], eager[:3]):
            assert torch.equal(a, b)
    _check(res, X, u, s)
