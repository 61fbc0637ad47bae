"""C-ABI and binding checks of the base losses and the top logits that need no
GPU: every call here fails validation before anything is launched."""
import ctypes
import os

import pytest
import torch

import paper_2602_05774_amd as vsd
from paper_2602_05774_amd import _lib

FAKE = 0x10000  # a 16-byte aligned stand-in address; never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libvsd.so not built (run __graft_entry__.build())")
    return _lib.load()


def _rows(**kw):
    return _lib.VsdRows(**{**dict(R=24, ld=1000, v=1000, dtype=_lib.VSD_F32, hidden_dim=0), **kw})


def _head(**kw):
    return _rows(**{**dict(dtype=_lib.VSD_BF16, hidden_dim=128), **kw})


LOGITS, HEAD = _lib.VsdSrc(FAKE, None, None), _lib.VsdSrc(None, FAKE, FAKE)
OUT = _lib.VsdLossOut(FAKE, FAKE, FAKE, FAKE)
HGRAD = _lib.VsdLossGrad(None, 0, FAKE, FAKE + 16, 0)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _ce(lib, rows=None, src=LOGITS, labels=FAKE, temp=1.0, scale=1.0, out=OUT, grad=None, ws=None, n=0):
    rows = _rows() if rows is None else rows
    return lib.vsd_cross_entropy(_ref(rows), _ref(src), labels, None, temp, scale, _ref(out), _ref(grad), ws, n, None)


def _kd(lib, rows=None, src=LOGITS, k=8, idx=FAKE, val=FAKE, dt=0, temps=(1.0, 1.0), out=OUT, grad=None, ws=None, n=0):
    rows = _rows() if rows is None else rows
    return lib.vsd_distill_loss(_ref(rows), _ref(src), k, idx, val, dt, None, None, *temps, 1.0, _ref(out), _ref(grad),
                                ws, n, None)


def _top(lib, rows=None, src=LOGITS, k=8, d2t=None, vd=0, temp=1.0, idx=FAKE, val=FAKE, ws=None, n=0, err=FAKE):
    rows = _rows() if rows is None else rows
    return lib.vsd_top_logits(_ref(rows), _ref(src), k, d2t, vd, temp, idx, val, None, ws, n, err, None)


@pytest.mark.parametrize("call", (_ce, _kd, _top))
@pytest.mark.parametrize("kw,code", [
    (dict(R=0), 2), (dict(R=1 << 24), 2), (dict(v=0), 2), (dict(v=(1 << 30) + 8, ld=1 << 31), 2), (dict(dtype=3), 3), (dict(ld=999), 2), (dict(ld=1001), 4),
    (dict(hidden_dim=-64), 2), (dict(hidden_dim=100), 2), (dict(hidden_dim=128), 6),
])
def test_bad_rows(lib, call, kw, code):
    assert call(lib, rows=_rows(**kw)) == code
    assert lib.vsd_last_error().decode() != ""


@pytest.mark.parametrize("call", (_ce, _kd, _top))
def test_bad_sources(lib, call):
    assert call(lib, src=None) == 1
    assert call(lib, src=_lib.VsdSrc(None, None, None)) == 1
    assert call(lib, src=_lib.VsdSrc(FAKE + 8, None, None)) == 4
    assert call(lib, src=HEAD) == 6                       # a head needs hidden_dim


@pytest.mark.parametrize("temp", (0.0, -1.0, float("inf"), float("nan"), 1e-45, 1e31))
def test_bad_temperatures(lib, temp):
    assert _ce(lib, temp=temp) == 3 and _top(lib, temp=temp) == 3
    assert _kd(lib, temps=(temp, 1.0)) == 3 and _kd(lib, temps=(1.0, temp)) == 3


def test_bad_outputs_and_gradients(lib):
    for call in (_ce, _kd):
        assert call(lib, out=None) == 1
        assert call(lib, out=_lib.VsdLossOut(None, FAKE, FAKE, FAKE)) == 1
        assert call(lib, out=_lib.VsdLossOut(FAKE, FAKE, FAKE, None)) == 1
        assert call(lib, grad=_lib.VsdLossGrad(None, 1000, None, None, 0)) == 1
        assert call(lib, grad=_lib.VsdLossGrad(FAKE + 4, 1000, None, None, 0)) == 4
        assert call(lib, grad=_lib.VsdLossGrad(FAKE, 999, None, None, 0)) == 2
        assert call(lib, grad=_lib.VsdLossGrad(FAKE + 16, 1002, None, None, 0)) == 4
        assert call(lib, grad=_lib.VsdLossGrad(FAKE, 1000, FAKE, None, 0)) == 6
        hg = lambda **kw: _lib.VsdLossGrad(**{**dict(grad_hidden=FAKE, grad_weight=FAKE + 16), **kw})  # noqa: E731
        # in the logits' place: their stride, the check of which comes before the alignment's
        assert call(lib, grad=_lib.VsdLossGrad(FAKE, 1002, None, None, 0)) == 3
        head = dict(rows=_head(), src=HEAD, ws=FAKE, n=1 << 40)
        assert call(lib, **head, grad=hg(grad_hidden=None)) == 1
        assert call(lib, **head, grad=hg(grad_hidden=FAKE + 8)) == 4
        assert call(lib, **head, grad=hg(grad_weight=FAKE + 8)) == 4
        assert call(lib, **head, grad=hg(weight_dtype=2)) == 3
        assert call(lib, **head, grad=hg(grad_weight=FAKE)) == 3    # the weight itself
        assert call(lib, **head, grad=hg(grad_logits=FAKE)) == 6
    assert _ce(lib, labels=None) == 1
    assert _ce(lib, scale=float("inf")) == 3
    assert _kd(lib, idx=None) == 1 and _kd(lib, val=None) == 1 and _kd(lib, dt=2) == 3
    assert _kd(lib, k=0) == 3 and _kd(lib, k=65) == 3
    assert _top(lib, k=0) == 3 and _top(lib, k=65) == 3
    assert _top(lib, idx=None) == 1 and _top(lib, val=None) == 1 and _top(lib, err=None) == 1
    assert _top(lib, rows=_rows(R=1 << 22)) == 2


def test_workspaces(lib):
    need = ctypes.c_size_t()
    for call, k in ((_ce, 0), (_kd, 8)):
        for grad in (None, HGRAD):
            assert lib.vsd_loss_workspace_bytes(ctypes.byref(_head()), k, int(grad is not None), ctypes.byref(need)) == 0
            head = dict(rows=_head(), src=HEAD, grad=grad)
            assert call(lib, **head, ws=FAKE, n=need.value - 1) == 7
            assert call(lib, **head, ws=None, n=need.value) == 7
            assert call(lib, **head, ws=FAKE + 4, n=need.value) == 4
    assert lib.vsd_loss_workspace_bytes(ctypes.byref(_rows()), 8, 1, ctypes.byref(need)) == 0 and need.value == 0
    assert lib.vsd_loss_workspace_bytes(ctypes.byref(_head()), 65, 1, ctypes.byref(need)) == 3
    assert lib.vsd_loss_workspace_bytes(ctypes.byref(_head()), 8, 1, None) == 1
    assert lib.vsd_top_workspace_bytes(ctypes.byref(_rows()), 1, None) == 1
    assert lib.vsd_top_workspace_bytes(ctypes.byref(_rows()), 0, ctypes.byref(need)) == 0 and need.value == 0
    assert lib.vsd_top_workspace_bytes(ctypes.byref(_rows()), 1, ctypes.byref(need)) == 0 and need.value >= 4125
    assert _top(lib, d2t=FAKE, vd=500, ws=FAKE, n=need.value - 1) == 7
    assert _top(lib, d2t=FAKE, vd=500, ws=FAKE + 8, n=need.value) == 4
    assert _top(lib, d2t=FAKE + 4, vd=500, ws=FAKE, n=need.value) == 4
    assert _top(lib, d2t=FAKE, vd=1001, ws=FAKE, n=need.value) == 2
    assert _top(lib, d2t=FAKE, vd=0, ws=FAKE, n=need.value) == 2


@pytest.mark.parametrize("R,v,H", ((1, 1, 64), (6144, 128256, 4096), (70000, 9000, 64), (1 << 20, 50000, 1024),
                                   (48, 32000, 4096), (300, 257, 65536)))
def test_workspace_is_bounded_by_its_parts(lib, R, v, H):
    """Never the logits of a large batch: about 1 GiB of their gradient at most, the hidden
    states, the products' fp32 partial sums (32 ranges or 2560 and 512 tiles of 256 x 256) and
    small per-row records."""
    got = vsd.loss_workspace_bytes(R, v, H, 16, True)
    pad, tiles = (R + 63) // 64 * 64, -(-v // 256)
    g = max(1 << 30, pad * 2 * 1024) + pad * 2 * (256 + 128)
    dh = 4 * min(32 * R * H, max(2560 << 16, R * H))
    parts = 16 * max(R, min(1024 * 256, R * tiles), R * -(-v // 64) if R <= 128 else 512 * 128)
    assert got <= g + dh + 4 * (512 << 16) + pad * H * 2 + parts + R * (16 * 12 + 64) + 16 * 256


@pytest.mark.parametrize("kw", (dict(R=(1 << 24) - 1, v=1 << 20), dict(v=(1 << 29) + 1, hidden_dim=64),
                                dict(R=1 << 23, v=8, hidden_dim=4096), dict(R=1 << 20, v=1 << 26, hidden_dim=64)))
def test_fused_launches_stay_within_32_bits(lib, kw):
    assert _ce(lib, rows=_head(**kw), src=HEAD, ws=FAKE, n=1 << 50) == 2


def test_binding_refuses_host_tensors():
    x, lab = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        vsd.cross_entropy(x, lab)
    with pytest.raises(ValueError, match="device tensor"):
        vsd.distill_loss(x, lab[:, None], x[:, :1])
    with pytest.raises(ValueError, match="device tensor"):
        vsd.top_logits(x, 2)
    with pytest.raises(ValueError, match="hidden"):
        vsd.cross_entropy(vsd.LmHead(x.bfloat16(), x.bfloat16()), lab)
    with pytest.raises(ValueError, match="materialised"):
        vsd.top_logits(vsd.LmHead(x, x), 2)
