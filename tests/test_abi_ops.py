"""C-ABI and binding checks of the filtered draws, the block matrices and the
gradients' clipping that need no GPU: every call here fails validation before
anything is launched."""
import ctypes
import os

import pytest
import torch

import paper_2602_05774_amd as vsd
from paper_2602_05774_amd import _lib

FAKE = 0x10000  # a 16-byte aligned stand-in address; never dereferenced
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libvsd.so not built (run __graft_entry__.build())")
    return _lib.load()


def _ref(x):
    return None if x is None else ctypes.byref(x)


LOGITS = _lib.VsdSrc(FAKE, None, None)


def _rows(**kw):
    return _lib.VsdRows(**{**dict(R=24, ld=1000, v=1000, dtype=_lib.VSD_F32, hidden_dim=0), **kw})


def _draw(lib, rows=None, src=LOGITS, setting=None, u=FAKE, tok=FAKE, ws=FAKE, n=1 << 40, err=FAKE):
    d = _lib.VsdDraw(*{**dict(t=1.0, k=0, p=1.0, m=0.0, rt=None, rk=None, rp=None, rm=None), **(setting or {})}.values())
    return lib.vsd_sample_rows(_ref(rows or _rows()), _ref(src), _ref(d), u, tok, None, None, ws, n, err, None)


@pytest.mark.parametrize("kw,code", [
    (dict(R=0), 2), (dict(R=1 << 22), 2), (dict(v=0), 2), (dict(dtype=3), 3), (dict(ld=999), 2), (dict(ld=1001), 4),
    (dict(hidden_dim=128, dtype=_lib.VSD_BF16), 6)])
def test_draw_rows(lib, kw, code):
    assert _draw(lib, rows=_rows(**kw)) == code and lib.vsd_last_error().decode() != ""


@pytest.mark.parametrize("setting", [dict(t=-1.0), dict(t=NAN), dict(t=1e-45), dict(t=INF), dict(k=-1), dict(p=0.0),
                                     dict(p=1.5), dict(p=NAN), dict(m=-0.1), dict(m=1.1), dict(m=NAN)])
def test_draw_settings(lib, setting):
    assert _draw(lib, setting=setting) == 3
    # a setting of each row takes the common one's place: that is not looked at (the workspace is what is missing)
    name = {"t": "rt", "k": "rk", "p": "rp", "m": "rm"}[next(iter(setting))]
    assert _draw(lib, setting={**setting, name: FAKE}, ws=None) == 7


def test_draw_pointers_and_workspace(lib):
    need = ctypes.c_size_t()
    assert lib.vsd_draw_workspace_bytes(_ref(_rows()), ctypes.byref(need)) == 0 and need.value > 24 * 80
    assert _draw(lib, n=need.value - 1) == 7 and _draw(lib, ws=None) == 7 and _draw(lib, ws=FAKE + 8) == 4
    for kw in (dict(u=None), dict(tok=None), dict(err=None), dict(src=None)):
        assert _draw(lib, **kw) == 1
    assert lib.vsd_draw_workspace_bytes(_ref(_rows()), None) == 1
    assert lib.vsd_draw_workspace_bytes(_ref(_rows(v=(1 << 18) + 1)), ctypes.byref(need)) == 0 and need.value == 0


def _blocks(**kw):
    return _lib.VsdBlocks(**{**dict(values=FAKE, scales=FAKE, rows=300, cols=500, ld=512, scale_ld=300, group=1), **kw})


BAD_BLOCKS = [(dict(values=None), 1), (dict(scales=None), 1), (dict(rows=0), 2), (dict(cols=0), 2), (dict(rows=1 << 31), 2),
              (dict(ld=500), 2), (dict(ld=384), 2), (dict(scale_ld=299), 2), (dict(group=64), 3), (dict(values=FAKE + 8), 4),
              (dict(scales=FAKE + 2), 4)]


@pytest.mark.parametrize("kw,code", BAD_BLOCKS)
def test_bad_block_matrices(lib, kw, code):
    n = ctypes.c_size_t()
    good, bad = _blocks(), _blocks(**kw)
    assert lib.vsd_block_product(_ref(bad), _ref(good), FAKE, 304, 0, FAKE, 1 << 40, None) == code
    assert lib.vsd_block_product(_ref(good), _ref(bad), FAKE, 304, 0, FAKE, 1 << 40, None) == code
    assert lib.vsd_product_workspace_bytes(_ref(good), _ref(bad), 0, ctypes.byref(n)) == code
    assert lib.vsd_quantize_blocks(FAKE, bad.rows, bad.cols, bad.cols, 0, 0, _ref(bad), None) == code


def test_bad_products(lib):
    a, b = _blocks(), _blocks(rows=200, scale_ld=2, group=128)
    call = lambda a=a, b=b, out=FAKE, ld=200, dt=0, ws=FAKE, n=1 << 40: lib.vsd_block_product(  # noqa: E731
        _ref(a), _ref(b), out, ld, dt, ws, n, None)
    assert call(a=None) == 1 and call(b=None) == 1 and call(out=None) == 1
    assert call(a=b) == 6                                  # the rows' factor has a scale per row
    assert call(b=_blocks(cols=400)) == 2
    assert call(ld=199) == 2 and call(ld=201) == 4 and call(out=FAKE + 4) == 4 and call(dt=2) == 3
    assert call(b=_blocks(rows=1 << 30, scale_ld=1 << 30), a=_blocks(rows=1 << 30, scale_ld=1 << 30), ld=1 << 30) == 2
    n = ctypes.c_size_t()
    few = _blocks(rows=300, cols=4096, ld=4096)
    assert lib.vsd_product_workspace_bytes(_ref(few), _ref(_blocks(rows=520, cols=4096, ld=4096, scale_ld=520)), 1, ctypes.byref(n)) == 0
    assert n.value > 0                                     # few tiles: the sum in ranges
    assert lib.vsd_block_product(_ref(few), _ref(_blocks(rows=520, cols=4096, ld=4096, scale_ld=520)), FAKE, 520, 1, FAKE,
                                 n.value - 1, None) == 7
    assert lib.vsd_product_workspace_bytes(_ref(a), _ref(b), 0, None) == 1
    assert lib.vsd_product_workspace_bytes(_ref(a), _ref(b), 2, ctypes.byref(n)) == 3


def test_bad_quantising(lib):
    out = _blocks()
    call = lambda x=FAKE, r=300, c=500, ld=500, dt=0, tr=0, out=out: lib.vsd_quantize_blocks(x, r, c, ld, dt, tr, _ref(out), None)  # noqa: E731
    assert call(x=None) == 1 and call(dt=2) == 3 and call(r=299) == 2 and call(c=501) == 2 and call(ld=499) == 2
    assert call(tr=1) == 2 and call(x=FAKE + 2) == 4 and call(x=FAKE + 1, dt=1) == 4
    big = _blocks(rows=1 << 30, cols=1 << 30, ld=1 << 30, scale_ld=1 << 30)
    assert call(r=1 << 30, c=1 << 30, ld=1 << 30, out=big) == 2


def _tensors(*items):
    return (_lib.VsdTensor * len(items))(*[_lib.VsdTensor(*i) for i in items])


def _clip(lib, g, out=None, n=None, bound=1.0, norm=None, norm_out=FAKE, scale=FAKE, ws=FAKE, size=1 << 40):
    return lib.vsd_clip_gradients(g, out, len(g) if n is None else n, bound, norm, norm_out, scale, ws, size, None)


def test_bad_gradients(lib):
    one = (FAKE, 1, 100, 100, 0)
    for bad, code in [((None, 1, 100, 100, 0), 1), ((FAKE, -1, 100, 100, 0), 2), ((FAKE, 1, -1, 100, 0), 2), ((FAKE, 2, 100, 99, 0), 2),
                      ((FAKE, 1, 1 << 45, 1 << 45, 0), 2), ((FAKE, 1, 1 << 44, 1 << 44, 0), 2), ((FAKE, 1, 100, 100, 2), 3),
                      ((FAKE + 2, 1, 100, 100, 0), 4), ((FAKE + 1, 1, 100, 100, 1), 4)]:
        assert _clip(lib, _tensors(bad)) == code
        assert lib.vsd_grad_norm(_tensors(bad), 1, FAKE, FAKE, 1 << 40, None) == code
    g = _tensors(one)
    for bound in (0.0, -1.0, NAN):
        assert _clip(lib, g, bound=bound) == 3
    assert _clip(lib, g, n=0) == 2 and lib.vsd_grad_norm(g, 0, FAKE, FAKE, 1 << 40, None) == 2
    assert lib.vsd_grad_norm(None, 1, FAKE, FAKE, 1 << 40, None) == 1 and lib.vsd_grad_norm(g, 1, None, FAKE, 1 << 40, None) == 1
    need = ctypes.c_size_t()
    assert lib.vsd_norm_workspace_bytes(1, ctypes.byref(need)) == 0
    assert _clip(lib, g, size=need.value - 1) == 7 and _clip(lib, g, ws=None) == 7 and _clip(lib, g, ws=FAKE + 8) == 4
    assert lib.vsd_norm_workspace_bytes(0, ctypes.byref(need)) == 2 and lib.vsd_norm_workspace_bytes(1, None) == 1
    assert _clip(lib, g, norm=FAKE) == 3                   # the result in the given norm's place
    assert _clip(lib, g, out=_tensors((FAKE + 4096, 1, 99, 99, 0))) == 2
    assert _clip(lib, g, out=_tensors((FAKE, 1, 100, 100, 1))) == 3


def test_what_is_written_overlaps_nothing(lib):
    A = FAKE
    assert _clip(lib, _tensors((A, 1, 100, 100, 0), (A, 1, 100, 100, 0))) == 3            # one gradient twice
    assert _clip(lib, _tensors((A, 1, 100, 100, 0), (A + 396, 1, 100, 100, 0))) == 3      # the last element
    # out of place: onto another gradient, or onto each other
    g = _tensors((A, 1, 100, 100, 0), (A + 400, 1, 100, 100, 0))
    assert _clip(lib, g, out=_tensors((A + 400, 1, 100, 100, 0), (A + 4000, 1, 100, 100, 0))) == 3
    assert _clip(lib, g, out=_tensors((A + 4000, 1, 100, 100, 0), (A + 4000, 1, 100, 100, 0))) == 3
    assert _clip(lib, g, out=_tensors((A + 4, 1, 100, 100, 0), (A + 4000, 1, 100, 100, 0))) == 3
    # rows of one buffer: shared columns
    assert _clip(lib, _tensors((A, 10, 60, 100, 0), (A + 200, 10, 50, 100, 0))) == 3
    assert _clip(lib, _tensors((A, 10, 60, 100, 0), (A + 4 * 90, 10, 20, 100, 0))) == 3   # ... around the row's end
    # apart (what is missing then is the workspace)
    for ok in (g, _tensors((A, 10, 60, 100, 0), (A + 240, 10, 40, 100, 0)), _tensors((A, 0, 5, 5, 0), (A, 1, 5, 5, 0))):
        assert _clip(lib, ok, ws=None) == 7


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 8)
    for call, what in [(lambda: vsd.sample_rows(x, x[:, 0]), "device"), (lambda: vsd.quantize_blocks(x), "device"),
                       (lambda: vsd.grad_norm([x]), "device"), (lambda: vsd.clip_gradients([], 1.0), "one or more"),
                       (lambda: vsd.sample_rows(vsd.LmHead(x, x), x[:, 0]), "materialised"),
                       (lambda: vsd.block_product(vsd.BlockMatrix(x, x, 8), vsd.BlockMatrix(x, x, 8)), "float8")]:
        with pytest.raises(ValueError, match=what):
            call()
