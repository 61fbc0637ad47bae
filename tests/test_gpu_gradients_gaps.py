"""Gradients that lie in the gaps of another one's rows."""
import math

import pytest
import torch

import paper_2602_05774_amd as vsd
from tests.test_gpu_gradients import _check_clipped, _norm

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("kind", (torch.float32, torch.bfloat16))
def test_pieces_beside_a_gradients_columns(kind):
    buf = torch.randn(50, 80, device=DEV).to(kind)
    grads = [buf[:, :40], buf[5, 50:60], buf[9::3, 60:70], buf.view(-1)[46 * 80 + 40:47 * 80]]
    keep, before = buf.clone(), [t.clone() for t in grads]
    norm = _norm(grads)
    r = vsd.clip_gradients(grads, 0.2 * norm)
    assert abs(float(r.norm) - norm) <= 2.0 ** -24 * norm + 1e-12 * norm
    _check_clipped(grads, before, float(torch.tensor(0.2 * norm)) / norm)
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[:, :40] = rest[5, 50:60] = rest[46, 40:] = False
    rest[9::3, 60:70] = False
    assert torch.equal(buf[rest], keep[rest])
    with pytest.raises(vsd.VsdError, match="overlap"):
        vsd.clip_gradients([buf[:, :40], buf[5, 39:60]], math.inf)


def test_a_norm_of_the_tensors():
    """Refused where it would be scaled while it is read; read from a gradient that stays."""
    buf = torch.tensor([3.0, 4.0, 5.0, 0.0], device=DEV)
    for grads in ([buf], [buf[:2], buf[2:]]):
        with pytest.raises(vsd.VsdError, match="norm lies in tensor"):
            vsd.clip_gradients(grads, 1.0, norm=buf[2:3])
    out = torch.empty_like(buf)
    r = vsd.clip_gradients([buf], 1.0, norm=buf[2:3], out=[out])
    assert torch.equal(out, buf * r.scale) and float(r.norm) == 5.0
    r = vsd.clip_gradients([buf[:2]], 1.0, norm=buf[2:3])
    assert float(r.norm) == 5.0 and buf[2] == 5.0 and torch.equal(buf[:2], out[:2])
