"""What the bindings of the draws, block matrices and gradients refuse, before any launch."""
import math

import pytest
import torch

import paper_2602_05774_amd as vsd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
REFUSED = (ValueError, TypeError, vsd.VsdError)


def _each(call, good, bad):
    call(**good)
    for kw in bad:
        with pytest.raises(REFUSED):
            call(**{**good, **kw})
            pytest.fail(f"not refused: {kw}")


def test_draws_refuse():
    Y, u = torch.randn(4, 64, device=DEV), torch.rand(4, device=DEV)
    head = vsd.LmHead(torch.randn(4, 64, device=DEV, dtype=torch.bfloat16),
                      torch.randn(64, 64, device=DEV, dtype=torch.bfloat16))
    _each(vsd.sample_rows, dict(Y=Y, u=u), [
        dict(Y=head), dict(Y=Y.half()), dict(Y=Y[0]), dict(Y=Y[:, ::2]), dict(Y=Y[:0]), dict(Y=Y.cpu()),
        dict(u=None), dict(u=u[:3]), dict(u=u.double()), dict(u=u.cpu()),
        dict(temp_target=-1.0), dict(temp_target=1e-31), dict(temp_target=math.nan), dict(temp_target=u.double()),
        dict(temp_target=u[:3]), dict(top_k=-1), dict(top_k=2.5), dict(top_k=torch.ones(4, device=DEV)),
        dict(top_p=0.0), dict(top_p=1.5), dict(top_p=math.nan), dict(top_p=u[:1]), dict(min_p=-0.1), dict(min_p=1.5),
        dict(min_p=math.nan), dict(device_error=torch.zeros(1, device=DEV)), dict(workspace=torch.zeros(64, device=DEV)),
    ])


def test_block_matrices_refuse():
    x = torch.randn(200, 300, device=DEV)
    out = vsd.quantize_blocks(x)
    _each(vsd.quantize_blocks, dict(x=x), [
        dict(x=x.cpu()), dict(x=x.half()), dict(x=x[0]), dict(x=x[:, ::2]), dict(x=x[:0]), dict(group=64),
        dict(out=vsd.quantize_blocks(x[:199])), dict(out=vsd.quantize_blocks(x, 128)), dict(transpose=True, out=out),
        dict(out=out._replace(cols=299)), dict(out=out._replace(values=out.values.view(torch.int8))),
        dict(out=out._replace(scales=out.scales.double())), dict(out=out._replace(values=out.values[:, :300])),
    ])
    b = vsd.quantize_blocks(torch.randn(130, 300, device=DEV), 128)
    res = torch.full((200, 136), 5.0, device=DEV)
    _each(vsd.block_product, dict(a=out, b=b), [
        dict(a=b, b=out), dict(b=vsd.quantize_blocks(torch.randn(130, 290, device=DEV), 128)),
        dict(a=out._replace(scales=out.scales[:2])), dict(b=b._replace(scales=b.scales.cpu())), dict(dtype=torch.float16),
        dict(out=res), dict(out=res[:, 1:131]), dict(out=res[:, :130].half()), dict(out=res.cpu()[:, :130]),
        dict(out=torch.empty(200, 130, device=DEV)), dict(out=res.T[:130]), dict(out=[]),
    ])
    assert (res == 5).all()


def test_gradients_refuse():
    g = [torch.randn(40, device=DEV), torch.randn(6, 10, device=DEV)]
    keep = [t.clone() for t in g]
    _each(vsd.clip_gradients, dict(grads=g, max_norm=1e30), [
        dict(grads=[]), dict(grads=[None]), dict(grads=[g[0], None]), dict(grads=[g[0].half()]), dict(grads=[g[0], g[1].cpu()]),
        dict(grads=[g[0][::2]]), dict(grads=[g[1].T]), dict(grads=[g[1].expand(3, 6, 10)]), dict(max_norm=0.0),
        dict(max_norm=-1.0), dict(max_norm=math.nan), dict(out=[g[0]]), dict(out=[g[1], g[0]]), dict(out=[g[0], g[1].half()]),
        dict(norm=torch.ones((), device=DEV)), dict(norm=torch.ones(1)), dict(norm=torch.ones(1, device=DEV).double()),
        dict(grads=[g[0], g[0]]),
    ])
    assert all(torch.equal(a, b) for a, b in zip(g, keep))
    for bad in ([], [None], [g[0], g[0].cpu()], [g[0].long()]):
        with pytest.raises(REFUSED):
            vsd.grad_norm(bad)
