"""Draws, block matrices and gradients whose elements pass 2^31: their last parts
against calls on those alone."""
import pytest
import torch

import paper_2602_05774_amd as vsd

pytestmark = pytest.mark.gpu
DEV = "cuda"
R, V = 17000, 128256  # 2.18e9 elements
assert R * V > 1 << 31


@pytest.fixture(scope="module")
def logits():
    g = torch.Generator(device=DEV).manual_seed(1)
    Y = torch.empty(R, V, dtype=torch.bfloat16, device=DEV)
    for part in Y.split(1000):
        part.normal_(generator=g)
    yield Y
    del Y, part
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rule", (dict(), dict(top_k=50, top_p=0.9), dict(temp_target=0.2, top_p=0.99), dict(temp_target=0.0)))
def test_draws(logits, rule):
    u = torch.rand(R, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    all_rows, last = vsd.sample_rows(logits, u, **rule), vsd.sample_rows(logits[-32:], u[-32:], **rule)
    for a, b in zip(all_rows[:3], last[:3]):
        assert torch.equal(a[-32:], b)


@pytest.mark.parametrize("trans", (False, True))
@pytest.mark.parametrize("group", (1, 128))
def test_quantize(logits, group, trans):
    q = vsd.quantize_blocks(logits, group, trans)
    x = logits[:, -256:] if trans else logits[R // 128 * 128:]  # whole blocks
    part = vsd.quantize_blocks(x, group, trans)
    rows = part.values.shape[0]
    assert torch.equal(q.values[-rows:].view(torch.uint8), part.values.view(torch.uint8))
    assert torch.equal(q.scales[:, -part.scales.shape[1]:], part.scales)


@pytest.mark.parametrize("kind", (torch.bfloat16, torch.float32))
def test_product(kind):
    """Whole numbers, whose sums are exact in any order."""
    g = torch.Generator(device=DEV).manual_seed(3)
    one = lambda rows: torch.randint(-1, 2, (rows, 256), generator=g, device=DEV).float()  # noqa: E731
    A, B = one(R), one(V)
    a, b = (vsd.BlockMatrix(m.to(torch.float8_e4m3fn), torch.ones(2, m.shape[0], device=DEV), 256) for m in (A, B))
    out = vsd.block_product(a, b, kind)
    assert torch.equal(out[-300:], (A[-300:] @ B.T).to(kind))
    assert torch.equal(out[:, -300:], (A @ B[-300:].T).to(kind))
    del out
    torch.cuda.empty_cache()


def test_gradients(logits):
    g = logits.view(-1)
    norm = vsd.grad_norm([g])
    want = sum(float((p.double() ** 2).sum()) for p in logits.split(1000)) ** 0.5
    # 2^31 squares in 64 bits, the root's rounding to fp32
    assert abs(float(norm) - want) <= want * (2 ** -24 + 1e-12)
    out = torch.empty_like(g)
    res = vsd.clip_gradients([g], want / 3, out=[out])
    scale = res.scale.clone()
    assert float(res.norm) == float(norm)
    for at in (0, 1 << 31, g.numel() - (1 << 20)):
        assert torch.equal(out[at:at + (1 << 20)], (g[at:at + (1 << 20)].float() * scale).to(torch.bfloat16))
