"""Block products of matrices whose row stride the tiles' 32-bit offsets do not reach."""
import pytest
import torch

import paper_2602_05774_amd as vsd
from tests.test_gpu_blocks import _check_product, _matrix

pytestmark = pytest.mark.gpu
DEV = "cuda"
LD = (1 << 22) + 128


@pytest.mark.parametrize("M,N,K,a_wide,b_wide", [(65, 33, 128, True, False), (97, 70, 300, False, True), (130, 161, 1, True, True),
                                                 (20, 200, 700, True, True)])
@pytest.mark.parametrize("group", (1, 128))
@pytest.mark.parametrize("kind", ("f32", "bf16"))
def test_product_of_far_rows(M, N, K, a_wide, b_wide, group, kind):
    a, b = _matrix(M, K, 1, M), _matrix(N, K, group, N)

    def far(m):
        """The same matrix in rows LD apart, in front of bytes that are not its own."""
        width = m.values.shape[1]
        buf = torch.full((m.values.shape[0], LD), 0x7F, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)  # NaN
        buf[:, :width] = m.values
        return m._replace(values=buf[:, :width])

    near = vsd.block_product(a, b, dtype=torch.float32 if kind == "f32" else torch.bfloat16)
    wide = [far(m) if w else m for m, w in ((a, a_wide), (b, b_wide))]
    assert max(m.values.stride(0) for m in wide) == LD
    out = torch.full((M + 1, (N + 7) // 8 * 8 + 8), -7.0, dtype=near.dtype, device=DEV)
    vsd.block_product(*wide, out=out[:M, :N])
    _check_product(out[:M, :N], *wide, kind)
    _check_product(near, a, b, kind)
    assert (out[M] == -7).all() and (out[:, N:] == -7).all()
