"""Block products of more columns than one launch takes."""
import pytest
import torch

import paper_2602_05774_amd as vsd

pytestmark = pytest.mark.gpu
DEV = "cuda"
N = (1 << 29) + 100
PERIOD = 1000003  # the factor's rows repeat: no launch's first column is a multiple of it


@pytest.fixture(scope="module")
def wide():
    """(one period of b's rows, b's values): whole numbers, whose sums are exact in any order."""
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("b takes 69 GB")
    g = torch.Generator(device=DEV).manual_seed(1)
    part = torch.randint(-1, 2, (PERIOD, 128), generator=g, device=DEV).to(torch.float8_e4m3fn)
    val = torch.empty(N, 128, dtype=torch.float8_e4m3fn, device=DEV)
    for at in range(0, N, PERIOD):
        val[at:at + PERIOD].copy_(part[:min(PERIOD, N - at)])
    yield part.float(), val
    del val, part
    torch.cuda.empty_cache()


@pytest.mark.parametrize("group,kind", [(128, torch.bfloat16), (1, torch.float32)])
def test_few_rows_by_more_columns_than_a_launch(wide, group, kind):
    part, val = wide
    g = torch.Generator(device=DEV).manual_seed(2)
    A = torch.randint(-1, 2, (3, 128), generator=g, device=DEV).float()
    sb = torch.exp2(torch.randint(-3, 4, (1, -(-N // group)), generator=g, device=DEV, dtype=torch.int8).float())
    a = vsd.BlockMatrix(A.to(torch.float8_e4m3fn), torch.ones(1, 3, device=DEV), 128)
    out = vsd.block_product(a, vsd.BlockMatrix(val, sb, 128), kind)
    once = A @ part.T
    for at in range(0, N, PERIOD):
        n = min(PERIOD, N - at)
        cols = torch.arange(at, at + n, device=DEV) // group
        assert torch.equal(out[:, at:at + n], (once[:, :n] * sb[0][cols]).to(kind)), at
