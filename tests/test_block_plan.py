"""The block products' launches against their 32-bit count, compiled from the kernels' own header."""
import pytest

from tests.test_launch_bounds import _run

MAX = 2 ** 31 - 1
COLS = (1, 32, 33, 2 ** 24, 2 ** 28 - 1, 2 ** 28, 2 ** 28 + 1, 2 ** 29 - 32, 2 ** 29, 2 ** 29 + 100, 2 ** 30 + 7, MAX - 63)


@pytest.mark.parametrize("M", (1, 16, 17, 32, 33, 64, 65, 300))
def test_product_launches_fit_their_grids(tmp_path, M):
    cases = [(n, blocks, f32) for n in COLS for blocks in (1, 33) for f32 in (0, 1)
             if -(-M // 32) * -(-n // 32) < 2 ** 26]  # (more results than that are refused)
    got = _run(tmp_path, "".join(
        f"{{ const auto p = vsd::block_plan({M}, {n}ll, {blocks}, {blocks} * 128ll, {blocks} * 128ll, {f32});\n"
        'std::printf("%d %d %d %d %d %lld\\n", p.few, p.tiles, p.runs, p.ranges, p.waves, (long long)vsd::kBlockFewCols); }\n'
        for n, blocks, f32 in cases))
    for k, (n, blocks, f32) in enumerate(cases):
        few, tiles, runs, ranges, waves, cols = map(int, got[6 * k:6 * k + 6])
        if few:
            assert ranges == 1 or n <= cols  # (launches of part of the columns are of all of the sum)
            assert -(-min(n, cols) // 32) * ranges * waves * 64 < 2 ** 32, (M, n)
        elif tiles:
            assert -(-M // 256) * runs * ranges * 512 < 2 ** 32, (M, n)
        else:
            assert -(-M // 32) * -(-n // 32) * 64 <= 2 ** 32 - 64, (M, n)
