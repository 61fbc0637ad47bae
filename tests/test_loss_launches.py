"""Host-side arithmetic of the base losses' launches and workspaces, compiled from
the kernels' own header: a launch's size against its 32-bit count, the threads
of a row against the kernels there are, and the products' partial sums against
their regions for every number of rows in play."""
import math

import pytest

from tests.test_launch_bounds import _run

ROWS = (1, 63, 64, 512, 513, 2 ** 20, 2 ** 22 - 1, 2 ** 22, 2 ** 23, 2 ** 24 - 1)
VOCAB = (1, 7, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385, 32768, 32769, 65536, 65537, 131072, 131073, 2 ** 30)


def test_row_loss_launch(tmp_path):
    calls = [(r, v, w, g) for r in ROWS for v in VOCAB for w in (0, 1) for g in (0, 1)]
    got = _run(tmp_path, "vsd::RowThreads t;\n" + "".join(
        f't = vsd::row_loss_threads({r}ll, {v}, {w}, {g}); std::printf("%d %d %d\\n", t.threads, t.chunks, t.more);\n'
        for r, v, w, g in calls))
    kernels = {0: {(64, 0, 1), (256, 0, 1), (1024, 0, 1)},
               1: {(64, 4, 0), (256, 0, 1), (1024, 8, 0), (128, 4, 0), (256, 4, 0), (512, 4, 0), (512, 8, 0),
                   (1024, 16, 0), (1024, 16, 1)},
               2: {(64, 4, 0), (256, 0, 1), (1024, 8, 0), (256, 2, 0), (512, 2, 0), (1024, 2, 0), (1024, 4, 0),
                   (1024, 8, 1)}}
    for k, (r, v, w, g) in enumerate(calls):
        t = tuple(map(int, got[3 * k:3 * k + 3]))
        assert t in kernels[0 if not g else 1 + w]
        assert r * t[0] < 2 ** 32
        assert t[2] or t[0] * 8 * t[1] >= v


@pytest.mark.parametrize("R", (1, 100, 128, 129, 500, 1024, 6144, 8192, 8193, 70001, 300000))
@pytest.mark.parametrize("V", (1, 300, 32000, 128256))
@pytest.mark.parametrize("H", (64, 1024, 4096))
def test_partial_sums_fit_their_regions(tmp_path, R, V, H):
    """The plan's divisions (vsd_lm_loss.hpp: runs x row tiles within kLmLossRuns, ranges x tiles
    within kLmLossDh and kLmLossDw, at most kLmLossSplits) for every number n of rows in play."""
    ns = sorted({n for n in (1, 2, 63, 64, 255, 256, 257, R // 2, R - 1, R) if 1 <= n <= R})
    parts, sums, wsums, piece, runs_max, dh_max, dw_max, splits_max = map(int, _run(tmp_path, (
        f'std::printf("%lld %lld ", (long long)vsd::lm_loss_parts({R}ll, {V}), (long long)vsd::lm_loss_sums({R}ll, {H}));\n'
        f'const int piece = vsd::lm_loss_piece({R}ll, {V});\n'
        f'std::printf("%lld %d ", (long long)vsd::lm_loss_wsums({V}, {H}, piece), piece);\n'
        'std::printf("%d %d %d %d", vsd::kLmLossRuns, vsd::kLmLossDh, vsd::kLmLossDw, vsd::kLmLossSplits);\n')))
    assert piece % 256 == 0 and (piece >= V or piece >= 1024)
    cols = min(V, piece)
    for n in ns:
        nrt, nht, tiles = math.ceil(n / 256), math.ceil(H / 256), math.ceil(V / 256)
        few = R <= 128 or (R <= 8192 and math.ceil(R / 128) * math.ceil(V / 64) <= 512)
        runs = math.ceil(V / 64) if few else min(tiles, max(1, runs_max // nrt))
        assert 2 * runs * n <= parts
        splits = min(math.ceil(cols / 64), splits_max, max(1, dh_max // (nrt * nht)))
        assert splits * n * H <= sums
        wt = math.ceil(cols / 256) * nht
        wsplits = min(math.ceil(n / 64), splits_max, max(1, dw_max // wt)) if wsums else 1
        assert wsplits == 1 or wsplits * cols * H <= wsums
        assert wsums or 2 * wt > dw_max
