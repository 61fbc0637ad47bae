"""Rules of the base losses' launches that other rules rely on, compiled from the
kernels' own header."""
from tests.test_launch_bounds import _run

SIZES = [(v, k, h) for v in (1, 64, 130, 32000, 128256, 2 ** 20, 2 ** 29) for k in (0, 1, 64) for h in (64, 4096, 65536)]


def test_the_total_of_few_rows_is_formed_by_their_joins(tmp_path):
    """The counter that spares the total a launch is counted by workgroups of one row each."""
    body = "".join(f'std::printf("%d\\n", vsd::lm_by_workgroup({r}, {v}, {k}, {h}));\n'
                   for r in (1, 2, 63) for v, k, h in SIZES)
    body += "".join(f'std::printf("%d\\n", vsd::lm_by_workgroup(vsd::kTotalRows, {v}, {k}, {h}));\n' for v, k, h in SIZES)
    assert set(_run(tmp_path, body)) == {"1"}


def test_gradient_and_sums_come_from_the_same_products(tmp_path):
    """With a gradient the 64-column forward runs exactly where its logits are kept, and another
    forward's log-sum-exps (two per run and row, a run per tile at most) fit few rows' region."""
    cases = [(r, v) for r in (1, 16, 100, 128, 129, 900, 8192, 8193) for v in (1, 130, 6000, 524288, 524289, 700001, 2 ** 29)]
    got = _run(tmp_path, "".join(
        f'std::printf("%d %d %d %lld\\n", vsd::lm_few_forward({r}, {v}, true), vsd::lm_few_keeps({r}, {v}), '
        f'vsd::lm_few_forward({r}, {v}, false) == vsd::lm_few({r}, {v}), (long long)vsd::lm_loss_parts({r}, {v}));\n'
        for r, v in cases))
    runs_max = 1024
    for n, (r, v) in enumerate(cases):
        grad, keeps, same, parts = map(int, got[4 * n:4 * n + 4])
        assert grad == keeps and same
        if r <= 128 and not keeps:
            assert 2 * min(-(-v // 256), runs_max) * r <= parts
