"""The whole softmax's choice of a span, compiled from the kernels' own header, behind a
scan in the order of the kernel's: a span without weight is never taken, some span
is, and it holds u Z up to the sums' roundings."""
import pytest

from tests.test_launch_bounds import _run

# lane l's terms a[2 l] and a[2 l + 1], the sums of the lanes before in the wavefront's order
SCAN = """
auto scan = [](const double* a, double* before) {
  double v[64], w[64];
  for (int l = 0; l < 64; ++l) v[l] = a[2 * l] + a[2 * l + 1];
  for (int d = 1; d < 16; d *= 2) {  // in rows of 16 lanes
    for (int l = 0; l < 64; ++l) w[l] = l % 16 >= d ? v[l] + v[l - d] : v[l];
    for (int l = 0; l < 64; ++l) v[l] = w[l];
  }
  for (int l = 16; l < 32; ++l) v[l] += v[15];
  for (int l = 48; l < 64; ++l) v[l] += v[47];
  for (int l = 32; l < 64; ++l) v[l] += v[31];
  for (int l = 0; l < 64; ++l) before[l] = l > 0 ? v[l - 1] : 0.0;
  return v[63];
};
unsigned long long state = SEED;
auto uniform = [&]() {
  state = state * 6364136223846793005ull + 1442695040888963407ull;
  return (double)(state >> 11) / 9007199254740992.0;
};
long pairs = 0, none = 0, empty = 0, far = 0;
for (int row = 0; row < 400; ++row) {
  double a[128], before[64];
  const double same = 1.0 + 2047.0 * uniform();
  for (int s = 0; s < 128; ++s) a[s] = WEIGHT;
  const double z = scan(a, before);
  if (!(z > 0.0)) continue;
  for (int j = 0; j <= 64; ++j) {
    const double u = j < 64 ? j / 64.0 : 1.0 - 0x1p-24, target = u * z;
    int at = -1;
    for (int l = 63; l >= 0; --l) {
      const int which = vsd::draw_span(before[l], a[2 * l], a[2 * l + 1], target);
      if (which >= 0) at = 2 * l + which;
    }
    ++pairs;
    if (at < 0) { ++none; continue; }
    empty += !(a[at] > 0.0);
    long double upto = 0.0L;
    for (int s = 0; s < at; ++s) upto += a[s];
    far += upto > target + 1e-12 * z || upto + a[at] < target - 1e-12 * z;
  }
}
std::printf("%ld %ld %ld %ld\\n", pairs, none, empty, far);
"""


@pytest.mark.parametrize("weight", ["s % 2 ? same : 0.0",                      # equal spans behind masked ones
                                    "s % 2 ? 0.0 : same", "same", "s % 4 == 3 ? same : 0.0",
                                    "s % 3 == 1 ? 1.0 + 2047.0 * uniform() : 0.0",
                                    "uniform() < 0.5 ? same : 0.0", "uniform() < 0.2 ? same * uniform() : 0.0",
                                    "s == row % 128 ? same : 0.0", "s < 2 ? same : 1e-300"])
def test_span_has_weight(tmp_path, weight):
    pairs, none, empty, far = map(int, _run(tmp_path, SCAN.replace("SEED", "12345").replace("WEIGHT", weight)))
    assert pairs > 20000 and (none, empty, far) == (0, 0, 0)
