"""Which keys a walk counts, to the key: every score is 0, so that each key seen has the same weight, and values
are whole numbers, so that O times the number of keys is a whole number too.  A key too many or too few moves
the LSE by 1 / n, one taken for another moves O by 1 / n at least."""
import numpy as np
import pytest

import oracle.fp8 as ref
from tests.window_util import Case, bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(8, 1, 128), (4, 2, 64), (32, 8, 128)])
@pytest.mark.parametrize("prefix, chunk, window, sinks", [
    ([9000], [1], None, 0), ([9000], [130], None, 0), ([9001], [130], 4999, 33), ([8191], [64], 4096, 4),
    ([6000], [200], 5000, 64), ([0], [1500], 1100, 70), ([7007, 5000, 12], [1, 300, 40], 2500, 65),
    ([300] * 20, [1] * 20, 257, 5), ([5000, 4000], [1, 1], 3000, 31)])
@pytest.mark.parametrize("fp8", [False, True])
def test_every_key_counts_once(fp8, heads, prefix, chunk, window, sinks):
    """Probabilities are exactly 1 (scores and the reference point are 0), sums of them and of the values, up
    to 15 in magnitude, whole numbers below 2^24: exact.  What is rounded: a quotient, an LSE of each range
    (2^-20 near 10, and a logarithm's and an exponential's 2^-21), and with them the merge's weights, which
    move O by less than 15 * 2^-18 (the ranges' means differ by less than 15): 6e-5, below half of
    1 / 9200."""
    c = Case(*heads, prefix, chunk, window, sinks, fp8, seed=len(prefix) + chunk[0])
    rng = np.random.default_rng(sum(chunk))
    v = rng.integers(-15, 16, c.v.shape).astype(np.float64)
    if fp8:
        seen = c.k != 0x7f
        zero, byte = ref.quantise_rows(bits(np.zeros(c.k.shape)))
        c.k = np.where(seen, zero, c.k).astype(np.uint8)
        c.kv_scale[:, :, 0] = np.where(c.kv_scale[:, :, 0] == 255, 255, byte)
        code, byte = ref.quantise_rows(bits(v))
        c.v = np.where(seen, code, c.v).astype(np.uint8)
        c.kv_scale[:, :, 1] = np.where(c.kv_scale[:, :, 1] == 255, 255, byte)
        c.kf, c.vf = (ref.cache_values(x, c.kv_scale[:, :, w]) for w, x in enumerate((c.k, c.v)))
        assert np.array_equal(c.vf[np.isfinite(c.vf)], v[np.isfinite(c.vf)])
    else:
        seen = c.k != 0x7fc0
        c.k, c.v = np.where(seen, 0, c.k).astype(np.uint16), np.where(seen, bits(v), c.v).astype(np.uint16)
        c.kf, c.vf = ref.bf16_values(c.k), ref.bf16_values(c.v)
    if not fp8 and window is None:
        c.window = 2 ** 31 - 1  # (windowed calls over the bf16 cache need one)
    out, lse = (t.double().cpu().numpy() for t in c.run())
    ro, rl, _, _ = c.oracle()
    n = np.exp(rl).max()
    assert n < 9200
    print(f"O {np.abs(out - ro).max():.1e}, LSE {np.abs(lse - rl).max():.1e}, a key {1 / n:.1e}")
    assert np.abs(out - ro).max() < 6e-5
    assert np.abs(lse - rl).max() < 2.0 ** -17
