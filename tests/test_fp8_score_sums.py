"""Scores over the 8-bit cache are sums in fp32, whatever their products' sizes and whichever kernel takes
the rows: channels far larger than the others, whose products cancel."""
import numpy as np
import pytest

import oracle.fp8 as ref
from tests.window_util import Case, bits

pytestmark = pytest.mark.gpu


def _outliers(c, seed):
    """Two channels of 16 in every query against +-32 in every key: products of 512 that cancel, beside
    d - 2 products of order 1."""
    rng = np.random.default_rng(seed)
    lo, hi = 3, c.d - 6
    q = rng.standard_normal(c.q.shape)
    q[..., lo] = q[..., hi] = 16.0
    k = rng.standard_normal(c.k.shape)
    sign = np.where(rng.random(k.shape[:-1]) < 0.5, -32.0, 32.0)
    k[..., lo], k[..., hi] = sign, -sign
    c.q = bits(q)
    code, byte = ref.quantise_rows(bits(k))
    seen = c.k != 0x7f
    c.k = np.where(seen, code, c.k).astype(np.uint8)
    c.kv_scale[:, :, 0] = np.where(c.kv_scale[:, :, 0] == 255, 255, byte)
    c.kf = ref.cache_values(c.k, c.kv_scale[:, :, 0])
    return c


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 1, 128), (32, 8, 64), (4, 2, 64)])
@pytest.mark.parametrize("prefix, chunk, window, sinks", [
    ([30], [1], None, 0), ([30], [9], None, 0), ([0], [65], None, 0), ([200], [40], 70, 3),
    ([0, 500, 20], [300, 1, 17], None, 0), ([5000], [140], None, 0), ([5000], [300], 4100, 9)])
def test_products_that_cancel(heads, prefix, chunk, window, sinks):
    """A score's partial sums stay below 2^10 (512 and d - 2 products whose sum is rarely above 60), so an
    addition is off by at most 2^-15 and by 2^-14 / sqrt(12) = 1.8e-5 rms; d of them by sqrt(d) times that,
    2.0e-4 at d 128 and 1.4e-4 at 64, and by d^-1/2 of it behind the scale: 1.8e-5.  An LSE, a mean of such
    errors and a few roundings of its own (below 1e-6), is off by less than 2e-5 rms.  (Sums that keep 13
    bits below the largest product drop up to 0.06 a term: 1e-3 and more.)"""
    c = _outliers(Case(*heads, prefix, chunk, window, sinks, True, seed=chunk[0]), seed=chunk[0] + 1)
    out, lse = c.run()
    c.fp8 = False  # (for the bounds: of fp32 sums)
    want = c.oracle()
    c.check(out, lse, want)
    rms = np.sqrt(((lse.double().cpu().numpy() - want[1]) ** 2).mean())
    print(f"lse rms {rms:.1e}")
    assert rms < 2e-5


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64)])
def test_a_row_does_not_depend_on_the_chunk_it_comes_in(heads):
    """The last token's rows, as a decode, at the end of 8 tokens and at the end of 200: the sums differ by
    the order of additions only (1.8e-5 rms each, see above, so 8 times that apart at most for the rows
    here; probabilities that are rounded to bf16 against other reference points move O)."""
    p = 700
    c = _outliers(Case(*heads, [p - 200], [200], None, 0, True, seed=3), seed=4)
    q, cache, table = c.device()
    want = c.oracle()
    got = []
    for n in (1, 8, 200):
        o, l = c.run(dev=(q[-n:].contiguous(), cache, table), prefix=[p - n], chunk=[n])
        got.append(l[-1].double().cpu().numpy())
    for l in got:
        assert np.abs(l - want[1][-1]).max() < 8 * 1.8e-5
