"""Values of the smallest scales, attended to with small probabilities: decodes and chunks."""
import numpy as np
import pytest

import oracle.fp8 as ref
from tests.window_util import Case, bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(4, 2, 128), (8, 2, 64)])
@pytest.mark.parametrize("chunk", [1, 4, 60])
@pytest.mark.parametrize("power", [-112, -60, 100])
def test_one_key_of_no_value_outweighs_each_of_the_others(heads, chunk, power):
    """The first key's score lies 13 above all others', which are near 0, and its value is zero: the
    others' probabilities are near e^-13 = 2^-18.8 of the largest, and O is all theirs."""
    n = 4000
    c = Case(*heads, [n - chunk], [chunk], None, 0, True, seed=chunk)
    rng = np.random.default_rng(chunk)
    k, v = 0.02 * rng.standard_normal(c.k.shape), rng.uniform(0.5, 1.0, c.v.shape) * 2.0 ** power
    q = rng.standard_normal(c.q.shape)
    first = int(c.table[0])
    q[..., 0] = 8.0
    k[first, :, 0, 0] = 13.0 / (8.0 * c.scale)
    v[first, :, 0] = 0.0
    c.q = bits(q)
    seen = c.k != 0x7f
    for w, (name, x) in enumerate((("k", k), ("v", v))):
        code, byte = ref.quantise_rows(bits(x))
        setattr(c, name, np.where(seen, code, getattr(c, name)).astype(np.uint8))
        c.kv_scale[:, :, w] = np.where(c.kv_scale[:, :, w] == 255, 255, byte)
    c.kf, c.vf = (ref.cache_values(x, c.kv_scale[:, :, w]) for w, x in enumerate((c.k, c.v)))
    out, lse = c.run()
    # (the bounds of fp32 sums: scores near 13: products up to 150)
    c.fp8 = False
    ro, rl, bo, bl = c.oracle()
    eo = np.abs(out.double().cpu().numpy() - ro)
    print(f"largest error {np.max(eo / bo):.2f} of its bound, LSE {np.max(np.abs(lse.double().cpu().numpy() - rl) / bl):.2f}")
    assert (np.abs(ro) > 0.004 * np.ldexp(1.0, power)).all()
    assert (eo <= bo).all() and (np.abs(lse.double().cpu().numpy() - rl) <= bl).all()
