"""Windowed attention over the bf16 cache, and attention over the 8-bit cache with and without a
window, against the fp64 oracle."""
import ctypes

import numpy as np
import pytest
import torch

import oracle.fp8 as ref
import paper_2409_17264_amd as medha
from paper_2409_17264_amd import binding
from tests import helpers
from tests.window_util import Case, bits, from_bits

HEADS = [(32, 8, 128), (8, 1, 128), (8, 2, 64), (2, 1, 64), (6, 3, 128), (40, 1, 64), (5, 5, 128)]


# ----------------------------------------------------------------- the oracle itself (CPU)

def test_oracle_without_a_window_is_the_brute_force():
    c = Case(4, 2, 64, [5, 40], [7, 3], seed=1)
    ro, rl = helpers.brute_force_prefill(c.q, c.k, c.v, c.table, c.offs, c.prefix, c.chunk, c.scale)
    o, l, _, _ = c.oracle()
    assert np.abs(o - ro).max() < 1e-12 and np.abs(l - rl).max() < 1e-12


def test_oracle_window_key_by_key():
    c = Case(2, 1, 64, [50], [20], window=9, sinks=3, seed=2)
    o, l, _, _ = c.oracle()
    q = ref.bf16_values(c.q)
    for j in range(20):
        p = 50 + j
        t = [x for x in range(p + 1) if x > p - 9 or x < 3]
        k = np.stack([c.kf[c.table[x // 16], 0, x % 16] for x in t])
        v = np.stack([c.vf[c.table[x // 16], 0, x % 16] for x in t])
        w = np.exp(c.scale * k @ q[j, 1])
        assert np.abs(o[j, 1] - w @ v / w.sum()).max() < 1e-12
        assert abs(l[j, 1] - np.log(w.sum())) < 1e-12


# ----------------------------------------------------------------- refusals (CPU: nothing is enqueued)

def _host_call(fp8, **change):
    lib = medha.load_library()
    at = 1 << 20
    a = dict(q=at, k=at, v=at, s=at, pages=8, size=16, h_kv=2, d=64, table=at, offs=[0, 4], prefix=[30],
             chunk=[20], batch=1, h_q=4, scale=0.1, window=8, sinks=2, type=0, out=at, lse=at, ws=at,
             bytes=1 << 30)
    a.update(change)
    host = [np.array(a[n], t).tobytes() if a[n] is not None else None
            for n, t in (("offs", np.int64), ("prefix", np.int32), ("chunk", np.int32))]
    if fp8:
        kv, call = binding._KvCacheFp8(a["k"], a["v"], a["s"], a["pages"], a["size"], a["h_kv"], a["d"]), \
            lib.medha_chunked_prefill_attn_fp8
    else:
        kv, call = binding._KvCache(a["k"], a["v"], a["pages"], a["size"], a["h_kv"], a["d"]), \
            lib.medha_window_attn
    return call(a["q"], None if change.get("null") else ctypes.byref(kv), a["table"], *host, a["batch"],
                a["h_q"], a["scale"], a["window"], a["sinks"], a["type"], a["out"], a["lse"], a["ws"],
                a["bytes"], None)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("change, code", [
    (dict(null=True), -1), (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(table=None), -1),
    (dict(offs=None), -1), (dict(prefix=None), -1), (dict(chunk=None), -1), (dict(out=None), -1),
    (dict(lse=None), -1), (dict(batch=-1), -1), (dict(h_q=5), -1), (dict(h_kv=0), -1), (dict(pages=0), -1),
    (dict(size=8), -2), (dict(d=96), -2), (dict(prefix=[-1]), -1), (dict(chunk=[0]), -1),
    (dict(prefix=[2 ** 31 - 10]), -1), (dict(offs=[0, 3]), -1), (dict(offs=[-1, 4]), -1),
    (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(type=2), -1), (dict(type=-1), -1),
    (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(q=(1 << 20) + 8), -1),
    (dict(out=(1 << 20) + 8), -1), (dict(lse=(1 << 20) + 2), -1), (dict(k=(1 << 20) + 8), -1),
    (dict(prefix=[30000], offs=[0, 4000], window=20000, ws=None, bytes=0), -3),
    (dict(prefix=[30000], offs=[0, 4000], window=20000, ws=(1 << 20) + 64), -3), (dict(batch=0), 0)])
def test_refusals(fp8, change, code):
    assert _host_call(fp8, **change) == code


def test_refusals_of_one_cache_only():
    assert _host_call(False, window=0) == -1
    assert _host_call(True, s=None) == -1
    assert _host_call(True, s=(1 << 20) + 8) == -1


def test_workspace_queries():
    for query, least in ((medha.window_workspace_bytes, 1), (medha.chunked_prefill_fp8_workspace_bytes, 0)):
        assert query([100000], [1], 32, 8, 128, least) > 0
        for bad in (([10], [0], 8, 2, 128, 5), ([10], [4], 7, 2, 128, 5), ([-1], [4], 8, 2, 128, 5),
                    ([10], [4], 8, 2, 96, 5), ([10], [4], 8, 2, 128, least - 1), ([10], [4], 8, 2, 128, 5, -1)):
            assert query(*bad) == 0
    # a window bounds what has to be kept
    assert medha.window_workspace_bytes([10 ** 6], [1], 8, 1, 128, 100) <= \
        medha.window_workspace_bytes([10 ** 6], [1], 8, 1, 128, 10 ** 6)


# ----------------------------------------------------------------- on the device

@pytest.mark.gpu
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("prefix, chunk, window, sinks", [
    ([0], [1], 1, 0), ([0], [5], 1, 0), ([700], [1], 1, 3), ([33], [70], 16, 0), ([1000], [1], 100, 4),
    ([0, 15, 16, 500, 1200], [40, 1, 2, 100, 1], 64, 1), ([900, 3], [33, 260], 200, 130),
    ([2000], [300], 511, 17), ([640], [64], 640, 640), ([100, 31], [50, 1], 1000, 5)])
def test_windows(heads, fp8, prefix, chunk, window, sinks):
    c = Case(*heads, prefix, chunk, window, sinks, fp8, seed=len(prefix) + window)
    c.check(*c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("prefix, chunk", [
    ([0], [1]), ([15], [1]), ([0], [17]), ([0], [300]), ([1025], [1]), ([4000], [9]), ([2500], [200]),
    ([0, 1, 15, 16, 17, 63, 300], [1, 1, 3, 64, 2, 1, 130])])
def test_the_8_bit_cache_without_a_window(heads, prefix, chunk):
    c = Case(*heads, prefix, chunk, None, 0, True, seed=len(prefix) + chunk[0])
    c.check(*c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(8, 1, 128), (4, 2, 64)])
@pytest.mark.parametrize("fp8, prefix, chunk, window, sinks", [
    (False, [9000], [130], 4999, 33), (False, [9000], [64], 7000, 0), (False, [0], [1500], 1100, 70),
    (False, [5000, 70], [1, 700], 2500, 4), (True, [9000], [130], 4999, 33), (True, [9000], [64], None, 0),
    (True, [0], [1500], None, 0), (True, [0], [1500], 1100, 70), (True, [5000, 70], [1, 700], None, 0)])
def test_long_walks(heads, fp8, prefix, chunk, window, sinks):
    c = Case(*heads, prefix, chunk, window, sinks, fp8, seed=sum(chunk))
    c.check(*c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("fp8, prefix, chunk, window", [
    (True, 6000, 200, None), (True, 9000, 130, None), (True, 9007, 130, 8000), (False, 9007, 130, 8000),
    (False, 6011, 200, 6000)])
def test_workgroups_in_pairs(fp8, prefix, chunk, window):
    """Launches that take two 128-row workgroups to a compute unit, with the short ring."""
    e, grid, _, _ = medha.describe_plan([prefix], [chunk], 32, 8, 128, 256)
    assert e[0].mode == 0 and e[0].rows_per_wg == 128 and grid > 256
    c = Case(32, 8, 128, [prefix], [chunk], window, 5, fp8, seed=chunk)
    c.check(*c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("k_std", [6.0, 0.0])
@pytest.mark.parametrize("fp8, window", [(False, 3000), (True, 3000), (True, None)])
def test_peaked_and_flat_rows(fp8, window, k_std):
    """Keys six times as long (one key carries its row, at places that shift from row to row), and keys
    that are all zero."""
    c = Case(4, 1, 128, [4000], [100], window, 5, fp8, seed=4, k_std=k_std)
    c.check(*c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64)])
@pytest.mark.parametrize("prefix, chunk, window, sinks", [
    ([776], [1], 129, 1), ([776], [8], 64, 0), ([299] * 8, [1] * 8, None, 0)])
def test_decodes_over_the_8_bit_cache_add_up_in_fp32(heads, prefix, chunk, window, sinks):
    """They turn keys into bf16 first, so a score is as exact as over the bf16 cache.  The partial sums of
    its d products stay below 16 but for rare ones, where a rounding is off by 2^-20 / sqrt(12) rms: d of
    them sqrt(d) times that, 2.8e-7 after the scale of d^-1/2.  A few roundings of the LSE (below 8: 1.4e-7
    rms each), an exponential and a logarithm beside them: below 1e-6 rms."""
    c = Case(*heads, prefix, chunk, window, sinks, True, seed=chunk[0])
    out, lse = c.run()
    c.fp8 = False  # (for the bounds: of fp32 sums)
    want = c.oracle()
    c.check(out, lse, want)
    assert np.sqrt(((lse.double().cpu().numpy() - want[1]) ** 2).mean()) < 1e-6
