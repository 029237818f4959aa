"""Windowed attention and the 8-bit cache with the least scratch that they accept."""
import pytest
import torch

import paper_2409_17264_amd as medha
from tests.window_util import Case

pytestmark = pytest.mark.gpu
GUARD = 1024


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads, prefix, chunk, window", [
    ((8, 1, 128), [5000, 4000], [64, 1], 4500), ((32, 8, 128), [9000, 300, 2000], [1, 1, 1], 8000),
    ((8, 2, 64), [3000], [200], 2500)])
def test_the_least_workspace(fp8, heads, prefix, chunk, window):
    c = Case(*heads, prefix, chunk, window, 3, fp8, seed=12)
    query = medha.chunked_prefill_fp8_workspace_bytes if fp8 else medha.window_workspace_bytes
    need = query(c.prefix, c.chunk, *heads, window, 3)
    want, dev = c.oracle(), c.device()
    shape = dev[0].shape

    def attempt(size):
        """Whether a workspace of that size is accepted; neither way is a byte outside it touched."""
        mem = torch.full((size + 2 * GUARD,), 0xff, dtype=torch.uint8, device="cuda")
        out, lse = torch.full(shape, 7.0, device="cuda"), torch.full(shape[:2], 7.0, device="cuda")
        try:
            c.run(out, lse, mem[GUARD:GUARD + size], dev=dev)
        except medha.MedhaError as e:
            assert e.code == -3
            assert (mem == 0xff).all() and (out == 7.0).all() and (lse == 7.0).all()
            return False
        torch.cuda.synchronize()
        assert (mem[:GUARD] == 0xff).all() and (mem[GUARD + size:] == 0xff).all()
        c.check(out, lse, want)
        return True

    assert attempt(need)
    low, high = 0, need // 256  # refused, accepted, in units of 256 bytes
    assert need % 256 == 0 and not attempt(256 * low)
    while high - low > 1:
        mid = (low + high) // 2
        low, high = (low, mid) if attempt(256 * mid) else (mid, high)
    print(f"needs {need}, takes {256 * high}")
    for size in (256 * high, 256 * high + 256, (need + 256 * high) // 512 * 256, need - 256):
        assert size < 256 * high or attempt(size)
    assert not attempt(256 * high - 256) and not attempt(256 * high - 1)
