"""Chunks whose windows lie in the last tile of the positions' range."""
import pytest
import torch

import paper_2409_17264_amd as medha
from tests.window_util import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("h_q, h_kv, d, chunk, window, sinks", [
    (4, 2, 64, 20, 10, 3), (16, 2, 128, 5, 1, 17), (16, 2, 128, 40, 20, 70), (4, 1, 64, 9, 50, 1)])
def test_windows_inside_the_last_64_positions(fp8, h_q, h_kv, d, chunk, window, sinks):
    """A stream of 2^31 - 1 tokens, of which the last ones and the first ones are left: the same rows over
    the same pages as near the start of a stream, whatever stands in the slots that no row sees."""
    assert chunk + window <= 64
    prefix = 2 ** 31 - 1 - chunk
    shift = (prefix - 400) % 64
    near = Case(h_q, h_kv, d, [400 + shift], [chunk], window, sinks, fp8, seed=7)
    q, cache, table = near.device()
    last, near_last = (prefix + chunk - 1) // 16, (400 + shift + chunk - 1) // 16
    far = torch.full((last + 1,), near.dead_page, dtype=torch.int32, device="cuda")
    live, first = (window + chunk) // 16 + 3, (sinks + 15) // 16
    far[last - live:] = table[near_last - live:near_last + 1]
    far[:first] = table[:first]
    call = medha.chunked_prefill_attn_fp8 if fp8 else medha.window_attn
    near.check(*call(q, *cache, far, [0, last + 1], [prefix], [chunk], near.scale, window, sinks))
