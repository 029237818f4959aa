"""Window arguments at the edge of what the calls take (CPU: nothing is enqueued)."""
import pytest

import paper_2409_17264_amd as medha
from tests.test_window_fp8_attn import _host_call

BIG = dict(prefix=[30000], offs=[0, 4000], ws=None, bytes=0)  # a call that is refused for its scratch only


@pytest.mark.parametrize("sinks", [0, 5, 2 ** 31 - 1, -1, -2 ** 31])
def test_without_a_window_the_first_tokens_are_not_looked_at(sinks):
    assert _host_call(True, window=0, sinks=sinks, **BIG) == -3
    want = medha.chunked_prefill_fp8_workspace_bytes([30000], [20], 4, 2, 64, 0, 0)
    assert want > 256
    assert medha.chunked_prefill_fp8_workspace_bytes([30000], [20], 4, 2, 64, 0, sinks) == want


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window, sinks, code", [
    (1, 0, 0), (2 ** 31 - 1, 2 ** 31 - 1, -3), (2 ** 31 - 1, -1, -1), (-1, 0, -1), (-2 ** 31, 5, -1), (20000, -1, -1)])
def test_windows_and_first_tokens(fp8, window, sinks, code):
    if code == 0:  # (would be enqueued: ask for the scratch instead)
        query = medha.chunked_prefill_fp8_workspace_bytes if fp8 else medha.window_workspace_bytes
        assert query([30000], [20], 4, 2, 64, window, sinks) > 0
    else:
        assert _host_call(fp8, window=window, sinks=sinks, **BIG) == code
