"""Streams of 2^31 - 1 tokens, all of them seen: every key scores 0 and has the value 1, so O is 1 and the LSE
the logarithm of the number of keys; the one slot behind the last token holds NaN."""
import math

import pytest
import torch

import paper_2409_17264_amd as medha
from tests.window_util import FP8

pytestmark = pytest.mark.gpu
LAST = 2 ** 31 - 1  # tokens


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("chunk", [1, 40])
def test_the_longest_stream(fp8, chunk):
    """Partial sums are whole numbers below 2^24 (a range of keys has 2^23 at most), hence exact; an LSE near
    21 has a spacing of 2^-19 and takes a logarithm and a few roundings (2^-17), by which the merge's
    weights, and so O's two sums, are off relatively."""
    h_q, h_kv, d, end = 2, 1, 64, LAST % 16
    table = torch.zeros(LAST // 16 + 1, dtype=torch.int32, device="cuda")
    table[-1] = 1  # two pages, of which the second ends the stream
    q = torch.randn(chunk, h_q, d, device="cuda").to(torch.bfloat16)
    where = (table, [0, len(table)], [LAST - chunk], [chunk], 0.125)
    if fp8:
        k = torch.zeros(2, h_kv, 16, d, dtype=torch.uint8, device="cuda")
        v = torch.full_like(k, 0x70)  # 128
        scale = torch.full((2, h_kv, 2, 16), 120, dtype=torch.uint8, device="cuda")
        k[1, :, end:], v[1, :, end:], scale[1, :, :, end:] = 0x7f, 0x7f, 255
        o, l = medha.chunked_prefill_attn_fp8(q, k.view(FP8), v.view(FP8), scale, *where)
    else:
        k = torch.zeros(2, h_kv, 16, d, dtype=torch.bfloat16, device="cuda")
        v = torch.ones_like(k)
        k[1, :, end:] = v[1, :, end:] = float("nan")
        o, l = medha.window_attn(q, k, v, *where, LAST)
    want = torch.tensor([math.log(LAST - chunk + j + 1) for j in range(chunk)], dtype=torch.float64)
    assert (o.double().cpu() - 1).abs().max() <= 2.0 ** -16
    assert (l.double().cpu() - want[:, None]).abs().max() <= 2.0 ** -17
