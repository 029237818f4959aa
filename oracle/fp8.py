"""fp64 oracle of the 8-bit KV cache and of windowed attention (TEST INFRASTRUCTURE ONLY), written
from the definitions in include/medha.h.  numpy throughout; bf16 data travels as uint16 bit patterns,
e4m3 values as uint8 codes.
"""
import numpy as np

PAGE = 16


def bf16_values(bits):
    with np.errstate(invalid="ignore"):  # (signalling NaN)
        return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def e4m3_values(codes):
    """OCP e4m3: 1 sign, 4 exponent (bias 7), 3 mantissa bits, no infinity, S.1111.111 is NaN."""
    c = np.asarray(codes).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, np.ldexp(8.0 + m, e - 10), np.ldexp(m.astype(np.float64), -9))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(c & 128, -v, v)


_MAGNITUDES = e4m3_values(np.arange(127))  # ascending


def e4m3_codes(values):
    """The nearest e4m3 code of every value (magnitudes up to 448), the even one of two as near."""
    a = np.abs(values)
    hi = np.searchsorted(_MAGNITUDES, np.where(np.isnan(a), 0.0, a))   # first code >= a
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _MAGNITUDES[hi] - a, a - _MAGNITUDES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isnan(a), 127, code)
    return (code + 128 * np.signbit(values)).astype(np.uint8)


def quantise_rows(bits):
    """bf16 rows [..][d] -> (codes [..][d], scale bytes [..])."""
    x = bf16_values(bits)
    finite = np.isfinite(x)
    top = np.where(finite, np.abs(x), 0.0).max(-1)
    e = np.frexp(top)[1] - 1 + 127                     # exponent field of a normal bf16 number
    byte = np.maximum(np.where(top > 0, e, 0) - 7, 10)
    x = np.where(finite, np.clip(x, -1.875 * 2.0 ** 127, 1.875 * 2.0 ** 127), np.copysign(np.nan, x))
    return e4m3_codes(np.ldexp(x, (127 - byte)[..., None])), byte.astype(np.uint8)


def cache_values(codes, scale):
    """Pool codes [pages][h_kv][16][d] and their scale bytes [pages][h_kv][16] -> fp64."""
    return np.ldexp(e4m3_values(codes), scale.astype(np.int64)[..., None] - 127)


def _places(table, offs, first, count):
    for b in range(len(first)):
        for t in range(int(first[b]), int(first[b]) + int(count[b])):
            yield int(table[int(offs[b]) + t // PAGE]), t % PAGE


def kv_append_fp8(k_new, v_new, k_pool, v_pool, scale, table, offs, prefix_len, chunk_len):
    """k_new, v_new uint16 [tokens][h_kv][d]; the pools (uint8) and scale are written IN PLACE."""
    new = [quantise_rows(k_new), quantise_rows(v_new)]
    for row, (page, slot) in enumerate(_places(table, offs, prefix_len, chunk_len)):
        if not 0 <= page < len(k_pool):
            continue
        for w, pool in enumerate((k_pool, v_pool)):
            pool[page, :, slot] = new[w][0][row]
            scale[page, :, w, slot] = new[w][1][row]


def kv_read_fp8(k_pool, v_pool, scale, table, offs, first, count):
    """fp64 [sum count][h_kv][d] for K and for V."""
    n, h_kv, d = int(np.sum(count)), k_pool.shape[1], k_pool.shape[3]
    out = np.zeros((2, n, h_kv, d))
    for row, (page, slot) in enumerate(_places(table, offs, first, count)):
        if 0 <= page < len(k_pool):
            for w, pool in enumerate((k_pool, v_pool)):
                out[w, row] = cache_values(pool[page, :, slot], scale[page, :, w, slot])
    return out


def window_attn(q, k, v, table, offs, prefix_len, chunk_len, scale, window=None, sinks=0):
    """q uint16 [tokens][h_q][d], pools k and v fp64 [pages][h_kv][16][d].  The row at position p
    sees key t if t <= p and (t > p - window or t < sinks); no window: all t <= p.
    Returns (out [tokens][h_q][d], lse [tokens][h_q]) in fp64.  Only pages of seen keys are read."""
    tokens, h_q, d = q.shape
    h_kv = k.shape[1]
    qf = bf16_values(q)
    out, lse = np.zeros((tokens, h_q, d)), np.zeros((tokens, h_q))
    start = 0
    for b in range(len(prefix_len)):
        p0, c = int(prefix_len[b]), int(chunk_len[b])
        t = np.arange(p0 + c)
        pos = p0 + np.arange(c)[:, None]
        seen = t <= pos
        if window is not None:
            seen &= (t > pos - int(window)) | (t < int(sinks))
        t = t[seen.any(0)]
        seen = seen[:, seen.any(0)]
        page = np.asarray(table)[int(offs[b]) + t // PAGE]
        for h in range(h_q):
            g = h // (h_q // h_kv)
            s = float(scale) * (qf[start:start + c, h] @ k[page, g, t % PAGE].T)
            s = np.where(seen, s, -np.inf)
            top = s.max(1, keepdims=True)
            p = np.exp(s - top)
            total = p.sum(1, keepdims=True)
            out[start:start + c, h] = (p / total) @ v[page, g, t % PAGE]
            lse[start:start + c, h] = (top + np.log(total))[:, 0]
        start += c
    return out, lse
