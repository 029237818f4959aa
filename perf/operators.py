"""Workloads of the 8-bit KV cache and of windowed attention, each with its plain form.

Four operators of a paged KV cache of 16-token pages:

  append   a batch's new keys and values are quantised into the 8-bit cache;
  read     a range of tokens of each sequence comes back from it, in bf16;
  fp8      attention of chunks and decodes over it, optionally windowed;
  window   attention over the bf16 cache in which a row sees the last `window` tokens up to
           itself and the sequence's first `sinks`.

The 8-bit cache holds e4m3 values, [pages][kv heads][16][d] for K and for V, and one exponent byte
for each (token, head) row, [pages][kv heads][2][16], K's before V's: value * 2^(byte - 127).

``own`` False computes the operators from elementary tensor operations, True through the
library's entry points.  A case holds every size; the seed draws values and page tables.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
# (query heads, KV heads, head dim): the full 8B-sized layer, one GPU's share of the 70B-sized one,
# and the small-head shapes of the tests
HEADS = [(32, 8, 128), (32, 8, 128), (8, 1, 128), (8, 1, 128), (8, 2, 128), (32, 8, 64), (8, 2, 64),
         (2, 1, 64)]
MAX_SCORES = 4.4e9    # (row, key) pairs, padded, times heads: what the plain form holds at once
MAX_FLOPS = 2.3e12    # the largest listed case: 2048 tokens at a prefix of 262144
MAX_GATHERED = 2.2e9  # gathered key elements, padded (the plain form's copies)


def _case(name, op, heads, prefix=0, chunk=0, prompts=0, decodes=0, median=0, lengths=0, window=0, sinks=0):
    c = dict(op=op, h_q=heads[0], h_kv=heads[1], d=heads[2], prefix=prefix, chunk=chunk, prompts=prompts,
             decodes=decodes, median=median, lengths=lengths, window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def listed():
    full, share, small = (32, 8, 128), (8, 1, 128), (8, 2, 64)
    return [
        # the new token of one chat request: launch latency and host work
        _case("append_one", "append", full, decodes=1, median=2048),
        # eight fresh prompts of assorted lengths entering together
        _case("append_prompts", "append", full, prompts=8, median=1024, lengths=11),
        # a few hundred tokens of a small-head sequence, from the middle of a page
        _case("read_odd", "read", small, prefix=1003, chunk=300),
        # a 32K prefix handed to another request's cache
        _case("read_32k", "read", full, prefix=0, chunk=32768),
        # one chat request generating its next token
        _case("fp8_decode_one", "fp8", full, decodes=1, median=2048),
        # a decode-only iteration of a busy server
        _case("fp8_decode_batch", "fp8", full, decodes=64, median=4096, lengths=5007),
        # the 8B-sized layer at a 32K prefix
        _case("fp8_chunk_32k", "fp8", full, prefix=32768, chunk=2048),
        # one GPU's share of the 70B-sized layer: a small chunk at a long odd prefix, and a large one
        _case("fp8_chunk_long", "fp8", share, prefix=524291, chunk=111),
        _case("fp8_chunk_large", "fp8", share, prefix=262144, chunk=2048),
        # decodes far into their contexts, each behind a window of 4096 and 4 first tokens
        _case("window_decode_batch", "window", full, decodes=64, median=8192, lengths=77, window=4096, sinks=4),
        # a long request's chunk packed with decodes, windowed
        _case("window_mixed", "window", full, prefix=131071, chunk=2048, decodes=16, median=8192, lengths=5,
              window=4096, sinks=4),
        # fresh prompts at head dim 64 and a window that is no multiple of anything
        _case("window_prompts_d64", "window", (32, 8, 64), prompts=8, median=1024, lengths=0, window=1000, sinks=17),
    ]


def _log_int(rng, lo, hi):
    """Integer spread over its logarithm in [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["append", "read", "fp8", "fp8", "fp8", "window", "window", "window"])
    case = _case("", op, rng.choice(HEADS), lengths=rng.randrange(1 << 20))
    if op in ("append", "read"):
        kind = rng.choice(["chunk", "prompts", "decodes"] if op == "append" else ["chunk"])
        if kind == "chunk":
            case.update(prefix=_log_int(rng, 1, 32768), chunk=_log_int(rng, 1, 32768 if op == "read" else 8192))
        else:
            case.update({kind: _log_int(rng, 1, 16 if kind == "prompts" else 128),
                         "median": _log_int(rng, 128, 4096)})
        return case
    if op == "window" or rng.random() < 0.25:
        case.update(window=_log_int(rng, 64, 8192), sinks=rng.choice([0, 1, 4, 4, 16, rng.randrange(1, 129)]))
    mix = rng.choice(["decodes", "prompts", "chunk", "chunk", "mixed"])
    if mix == "prompts":
        case.update(prompts=_log_int(rng, 1, 16), median=_log_int(rng, 64, 4096))
    if mix in ("decodes", "mixed"):
        case.update(decodes=_log_int(rng, 1, 128), median=_log_int(rng, 256, 8192))
    if mix in ("chunk", "mixed"):
        case.update(prefix=_log_int(rng, 256, 524288), chunk=_log_int(rng, 2, 2048))
    # no dearer than the largest listed cases
    while _dear(case):
        big = max(("prefix", "chunk", "median", "decodes", "prompts"), key=lambda k: case[k] if k != "chunk" else 16 * case[k])
        case[big] = max(1, case[big] * 3 // 4)
    return case


def _lengths(case):
    """(prefix_len, chunk_len) of every sequence of the batch, the long request first."""
    prefix, chunk = [], []
    if case["chunk"]:
        prefix.append(case["prefix"])
        chunk.append(case["chunk"])
    rng = np.random.default_rng(case["lengths"])
    z = np.exp(rng.standard_normal(case["prompts"]))
    chunk += [int(n) for n in np.clip(np.rint(case["median"] * z), 16, 8192)]
    prefix += [0] * case["prompts"]
    z = np.exp(rng.standard_normal(case["decodes"]) * (case["decodes"] > 1))
    prefix += [int(n) - 1 for n in np.clip(np.rint(case["median"] * z), min(256, case["median"]), 8 * max(2048, case["median"]))]
    chunk += [1] * case["decodes"]
    return np.array(prefix, np.int64), np.array(chunk, np.int64)


def _window(case):
    return case["window"] or 1 << 30


def _live(case):
    """First key that a sequence's window reaches, and the first tokens before it that stay visible."""
    prefix, _ = _lengths(case)
    lo = np.maximum(0, prefix + 1 - _window(case))
    return lo, np.minimum(lo, case["sinks"])


def _groups(case):
    """The batch's chunks and its single tokens, as lists of sequences."""
    _, chunk = _lengths(case)
    return [g for g in (np.flatnonzero(chunk > 1), np.flatnonzero(chunk == 1)) if len(g)]


def _dear(case):
    prefix, chunk = _lengths(case)
    lo, first = _live(case)
    keys = prefix + chunk - lo + first
    padded = sum(len(g) * int(chunk[g].max()) * int(keys[g].max()) for g in _groups(case))
    gathered = sum(len(g) * int(keys[g].max()) for g in _groups(case))
    return (padded * case["h_q"] > MAX_SCORES or gathered * case["h_kv"] * case["d"] > MAX_GATHERED
            or work(case)["flops"] > MAX_FLOPS)


# ---------------------------------------------------------------------------- inputs

def _pow2(byte):
    """2^(byte - 127) in fp32, for whole numbers 1 to 254."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _quantise(x):
    """bf16 [..][d] -> e4m3 [..][d] and exponent bytes [..]: the largest finite magnitude of a row
    lies in [128, 256) of its scale, no scale is below 2^-117, and NaN and infinities become NaN."""
    a = x.abs().float()
    top = torch.where(a.isfinite(), a, 0.0).amax(-1)
    byte = ((top.view(torch.int32) >> 23) - 7).clamp_min(10)
    x = torch.where(a.isfinite(), x.float().clamp(-1.875 * 2.0 ** 127, 1.875 * 2.0 ** 127), math.nan)
    return (x * _pow2(254 - byte).unsqueeze(-1)).to(torch.float8_e4m3fn), byte.to(torch.uint8)


def _tables(case, seed):
    """Page table, offsets and number of pages.  A server with windows frees what no window reaches:
    those entries point at a page that holds something else."""
    prefix, chunk = _lengths(case)
    lo, first = _live(case)
    n_pages = -(-(prefix + chunk) // PAGE)
    offs = np.concatenate([[0], np.cumsum(n_pages)]).astype(np.int64)
    live = np.concatenate([(np.arange(n) >= lo[b] // PAGE) | (np.arange(n) * PAGE < first[b]) for b, n in enumerate(n_pages)])
    table = np.zeros(len(live), np.int32)
    table[live] = np.random.default_rng(seed).permutation(int(live.sum())).astype(np.int32)
    return torch.from_numpy(table).cuda(), offs, int(live.sum())


def prepare(case, seed):
    h_q, h_kv, d = case["h_q"], case["h_kv"], case["d"]
    prefix, chunk = _lengths(case)
    tokens = int(chunk.sum())
    table, offs, pages = _tables(case, seed)
    gen = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    s = dict(op=case["op"], table=table, offs=offs, prefix=prefix.astype(np.int32), chunk=chunk.astype(np.int32),
             scale=1.0 / math.sqrt(d), window=case["window"], sinks=case["sinks"], groups=_groups(case),
             live=_live(case))
    # tokens differ in magnitude, and a key's channels too, as behind a rotary embedding
    channel = torch.exp(0.4 * normal(h_kv, 1, d))
    channel /= channel.square().mean(-1, keepdim=True).sqrt()
    rows = (pages, h_kv, PAGE)
    k = (normal(*rows, d) * channel * torch.exp(0.2 * normal(*rows, 1))).bfloat16()
    v = (normal(*rows, d) * torch.exp(0.5 * normal(*rows, 1))).bfloat16()
    if case["op"] == "window":
        s.update(k=k, v=v)
    else:
        (k8, kb), (v8, vb) = _quantise(k), _quantise(v)
        s.update(k=k8, v=v8, kv_scale=torch.stack([kb, vb], 2).contiguous())
    if case["op"] == "append":
        s["k_new"] = (normal(tokens, h_kv, d) * channel[:, 0]).bfloat16()
        s["v_new"] = (normal(tokens, h_kv, d) * torch.exp(0.5 * normal(tokens, h_kv, 1))).bfloat16()
    elif case["op"] != "read":
        s["q"] = normal(tokens, h_q, d).bfloat16()
    return s


# ---------------------------------------------------------------------------- one pass

def run(s):
    if own:
        return _own(s)
    if s["op"] == "append":
        page, slot = _places(s)
        (s["k"][page, :, slot], kb), (s["v"][page, :, slot], vb) = _quantise(s["k_new"]), _quantise(s["v_new"])
        s["kv_scale"][page, :, 0, slot] = kb
        s["kv_scale"][page, :, 1, slot] = vb
        return {"k": s["k"], "v": s["v"], "kv_scale": s["kv_scale"]}
    if s["op"] == "read":
        k, v = _keys(s, *_places(s))
        return {"k": k.bfloat16(), "v": v.bfloat16()}
    return _attention(s)


def _own(s):
    import paper_2409_17264_amd as medha

    where = (s["table"], s["offs"], s["prefix"], s["chunk"])
    if s["op"] == "append":
        medha.kv_append_fp8(s["k_new"], s["v_new"], s["k"], s["v"], s["kv_scale"], *where)
        return {"k": s["k"], "v": s["v"], "kv_scale": s["kv_scale"]}
    if s["op"] == "read":
        k, v = medha.kv_read_fp8(s["k"], s["v"], s["kv_scale"], *where)
        return {"k": k, "v": v}
    out = torch.empty_like(s["q"])  # bf16, as the next layer takes it
    if s["op"] == "fp8":
        out, lse = medha.chunked_prefill_attn_fp8(s["q"], s["k"], s["v"], s["kv_scale"], *where, s["scale"],
                                                  window=s["window"], sinks=s["sinks"], out=out)
    else:
        out, lse = medha.window_attn(s["q"], s["k"], s["v"], *where, s["scale"], s["window"], s["sinks"], out=out)
    return {"out": out, "lse": lse}


def _places(s):
    """Page and slot of every token of the batch's chunks."""
    seq = np.repeat(np.arange(len(s["chunk"])), s["chunk"])
    start = np.cumsum(s["chunk"]) - s["chunk"]
    at = s["prefix"][seq] + np.arange(len(seq)) - start[seq]
    index = torch.from_numpy(np.stack([s["offs"][seq] + at // PAGE, at % PAGE])).cuda()
    return s["table"][index[0]].long(), index[1]


def _keys(s, page, slot):
    """Keys and values at (page, slot) pairs, in fp32 (exactly what the cache holds)."""
    k, v = s["k"][page, :, slot].float(), s["v"][page, :, slot].float()
    if "kv_scale" in s:
        k *= _pow2(s["kv_scale"][page, :, 0, slot]).unsqueeze(-1)
        v *= _pow2(s["kv_scale"][page, :, 1, slot]).unsqueeze(-1)
    return k, v


def _attention(s):
    out, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")
    starts = np.cumsum(s["chunk"]) - s["chunk"]
    for group in s["groups"]:
        _attend(s, group, starts[group], out, lse)
    return {"out": out, "lse": lse}


def _attend(s, group, start, out, lse):
    """Softmax attention of a group of sequences, padded to the longest chunk and the most keys."""
    h_q, d = s["q"].shape[1:]
    h_kv = s["k"].shape[1]
    b, c = len(group), int(s["chunk"][group].max())
    host = np.stack([s["prefix"][group], s["chunk"][group], s["live"][0][group], s["live"][1][group], start, s["offs"][group]])
    prefix, chunk, lo, first, start, offs = torch.from_numpy(host.astype(np.int64)).cuda().unsqueeze(-1)
    n_keys = s["prefix"][group] + s["chunk"][group] - s["live"][0][group] + s["live"][1][group]
    j, i = torch.arange(int(n_keys.max()), device="cuda"), torch.arange(c, device="cuda")
    # key j of a sequence: its first tokens, then what its rows' windows reach
    at = torch.where(j < first, j, lo + j - first)
    there = at < prefix + chunk
    at = torch.minimum(at, prefix + chunk - 1)
    k, v = _keys(s, s["table"][offs + at // PAGE].long(), at % PAGE)
    row = torch.minimum(start + i, start + chunk - 1)
    q = s["q"][row].float().reshape(b, c, h_kv, h_q // h_kv, d).transpose(1, 2).reshape(b, h_kv, -1, d)
    pos = (prefix + i).unsqueeze(-1)
    at = at.unsqueeze(1)
    sees = there.unsqueeze(1) & (at <= pos)
    if s["window"]:
        sees &= (at > pos - s["window"]) | (at < s["sinks"])
    p = torch.matmul(q, k.permute(0, 2, 3, 1)).reshape(b, h_kv, c, -1, len(j))
    p.mul_(s["scale"]).masked_fill_(~sees[:, None, :, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(b, h_kv, -1, len(j)), v.transpose(1, 2)).reshape(b, h_kv, c, -1, d) / total
    here = i < chunk
    out[row[here]] = o.transpose(1, 2).reshape(b, c, h_q, d)[here].bfloat16()
    lse[row[here]] = (top + total.log()).squeeze(-1).transpose(1, 2).reshape(b, c, h_q)[here]


# ---------------------------------------------------------------------------- what a pass needs

def work(case):
    prefix, chunk = _lengths(case)
    h_q, h_kv, d = case["h_q"], case["h_kv"], case["d"]
    tokens = float(chunk.sum())
    pages = float((-(-(prefix + chunk) // PAGE) - prefix // PAGE).sum())
    if case["op"] in ("append", "read"):
        return {"bytes": tokens * 2 * h_kv * (2 * d + d + 1) + 4 * pages, "flops": 0.0}
    lo, first = _live(case)
    keys = float((prefix + chunk - lo + first).sum())
    n_bytes = tokens * h_q * (2 * d + 2 * d + 4)  # q, out, lse
    n_bytes += keys * (2 * h_kv * (2 * d if case["op"] == "window" else d + 1) + 4 / PAGE)
    # pairs: every key up to the row's own, less those that lie between the first tokens and its window
    def below(n):  # sum over the rows at positions [prefix, prefix + chunk) of max(0, position + 1 - n)
        hi, lo_ = np.maximum(0, prefix + chunk - n).astype(float), np.maximum(0, prefix - n).astype(float)
        return hi * (hi + 1) / 2 - lo_ * (lo_ + 1) / 2
    pairs = float((below(0) - below(_window(case) + min(case["sinks"], 1 << 29))).sum())
    return {"bytes": n_bytes, "flops": pairs * 4.0 * d * h_q}


# ---------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    h_kv = s["k"].shape[1]
    ends = np.cumsum(s["chunk"])
    if case["op"] in ("append", "read"):
        cache = [s["k"].double(), s["v"].double()]
        byte = s["kv_scale"].long()
        new = [_code(s[n]) for n in ("k_new", "v_new")] if case["op"] == "append" else None
        got = [[], []]
        for b, n in enumerate(s["chunk"].tolist()):
            at = torch.arange(n, device="cuda") + int(s["prefix"][b])
            page = s["table"][int(s["offs"][b]):][at // PAGE].long()
            for w in (0, 1):
                if new is None:
                    got[w].append(cache[w][page, :, at % PAGE] * _two(byte[page, :, w, at % PAGE] - 127)[..., None])
                else:
                    cache[w][page, :, at % PAGE] = new[w][int(ends[b]) - n:int(ends[b])]
        if new is None:
            return {"k": torch.cat(got[0]), "v": torch.cat(got[1])}
        return {"k": cache[0], "v": cache[1], "kv_scale": None}
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = out.new_empty(out.shape[:2])
    group = out.shape[1] // h_kv
    for b, c in enumerate(s["chunk"].tolist()):
        p0, first_row, lo = int(s["prefix"][b]), int(ends[b]) - c, int(s["live"][0][b])
        t = torch.cat([torch.arange(int(s["live"][1][b]), device="cuda"), torch.arange(lo, p0 + c, device="cuda")])
        page = s["table"][int(s["offs"][b]):][t // PAGE].long()
        for h in range(h_kv):
            k, v = (s[n][page, h, t % PAGE].double() for n in ("k", "v"))
            if "kv_scale" in s:
                e = _two(s["kv_scale"][page, h, :, t % PAGE].long() - 127)
                k, v = k * e[:, :1], v * e[:, 1:]
            heads = slice(h * group, (h + 1) * group)
            step = max(1, (1 << 28) // (len(t) * group))
            for r in range(0, c, step):
                rows = slice(first_row + r, first_row + min(c, r + step))
                x = torch.einsum("rgd,td->rgt", s["q"][rows, heads].double(), k) / math.sqrt(case["d"])
                pos = p0 + r + torch.arange(x.shape[0], device="cuda")[:, None]
                hidden = (t > pos) | ((t <= pos - _window(case)) & (t >= case["sinks"]))
                x = x.masked_fill(hidden[:, None], -math.inf)
                z = torch.logsumexp(x, -1)
                lse[rows, heads] = z
                out[rows, heads] = torch.einsum("rgt,td->rgd", torch.exp(x - z[..., None]), v)
    return {"out": out, "lse": lse}


def _code(x):
    """The e4m3 values that stand for bf16 rows [..][d] of finite numbers: a multiple of the step that
    belongs to the value's binade, the even one of two that are as near."""
    x = x.double()
    _, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    y = x * _two(8 - torch.clamp_min(e, -109))
    _, e = torch.frexp(y)
    step = _two(torch.clamp_min(e - 1, -6) - 3)
    return torch.round(y / step) * step


def _two(e):
    """2^e in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)
