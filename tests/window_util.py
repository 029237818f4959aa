"""Inputs, oracle results and error bounds for windowed attention and attention over the 8-bit cache."""
import numpy as np
import torch

import oracle.fp8 as ref
import paper_2409_17264_amd as medha
from paper_2409_17264_amd import workloads as wl

FP8 = torch.float8_e4m3fn


def bits(x):
    t = torch.as_tensor(x).to(torch.bfloat16)
    return t.contiguous().view(torch.int16).numpy().view(np.uint16)


def from_bits(b):
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).view(torch.bfloat16)


class Case:
    """A batch over a cache in which all that no row sees is NaN: slots of no token, tokens between
    the first ones and the windows, and the pages that their table entries point at."""

    def __init__(self, h_q, h_kv, d, prefix, chunk, window=None, sinks=0, fp8=False, seed=0,
                 k_std=1.0, spare=2):
        self.h_q, self.h_kv, self.d, self.fp8 = h_q, h_kv, d, fp8
        self.prefix, self.chunk = np.array(prefix, np.int32), np.array(chunk, np.int32)
        self.window, self.sinks = window, sinks
        self.scale = d ** -0.5
        rng = np.random.default_rng(seed)
        n_pages = [wl.pages_for(p + c) for p, c in zip(prefix, chunk)]
        self.offs = np.concatenate([[0], np.cumsum(n_pages)]).astype(np.int64)
        pages = int(self.offs[-1]) + spare
        self.table = rng.permutation(pages)[:self.offs[-1]].astype(np.int32)
        self.dead_page = int(np.setdiff1d(np.arange(pages), self.table)[0])
        tokens = int(self.chunk.sum())
        self.q = bits(rng.standard_normal((tokens, h_q, d)))
        shape = (pages, h_kv, 16, d)
        k = rng.standard_normal(shape) * k_std * np.exp(0.3 * rng.standard_normal((*shape[:3], 1)))
        v = rng.standard_normal(shape) * np.exp(0.5 * rng.standard_normal((*shape[:3], 1)))
        seen = np.zeros((pages, 16), bool)
        for b, (p, c) in enumerate(zip(prefix, chunk)):
            t = np.arange(p + c)
            if window is not None:
                t = t[(t > p - window) | (t < sinks)]
            at = self.table[self.offs[b] + t // 16]
            seen[at, t % 16] = True
        live = seen.any(1)
        self.table = np.where(live[self.table], self.table, self.dead_page).astype(np.int32)
        hide = ~seen[:, None, :, None]
        kb, vb = bits(k), bits(v)
        if fp8:
            (self.k, ks), (self.v, vs) = ref.quantise_rows(kb), ref.quantise_rows(vb)
            self.kv_scale = np.stack([ks, vs], 2)
            self.kv_scale[np.broadcast_to(~seen[:, None, None, :], self.kv_scale.shape)] = 255
            for x in (self.k, self.v):
                x[np.broadcast_to(hide, x.shape)] = 0x7f
            self.kf, self.vf = (ref.cache_values(x, self.kv_scale[:, :, w]) for w, x in
                                enumerate((self.k, self.v)))
        else:
            for x in (kb, vb):
                x[np.broadcast_to(hide, x.shape)] = 0x7fc0
            self.k, self.v = kb, vb
            self.kf, self.vf = ref.bf16_values(kb), ref.bf16_values(vb)

    def device(self):
        conv = (lambda x: torch.from_numpy(x).cuda().view(FP8)) if self.fp8 else (lambda x: from_bits(x).cuda())
        cache = [conv(self.k), conv(self.v)]
        if self.fp8:
            cache.append(torch.from_numpy(self.kv_scale).cuda())
        return from_bits(self.q).cuda(), cache, torch.from_numpy(self.table).cuda()

    def run(self, out=None, lse=None, workspace=None, dev=None, **lengths):
        q, cache, table = dev or self.device()
        call = medha.chunked_prefill_attn_fp8 if self.fp8 else medha.window_attn
        got = call(q, *cache, table, self.offs, lengths.get("prefix", self.prefix),
                   lengths.get("chunk", self.chunk), self.scale, self.window or 0, self.sinks, out,
                   lse, workspace)
        return got

    def oracle(self):
        """(out, lse, bound on |out - result| in fp32, bound on |lse - result|)."""
        args = (self.table, self.offs, self.prefix, self.chunk)
        out, lse = ref.window_attn(self.q, self.kf, self.vf, *args, self.scale, self.window, self.sinks)
        mean_abs, _ = ref.window_attn(self.q, self.kf, np.abs(self.vf), *args, self.scale, self.window,
                                      self.sinks)
        # A score's error: the matrix instructions add up d products.  With bf16 operands in fp32:
        # d roundings of at most the sum of the magnitudes.  The 8-bit one keeps about 13 bits below
        # its largest product (2^-12.8 of the sum of magnitudes, measured over random operands).
        # (Magnitudes of a row and a key at most the product of their 2-norms; the longest key.)
        qn = np.sqrt((ref.bf16_values(self.q) ** 2).sum(-1))
        kn = np.sqrt(np.nansum(np.where(np.isfinite(self.kf), self.kf, 0) ** 2, -1)).max()
        unit = 2.0 ** -12 if self.fp8 else (self.d + 4) * 2.0 ** -24
        score = unit * abs(self.scale) * qn * kn
        keys = int((self.prefix + self.chunk).max())
        total = (keys / 32 + 64) * 2.0 ** -24 + 2.0 ** -21     # adding up, exponential, logarithm
        lse_bound = score + total + 2.0 ** -22 * np.abs(lse)
        # probabilities are rounded to bf16 (2^-8 of each); both sums have the scores' errors
        out_bound = mean_abs * (2.0 ** -8 + 2 * (score + total))[..., None]
        return out, lse, out_bound, lse_bound

    def check(self, out, lse, want=None):
        ro, rl, bo, bl = want or self.oracle()
        o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
        if out.dtype == torch.bfloat16:
            bo = bo * (1 + 2.0 ** -8) + np.abs(ro) * 2.0 ** -8
        assert np.isfinite(o).all() and np.isfinite(l).all()
        eo, el = np.abs(o - ro), np.abs(l - rl)
        print(f"max|dO|={eo.max():.2e} ({(eo / bo).max():.2f} of its bound) max|dLSE|={el.max():.2e} "
              f"({(el / bl).max():.2f}) rel {np.linalg.norm(o - ro) / np.linalg.norm(ro):.1e}", flush=True)
        assert (eo <= bo).all() and (el <= bl).all()
