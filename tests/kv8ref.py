"""The 8-bit cache operators from their definitions in 64 bits (numpy / torch on the CPU), for the tests."""
import math

import numpy as np
import torch

SCALE_MIN = 2.0 ** -60


def quantise(x):
    """x [..., dim] (any float type) -> int codes (float64), scales (float32)."""
    x = x.double()
    amax = x.abs().amax(-1)
    s = (amax.float() * torch.tensor(1 / 127, dtype=torch.float32)).clamp_min(SCALE_MIN)
    bad = ~torch.isfinite(x).all(-1)
    s = torch.where(bad, torch.nan, s)
    # 53 bits hold the quotient of two 24-bit numbers far enough to tell a half; an integer has no -0
    c = torch.round(x / s.double().unsqueeze(-1)) + 0.0
    return torch.where(bad.unsqueeze(-1), 0.0, c), s


class Cache:
    """Codes and scales of sequences with capacities caps, as the library lays them out, on the CPU."""

    def __init__(self, caps, kv_heads, dim, gap=0):
        self.cap = list(caps)
        self.off = [gap + sum(caps[:j]) + gap * j for j in range(len(caps))]
        self.tokens = self.off[-1] + caps[-1] + gap
        self.k = torch.zeros(kv_heads, self.tokens, dim, dtype=torch.int8)
        self.v = torch.zeros_like(self.k)
        self.ks = torch.zeros(kv_heads, self.tokens)
        self.vs = torch.zeros_like(self.ks)

    def fill(self, seed, spread=0.5):
        g = torch.Generator().manual_seed(seed)
        for c, s in ((self.k, self.ks), (self.v, self.vs)):
            x = torch.randn(c.shape, generator=g) * torch.exp(spread * torch.randn(s.shape, generator=g)).unsqueeze(-1)
            codes, scale = quantise(x)
            c.copy_(codes.to(torch.int8)), s.copy_(scale)
        return self

    def to_gpu(self):
        from paper_2505_08600_amd import api
        d = lambda t: t.cuda()
        return api.Kv8Cache(d(self.k), d(self.v), d(self.ks), d(self.vs), torch.tensor(self.off, dtype=torch.int64).cuda(),
                            torch.tensor(self.cap, dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda())

    def held(self, b, h, n):
        o = self.off[b]
        return (self.k[h, o:o + n].double() * self.ks[h, o:o + n, None].double(),
                self.v[h, o:o + n].double() * self.vs[h, o:o + n, None].double())


def visible(length, i, cap, causal, window, sinks):
    """Tokens that row i sees, as a list."""
    end = length + i + 1 if causal else length
    seen = range(max(0, min(end, cap)))
    return [t for t in seen if not window or t >= end - window or t < sinks]


def attend(cache, q, parts, scale, causal=True, window=0, sinks=0):
    """q [rows][heads][dim]; parts: (sequence, length, first row, rows) of each sequence.  -> out, lse, and a bound on the error of
    each for `dtype` rows, in float64.

    Bound, from the half steps of what is rounded.  Scores: fp32 queries enter as two 11-bit terms (2^-22 of the row's largest
    element each), products add up in 32 bits (dim + 8 steps of 2^-24 of the sum of magnitudes), so s is off by at most
      ds = scale * (2^-22 max|q| sum|k| + (dim + 8) 2^-24 sum|q k|) + 2^-22 |s|.
    A probability is off by its exponent's ds and by the exponential (2^-22); two terms add 2^-22, one term (bf16 rows) 2^-11; sums
    over n tokens in 32 bits n 2^-24.  Numerator and denominator both carry it: twice, against sum p|v|.  A bf16 result adds 2^-8.
    Below all that: probabilities enter the products as halves of p * (vs / E) * 2^10 or more with E a power of two not above the
    largest scale seen, whose smallest steps are 2^-24, so each token's share of an element may be off by 2^-25 2^-10 E |code|, against a
    denominator of at least 1 (and an exponential below 2^-126 is 0, which is less)."""
    heads, dim = q.shape[1:]
    grp = heads // cache.k.shape[0]
    out = torch.full((q.shape[0], heads, dim), math.nan, dtype=torch.float64)
    lse = torch.full((q.shape[0], heads), math.nan, dtype=torch.float64)
    b_out, b_lse = torch.zeros_like(out), torch.zeros_like(lse)
    p16 = 2.0 ** -11 if q.dtype == torch.bfloat16 else 2.0 ** -22
    for b, length, row0, n in parts:
        for h in range(heads):
            k, v = cache.held(b, h // grp, cache.cap[b])
            for i in range(n):
                see = visible(length, i, cache.cap[b], causal, window, sinks)
                r = row0 + i
                if not see:
                    out[r, h], lse[r, h] = 0.0, -math.inf
                    continue
                kk, vv, qq = k[see], v[see], q[r, h].double()
                s = scale * (kk @ qq)
                p = torch.softmax(s, 0)
                out[r, h], lse[r, h] = p @ vv, torch.logsumexp(s, 0)
                ds = (abs(scale) * (2.0 ** -22 * qq.abs().max() * kk.abs().sum(1) + (dim + 8) * 2.0 ** -24 * (kk.abs() @ qq.abs()))
                      + 2.0 ** -22 * s.abs()).max()
                rel = ds + 2.0 ** -21 + len(see) * 2.0 ** -24
                o = cache.off[b]
                codes, vs = cache.v[h // grp, o:o + cache.cap[b]][see].double(), cache.vs[h // grp, o:o + cache.cap[b]][see]
                floor = 2.0 ** -35 * vs.max().double() * codes.abs().sum(0)
                b_out[r, h] = floor + 2 * (rel + p16) * (p @ vv.abs()) + (2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -23) * out[r, h].abs()
                b_lse[r, h] = rel + 2.0 ** -22 * lse[r, h].abs()
    return out, lse, b_out, b_lse


def rope(x, pos, freq, interleaved=False, inverse=False, gain=1.0):
    x = x.double().numpy()
    rot = 2 * len(freq)
    a = np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64)
    c, s = gain * np.cos(a)[:, None], (-1 if inverse else 1) * gain * np.sin(a)[:, None]
    y = x.copy()
    i0, i1 = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., i0] = x[..., i0] * c - x[..., i1] * s
    y[..., i1] = x[..., i1] * c + x[..., i0] * s
    return torch.from_numpy(y)
