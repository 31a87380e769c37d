"""The operators on heads from their definitions, in 64 bits on the CPU, one sequence and one block after the other."""
import math

import numpy as np
import torch

E_MIN, E_MAX = -40, 40


def decode_table():
    """The 256 E4M3 values: sign, four exponent bits of bias 7, three fraction bits; 0x7f and 0xff are NaN."""
    out = np.zeros(256)
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        mag = math.nan if c & 0x7F == 0x7F else f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        out[c] = -mag if c & 0x80 else mag
    return out


VALUES = decode_table()


def encode(x):
    """Nearest code, ties to the even one; NaN as 0, beyond the largest that one.  The sign of a zero is not compared."""
    x = np.where(np.isnan(x), 0.0, np.clip(x, -448.0, 448.0))
    mags = VALUES[:127]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(mags, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - mags[lo], mags[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code + np.where((x < 0) & (code > 0), 128, 0)).astype(np.uint8)


def exponent(amax):
    """The smallest whole e with amax <= 448 * 2^e, inside the range; by trying them."""
    for e in range(E_MIN, E_MAX):
        if amax <= 448.0 * 2.0 ** e:
            return e
    return E_MAX


def rope(x, w, positions, inv_freq, rot, interleaved, eps, norm):
    """x [M, heads, dim] -> (result in float64, |y_a| + |y_b| of each element's pair)"""
    x = x.double().numpy().copy()
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if w is not None:
            x = x * w.double().numpy()
    y, size = x.copy(), np.abs(x)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        t = positions.double().numpy() * float(inv_freq[i])
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


class Cache:
    """A cache on the CPU: codes [blocks, heads, block, dim] for both sides, exponents [blocks, heads]."""

    def __init__(self, blocks, heads, block, dim, fill=0x7F):
        self.sizes = (blocks, heads, block, dim)
        self.k, self.v = (np.full(self.sizes, fill, dtype=np.uint8) for _ in range(2))
        self.ke, self.ve = (np.zeros((blocks, heads), dtype=np.int64) for _ in range(2))

    def write(self, K, V, table, lens, cu, batch):
        """K, V float64 [M, heads, dim]"""
        blocks, heads, block, _ = self.sizes
        for b in range(batch):
            n = int(cu[b + 1] - cu[b])
            start = int(lens[b]) - n
            touched = {}
            for i in range(n):
                if start + i >= 0:
                    touched.setdefault((start + i) // block, []).append(i)
            for o, rows in touched.items():
                page = int(table[b, o])
                if not 0 <= page < blocks:
                    continue
                slots = [(start + i) % block for i in rows]
                for codes, exps, X in ((self.k, self.ke, K), (self.v, self.ve, V)):
                    for h in range(heads):
                        x = X[[cu[b] + i for i in rows], h]
                        e = exponent(np.max(np.abs(np.where(np.isfinite(x), x, 0.0))))
                        if slots[0] > 0:
                            e = max(e, exps[page, h])
                            if e > exps[page, h]:
                                old = codes[page, h]  # the whole block, a NaN where nothing was written yet stays one
                                codes[page, h] = np.where(old & 0x7F == 0x7F, old, encode(VALUES[old] * 2.0 ** float(exps[page, h] - e)))
                        codes[page, h, slots] = encode(x * 2.0 ** float(-e))
                        exps[page, h] = e

    def rows(self, table, b, n):
        """(keys, values, whether each is there) of the first n tokens of sequence b, float64 [n, heads, dim]"""
        blocks, heads, block, dim = self.sizes
        K, V, there = np.zeros((n, heads, dim)), np.zeros((n, heads, dim)), np.zeros(n, dtype=bool)
        for o in range(-(-n // block)):
            page, lo, hi = int(table[b, o]), o * block, min(n, (o + 1) * block)
            if 0 <= page < blocks:
                there[lo:hi] = True
                for codes, exps, out in ((self.k, self.ke, K), (self.v, self.ve, V)):
                    out[lo:hi] = (VALUES[codes[page]] * 2.0 ** exps[page][:, None, None].astype(float)).transpose(1, 0, 2)[:hi - lo]
        return K, V, there

    def device(self, B, dev="cuda:0"):
        k = torch.from_numpy(self.k.copy()).to(dev)
        v = torch.from_numpy(np.ascontiguousarray(self.v.transpose(0, 1, 3, 2))).to(dev)
        return B.make_cache(k, v, *(torch.from_numpy(2.0 ** e.astype(np.float32)).float().to(dev) for e in (self.ke, self.ve)))

    def back(self, cache):
        """What a device cache holds, as one of these."""
        c = Cache(*self.sizes)
        k, v, ks, vs = (t.cpu().numpy() for t in cache.tensors)
        c.k, c.v = k, np.ascontiguousarray(v.transpose(0, 1, 3, 2))
        c.ke, c.ve = (np.log2(s.astype(np.float64)).astype(np.int64) for s in (ks, vs))
        assert all((2.0 ** e == s).all() for e, s in ((c.ke, ks), (c.ve, vs)))
        return c


def attention(cache, Q, table, lens, cu, batch, alpha, causal, window):
    """Q float64 [M, heads, dim] -> out, lse, and what bounds a kernel's error:
    near   sum_j p_j |v_j| (errors relative to the weights), far   sum_j |v_j| / sum_j exp(s_j - max s) (absolute ones),
    score  the largest alpha sum |q_i k_i| of a row (errors of scores)"""
    M, heads, dim = Q.shape
    out, lse = np.zeros(Q.shape), np.full((M, heads), -np.inf)
    near, far, score = np.zeros(Q.shape), np.zeros(Q.shape), np.zeros((M, heads))
    group = heads // cache.sizes[1]
    for b in range(batch):
        n, m = int(cu[b + 1] - cu[b]), int(lens[b])
        K, V, there = cache.rows(table, b, m)
        j = np.arange(m)
        for i in range(n):
            p = m - n + i
            see = there & (j <= p) if causal else there.copy()
            if window:
                see &= j > p - window
            if not see.any():
                continue
            for h in range(heads):
                q, k, v = Q[cu[b] + i, h], K[see, h // group], V[see, h // group]
                s = alpha * (k @ q)
                w = np.exp(s - s.max())
                out[cu[b] + i, h] = (w @ v) / w.sum()
                lse[cu[b] + i, h] = s.max() + np.log(w.sum())
                near[cu[b] + i, h] = (w @ np.abs(v)) / w.sum()
                far[cu[b] + i, h] = np.abs(v).sum(0) / w.sum()
                score[cu[b] + i, h] = (alpha * (np.abs(k) @ np.abs(q))).max()
    return out, lse, near, far, score


def attention_tolerance(dtype, out, lse, near, far, score):
    """(of out, of lse).  Scores are fp32 sums of up to 256 exact products: at most 256 * 2^-24 of sum |q_i k_i| off, the
    factor alpha and the power add 2^-21.  Weights are rounded to fp16, 2^-11 of each while it is normal; relative to the
    row's largest weight one is at least 2^-4 / 1 of its stored size (a block's value scale may be 4 bits off the sums'
    unit), so below the normal range it is off by at most 2^-25 * 2^4 of the largest.  Sums in fp32 and the split's
    rescaling add less than 2^-16 of what is summed.  Then one rounding."""
    ds = score * 2.0 ** -16 + 2.0 ** -20
    eps = torch.finfo(dtype).eps / 2
    tol = eps * np.abs(out) + near * (2.0 ** -11 + 2 * ds[..., None] + 2.0 ** -16) * 1.01 + far * 2.0 ** -21 + float(torch.finfo(dtype).smallest_normal) * eps
    return tol, ds + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0.0)) + 2.0 ** -20
