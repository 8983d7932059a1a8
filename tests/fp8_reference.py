"""The 8-bit cache in 64 bits, from its definition, one sequence at a time: what the GPU tests compare with.  numpy only."""
import math

import numpy as np


def e4m3_values():
    """What the 256 codes stand for (NaN for 0x7f and 0xff)."""
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[b] = math.nan if (b & 127) == 127 else (-v if b & 128 else v)
    return out


VALUES = e4m3_values()
GRID = VALUES[:127]          # the non-negative ones, growing


def nearest_codes(x):
    """Code of the nearest e4m3 value of every x (|x| <= 448), ties to the even code; NaN stays."""
    a = np.abs(x)
    bad = ~np.isfinite(a)
    a = np.where(bad, 0.0, a)
    hi = np.searchsorted(GRID, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = GRID[hi] - a, a - GRID[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(GRID[hi] == a, hi, code).astype(np.uint8)
    code = np.where(np.signbit(x), code | 128, code).astype(np.uint8)
    return np.where(bad, np.uint8(127), code)


def block_exponent(x):
    """Smallest e >= -126 with max |x| <= 448 * 2^e over the finite values."""
    a = np.abs(x[np.isfinite(x)])
    top = a.max() if a.size else 0.0
    e = -126
    if top > 0:
        e = max(-126, math.frexp(top / 448.0)[1] - 2)
        while top > 448.0 * 2.0 ** e:
            e += 1
    return e


class Stream:
    """K or V of one (sequence, head)."""

    def __init__(self, block, d):
        self.block, self.d, self.codes, self.exp, self.flag = block, d, np.zeros((0, d), np.uint8), [], []

    def append(self, x):
        B = self.block
        at = 0
        while at < len(x):
            held = len(self.codes) % B
            new = x[at:at + B - held]
            e = block_exponent(new)
            flag = bool((~np.isfinite(new)).any())
            if held:
                if e > self.exp[-1]:
                    old = VALUES[self.codes[-held:]] * 2.0 ** (self.exp[-1] - e)
                    self.codes[-held:] = nearest_codes(old)
                    self.exp[-1] = e
                e = self.exp[-1]
                self.flag[-1] |= flag
            else:
                self.exp.append(e)
                self.flag.append(flag)
            self.codes = np.concatenate([self.codes, nearest_codes(new * 2.0 ** -e)])
            at += len(new)

    def values(self):
        if not len(self.codes):
            return np.zeros((0, self.d))
        return VALUES[self.codes] * np.repeat(2.0 ** np.array(self.exp, float), self.block)[:len(self.codes), None]


class Sequence:
    def __init__(self, hkv, block, d):
        self.hkv, self.block, self.d = hkv, block, d
        self.k, self.v = [Stream(block, d) for _ in range(hkv)], [Stream(block, d) for _ in range(hkv)]
        self.pos = [np.zeros(0, np.int64) for _ in range(hkv)]
        self.weight = [np.zeros(0) for _ in range(hkv)]
        self.next = 0

    @property
    def length(self):
        return len(self.pos[0])

    def append(self, k, v):
        """k, v [hkv][n][d] in 64 bits"""
        n = k.shape[1]
        for h in range(self.hkv):
            self.k[h].append(k[h])
            self.v[h].append(v[h])
            self.pos[h] = np.concatenate([self.pos[h], self.next + np.arange(n)])
            self.weight[h] = np.concatenate([self.weight[h], np.zeros(n)])
        self.next += n

    def scores(self, q, scale, cap=0.0, window=0, slopes=None):
        """q [hq][n][d] -> [hq][n][length], masked ones -inf; and the largest sum of magnitudes of a row's products"""
        hq, n, _ = q.shape
        r = hq // self.hkv
        s = np.empty((hq, n, self.length))
        size = np.zeros((hq, n))
        i = np.arange(n)[:, None]
        for h in range(hq):
            k = self.k[h // r].values()
            x = q[h] @ k.T * scale
            if self.length:
                size[h] = (np.abs(q[h]) @ np.abs(np.nan_to_num(k)).T * abs(scale)).max(1)
            if cap:
                x = cap * np.tanh(x / cap)
            back = self.next - n + i - self.pos[h // r][None]
            if slopes is not None:
                x = x - slopes[h] * back
                if self.length:
                    size[h] += np.abs(slopes[h] * back).max()
            seen = np.arange(self.length)[None] <= self.length - n + i
            if window:
                seen = seen & (back < window)
            s[h] = np.where(seen, x, -np.inf)
        return s, size

    def attention(self, q, scale, **how):
        """-> out [hq][n][d], lse [hq][n], softmax [hq][n][length], sum p |v|, size of the scores"""
        s, size = self.scores(q, scale, **how)
        hq, n, t = s.shape
        r = hq // self.hkv
        out, mag, lse, soft = np.zeros((hq, n, self.d)), np.zeros((hq, n, self.d)), np.full((hq, n), -np.inf), np.zeros((hq, n, t))
        for h in range(hq):
            v = self.v[h // r].values()
            for i in range(n):
                seen = s[h, i] != -np.inf
                if not seen.any():
                    continue
                x = s[h, i, seen]
                top = x.max()
                e = np.exp(x - top)
                lse[h, i] = top + np.log(e.sum())
                soft[h, i, seen] = e / e.sum()
                out[h, i] = soft[h, i, seen] @ v[seen]
                mag[h, i] = soft[h, i, seen] @ np.abs(v[seen])
        return out, lse, soft, mag, size

    def evict(self, budget, first, last):
        out = Sequence(self.hkv, self.block, self.d)
        out.next = self.next
        t = self.length
        for h in range(self.hkv):
            w = self.weight[h].copy()
            if t <= budget:
                keep = np.arange(t)
            else:
                middle = np.arange(first, t - last)
                w = np.where(np.isnan(w), -np.inf, w)[middle]
                nan = np.isnan(self.weight[h])[middle]
                order = np.lexsort((middle, nan, -w))
                keep = np.sort(np.concatenate([np.arange(first), middle[order[:budget - first - last]], np.arange(t - last, t)]))
            out.k[h].append(self.k[h].values()[keep])
            out.v[h].append(self.v[h].values()[keep])
            out.pos[h], out.weight[h] = self.pos[h][keep], self.weight[h][keep]
        return out
