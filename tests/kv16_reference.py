"""The paged 16-bit cache, its pages and the attention of prompts from their definitions: page lists in Python, attention in 64 bits with numpy."""
import math

import numpy as np


class Pool:
    """Pages of every sequence and the stack of free ones, one list each."""

    def __init__(self, n_seq, page, n_pages, per_seq, order):
        self.page, self.n_pages, self.per_seq = page, n_pages, per_seq
        self.free = list(order)
        self.pages = [[] for _ in range(n_seq)]
        self.length, self.next = [0] * n_seq, [0] * n_seq

    def update(self, counts, n_tokens):
        """-> starts, slots, positions, taken"""
        P, cap = self.page, self.per_seq * self.page
        # the rows of the packed tensors
        starts, fresh = [0], []
        for c in counts:
            fresh.append(min(max(c, 0), n_tokens - starts[-1]))
            starts.append(starts[-1] + fresh[-1])
        # what comes back
        for i, c in enumerate(counts):
            if c < 0:
                gone = min(-c, self.length[i])
                self.length[i] -= gone
                self.next[i] -= gone
                keep = -(-self.length[i] // P)
                self.free += self.pages[i][keep:]
                del self.pages[i][keep:]
        # what is needed
        taken, slots, positions = [], [-1] * n_tokens, [0] * n_tokens
        for i, c in enumerate(counts):
            taken.append(0)
            if c <= 0:
                continue
            want = min(self.length[i] + fresh[i], cap)
            while len(self.pages[i]) * P < want and self.free:
                self.pages[i].append(self.free.pop())
            taken[i] = min(want, len(self.pages[i]) * P) - self.length[i]
            for k in range(fresh[i]):
                positions[starts[i] + k] = self.next[i] + k
                if k < taken[i]:
                    t = self.length[i] + k
                    slots[starts[i] + k] = self.pages[i][t // P] * P + t % P
            self.length[i] += taken[i]
            self.next[i] += taken[i]
        return starts, slots, positions, taken


def attention(q, k, v, place, scale, cap=0.0, window=0, slopes=None):
    """q [heads][rows][d] at positions place [rows], k and v [keys][d] at positions 0, 1, ..: -> out [heads][rows][d], lse, sum p |v|, size of the scores
    (the largest sum of magnitudes of a row's products), and the smallest weight, relative to the row's largest, of a seen key whose values are not
    finite (1: none).  Only keys that a row sees are looked at."""
    heads, rows, d = q.shape
    out, mag = np.zeros((heads, rows, d)), np.zeros((heads, rows, d))
    lse, size, weak = np.full((heads, rows), -math.inf), np.zeros((heads, rows)), np.ones((heads, rows))
    odd = ~np.isfinite(v).all(1)
    with np.errstate(all="ignore"):
        for i in range(rows):
            lo = max(0, place[i] - window + 1) if window else 0
            hi = min(place[i] + 1, len(k))
            if lo >= hi:
                continue
            back = place[i] - np.arange(lo, hi)
            s = q[:, i] @ k[lo:hi].T * scale
            size[:, i] = np.nan_to_num(np.abs(q[:, i]) @ np.abs(k[lo:hi]).T * abs(scale), posinf=0.0).max(1)
            if cap:
                s = cap * np.tanh(s / cap)
            if slopes is not None:
                s = s - slopes[:, None] * back
                size[:, i] += np.abs(slopes) * back.max()
            top = s.max(1, keepdims=True)
            e = np.exp(s - top)
            total = e.sum(1, keepdims=True)
            weak[:, i] = e[:, odd[lo:hi]].min(1, initial=1.0)
            lse[:, i] = (top + np.log(total))[:, 0]
            out[:, i] = e / total @ v[lo:hi]
            mag[:, i] = e / total @ np.abs(v[lo:hi])
    return out, lse, mag, size, weak
