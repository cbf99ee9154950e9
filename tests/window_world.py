"""A world of sequences whose rows see a window and a few first tokens: the
definition in 64 bits, of outputs, logarithms of sums, and tokens' weights."""

import math

import numpy as np

from attend_world import World


class WindowWorld(World):
    def __init__(self, torch, *, window=None, sinks=0, **kw):
        super().__init__(torch, **kw)
        self.window, self.sinks = window, sinks

    def seen(self, P):
        """Which of positions 0..P the row at P sees."""
        p = np.arange(P + 1)
        return p >= 0 if self.window is None else (p > P - self.window) | (p < self.sinks)

    def set_lengths(self, lengths):
        self.length = list(lengths)
        self.lengths = self.torch.tensor(self.length, dtype=self.torch.int32)

    def rows_of(self, scale=None):
        """For each row and query head that sees something: (row, head, its
        sequence, KV head, positions seen, whether all have a block, scores,
        the largest sum of magnitudes of a score, values)."""
        scale = self.dim**-0.5 if scale is None else scale
        q, row = self.q.double().numpy(), 0
        for s, (n, _) in enumerate(self.seqs):
            L = self.length[s]
            for h in range(self.heads if n else 0):
                k, v, fine = self.values(s, h)
                for i in range(n):
                    P = L - n + i
                    if P < 0:
                        continue
                    p = np.nonzero(self.seen(P))[0]
                    for g in range(self.group):
                        x = h * self.group + g
                        with np.errstate(invalid="ignore", over="ignore"):
                            a = k[p] @ q[row + i, x] * scale
                            big = np.abs(k[p]) @ np.abs(q[row + i, x]) * scale
                        yield row + i, x, s, p, bool(fine[p].all()), a, big.max(), v[p]
            row += n

    def expected(self, scale=None):
        """(outputs, bounds, logarithms of sums, their bounds).

        Outputs' bounds are the ones of attention without a window.  A
        logarithm moves as far as the scores do, which are off by at most
        (dim + 8) 2^-24 of the largest sum of magnitudes, twice for the
        maximum and a score; a sum of M weights in any order is off by at
        most M 2^-24 of itself, a weight by 2^-22; the last step by 2^-23 of
        the result and of the maximum."""
        out = np.zeros((self.rows, self.heads * self.group, self.dim))
        bound, lse = np.zeros_like(out), np.full(out.shape[:2], -math.inf)
        room = np.zeros_like(lse)
        for row, x, _, p, fine, a, big, v in self.rows_of(scale):
            if not fine:
                out[row, x] = lse[row, x] = math.nan
                continue
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                w = np.exp(a - a.max())
                lse[row, x] = a.max() + np.log(w.sum()) if a.max() > -math.inf else -math.inf
                w /= w.sum()
                out[row, x] = w @ v
                delta = 2 * (self.dim + 8) * 2.0**-24 * big
                bound[row, x] = (2.0**-8 * np.abs(out[row, x])
                                 + (2.0**-8 + delta + 2.0**-20) * (w @ np.abs(v)))
                room[row, x] = (delta + (len(p) + 8) * 2.0**-24
                                + 2.0**-22 * (1 + abs(lse[row, x]) + abs(a.max())))
        return out, 1.01 * bound + 1e-30, lse, 1.01 * room

    def weights(self, lse, scale=None):
        """(what every position of every sequence gets, bounds) for given
        logarithms.  A weight is off by its score's error (as above, and 2^-23
        of the score's and the logarithm's size, and 2^-22), a sum of N by N
        2^-24 of itself."""
        got = np.zeros((len(self.tables), self.tables.shape[1] * self.bs))
        room, count = np.zeros_like(got), np.zeros_like(got)
        lse = lse.double().cpu().numpy()
        for row, x, s, p, fine, a, big, _ in self.rows_of(scale):
            if not np.isfinite(lse[row, x]) or not fine:
                continue
            with np.errstate(over="ignore"):
                w = np.exp(a - lse[row, x])
            got[s, p] += w
            room[s, p] += w * ((self.dim + 8) * 2.0**-24 * big + 2.0**-22
                               + 2.0**-23 * (np.abs(a) + abs(lse[row, x])))
            count[s, p] += 1
        return got, 1.01 * (room + (count + 2) * 2.0**-24 * got) + 1e-37


def check_lse(lse, expected, room):
    got = lse.double().cpu().numpy()
    assert got.shape == expected.shape
    assert np.array_equal(np.isnan(got), np.isnan(expected))
    finite = np.isfinite(expected)
    assert np.array_equal(got[~finite], expected[~finite], equal_nan=True)
    off = np.abs(got - expected)[finite]
    assert (off <= room[finite]).all(), (off / room[finite]).max()
