"""Scores of -infinity: such keys have weight 0, and a row that sees no others
has 0 / 0, not the 0 of a row that sees nothing."""

import math

import numpy as np
import pytest

from attend_world import World, check

pytestmark = pytest.mark.gpu

COLUMN = 5


def world(torch, seqs, dead, **kw):
    """Keys of head 0 at the positions ``dead(sequence)`` are -infinity in a
    column where every query is 1 (and every other key positive)."""
    w = World(torch, seqs=seqs, **kw)
    w.q[:, :, COLUMN] = 1.0
    P = w.prefix_blocks * w.bs
    for s in range(len(seqs)):
        for p in dead(s, w.length[s]):
            b = w.prefix[p // w.bs] if p < P else w.tables[s, p // w.bs]
            w.kv[2 * w.layer, b, p % w.bs, 0, COLUMN] = -math.inf
    return w


def expected(w):
    """As World.expected, over the keys whose score is finite."""
    out = np.zeros((w.rows, w.heads * w.group, w.dim))
    bound = np.zeros_like(out)
    q, row = w.q.double().numpy(), 0
    for s, (n, _) in enumerate(w.seqs):
        for h in range(w.heads):
            k, v, _ = w.values(s, h)
            live = np.isfinite(k).all(1)
            for i in range(n):
                seen = np.flatnonzero(live[:w.length[s] - n + i + 1])
                for x in range(h * w.group, (h + 1) * w.group):
                    if w.length[s] - n + i < 0:
                        continue
                    if not len(seen):
                        out[row + i, x] = np.nan
                        continue
                    a = k[seen] @ q[row + i, x] * w.dim**-0.5
                    big = np.abs(k[seen]) @ np.abs(q[row + i, x]) * w.dim**-0.5
                    p = np.exp(a - a.max())
                    p /= p.sum()
                    out[row + i, x] = p @ v[seen]
                    delta = 2 * (w.dim + 8) * 2.0**-24 * big.max()
                    bound[row + i, x] = (2.0**-8 * np.abs(out[row + i, x])
                                         + (2.0**-8 + delta + 2.0**-20) * (p @ np.abs(v[seen])))
        row += n
    return out, 1.01 * bound + 1e-30


def attend(ck, w, prefix=False):
    pool, seqs, d = w.to_gpu(ck)
    with pool:
        if prefix:
            return seqs.attend_shared(w.layer, d.q, d.prefix, offsets=d.offsets, **w.scales()).cpu()
        return seqs.attend(w.layer, d.q, offsets=d.offsets, **w.scales()).cpu()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("seqs", [[(1, 0), (1, 30)], [(9, 0), (1, 0)], [(200, 0), (70, 10)], [(1, 5000)], [(30, 4000)]],
                         ids=str)
@pytest.mark.parametrize("dead", ["all", "first", "last"])
def test_keys_of_minus_infinity(torch, ck, seqs, dim, dead):
    places = {"all": lambda s, n: range(n),
              "first": lambda s, n: range(max(1, 3 * n // 4)),  # tiles and splits of nothing else
              "last": lambda s, n: range(n // 4, n)}[dead]
    w = world(torch, seqs, places, group=4, dim=dim, heads=2, seed=40)
    want = expected(w)
    if dead == "all":
        assert np.isnan(want[0][:, :4]).all()
    assert not np.isnan(want[0][:, 4:]).any()
    check(attend(ck, w), *want)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("seqs, blocks", [([(1, 0), (1, 30), (1, 2)], 6), ([(1, 3)] * 100, 350)], ids=["few", "many"])
@pytest.mark.parametrize("all_of_it", [False, True])
def test_a_prefix_of_minus_infinity(torch, ck, seqs, blocks, dim, all_of_it):
    """What comes after a prefix of such keys; and rows behind it that end inside."""
    P = 16 * blocks
    w = world(torch, seqs, lambda s, n: range(n if all_of_it else P), group=8, dim=dim, heads=1,
              prefix_blocks=blocks, seed=41)
    w.length[1] = P - 21
    w.lengths[1] = P - 21
    want = expected(w)
    assert np.isnan(want[0][1]).all() and np.isnan(want[0][0]).all() == all_of_it
    check(attend(ck, w, prefix=True), *want)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("seqs", [[(1, 40)], [(90, 0)], [(1, 3000)], [(3, 7)]], ids=str)
def test_a_query_of_minus_infinity(torch, ck, seqs, e4m3):
    """One row's query, over keys that are positive there; a row that sees
    nothing stays 0."""
    w = World(torch, seqs=seqs + [(2, 0)], group=2, e4m3=e4m3, seed=42)
    raw = w.kv.view(torch.uint8) if e4m3 else w.kv
    raw[2 * w.layer, ..., COLUMN] = 0x38 if e4m3 else 1.0
    w.length[1] = 1
    w.lengths[1] = 1
    clean, bound = w.expected()
    w.q[0, 1, COLUMN] = -math.inf
    clean[0, 1] = np.nan
    assert (clean[-2] == 0).all()
    check(attend(ck, w), clean, bound)
