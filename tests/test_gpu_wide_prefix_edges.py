"""What a row does not see, misses or cannot see of a long shared prefix, by the
wide tiles that such a prefix is read with."""

import math

import numpy as np
import pytest

from attend_world import World, check

pytestmark = pytest.mark.gpu

# 20 sequences of 64 query heads behind 5600 tokens: 7.2 M pairs, twice what narrow
# tiles are taken for
HEADS, GROUP, TOKENS = 4, 16, 5600
SEQS = [(1, m) for m in (0, 1, 15, 40, 33, 0, 64, 7, 21, 3) * 2]
SHORT = {3: TOKENS - 1, 7: 2600, 10: 1, 11: 0, 15: 64 * 9 + 5, 19: TOKENS}  # lengths inside the prefix


def world(torch, **kw):
    w = World(torch, seqs=SEQS, heads=HEADS, group=GROUP, prefix_blocks=TOKENS // kw.get("block_size", 16), **kw)
    for s, n in SHORT.items():
        w.length[s] = n
    w.lengths = torch.tensor(w.length, dtype=torch.int32)
    return w


def expected(w):
    """World.expected, a sequence's query heads at a time."""
    out = np.zeros((w.rows, HEADS * GROUP, w.dim))
    bound = np.zeros_like(out)
    q = w.q.double().numpy()
    for s, L in enumerate(w.length):
        for h in range(HEADS if L else 0):
            k, v, fine = w.values(s, h)
            own = slice(h * GROUP, (h + 1) * GROUP)
            if not fine.all():
                out[s, own] = math.nan
                continue
            with np.errstate(invalid="ignore"):
                a = q[s, own] @ k.T * w.dim**-0.5
                big = (np.abs(q[s, own]) @ np.abs(k).T * w.dim**-0.5).max(1, keepdims=True)
                p = np.exp(a - a.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                out[s, own] = p @ v
                delta = 2 * (w.dim + 8) * 2.0**-24 * big
                bound[s, own] = 2.0**-8 * np.abs(out[s, own]) + (2.0**-8 + delta + 2.0**-20) * (p @ np.abs(v))
    return out, 1.01 * bound + 1e-30


def attend(ck, w):
    pool, seqs, d = w.to_gpu(ck)
    with pool:
        return seqs.attend_shared(w.layer, d.q, d.prefix, offsets=d.offsets, **w.scales()).cpu()


MAIN = [(128, False, 16), (128, True, 16), (64, False, 8)]
KINDS = pytest.mark.parametrize("dim, e4m3, block_size", MAIN)


@pytest.mark.parametrize("dim, e4m3, block_size", MAIN + [(64, True, 16), (128, False, 32)])
def test_rows_that_end_inside(torch, ck, dim, e4m3, block_size):
    w = world(torch, dim=dim, e4m3=e4m3, block_size=block_size, seed=60)
    want = expected(w)
    assert (want[0][11] == 0).all() and (want[0][10] != 0).any()
    check(attend(ck, w), *want)


@KINDS
@pytest.mark.parametrize("at", [2570, TOKENS - 70])
def test_a_missing_block(torch, ck, dim, e4m3, block_size, at):
    """NaN for the rows that see into it, the shorter ones exact."""
    w = world(torch, dim=dim, e4m3=e4m3, block_size=block_size, seed=61)
    w.prefix[at // block_size] = -1 if at == 2570 else w.blocks
    want = expected(w)
    nan = np.isnan(want[0]).any((1, 2))
    assert nan[0] and nan[19] and not nan[[10, 11, 15]].any() and nan[7] == (at == 2570)
    check(attend(ck, w), *want)


@KINDS
def test_hidden_and_seen_nans(torch, ck, dim, e4m3, block_size):
    """NaN in a value near the end of the prefix, and one further in."""
    w = world(torch, dim=dim, e4m3=e4m3, block_size=block_size, seed=62)
    raw = w.kv.view(torch.uint8) if e4m3 else w.kv
    for at, column in ((TOKENS - 1, 3), (2610, dim - 1)):
        raw[2 * w.layer + 1, w.prefix[at // block_size], at % block_size, 0, column] = 0x7F if e4m3 else math.nan
    want = expected(w)
    nan = np.isnan(want[0])
    assert nan[0, :GROUP, 3].all() and not nan[3, :, 3].any() and nan[3, :GROUP, dim - 1].all()
    assert not nan[7].any() and not nan[:, :, 5].any() and not nan[:, GROUP:].any()
    check(attend(ck, w), *want)
