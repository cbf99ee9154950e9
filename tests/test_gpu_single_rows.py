"""One row, or one head, of a wider tensor: the stride that leads nowhere may
be any."""

import pytest

from attend_world import World, check

pytestmark = pytest.mark.gpu


def strided(torch, x, row, head):
    """x with those strides in elements, its data first in a tensor of its own."""
    n = 1 + sum((size - 1) * step for size, step in zip(x.shape, (row, head, 1)))
    wide = torch.zeros(n + 7, dtype=x.dtype, device="cuda").as_strided(x.shape, (row, head, 1))
    wide.copy_(x)
    return wide


@pytest.mark.parametrize("seqs, heads, group, row, head", [
    ([(1, 40)], 2, 2, 259, 64),  # one row
    ([(1, 0)], 1, 1, 1, 3),  # one row of one head
    ([(7, 20)], 1, 1, 72, 5)], ids=str)  # rows of one head
def test_attention(torch, ck, seqs, heads, group, row, head):
    w = World(torch, seqs=seqs, heads=heads, group=group, seed=50)
    pool, s, d = w.to_gpu(ck)
    with pool:
        q = strided(torch, w.q, row, head)
        out = strided(torch, torch.zeros_like(w.q), row, head)
        assert s.attend(w.layer, q, offsets=d.offsets, out=out) is out
        check(out, *w.expected())


@pytest.mark.parametrize("rows, heads, row, head", [(1, 2, 131, 64), (1, 1, 1, 3), (9, 1, 72, 5)])
def test_write(torch, ck, rows, heads, row, head):
    w = World(torch, seqs=[(rows, 13)], heads=heads, seed=51)
    pool, s, d = w.to_gpu(ck)
    with pool:
        g = torch.Generator().manual_seed(1)
        k, v = torch.randn(2, rows, heads, 64, generator=g).to(torch.bfloat16)
        s.write(w.layer, strided(torch, k, row, head), strided(torch, v, row, head), offsets=d.offsets)
        pos = torch.arange(13, 13 + rows)
        block = w.tables[0].long()[pos // w.bs]
        for plane, x in ((0, k), (1, v)):
            assert torch.equal(d.kv[2 * w.layer + plane].cpu()[block, pos % w.bs], x)


def test_strides_that_matter_are_refused(torch, ck):
    w = World(torch, seqs=[(3, 4)], heads=2, seed=52)
    pool, s, d = w.to_gpu(ck)
    with pool:
        for row, head in ((259, 64), (264, 65)):
            with pytest.raises(ck.ClaimError):
                s.attend(w.layer, strided(torch, w.q, row, head), offsets=d.offsets)
