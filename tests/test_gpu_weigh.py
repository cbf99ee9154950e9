"""What cached tokens weigh for query rows, against the definition in 64 bits."""

import numpy as np
import pytest

from window_world import WindowWorld

pytestmark = pytest.mark.gpu


def column(w, extra=0):
    return w.tables.shape[1] * w.bs + extra


def weigh(ck, w, stream=None, start=0.0, lse=None, extra=0, **kw):
    """(weights after one call, the logarithms it was given)."""
    torch = w.torch
    pool, seqs, d = w.to_gpu(ck, stream)
    got = torch.full((len(w.tables), column(w, extra)), start, device="cuda")
    sums = torch.empty(w.rows, w.heads * w.group, device="cuda")
    with pool:
        seqs.attend_window(w.layer, d.q, w.window, sinks=w.sinks, offsets=d.offsets, lse=sums, **w.scales())
        if lse is not None:
            sums = lse(sums)
        seqs.weigh(w.layer, d.q, sums, got, window=w.window, sinks=w.sinks, offsets=d.offsets,
                   k_scale=w.k_scale, **kw)
        torch.cuda.synchronize()
    return got, sums


def compare(w, got, lse, start=0.0, ids=None):
    want, room = w.weights(lse)
    got = got.double().cpu().numpy()
    rest = got[:, want.shape[1]:]
    assert (rest == start).all()
    got = got[:, :want.shape[1]]
    touched = want > 0
    assert (got[~touched & (room <= 1e-36)] == start).all()
    off = np.abs(got - start - want)
    room = room + 2.0**-23 * np.abs(got)
    assert (off <= room).all(), (off / room).max()


def both(ck, w, **kw):
    got, lse = weigh(ck, w, **kw)
    compare(w, got, lse)


SEQS = {
    "one": [(1, 0)],
    "short": [(3, 0), (1, 7), (0, 5), (16, 0), (17, 1)],
    "tile-edges": [(32, 0), (33, 31), (64, 0), (63, 1), (65, 64)],
    "long": [(257, 0), (5, 300), (130, 577)],
    "steps": [(1, 700), (1, 65), (1, 64), (1, 63), (1, 0)],
    "few-rows": [(4, 500), (2, 3), (3, 129)],
}


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window,sinks", [(None, 0), (1, 0), (64, 4), (100, 70), (600, 0)])
@pytest.mark.parametrize("seqs", SEQS.values(), ids=SEQS)
def test_weights(torch, ck, seqs, window, sinks, dim, e4m3):
    both(ck, WindowWorld(torch, seqs=seqs, dim=dim, e4m3=e4m3, window=window, sinks=sinks, seed=1))


@pytest.mark.parametrize("block_size", [1, 5, 8, 24, 64, 100])
@pytest.mark.parametrize("dim", [64, 128])
def test_block_sizes(torch, ck, block_size, dim):
    if block_size * dim * 2 * 3 % 16:
        pytest.skip("chunks are multiples of 16 bytes")
    for seqs in ([(40, 0), (1, 170), (90, 130)], [(1, 170), (1, 20), (2, 3)]):
        both(ck, WindowWorld(torch, seqs=seqs, heads=3, block_size=block_size, dim=dim, seed=2))


@pytest.mark.parametrize("heads,group", [(1, 1), (1, 16), (2, 5), (3, 7), (8, 4), (5, 1), (1, 33), (1, 64)])
def test_head_groups(torch, ck, heads, group):
    for seqs in ([(90, 120), (1, 50), (40, 3)], [(1, 300), (1, 3)]):
        both(ck, WindowWorld(torch, seqs=seqs, heads=heads, group=group, seed=3))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("seqs", [[(1, 5000)], [(600, 600)], [(1200, 0), (2, 900)]], ids=str)
def test_long(torch, ck, seqs, e4m3):
    both(ck, WindowWorld(torch, seqs=seqs, heads=1, group=4, dim=128, e4m3=e4m3, seed=4))
    both(ck, WindowWorld(torch, seqs=seqs, heads=1, group=4, dim=128, e4m3=e4m3, window=333, sinks=5, seed=4))


@pytest.mark.parametrize("seqs", [SEQS["long"], SEQS["steps"]], ids=str)
def test_it_adds_and_leaves_the_rest(torch, ck, seqs):
    """To what is there; columns past the table, and positions past the
    sequence or that no row sees, stay."""
    w = WindowWorld(torch, seqs=seqs, window=50, sinks=2, seed=5)
    got, lse = weigh(ck, w, start=3.0, extra=13)
    compare(w, got, lse, start=3.0)


@pytest.mark.parametrize("seqs", [SEQS["long"], SEQS["steps"]], ids=str)
def test_logarithms_that_are_not_finite_add_nothing(torch, ck, seqs):
    w = WindowWorld(torch, seqs=seqs, seed=6)

    def spoil(lse):
        lse[0, 0], lse[0, 1], lse[0, 2] = float("nan"), float("inf"), -float("inf")
        return lse
    both(ck, w, lse=spoil)


@pytest.mark.parametrize("kind", ["none", "out of range"])
@pytest.mark.parametrize("seqs", [[(140, 30), (5, 0)], [(1, 199), (1, 4)]], ids=str)
def test_missing_blocks(torch, ck, seqs, kind):
    """Behind a window, or seen by rows that are NaN for it: nothing is added
    there, and those rows add nothing anywhere."""
    w = WindowWorld(torch, seqs=seqs, window=20, sinks=3, seed=7)
    w.tables[0, 2] = w.tables[0, 5] = -1 if kind == "none" else w.blocks
    got, lse = weigh(ck, w)
    compare(w, got, lse)
    # and where the logarithms say otherwise, a position without a block is left
    got, lse = weigh(ck, w, lse=lambda x: torch.where(torch.isnan(x), 1.0, x))
    gone = got[0].view(-1, w.bs)[[2, 5]]
    assert bool((gone == 0).all()) and bool(torch.isfinite(got).all())


@pytest.mark.parametrize("seqs", [[(140, 60)], [(1, 199)]], ids=str)
def test_hidden_keys_have_no_effect(torch, ck, seqs):
    w = WindowWorld(torch, seqs=seqs, window=40, sinks=5, seed=8)
    got, lse = weigh(ck, w)
    first = w.length[0] - seqs[0][0] - 40 + 1
    for pos in (5, first - 1):
        w.kv[2 * w.layer, w.tables[0, pos // w.bs], pos % w.bs] = float("nan")
    again, _ = weigh(ck, w)
    assert torch.equal(got, again)
    compare(w, again, lse)


def test_lengths_out_of_range(torch, ck):
    """More rows than tokens; lengths past the table, whose rows are NaN."""
    for seqs in ([(140, 0), (3, 10)], [(3, 0), (1, 10)]):
        w = WindowWorld(torch, seqs=seqs, seed=9)
        w.set_lengths([seqs[0][0] - 2, w.length[1]])
        both(ck, w)
        for wild in (w.tables.shape[1] * w.bs + seqs[0][0], 2**31 - 1):
            w.lengths[0] = wild
            got, lse = weigh(ck, w)
            assert bool(torch.isnan(lse[:seqs[0][0]]).all())
            assert bool((got[0] == 0).all()) and bool((got[1, :w.length[1]] > 0).all())


@pytest.mark.parametrize("seqs", [[(140, 60), (30, 9), (80, 0)], [(1, 299), (2, 40), (1, 0)]], ids=str)
def test_ids_and_last_rows(torch, ck, seqs):
    """Sequences by number, and the last rows of a batch with their logarithms."""
    w = WindowWorld(torch, seqs=seqs, seed=10)
    got, lse = weigh(ck, w)
    order = [2, 0, 1]
    pool, s, d = w.to_gpu(ck)
    with pool:
        rows, off, ids = [], [0], []
        for k in order:
            n, a = seqs[k][0], int(w.offsets[k])
            rows += list(range(a, a + n))
            off.append(off[-1] + n)
            ids.append(k)
        t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        again = torch.zeros_like(got)
        s.weigh(w.layer, d.q[rows].contiguous(), lse[rows].contiguous(), again, ids=t(ids), offsets=t(off))
        assert torch.equal(again, got)
        last = [int(w.offsets[k + 1]) - 1 for k in range(3)]
        again.zero_()
        s.weigh(w.layer, d.q[last].contiguous(), lse[last].contiguous(), again)
        torch.cuda.synchronize()
    w2 = WindowWorld(torch, seqs=[(1, n + m - 1) for n, m in seqs], seed=10)
    w2.kv, w2.tables, w2.q, w2.blocks = w.kv, w.tables, w.q[last], w.blocks
    compare(w2, again, lse[last])


@pytest.mark.parametrize("seqs", [[(140, 60), (80, 900)], [(1, 1999), (2, 40)]], ids=str)
def test_equal_bits_streams_and_graphs(torch, ck, seqs):
    w = WindowWorld(torch, seqs=seqs, heads=4, seed=11)
    first, lse = weigh(ck, w)
    again, _ = weigh(ck, w, stream=torch.cuda.Stream())
    assert torch.equal(first, again)
    pool, s, d = w.to_gpu(ck, torch.cuda.Stream())
    got = torch.zeros_like(first)
    with pool:
        s.weigh(w.layer, d.q, lse, got, offsets=d.offsets)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=pool.stream):
            s.weigh(w.layer, d.q, lse, got, offsets=d.offsets)
        for _ in range(3):
            got.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(first, got)
            s.attend(w.layer, d.q, offsets=d.offsets)


def test_a_sequence_named_twice_counts_twice(torch, ck):
    w = WindowWorld(torch, seqs=[(1, 200)], heads=1, group=1, seed=12)
    once, lse = weigh(ck, w)
    pool, s, d = w.to_gpu(ck)
    got = torch.zeros_like(once)
    with pool:
        q, sums = torch.cat([d.q, d.q]), torch.cat([lse, lse])
        w2 = torch.zeros(2, once.shape[1], device="cuda")
        from paper_2606_01387_amd.sequences import Sequences

        s = Sequences(pool, tables=torch.cat([d.tables, d.tables]), lengths=torch.cat([d.lengths, d.lengths]))
        s.weigh(w.layer, q, sums, w2, ids=torch.zeros(2, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
    assert torch.equal(w2[0], 2 * once[0]) and bool((w2[1] == 0).all())
    del got


def test_refusals(torch, ck):
    w = WindowWorld(torch, seqs=[(4, 9), (2, 0)], seed=13)
    pool, s, d = w.to_gpu(ck)
    with pool:
        lse = torch.zeros(6, 4, device="cuda")
        good = torch.zeros(2, column(w), device="cuda")
        for bad in (good[:, :-1], good[:1], good.half(), good.cpu(), good.T.contiguous().T, good[0]):
            with pytest.raises(ValueError):
                s.weigh(w.layer, d.q, lse, bad, offsets=d.offsets)
        for bad in (lse[:5], lse.double(), lse.cpu(), lse.T.contiguous().T):
            with pytest.raises(ValueError):
                s.weigh(w.layer, d.q, bad, good, offsets=d.offsets)
        with pytest.raises(ValueError):
            s.weigh(w.layer, d.q, lse, good, offsets=d.offsets, window=0)
        for bad in (dict(scale=0.0), dict(scale=float("inf")), dict(k_scale=2.0)):
            with pytest.raises(ck.ClaimError):
                s.weigh(w.layer, d.q, lse, good, offsets=d.offsets, **bad)
        with pytest.raises(ck.ClaimError):
            s.weigh(9, d.q, lse, good, offsets=d.offsets)
        s.weigh(w.layer, d.q[:0], lse[:0], good, offsets=d.offsets[:1] * 0)
        torch.cuda.synchronize()
        assert bool((good == 0).all())
