"""Attention in a sliding window behind a few first tokens, against the definition in 64 bits."""

import numpy as np
import pytest

from attend_world import check
from window_world import WindowWorld, check_lse

pytestmark = pytest.mark.gpu


def attend(ck, w, stream=None, want_lse=True, **kw):
    pool, seqs, d = w.to_gpu(ck, stream)
    torch = w.torch
    lse = torch.full((w.rows, w.heads * w.group), 7.0, device="cuda") if want_lse else None
    with pool:
        out = seqs.attend_window(w.layer, d.q, w.window, sinks=w.sinks, offsets=d.offsets, lse=lse,
                                 **w.scales(), **kw)
        torch.cuda.synchronize()
    return out, lse


def both(ck, w, **kw):
    out, lse = attend(ck, w, **kw)
    want, bound, sums, room = w.expected()
    check(out, want, bound)
    check_lse(lse, sums, room)


SEQS = {
    "one": [(1, 0)],
    "short": [(3, 0), (1, 7), (0, 5), (16, 0), (17, 1)],
    "tile-edges": [(32, 0), (33, 31), (64, 0), (63, 1), (65, 64)],
    "long": [(257, 0), (5, 300), (130, 77)],
    "steps": [(1, 700), (1, 65), (1, 64), (1, 63), (1, 0)],
    "few-rows": [(4, 500), (2, 3), (3, 129)],
}


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 1), (64, 4), (100, 70), (130, 0), (1000, 3)])
@pytest.mark.parametrize("seqs", SEQS.values(), ids=SEQS)
def test_windows(torch, ck, seqs, window, sinks, dim, e4m3):
    both(ck, WindowWorld(torch, seqs=seqs, dim=dim, e4m3=e4m3, window=window, sinks=sinks, seed=1))


@pytest.mark.parametrize("block_size", [1, 5, 8, 24, 64, 100])
@pytest.mark.parametrize("dim", [64, 128])
def test_block_sizes(torch, ck, block_size, dim):
    if block_size * dim * 2 * 3 % 16:
        pytest.skip("chunks are multiples of 16 bytes")
    for seqs in ([(40, 0), (1, 170), (90, 130)], [(1, 170), (1, 20), (2, 3)]):
        both(ck, WindowWorld(torch, seqs=seqs, heads=3, block_size=block_size, dim=dim, window=50, sinks=9,
                             seed=2))


@pytest.mark.parametrize("heads,group", [(1, 1), (1, 16), (2, 5), (3, 7), (8, 4), (1, 33), (1, 64)])
def test_head_groups(torch, ck, heads, group):
    for seqs in ([(9, 120), (1, 50), (40, 3)], [(1, 200), (1, 3)]):
        both(ck, WindowWorld(torch, seqs=seqs, heads=heads, group=group, window=33, sinks=2, seed=3))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("window,sinks", [(None, 0), (4000, 5), (2500, 700), (300, 3000)])
@pytest.mark.parametrize("seqs", [[(1, 5000)], [(1, 3000), (1, 1), (1, 800)], [(20, 4000)], [(200, 2900)]],
                         ids=str)
def test_long_axis_is_split(torch, ck, seqs, window, sinks, e4m3):
    both(ck, WindowWorld(torch, seqs=seqs, heads=1, group=4, dim=128, e4m3=e4m3, window=window, sinks=sinks,
                         seed=5))


@pytest.mark.parametrize("seqs", [SEQS["long"], SEQS["steps"]], ids=str)
def test_no_window_is_attention(torch, ck, seqs):
    w = WindowWorld(torch, seqs=seqs, seed=6)
    pool, s, d = w.to_gpu(ck)
    with pool:
        plain = s.attend(w.layer, d.q, offsets=d.offsets)
    check(plain, *w.expected()[:2])
    both(ck, w)
    w.window = 2**32 - 1
    assert torch.equal(attend(ck, w)[0], attend(ck, w, want_lse=False)[0])


def test_more_rows_than_tokens(torch, ck):
    """Rows before position 0 see nothing: 0, and a logarithm of -infinity."""
    for seqs, short in (([(40, 0), (3, 10)], 11), ([(3, 0), (1, 10)], 2)):
        w = WindowWorld(torch, seqs=seqs, window=6, sinks=2, seed=7)
        w.set_lengths([short] + w.length[1:])
        out, _, lse, _ = w.expected()
        assert (out[:seqs[0][0] - short] == 0).all() and np.isneginf(lse[0]).all()
        both(ck, w)


def test_sequences_without_rows_or_length(torch, ck):
    w = WindowWorld(torch, seqs=[(0, 30), (1, 0), (0, 0), (1, 9)], window=4, sinks=1, seed=8)
    w.set_lengths([30, 0, 0, 10])
    both(ck, w)


@pytest.mark.parametrize("seqs", [[(1, 60), (2, 9)], [(90, 30), (5, 0)], [(1, 3000)], [(200, 2500)]], ids=str)
def test_rows_behind_the_last_sequence_are_left(torch, ck, seqs):
    """A padded batch, with parts to join and without."""
    w = WindowWorld(torch, seqs=seqs, heads=1, group=4, window=2000, sinks=2, seed=17)
    want, bound, lse, room = w.expected()
    pool, s, d = w.to_gpu(ck)
    out = torch.full((w.rows + 9, 4, w.dim), 5.0, dtype=torch.bfloat16, device="cuda")
    sums = torch.full((w.rows + 9, 4), 5.0, device="cuda")
    with pool:
        q = torch.cat([d.q, torch.full_like(out[:9], float("nan"))])
        s.attend_window(w.layer, q, w.window, sinks=w.sinks, offsets=d.offsets, lse=sums, out=out)
        weights = torch.zeros(len(seqs), w.tables.shape[1] * w.bs, device="cuda")
        s.weigh(w.layer, q, sums, weights, window=w.window, sinks=w.sinks, offsets=d.offsets)
        torch.cuda.synchronize()
    check(out[:w.rows], want, bound)
    check_lse(sums[:w.rows], lse, room)
    assert bool((out[w.rows:] == 5).all()) and bool((sums[w.rows:] == 5).all())
    got, off = w.weights(sums[:w.rows])
    assert (np.abs(weights.double().cpu().numpy() - got) <= off).all()


@pytest.mark.parametrize("kind", ["none", "out of range"])
@pytest.mark.parametrize("seqs", [[(70, 30), (5, 0)], [(1, 99), (1, 4)]], ids=str)
def test_blocks_behind_the_window_may_be_missing(torch, ck, seqs, kind):
    """Rows that do not see a missing block are exact, those that do are NaN."""
    w = WindowWorld(torch, seqs=seqs, window=20, sinks=3, seed=9)
    for entry in range(1, 4):
        w.tables[0, entry] = -1 if kind == "none" else w.blocks
    out = w.expected()[0]
    assert not np.isnan(out[seqs[0][0] - 1]).any() and (seqs[0][0] == 1) != np.isnan(out).any()
    both(ck, w)
    w.tables[0, 0] = -1  # the first tokens' own
    assert np.isnan(w.expected()[0][0]).all()
    both(ck, w)


@pytest.mark.parametrize("window", [1, 20, 1000, None])
@pytest.mark.parametrize("sinks", [0, 5])
def test_lengths_past_the_table(torch, ck, window, sinks):
    """Rows at positions that the table does not have are NaN, at once."""
    for seqs in ([(1, 40), (1, 7)], [(70, 30), (5, 0)]):
        w = WindowWorld(torch, seqs=seqs, window=window, sinks=sinks, seed=10)
        n = seqs[0][0]
        want, bound, lse, room = w.expected()
        for length in (w.tables.shape[1] * w.bs + n, 2**31 - 1, 2**32 - 1):
            w.lengths[0] = length - 2**32 if length >= 2**31 else length
            want[:n], lse[:n] = np.nan, np.nan
            out, got = attend(ck, w)
            check(out, want, bound)
            check_lse(got, lse, room)


@pytest.mark.parametrize("plane", [0, 1])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("seqs", [[(90, 110)], [(4, 160)], [(1, 199)]], ids=str)
def test_hidden_values_have_no_effect(torch, ck, seqs, e4m3, dim, value, plane):
    """Infinities and NaN in keys and values that no row sees, on both sides
    of the window's beginning and of the first tokens' end."""
    if e4m3 and value == value:
        pytest.skip("e4m3 has no infinity")
    w = WindowWorld(torch, seqs=seqs, dim=dim, e4m3=e4m3, window=40, sinks=5, seed=11)
    want, bound, lse, room = w.expected()
    first = w.length[0] - seqs[0][0] - 40 + 1  # the first row's window
    for pos in [5, 6, first - 1, first - 2, 30]:
        w.kv[2 * w.layer + plane, w.tables[0, pos // w.bs], pos % w.bs, :, :] = value
    out, got = attend(ck, w)
    check(out, want, bound)
    check_lse(got, lse, room)


@pytest.mark.parametrize("seqs", [[(90, 30)], [(4, 60)]], ids=str)
def test_values_seen_by_some_rows(torch, ck, seqs):
    """A NaN value reaches the rows that see it, in its column, and no others."""
    w = WindowWorld(torch, seqs=seqs, window=10, sinks=0, seed=12)
    pos = w.length[0] - 3
    clean, bound, _, _ = w.expected()
    w.kv[2 * w.layer + 1, w.tables[0, pos // w.bs], pos % w.bs, 0, 5] = float("nan")
    want = w.expected()[0]
    assert np.isnan(want).any() and not np.isnan(want[:, w.group:]).any()
    check(attend(ck, w)[0], want, bound)
    gone = w.length[0] - seqs[0][0] - 0  # the first row's own: later rows pass it
    w.kv[2 * w.layer + 1, w.tables[0, gone // w.bs], gone % w.bs, 1, 7] = float("inf")
    want = w.expected()[0]
    got = attend(ck, w)[0].double().cpu().numpy()
    hurt = ~np.isfinite(want)
    assert np.array_equal(~np.isfinite(got), hurt)
    assert (np.abs(got - clean)[~hurt] <= bound[~hurt]).all()


def test_scores_of_minus_infinity(torch, ck):
    """-infinity hides a key; a row with nothing else is NaN, its logarithm -infinity."""
    for seqs in ([(40, 30)], [(1, 69)]):
        w = WindowWorld(torch, seqs=seqs, window=8, sinks=2, heads=1, group=1, seed=13)
        w.q[:, :, 0] = 1.0
        n, L = seqs[0][0], w.length[0]
        for pos in range(L):
            if pos < 2 or L - 12 <= pos < L:
                b = w.tables[0, pos // w.bs]
                w.kv[2 * w.layer, b, pos % w.bs, :, 0] = float("-inf")
        want, bound, lse, room = w.expected()
        assert np.isnan(want[n - 1]).all() and np.isneginf(lse[n - 1]).all()
        out, got = attend(ck, w)
        check(out, want, bound)
        check_lse(got, lse, room)


def test_strides_ids_and_output_over_the_queries(torch, ck):
    w = WindowWorld(torch, seqs=[(5, 60), (1, 90), (30, 0)], window=25, sinks=3, seed=14)
    want, bound, lse, room = w.expected()
    wide = torch.zeros(w.rows, 9, w.dim, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:2 + w.heads * w.group] = w.q.cuda()
    q = wide[:, 2:2 + w.heads * w.group]
    w.tables, w.lengths = w.tables[[2, 0, 1]].contiguous(), w.lengths[[2, 0, 1]].contiguous()
    pool, seqs, d = w.to_gpu(ck)
    got = torch.empty(w.rows, w.heads * w.group, device="cuda")
    with pool:
        ids = torch.tensor([1, 2, 0], dtype=torch.int32, device="cuda")
        out = seqs.attend_window(w.layer, q, w.window, sinks=w.sinks, ids=ids, offsets=d.offsets, lse=got, out=q)
        torch.cuda.synchronize()
    assert out is q and (wide[:, :2] == 0).all() and (wide[:, 2 + w.heads * w.group:] == 0).all()
    check(out, want, bound)
    check_lse(got, lse, room)


@pytest.mark.parametrize("seqs", [[(1, 2000), (1, 900)], [(300, 500)]], ids=str)
def test_streams_and_graphs(torch, ck, seqs):
    w = WindowWorld(torch, seqs=seqs, heads=1, group=4, dim=128, window=700, sinks=4, seed=15)
    want, bound, lse, room = w.expected()
    pool, s, d = w.to_gpu(ck, torch.cuda.Stream())
    out, got = torch.empty_like(d.q), torch.empty(w.rows, 4, device="cuda")
    kw = dict(sinks=w.sinks, offsets=d.offsets, lse=got, out=out)
    with pool:
        first = s.attend_window(w.layer, d.q, w.window, **kw).clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=pool.stream):
            s.attend_window(w.layer, d.q, w.window, **kw)
        for _ in range(3):
            out.zero_()
            got.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, first)
            check(out, want, bound)
            check_lse(got, lse, room)
            s.attend(w.layer, d.q, offsets=d.offsets)  # eager work with the same scratch


def test_refusals(torch, ck):
    w = WindowWorld(torch, seqs=[(4, 9)], window=3, seed=16)
    pool, s, d = w.to_gpu(ck)
    with pool:
        for window, sinks in ((0, 0), (-1, 0), (2**32, 0), (5, -1), (5, 2**32)):
            with pytest.raises(ValueError):
                s.attend_window(w.layer, d.q, window, sinks=sinks, offsets=d.offsets)
        for lse in (torch.empty(4, 3, device="cuda"), torch.empty(4, 4, device="cuda").half(), torch.empty(4, 4),
                    torch.empty(4, 8, device="cuda")[:, :4]):
            with pytest.raises(ValueError):
                s.attend_window(w.layer, d.q, 5, lse=lse, offsets=d.offsets)
        with pytest.raises(ck.ClaimError):
            s.attend_window(9, d.q, 5, offsets=d.offsets)
        with pytest.raises(ck.ClaimError):
            s.attend_window(w.layer, d.q, 5, offsets=d.offsets, scale=0.0)
        assert s.attend_window(w.layer, d.q[:0], 5, offsets=d.offsets[:1] * 0).shape == (0, *d.q.shape[1:])
