"""Sequences of a pool on a stream of its own: the object's tensors are made on
the current stream and used on the pool's."""

import pytest

pytestmark = pytest.mark.gpu


def side_pool(torch, ck):
    """A pool on a side stream, with nothing queued anywhere."""
    from paper_2606_01387_amd.synth import Geometry

    g = Geometry(2, 2, 16, 2, 64, 2, 400)
    kv = torch.arange(g.pool_bytes // 8, device="cuda").view(torch.uint8)
    side = torch.cuda.Stream()
    pool = ck.Pool(g, 3, kv, stream=side, max_claims=16, max_footprint=64, event_capacity=64)
    x = torch.ones(8192, 8192, dtype=torch.bfloat16, device="cuda")
    for stream in (torch.cuda.current_stream(), side):  # each has its library's workspace
        with torch.cuda.stream(stream):
            torch.mm(x, x)
    torch.cuda.synchronize()
    return pool, side, x


def keep_busy(torch, x):
    """Tens of milliseconds of products on the current stream."""
    for _ in range(40):
        torch.mm(x, x)


def test_made_behind_work_of_the_current_stream(torch, ck):
    """Tables that are filled late on the current stream, used on the pool's."""
    from paper_2606_01387_amd.sequences import NONE, Sequences

    pool, side, x = side_pool(torch, ck)
    with pool:
        ids = torch.arange(5, dtype=torch.int32, device="cuda")
        tokens = torch.tensor([16, 1, 0, 40, 100], dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        keep_busy(torch, x)
        seqs = Sequences(pool, 40, 12)
        with torch.cuda.stream(side):
            status = seqs.grow(ids, tokens)
        torch.cuda.synchronize()
        assert status.tolist() == [0] * 5
        want = torch.full((40, 12), NONE, dtype=torch.int32)
        at = 0
        for s, n in enumerate((1, 1, 0, 3, 7)):
            want[s, :n] = torch.arange(at, at + n)
            at += n
        assert torch.equal(seqs.tables.cpu(), want)
        assert seqs.lengths.tolist() == [16, 1, 0, 40, 100] + [0] * 35
        assert seqs.refs.tolist() == [1] * at + [0] * (400 - at)


def test_dropped_behind_work_of_the_pools_stream(torch, ck):
    """Memory of an object that is dropped stays its own until the work queued
    on the pool's stream is done."""
    from paper_2606_01387_amd.sequences import Sequences

    pool, side, x = side_pool(torch, ck)
    with pool:
        seqs = Sequences(pool, 1000, 300)
        ids = torch.arange(3, dtype=torch.int32, device="cuda")
        tokens = ids + 20
        held = {t.data_ptr(): t.numel() for t in (seqs._scratch, seqs.tables)}

        def others():
            return [torch.empty(n, dtype=torch.int32, device="cuda") for n in held.values() for _ in range(4)]

        others()  # there is room for them, as taking memory from the device may wait
        with torch.cuda.stream(side):
            seqs.grow(ids, tokens)  # kernels are loaded by their first launch
            torch.cuda.synchronize()
            keep_busy(torch, x)
            seqs.grow(ids, tokens)
        del seqs
        again = others()
        busy = not side.query()
        torch.cuda.synchronize()
        assert busy  # else the memory is free by now and nothing was tested
        assert not held.keys() & {t.data_ptr() for t in again}
