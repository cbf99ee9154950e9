"""Sequences made over tables that a program has already."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture
def pool(torch, ck):
    from paper_2606_01387_amd.synth import Geometry

    g = Geometry(1, 2, 16, 2, 64, 2, 20)
    kv = torch.zeros(g.pool_bytes, dtype=torch.uint8, device="cuda")
    with ck.Pool(g, 3, kv, max_claims=16, max_footprint=64, event_capacity=64) as p:
        yield p


def test_counts_follow_the_tables(torch, pool):
    """Without counts, the blocks that tables name are not handed out."""
    from paper_2606_01387_amd.sequences import NONE, SEQ_NO_BLOCKS, SEQ_OK, Sequences

    rows = [[3, 0, 19, NONE], [3, 7, NONE, NONE], [20, -7, 5, NONE], [NONE] * 4]
    tables = torch.tensor(rows, dtype=torch.int32, device="cuda")
    lengths = torch.tensor([40, 17, 48, 0], dtype=torch.int32, device="cuda")
    seqs = Sequences(pool, tables=tables, lengths=lengths)
    want = [0] * 20
    want[0] = want[5] = want[7] = want[19] = 1
    want[3] = 2
    assert seqs.refs.tolist() == want and seqs.refs.dtype == torch.int32
    ids = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    assert seqs.grow(ids, torch.tensor([64, 32], dtype=torch.int32, device="cuda")).tolist() == [SEQ_OK] * 2
    assert seqs.tables[3].tolist() == [1, 2, 4, 6] and seqs.tables[1].tolist() == [3, 7, 8, 9]
    full = torch.arange(20, dtype=torch.int32, device="cuda").view(4, 5)
    seqs = Sequences(pool, tables=full, lengths=torch.full((4,), 79, dtype=torch.int32, device="cuda"))
    assert seqs.refs.tolist() == [1] * 20
    seqs = Sequences(pool, tables=torch.cat([full, full.new_full((1, 5), NONE)]),
                     lengths=torch.tensor([79] * 4 + [0], dtype=torch.int32, device="cuda"))
    one = torch.tensor([4], dtype=torch.int32, device="cuda")
    assert seqs.grow(one, one).tolist() == [SEQ_NO_BLOCKS]


def test_tables_need_lengths(torch, pool):
    from paper_2606_01387_amd.sequences import Sequences

    t = torch.zeros(3, 4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        Sequences(pool, tables=t)
    with pytest.raises(ValueError):
        Sequences(pool, tables=t, refs=torch.ones(20, dtype=torch.int32, device="cuda"))
