"""The two forms of the plans (entries in registers, entries in scratch) give
the same answers."""

import random

import pytest

from test_gpu_blocks import Pair, geometry

pytestmark = pytest.mark.gpu


def tiny(blocks):
    return geometry(num_layers=1, planes_per_layer=1, block_size=4, num_kv_heads=1, head_dim=8, elem_bytes=1,
                    num_blocks=blocks)


# rows of tables that fit the form in registers, and more
@pytest.mark.parametrize("max_seqs", [8192, 8193])
def test_entries_after_more_than_there_is(torch, ck, max_seqs):
    """With every block free, an entry that needs none comes after others that
    need more blocks than the pool has."""
    p = Pair(torch, ck, max_seqs, 8, tiny(30))
    with p.pool:
        p.do("grow", list(range(6)), [32, 0, 32, 32, 32, 0])  # 32 of 30 blocks
        p.do("free", list(range(6)))
        p.do("grow", list(range(6)), [32, 32, 32, 32, 0, 1])
        p.do("free", list(range(6)))
        p.do("grow", [7000, 3, 4, 5, 6], [24, 32, 32, 32, 0])  # 30 of 30
        p.do("free", list(range(8)) + [7000])
        # nothing is handed out at all, the pool stays free
        p.do("grow", [0, 0, 9000], [0, 0, 0])


@pytest.mark.parametrize("max_seqs", [8192, 8193])
def test_nothing_is_given_and_nothing_needed(torch, ck, max_seqs):
    p = Pair(torch, ck, max_seqs, 64, tiny(30))
    with p.pool:
        p.do("grow", [1, 2, 3], [124, 0, 0])  # 31 of 30 blocks: all of them stay free
        p.do("grow", [1, 2, 3], [256, 0, 120])
        p.do("grow", [2, 1, 3], [0, 120, 0])  # 30 of 30


@pytest.mark.parametrize("max_seqs", [8192, 8193])
@pytest.mark.parametrize("seed", range(3))
def test_random_requests_near_the_end(torch, ck, max_seqs, seed):
    rng = random.Random(seed)
    p = Pair(torch, ck, max_seqs, 16, tiny(40))
    with p.pool:
        for _ in range(10):
            ids = rng.sample(range(20), 8)
            p.do("grow", ids, [rng.choice([0, 0, 1, 4, 30, 64]) for _ in ids])
            p.do("fork", [rng.randrange(20) for _ in range(4)], rng.sample(range(20), 4))
            p.do("free", rng.sample(range(20), 12))
