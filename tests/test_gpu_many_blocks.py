"""Pools of so many blocks that a planning thread's share is more than it keeps
in registers."""

import random

import pytest

from test_gpu_blocks import Pair, geometry
from test_gpu_held_blocks import holding_pair

pytestmark = pytest.mark.gpu


def tiny(blocks):
    return geometry(num_layers=1, planes_per_layer=1, block_size=2, num_kv_heads=1, head_dim=8, elem_bytes=1,
                    num_blocks=blocks)


@pytest.mark.parametrize("blocks", [32767, 32769, 40003])
@pytest.mark.parametrize("seed", range(2))
def test_lifecycles(torch, ck, blocks, seed):
    rng = random.Random(seed)
    p = Pair(torch, ck, 30, 3000, tiny(blocks))
    with p.pool:
        # ragged sequences that leave holes all over the pool
        for _ in range(3):
            p.do("grow", rng.sample(range(30), 12), [rng.randint(1, 2500) for _ in range(12)])
            p.do("free", rng.sample(range(30), 5))
        p.do("fork", [rng.randrange(30) for _ in range(6)], rng.sample(range(30), 6))
        p.do("free", rng.sample(range(30), 4))
        p.do("compact")
        p.do("grow", list(range(30)), [rng.randint(0, 400) for _ in range(30)])
        p.do("free", rng.sample(range(30), 3))
        p.do("compact")


def test_a_full_pool(torch, ck):
    p = Pair(torch, ck, 14, 3000, tiny(40003))
    with p.pool:
        p.do("grow", list(range(14)), [6000] * 13 + [2006])  # the last block too
        p.do("free", [0, 6])
        p.do("grow", [0, 6], [5999, 6000])
        p.do("grow", [13], [1])  # none is left
        p.do("free", [1, 3])
        p.do("fork", [2], [1])
        p.do("compact")


def test_held_blocks(torch, ck):
    p, hold = holding_pair(torch, ck, 20, 3000, tiny(40003))
    rng = random.Random(5)
    with p.pool:
        p.do("grow", list(range(20)), [rng.randint(1, 3000) for _ in range(20)])
        kept = sorted(rng.sample(range(40003), 3000))
        hold(kept, 1)
        p.do("free", rng.sample(range(20), 10))
        p.do("compact")
        hold(kept, -1)
        p.do("compact")
