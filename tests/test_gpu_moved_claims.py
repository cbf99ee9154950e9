"""Claims whose blocks' sequences were moved by compaction."""

from types import SimpleNamespace

import numpy as np
import pytest

from test_gpu_blocks import Pair, geometry
from test_gpu_example import example  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_moved_claims_old_blocks(torch, ck):
    """They hit and check like freed blocks until they are handed out and
    written."""
    p = Pair(torch, ck, 4, 8, geometry(num_layers=1))
    with p.pool:
        p.do("grow", [0, 1], [48, 48])
        blocks, tokens = p.model.tables[1, :3].copy(), np.arange(48)
        row = ck.DeviceBatch(SimpleNamespace(claim_ids=[5], block_offsets=[0, 3], block_ids=blocks,
                                             token_offsets=[0, 48], tokens=tokens))

        def judged():
            p.pool.check(row)
            return p.pool.lookup(row)["hit_blocks"][0], p.pool.read()[0][-1]["code"]

        p.pool.offload(row)
        p.pool.restore(row)
        p.do("free", [0])
        p.do("compact")
        assert p.model.tables[1, :3].tolist() == [0, 1, 2]
        assert judged() == (3, ck.MATERIALIZED)
        p.do("grow", [2], [48])  # the same blocks, not written yet
        assert p.model.tables[2, :3].tolist() == blocks.tolist()
        assert judged() == (0, ck.MATERIALIZED)
        k = torch.ones(1, 2, 64, dtype=torch.bfloat16, device="cuda")
        p.seqs.write(0, k, k, ids=p.ints([2]))
        assert judged() == (0, ck.RESTORE_FAILED_FAIL_CLOSED)


@pytest.mark.parametrize("prompt,samples,steps", [(300, 6, 20), (16, 3, 5), (5, 2, 30), (100, 1, 1)])
def test_the_examples_claim_at_the_end(torch, ck, example, prompt, samples, steps):  # noqa: F811
    """The shared full blocks still hit; the last, partly filled one was freed
    and moved into."""
    r = example.serve(prompt=prompt, samples=samples, steps=steps)
    assert r["moved"] > 0
    assert r["hit_blocks_after"] == prompt // 16
