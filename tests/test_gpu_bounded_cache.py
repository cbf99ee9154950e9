"""The calls that keep a cache bounded, together: a few sequences are written,
attended to, weighed, cut and grown again, step after step."""

import os
import sys

import numpy as np
import pytest

from attend_world import check
from test_gpu_evict import choose
from window_world import check_lse

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class View:
    """The pool's present state, as tests/window_world.py takes its worlds."""

    def __init__(self, torch, seqs, kv, layer, q, rows, window, sinks, heads, group, dim, bs):
        from window_world import WindowWorld

        self.__class__ = type("View", (WindowWorld,), {})
        self.torch, self.layer, self.window, self.sinks = torch, layer, window, sinks
        self.heads, self.group, self.dim, self.bs, self.e4m3 = heads, group, dim, bs, False
        self.k_scale = self.v_scale = 1.0
        self.prefix_blocks = 0
        self.tables, self.lengths = seqs.tables.cpu(), seqs.lengths.cpu()
        self.length = self.lengths.tolist()
        self.seqs = [(n, L - n) for n, L in zip(rows, self.length)]
        self.kv, self.q, self.rows = kv.cpu(), q.cpu(), sum(rows)
        self.blocks = kv.shape[1]


def test_steps(torch, ck):
    """Attention, logarithms, weights and what is kept follow the definitions
    from the pool's own bytes at every step, and a token's key and value are
    those that were written for it, wherever cuts have moved it."""
    from paper_2606_01387_amd.sequences import Sequences
    from paper_2606_01387_amd.synth import Geometry

    H, G, D, bs, layers, budget = 2, 2, 64, 8, 2, 40
    geometry = Geometry(layers, 2, bs, H, D, 2, 60)
    kv = torch.full((2 * layers, 60, bs, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    freqs = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") / (D // 2))
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    with ck.Pool(geometry, 3, kv.view(torch.uint8), max_claims=16, max_footprint=64, event_capacity=64) as pool:
        seqs = Sequences(pool, max_seqs=3, max_blocks=12)
        weights = torch.zeros(3, 12 * bs, device="cuda")
        had, who = [0, 0, 0], [[], [], []]  # tokens of a sequence, and which of them it holds
        written = [{}, {}, {}]
        for step in range(12):
            rows = [(60, 33, 0), (1, 1, 70), (1, 1, 1), (5, 1, 2)][step if step < 2 else 2 + step % 2]
            assert (seqs.grow(None, ints(rows)) == 0).all()
            offsets = ints([0, *np.cumsum(rows)])
            positions = ints([had[s] + i for s in range(3) for i in range(rows[s])])
            for s in range(3):
                who[s] += range(had[s], had[s] + rows[s])
                had[s] += rows[s]
            before = weights.clone()
            total, room = 0, 0
            for layer, window in ((0, 24), (1, None)):
                T = sum(rows)
                q, k, v = (torch.randn(T, h, D, generator=gen, device="cuda").bfloat16() for h in (H * G, H, H))
                q = seqs.write_rotated(layer, q, k, v, freqs, positions=positions, offsets=offsets)
                lse = torch.empty(T, H * G, device="cuda")
                out = seqs.attend_window(layer, q, window, sinks=3, offsets=offsets, lse=lse)
                seqs.weigh(layer, q, lse, weights, window=window, sinks=3, offsets=offsets)
                w = View(torch, seqs, kv, layer, q, rows, window, 3, H, G, D, bs)
                want, bound, sums, sums_room = w.expected()
                check(out, want, bound)
                check_lse(lse, sums, sums_room)
                got, more = w.weights(lse)
                total, room = total + got, room + more
            off = np.abs((weights - before).double().cpu().numpy() - total)
            assert (off <= room + 2.0**-22 * weights.double().cpu().numpy()).all()
            for s in range(3):  # keys and values are where their tokens are
                L = int(seqs.lengths[s])
                assert len(who[s]) == L
                at = torch.arange(L, device="cuda")
                held = kv[:, seqs.tables[s].long()[at // bs], at % bs].cpu()
                for slot, token in enumerate(who[s]):
                    first = written[s].setdefault(token, held[:, slot])
                    assert torch.equal(first, held[:, slot]), (s, slot, token)
            if step % 3 == 2 or step == 1:
                w = weights.cpu().numpy()
                status, kept = seqs.evict(None, weights, budget, sinks=3, recent=10)
                assert status.tolist() == [0, 0, 0]
                for s in range(3):
                    keep = choose(w[s], len(who[s]), budget, 3, 10)
                    assert kept[s].tolist() == keep + [-1] * (budget - len(keep))
                    assert np.array_equal(weights[s, :len(keep)].cpu().numpy(), w[s][keep])
                    who[s] = [who[s][p] for p in keep]
                assert int((seqs.refs > 0).sum()) == sum(-(-len(x) // bs) for x in who)


def test_example(torch, ck):
    """The example runs, stays within its budget, and gives the same on every run."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import long_chat
    finally:
        sys.path.pop(0)
    a, b = (long_chat.chat(chats=3, prompt=150, steps=70, budget=96, slack=16, blocks=64) for _ in range(2))
    assert a["had"] == [220] * 3 and a["held"] == [96 + 6] * 3 and a["cuts"] == 5
    assert a["used"] == 3 * -(-102 // 16)
    assert torch.equal(a["said"], b["said"]) and torch.equal(a["hidden"], b["hidden"])
    assert torch.equal(a["weights"], b["weights"]) and bool(torch.isfinite(a["hidden"]).all())
    # the budget is kept in weights too: what every row gave, 1 a head and layer, less what was cut
    assert bool((a["weights"][:, 102:] == 0).all()) and float(a["weights"].sum()) <= 3 * 220 * 4 * 3 * 1.001
