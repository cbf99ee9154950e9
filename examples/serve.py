"""A small serving loop on one claim pool: a prompt is written and attended to,
claimed, offloaded and checked; samples are forked from it and decoded behind
the prompt's shared blocks; finished samples are freed and the pool is
compacted.

The model is a stand-in: random projections, attention and an output layer, so
that the calls are made as a serving program makes them.

    python examples/serve.py --prompt 300 --samples 6 --steps 20
"""

from __future__ import annotations

import argparse
import os
import sys
from types import SimpleNamespace

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_01387_amd import claimkv as ck  # noqa: E402
from paper_2606_01387_amd.sequences import SEQ_OK, Sequences  # noqa: E402
from paper_2606_01387_amd.synth import Geometry  # noqa: E402


class Model:
    """Attention layers over a pool's sequences, with random weights."""

    def __init__(self, geometry, group, vocab, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.geometry, self.heads = geometry, geometry.num_kv_heads * group
        self.kv_heads, self.dim = geometry.num_kv_heads, geometry.head_dim
        width, out = 128, (self.heads + 2 * self.kv_heads) * self.dim

        def weights(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") * shape[0] ** -0.5).bfloat16()

        self.embed = torch.randn(vocab, width, generator=g, device="cuda").bfloat16()
        self.head = weights(width, vocab)
        self.qkv = [weights(width, out) for _ in range(geometry.num_layers)]
        self.back = [weights(self.heads * self.dim, width) for _ in range(geometry.num_layers)]

    def __call__(self, seqs, tokens, attend, ids, offsets=None):
        """Hidden rows of ``tokens``, the last tokens of sequences ``ids``."""
        h = self.embed[tokens]
        q_end, k_end = self.heads * self.dim, (self.heads + self.kv_heads) * self.dim
        for layer in range(self.geometry.num_layers):
            rows = h @ self.qkv[layer]
            q = rows[:, :q_end].view(-1, self.heads, self.dim)
            k = rows[:, q_end:k_end].view(-1, self.kv_heads, self.dim)
            v = rows[:, k_end:].view(-1, self.kv_heads, self.dim)
            seqs.write(layer, k, v, ids=ids, offsets=offsets)
            out = attend(layer, q, ids=ids, offsets=offsets)
            h = h + out.flatten(1) @ self.back[layer]
        return h


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def claim(claim_id, blocks, tokens):
    return ck.DeviceBatch(SimpleNamespace(
        claim_ids=[claim_id], block_offsets=[0, len(blocks)], block_ids=blocks,
        token_offsets=[0, len(tokens)], tokens=tokens))


def serve(prompt=300, samples=6, steps=20, blocks=256, block_size=16, group=2, vocab=1000, seed=0):
    geometry = Geometry(2, 2, block_size, 2, 64, 2, blocks)
    kv = torch.zeros(geometry.pool_bytes, dtype=torch.uint8, device="cuda")
    model = Model(geometry, group, vocab, seed)
    rng = np.random.default_rng(seed)
    text = rng.integers(0, vocab, prompt)
    noise = torch.randn(steps, samples, vocab, generator=torch.Generator().manual_seed(seed)).cuda()
    report = {}
    with ck.Pool(geometry, 11, kv, max_claims=64, max_footprint=4096, event_capacity=256) as pool:
        seqs = Sequences(pool, max_seqs=2 * samples + 1, max_blocks=blocks)

        # the prompt, as one packed row of the batch
        first = ints([0])
        assert seqs.grow(first, ints([prompt])).item() == SEQ_OK
        hidden = model(seqs, torch.from_numpy(text).cuda(), seqs.attend, first, ints([0, prompt]))[-1:]

        # it is claimed and goes out; coming back it is checked before it is used again
        held = seqs.tables[0, : -(-prompt // block_size)].cpu().numpy()
        batch = claim(7, held, text)
        pool.offload(batch)
        pool.restore(batch)
        pool.check(batch)
        outcome = pool.read()[0][0]
        if outcome["code"] != ck.MATERIALIZED:
            raise RuntimeError("the prompt's blocks did not come back: nothing is served from them")
        report["hit_blocks"] = int(pool.lookup(batch)["hit_blocks"][0])

        # samples share the prompt's full blocks; each step reads those once for all
        ids = torch.arange(1, samples + 1, dtype=torch.int32, device="cuda")
        assert (seqs.fork(ints([0] * samples), ids) == SEQ_OK).all()
        shared = seqs.tables[0, : prompt // block_size].clone()
        hidden = hidden.expand(samples, -1)
        said = []
        one = torch.ones(samples, dtype=torch.int32, device="cuda")
        for step in range(steps):
            token = (hidden @ model.head + noise[step]).argmax(-1)
            said.append(token)
            assert (seqs.grow(ids, one) == SEQ_OK).all()
            hidden = model(seqs, token, lambda layer, q, **kw: seqs.attend_shared(layer, q, shared, **kw), ids)
        said = torch.stack(said, 1)

        # the same texts as prompts of their own give the same last rows
        again = ids + samples
        length = prompt + steps
        assert (seqs.grow(again, ints([length] * samples)) == SEQ_OK).all()
        whole = torch.cat([torch.from_numpy(text).cuda().expand(samples, -1), said], 1)
        rows = model(seqs, whole.flatten(), seqs.attend, again, ints([length * i for i in range(samples + 1)]))
        last = rows.view(samples, length, -1)[:, -1].float()
        report["difference"] = ((hidden.float() - last).norm() / last.norm()).item()

        # they end; what is left moves to the front of the pool
        report["used"] = int((seqs.refs > 0).sum())
        seqs.free(torch.cat([ids[: samples // 2], again]))
        seqs.free(ints([0]))
        report["moved"] = seqs.compact().item()
        left = int((seqs.refs > 0).sum())
        report["left"] = left
        report["packed"] = bool((seqs.refs[:left] > 0).all())
        # the claim names blocks: the kept samples share the full ones; the last one was
        # freed, and what moved into its place is not the claim's
        report["hit_blocks_after"] = int(pool.lookup(batch)["hit_blocks"][0])
        report["said"] = said.cpu().numpy()
    return report


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("prompt", 300), ("samples", 6), ("steps", 20), ("blocks", 256), ("seed", 0)):
        p.add_argument("--" + name, type=int, default=value)
    r = serve(**vars(p.parse_args()))
    print(f"prompt verified, {r['hit_blocks']} of its blocks hit; "
          f"{r['said'].shape[0]} samples x {r['said'].shape[1]} tokens decoded behind them")
    print(f"decoded rows against the same texts as prompts: relative difference {r['difference']:.2g}")
    print(f"{r['used']} blocks in use at the end; freed, {r['left']} left, {r['moved']} moved to the front")


if __name__ == "__main__":
    main()
