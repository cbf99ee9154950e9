"""A few long chats on one claim pool whose caches stay bounded: new tokens'
keys are normed and turned on their way into the blocks, one layer attends in a
sliding window and the others over all that is cached, what each cached token
weighed is added up, and chats that grow past their budget are cut to the tokens
that weighed most.

The model is a stand-in: random projections, attention and an output layer, so
that the calls are made as a serving program makes them.

    python examples/long_chat.py --chats 4 --prompt 200 --steps 150 --budget 128
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_01387_amd import claimkv as ck  # noqa: E402
from paper_2606_01387_amd.sequences import SEQ_OK, Sequences  # noqa: E402
from paper_2606_01387_amd.synth import Geometry  # noqa: E402


class Model:
    """Attention layers with normed and turned heads, with random weights."""

    def __init__(self, geometry, group, vocab, window, sinks, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.kv_heads, self.dim, self.layers = geometry.num_kv_heads, geometry.head_dim, geometry.num_layers
        self.heads, self.window, self.sinks = self.kv_heads * group, window, sinks
        width, out = 128, (self.heads + 2 * self.kv_heads) * self.dim

        def weights(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") * shape[0] ** -0.5).bfloat16()

        self.embed = torch.randn(vocab, width, generator=g, device="cuda").bfloat16()
        self.head = weights(width, vocab)
        self.qkv = [weights(width, out) for _ in range(self.layers)]
        self.back = [weights(self.heads * self.dim, width) for _ in range(self.layers)]
        self.norms = [[1 + weights(self.dim, 1).flatten() for _ in "qk"] for _ in range(self.layers)]
        pairs = self.dim // 2
        self.freqs = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)

    def __call__(self, seqs, tokens, positions, weights, offsets=None):
        """Hidden rows of ``tokens``, the chats' last ones; ``positions`` count
        all tokens that a chat has had, whatever its cache has kept."""
        h = self.embed[tokens]
        q_end, k_end = self.heads * self.dim, (self.heads + self.kv_heads) * self.dim
        lse = torch.empty(len(tokens), self.heads, device="cuda")
        for layer in range(self.layers):
            rows = h @ self.qkv[layer]
            q = rows[:, :q_end].view(-1, self.heads, self.dim)
            k = rows[:, q_end:k_end].view(-1, self.kv_heads, self.dim)
            v = rows[:, k_end:].view(-1, self.kv_heads, self.dim)
            q_norm, k_norm = self.norms[layer]
            q = seqs.write_rotated(layer, q, k, v, self.freqs, positions=positions, q_norm=q_norm,
                                   k_norm=k_norm, offsets=offsets)
            span = dict(window=self.window, sinks=self.sinks) if layer == 0 else dict(window=None)
            out = seqs.attend_window(layer, q, offsets=offsets, lse=lse, **span)
            seqs.weigh(layer, q, lse, weights, offsets=offsets, **span)
            h = h + out.flatten(1) @ self.back[layer]
        return h


def chat(chats=4, prompt=200, steps=150, budget=128, slack=32, blocks=256, block_size=16, group=2, vocab=1000,
         window=64, sinks=4, seed=0):
    geometry = Geometry(3, 2, block_size, 2, 64, 2, blocks)
    kv = torch.zeros(geometry.pool_bytes, dtype=torch.uint8, device="cuda")
    model = Model(geometry, group, vocab, window, sinks, seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    report = {"cuts": 0}
    with ck.Pool(geometry, 11, kv, max_claims=64, max_footprint=4096, event_capacity=256) as pool:
        most = -(-(prompt + budget + slack + 1) // block_size)
        seqs = Sequences(pool, max_seqs=chats, max_blocks=most)
        weights = torch.zeros(chats, most * block_size, device="cuda")
        tokens = torch.randint(0, vocab, (chats * prompt,), generator=g, device="cuda")
        had = torch.full((chats,), prompt, dtype=torch.int32, device="cuda")
        assert (seqs.grow(None, had) == SEQ_OK).all()
        offsets = prompt * torch.arange(chats + 1, dtype=torch.int32, device="cuda")
        places = torch.arange(prompt, dtype=torch.int32, device="cuda").repeat(chats)
        hidden = model(seqs, tokens, places, weights, offsets)[offsets[1:].long() - 1]
        one = torch.ones_like(had)
        said = []
        for step in range(steps):
            # every `slack` tokens, and after the prompts, all chats are cut to their budget
            if step % slack == 0:
                status, _ = seqs.evict(None, weights, budget, sinks=sinks, recent=budget // 4)
                assert (status == SEQ_OK).all()
                report["cuts"] += 1
            token = (hidden @ model.head).argmax(-1)
            said.append(token)
            assert (seqs.grow(None, one) == SEQ_OK).all()
            hidden = model(seqs, token, had, weights)
            had += 1
        report.update(said=torch.stack(said, 1).cpu(), hidden=hidden.float().cpu(), had=had.tolist(),
                      held=seqs.lengths.tolist(), used=int((seqs.refs > 0).sum()), weights=weights.cpu(),
                      most=most)
    return report


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("chats", 4), ("prompt", 200), ("steps", 150), ("budget", 128), ("blocks", 256), ("seed", 0)):
        p.add_argument("--" + name, type=int, default=value)
    r = chat(**vars(p.parse_args()))
    print(f"{len(r['had'])} chats of {r['had'][0]} tokens hold {r['held'][0]} each after {r['cuts']} cuts, "
          f"{r['used']} blocks in all")


if __name__ == "__main__":
    main()
