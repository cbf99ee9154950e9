"""Norms, positions and writing of new queries and keys against the formula in 64 bits."""

import numpy as np
import pytest

from attend_world import World

pytestmark = pytest.mark.gpu


class Rotation:
    """Inputs of one call on a world, and what it should give."""

    def __init__(self, torch, w, *, rot, axes=0, norms="qk", neighbours=False, eps=1e-6, seed=0, far=1 << 20,
                 spread=2.0):
        g = torch.Generator().manual_seed(seed)
        T, D = w.rows, w.dim
        self.w, self.rot, self.neighbours, self.eps = w, rot, neighbours, eps
        self.q, self.k, self.v = (
            (spread * torch.randn(T, h, D, generator=g)).to(torch.bfloat16)
            for h in (w.heads * w.group, w.heads, w.heads))
        self.q_norm = (1 + torch.randn(D, generator=g)).to(torch.bfloat16) if "q" in norms else None
        self.k_norm = (1 + torch.randn(D, generator=g)).to(torch.bfloat16) if "k" in norms else None
        half = rot // 2
        self.freqs = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(1, half)) if half else None
        self.positions = self.sections = None
        if axes:
            self.positions = torch.randint(-far, far, (T, axes), generator=g).to(torch.int32)
            cuts = sorted(torch.randint(0, half + 1, (axes - 1,), generator=g).tolist())
            self.sections = tuple(b - a for a, b in zip([0] + cuts, cuts + [half]))

    def kwargs(self, dev=lambda x: x.cuda() if x is not None else None):
        return dict(freqs=dev(self.freqs), positions=dev(self.positions), sections=self.sections,
                    q_norm=dev(self.q_norm), k_norm=dev(self.k_norm), eps=self.eps,
                    neighbours=self.neighbours, **self.w.scales())

    def places(self):
        """Each row's sequence and position."""
        got = []
        for s, (n, _) in enumerate(self.w.seqs):
            got += [(s, self.w.length[s] - n + i) for i in range(n)]
        return got

    def turned(self, x, weight):
        """(values, magnitudes that went into them) in 64 bits."""
        x = x.double().numpy()
        if weight is not None:
            with np.errstate(divide="ignore", invalid="ignore"):
                x = x / np.sqrt((x**2).mean(-1, keepdims=True) + self.eps) * weight.double().numpy()
        y, big = x.copy(), np.abs(x)
        half = self.rot // 2
        axis = np.repeat(np.arange(len(self.sections or [0])), self.sections or [half]) if half else []
        own = np.array([p for _, p in self.places()])
        for i in range(half):
            pos = own if self.positions is None else self.positions[:, axis[i]].numpy()
            t = (pos.astype(np.float64) * float(self.freqs[i]))[:, None]
            a, b = (2 * i, 2 * i + 1) if self.neighbours else (i, i + half)
            y[..., a] = x[..., a] * np.cos(t) - x[..., b] * np.sin(t)
            y[..., b] = x[..., b] * np.cos(t) + x[..., a] * np.sin(t)
            big[..., a] = big[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
        return y, big

    def bound(self, y, big):
        """One rounding to bf16 (2^-8), and 32-bit steps before it: the mean
        of squares is off by at most (dim + 2) 2^-24 of itself, its root by
        half of that, the root and its inverse, two products, a product and a
        sum by 6 more, a sine or cosine of an angle that is off by 2^-24 turns
        by 8: taken together (dim / 2 + 15) 2^-24 of the pair's magnitudes."""
        return 2.0**-8 * np.abs(y) + 1.01 * (self.w.dim / 2 + 15) * 2.0**-24 * big + 1e-30

    def check(self, out, kv, rows=None):
        w, torch = self.w, self.w.torch
        y, big = self.turned(self.q, self.q_norm)
        off = np.abs(out.double().cpu().numpy() - y)
        assert (off <= self.bound(y, big)).all(), (off / self.bound(y, big)).max()
        k, big = self.turned(self.k, self.k_norm)
        v = self.v.double().numpy()
        kv = kv.cpu().view(w.kv.dtype)
        written = torch.zeros(kv.shape[:3], dtype=torch.bool)
        for row, (s, pos) in enumerate(self.places()):
            if pos < 0 or pos // w.bs >= w.tables.shape[1]:
                continue
            b, t = int(w.tables[s, pos // w.bs]), pos % w.bs
            if not 0 <= b < w.blocks:
                continue
            got = [x.double().numpy() for x in kv[2 * w.layer:2 * w.layer + 2, b, t]]
            written[2 * w.layer:2 * w.layer + 2, b, t] = True
            if w.e4m3:
                # one rounding to e4m3 (2^-4, or half of the least step, 2^-10) of x / scale
                for x, want, more, scale in ((got[0], k[row], self.bound(k[row], big[row]), w.k_scale),
                                             (got[1], v[row], 0, w.v_scale)):
                    want = np.clip(want / scale, -448, 448)
                    room = np.maximum(2.0**-4 * np.abs(want), 2.0**-10) + more / scale * 1.07
                    assert (np.abs(x - want) <= room).all(), row
            else:
                assert (np.abs(got[0] - k[row]) <= self.bound(k[row], big[row])).all(), row
                assert (got[1] == v[row]).all(), row
        # nothing else has changed
        same = kv.view(torch.uint8 if w.e4m3 else torch.int16) == w.kv.view(torch.uint8 if w.e4m3 else torch.int16)
        assert bool(same[~written].all())


def run(ck, w, r, stream=None, out=None, **kw):
    pool, seqs, d = w.to_gpu(ck, stream)
    with pool:
        got = seqs.write_rotated(w.layer, r.q.cuda(), r.k.cuda(), r.v.cuda(), offsets=d.offsets, out=out,
                                 **r.kwargs(), **kw)
        w.torch.cuda.synchronize()
        return got, d.kv


SEQS = {"one": [(1, 0)], "step": [(1, 3), (1, 0), (1, 100), (1, 15), (1, 16)],
        "ragged": [(3, 0), (1, 7), (0, 5), (16, 1), (17, 40)], "long": [(300, 20)]}


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim,rot", [(64, 64), (64, 16), (128, 128), (128, 64), (128, 0), (64, 48)])
@pytest.mark.parametrize("seqs", SEQS.values(), ids=SEQS)
def test_rotated(torch, ck, seqs, dim, rot, e4m3):
    w = World(torch, seqs=seqs, dim=dim, e4m3=e4m3, seed=1)
    r = Rotation(torch, w, rot=rot, seed=2)
    r.check(*run(ck, w, r))


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("norms", ["", "q", "k", "qk"])
def test_positions_and_norms(torch, ck, axes, norms, neighbours):
    w = World(torch, seqs=SEQS["ragged"], dim=128, seed=3)
    r = Rotation(torch, w, rot=96, axes=axes, norms=norms, neighbours=neighbours, seed=4)
    r.check(*run(ck, w, r))


@pytest.mark.parametrize("heads,group", [(1, 1), (1, 16), (3, 5), (8, 8), (2, 33)])
def test_heads(torch, ck, heads, group):
    w = World(torch, seqs=SEQS["step"], heads=heads, group=group, seed=5)
    r = Rotation(torch, w, rot=64, axes=1, seed=6)
    r.check(*run(ck, w, r))


def test_far_positions(torch, ck):
    """The largest positions that 32 bits hold, both signs."""
    w = World(torch, seqs=[(40, 0)], dim=128, seed=7)
    r = Rotation(torch, w, rot=128, axes=1, seed=8)
    ends = torch.tensor([2**31 - 1, -2**31, 2**31 - 2, 2**30 + 1, 16777217, -16777217, 0, 1])
    r.positions[:8, 0] = ends.to(torch.int32)
    r.check(*run(ck, w, r))


def test_rows_without_a_block(torch, ck):
    """Missing blocks, lengths past the table, rows before position 0: not
    written, queries given all the same."""
    w = World(torch, seqs=[(20, 30), (9, 0), (4, 60)], seed=9)
    w.tables[0, 2] = -1
    w.tables[2, 3] = w.blocks
    w.length[1] = 5
    w.lengths = torch.tensor(w.length, dtype=torch.int32)
    r = Rotation(torch, w, rot=64, seed=10)
    r.check(*run(ck, w, r))


def test_rows_behind_the_last_sequence_are_left(torch, ck):
    w = World(torch, seqs=[(3, 0), (5, 2)], seed=11)
    r = Rotation(torch, w, rot=64, seed=12)
    pad = [torch.cat([x, x[:4] * 0 + 7]).cuda() for x in (r.q, r.k, r.v)]
    out = torch.full_like(pad[0], 3)
    pool, seqs, d = w.to_gpu(ck)
    with pool:
        seqs.write_rotated(w.layer, *pad, offsets=d.offsets, out=out, **r.kwargs())
        torch.cuda.synchronize()
    assert bool((out[8:] == 3).all())
    r.check(out[:8], d.kv)


def test_in_place_and_from_a_projection(torch, ck):
    """Slices of one fused projection, the queries turned where they lie."""
    w = World(torch, seqs=SEQS["ragged"], heads=2, group=3, dim=128, seed=13)
    r = Rotation(torch, w, rot=128, axes=3, seed=14)
    T = w.rows
    flat = torch.cat([x.flatten(1) for x in (r.q, r.k, r.v)], 1).cuda()
    q, k, v = flat[:, :768].view(T, 6, 128), flat[:, 768:1024].view(T, 2, 128), flat[:, 1024:].view(T, 2, 128)
    pool, seqs, d = w.to_gpu(ck)
    kw = r.kwargs()
    kw["positions"] = kw["positions"].T.contiguous().T  # [axes, rows] in memory
    with pool:
        got = seqs.write_rotated(w.layer, q, k, v, offsets=d.offsets, out=q, **kw)
        torch.cuda.synchronize()
    assert got is q and torch.equal(flat[:, 768:].cpu(), torch.cat([r.k.flatten(1), r.v.flatten(1)], 1))
    r.check(q, d.kv)


def test_norm_of_zeros_and_nan(torch, ck):
    """A head of zeros stays zero with eps, is NaN without; NaN stays in its head."""
    w = World(torch, seqs=[(4, 0)], seed=15)
    for eps, want in ((1e-6, 0.0), (0.0, float("nan"))):
        r = Rotation(torch, w, rot=64, eps=eps, seed=16)
        r.q[1, 2] = 0
        r.k[2, 1, 5] = float("nan")
        out, kv = run(ck, w, r)
        zero = out[1, 2].float().cpu()
        assert bool(torch.isnan(zero).all()) if want != want else bool((zero == 0).all())
        clean = out.float().cpu()
        clean[1, 2] = 0
        assert bool(torch.isfinite(clean).all())
        b = int(w.tables[0, 0])
        key = kv.cpu()[2 * w.layer, b, 2].float()
        assert bool(torch.isnan(key[1]).all()) and bool(torch.isfinite(key[0]).all())


def test_unturned_elements_ignore_the_others(torch, ck):
    """Without norms, an infinity among the turned elements stays there."""
    w = World(torch, seqs=[(2, 0)], dim=64, seed=17)
    for neighbours in (False, True):
        r = Rotation(torch, w, rot=32, norms="", neighbours=neighbours, seed=18)
        r.q[0, 1, 3] = float("inf")
        out, _ = run(ck, w, r)
        mate = 2 if neighbours else 19
        rest = out[0, 1].float().cpu()
        rest[[3, mate]] = 0
        assert bool(torch.isfinite(rest).all()) and not bool(torch.isfinite(out[0, 1, 3]))


def test_another_stream_and_a_graph(torch, ck):
    """The pool's stream apart from the current one, then replays of a capture."""
    w = World(torch, seqs=SEQS["step"], seed=19)
    r = Rotation(torch, w, rot=64, axes=2, seed=20)
    out, kv = run(ck, w, r, stream=torch.cuda.Stream())
    r.check(out, kv)

    pool, seqs, d = w.to_gpu(ck, torch.cuda.Stream())
    q, k, v = r.q.cuda(), r.k.cuda(), r.v.cuda()
    kw, got = r.kwargs(), torch.empty_like(q)
    with pool, torch.cuda.stream(pool.stream):
        pool.stream.wait_stream(torch.cuda.default_stream())
        seqs.write_rotated(w.layer, q, k, v, offsets=d.offsets, out=got, **kw)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=pool.stream):
            seqs.write_rotated(w.layer, q, k, v, offsets=d.offsets, out=got, **kw)
        for step in range(3):
            r.q, r.k = r.q.roll(1, 0), r.k.roll(1, 0)
            q.copy_(r.q)
            k.copy_(r.k)
            got.zero_()
            graph.replay()
            torch.cuda.synchronize()
            r.check(got, d.kv)


def test_refusals(torch, ck):
    w = World(torch, seqs=[(4, 0)], dim=64, seed=21)
    r = Rotation(torch, w, rot=32, axes=2, seed=22)
    pool, seqs, d = w.to_gpu(ck)
    q, k, v = r.q.cuda(), r.k.cuda(), r.v.cuda()
    good = r.kwargs()
    with pool:
        def refused(error, *rows, **change):
            before = d.kv.clone()
            with pytest.raises(error):
                seqs.write_rotated(change.pop("layer", w.layer), *(rows or (q, k, v)), offsets=d.offsets,
                                   **{**good, **change})
            torch.cuda.synchronize()
            assert torch.equal(before.view(torch.int16), d.kv.view(torch.int16))

        refused(ck.ClaimError, layer=9)
        refused(ck.ClaimError, eps=-1.0)
        refused(ck.ClaimError, eps=float("nan"))
        refused(ck.ClaimError, freqs=good["freqs"][:12].contiguous(), sections=(6, 6))  # 24 dimensions
        refused(ck.ClaimError, freqs=torch.ones(48, dtype=torch.float64, device="cuda"), sections=(24, 24))
        refused(ck.ClaimError, k_scale=2.0)  # a bf16 pool
        refused(ValueError, freqs=good["freqs"].float())
        refused(ValueError, sections=(8, 9))
        refused(ValueError, sections=(16,))
        refused(ValueError, sections=(-1, 17))
        refused(ValueError, positions=good["positions"].long())
        refused(ValueError, positions=good["positions"][:3])
        refused(ValueError, positions=good["positions"].cpu())
        refused(ValueError, q_norm=torch.ones(32, dtype=torch.bfloat16, device="cuda"))
        refused(ValueError, k_norm=torch.ones(64, device="cuda"))
        refused(ValueError, q, k[:3], v)
        refused(ValueError, q.float(), k, v)
        refused(ValueError, q, k, v, out=q[:, :2])
        got = seqs.write_rotated(w.layer, q[:0], k[:0], v[:0], offsets=d.offsets[:1] * 0,
                                 **{**good, "positions": good["positions"][:0]})
        assert got.shape == (0, *q.shape[1:])
