"""Norms of heads whose squares leave 32 bits at the lower end."""

import pytest

from attend_world import World
from test_gpu_rotated import SEQS, Rotation, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-36, 1e-20])
@pytest.mark.parametrize("power", [-20, -45, -62, -70, -100, -125])
@pytest.mark.parametrize("dim,rot,norms,e4m3", [(64, 64, "qk", False), (128, 64, "q", False), (128, 128, "k", True)])
def test_small_heads_are_normed(torch, ck, dim, rot, norms, e4m3, power, eps):
    """Heads of about 2^power beside ordinary ones: x w / sqrt(mean(x^2) + eps)
    holds for them too, with an eps that is small beside them or none.  The
    bounds are those of ordinary heads, as a power of two rounds nothing."""
    w = World(torch, seqs=SEQS["ragged"], dim=dim, e4m3=e4m3, seed=31)
    r = Rotation(torch, w, rot=rot, axes=1, norms=norms, neighbours=e4m3, seed=32,
                 eps=float(torch.tensor(eps, dtype=torch.float32)))
    for x in (r.q, r.k):
        x[::2] *= 2.0**power
        x[1, 0] *= 2.0**(power // 2)
    r.check(*run(ck, w, r))
