"""What the sequence calls refuse, and that refused calls change nothing."""

import ctypes

import pytest

pytestmark = pytest.mark.gpu


def world(torch, ck, **kw):
    from paper_2606_01387_amd.sequences import Sequences
    from paper_2606_01387_amd.synth import Geometry

    d = dict(num_layers=2, planes_per_layer=2, block_size=16, num_kv_heads=2, head_dim=64, elem_bytes=2,
             num_blocks=20)
    d.update(kw)
    g = Geometry(**d)
    kv = torch.zeros(g.pool_bytes, dtype=torch.uint8, device="cuda")
    pool = ck.Pool(g, 3, kv, max_claims=16, max_footprint=64, event_capacity=64)
    return pool, Sequences(pool, 4, 8), kv


def call(ck, seqs, what, change=None, seqs_change=None):
    """claim_attend or claim_kv_write with one field changed."""
    torch = ck._torch()
    x = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    rows = ck.CRows(data=x.data_ptr(), row_stride=256, head_stride=64)
    kv = ck.CKvDesc(layer=0, num_seqs=2, num_rows=2, k_scale=1.0, v_scale=1.0)
    d = ck.CAttendDesc(kv=kv, q=rows, out=rows, num_heads=4, scale=0.125)
    s = ck.CSeqs.from_buffer_copy(seqs._seqs)
    for struct, fields in ((d, change or {}), (s, seqs_change or {})):
        for path, value in fields.items():
            at = struct
            *where, last = path.split(".")
            for name in where:
                at = getattr(at, name)
            setattr(at, last, value)
    h = seqs.pool._h
    if what == "attend":
        return ck.lib().claim_attend(h, ctypes.addressof(s), ctypes.addressof(d))
    return ck.lib().claim_kv_write(h, ctypes.addressof(s), ctypes.addressof(d.kv), ctypes.addressof(d.q),
                                   ctypes.addressof(d.out))


SHARED = [{"kv.layer": 2}, {"kv.reserved": 1}, {"kv.num_seqs": 5}, {"kv.num_rows": 3}, {"kv.k_scale": 2.0},
          {"kv.v_scale": 0.0}, {"q.data": 0}, {"q.data": 8}, {"q.row_stride": 4}, {"out.head_stride": 68},
          {"out.data": 0}]


@pytest.mark.parametrize("what", ["attend", "write"])
@pytest.mark.parametrize("change", SHARED, ids=str)
def test_bad_rows_and_layers(torch, ck, what, change):
    pool, seqs, _ = world(torch, ck)
    with pool:
        assert call(ck, seqs, what) == ck.OK
        assert call(ck, seqs, what, change) == ck.EINVAL


@pytest.mark.parametrize("change", [{"num_heads": 0}, {"num_heads": 3}, {"num_heads": 130}, {"scale": 0.0},
                                    {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")},
                                    {"reserved": 1}, {"prefix_blocks": 1}, {"prefix_blocks": 2**31}], ids=str)
def test_bad_attention(torch, ck, change):
    pool, seqs, _ = world(torch, ck)
    with pool:
        assert call(ck, seqs, "attend", change) == ck.EINVAL


@pytest.mark.parametrize("change", [{"max_seqs": 0}, {"max_blocks": 0}, {"tables": None}, {"lengths": None},
                                    {"refs": None}, {"max_seqs": 2**31}], ids=str)
def test_bad_sequences(torch, ck, change):
    pool, seqs, _ = world(torch, ck)
    with pool:
        assert call(ck, seqs, "attend", seqs_change=change) == ck.EINVAL
        assert call(ck, seqs, "write", seqs_change=change) == ck.EINVAL


@pytest.mark.parametrize("scale", [0.0, -1.0, 1e-31, 1e31, float("inf"), float("nan")])
def test_bad_e4m3_scales(torch, ck, scale):
    pool, seqs, _ = world(torch, ck, elem_bytes=1)
    with pool:
        assert call(ck, seqs, "attend", {"kv.k_scale": 0.5, "kv.v_scale": 2.0}) == ck.OK
        for name in ("kv.k_scale", "kv.v_scale"):
            assert call(ck, seqs, "attend", {name: scale}) == ck.EINVAL
            assert call(ck, seqs, "write", {name: scale}) == ck.EINVAL


@pytest.mark.parametrize("kw", [dict(planes_per_layer=1), dict(head_dim=80), dict(head_dim=256),
                                dict(elem_bytes=4)], ids=str)
def test_pools_without_attention(torch, ck, kw):
    """Latents, other head sizes and other types are refused; their blocks
    can be moved all the same."""
    pool, seqs, _ = world(torch, ck, **kw)
    with pool:
        assert call(ck, seqs, "attend") == ck.EINVAL
        ids = torch.arange(2, dtype=torch.int32, device="cuda")
        assert seqs.grow(ids, ids + 17).tolist() == [0, 0]
        seqs.free(ids)
        assert seqs.compact().item() == 0


def test_too_little_scratch(torch, ck):
    """A call whose parts do not fit is refused, and told how many bytes do."""
    pool, seqs, _ = world(torch, ck, num_blocks=400)
    from paper_2606_01387_amd.sequences import Sequences

    with pool:
        seqs = Sequences(pool, 2, 400)
        d = ck.CAttendDesc(kv=ck.CKvDesc(num_seqs=2, num_rows=2, k_scale=1.0, v_scale=1.0), num_heads=4, scale=0.1)
        x = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
        d.q = d.out = ck.CRows(data=x.data_ptr(), row_stride=256, head_stride=64)
        need = ctypes.c_uint64()
        s, a = ctypes.addressof(seqs._seqs), ctypes.addressof(d)
        assert ck.lib().claim_attend_work(pool._h, s, a, ctypes.byref(need)) == ck.OK and need.value > 0
        assert ck.lib().claim_attend(pool._h, s, a) == ck.ENOSPC
        work = torch.empty(need.value + 256, dtype=torch.uint8, device="cuda")
        d.work, d.work_bytes = work.data_ptr(), need.value - 1
        assert ck.lib().claim_attend(pool._h, s, a) == ck.ENOSPC
        d.work, d.work_bytes = work.data_ptr() + 8, need.value
        assert ck.lib().claim_attend(pool._h, s, a) == ck.EINVAL
        d.work = work.data_ptr()
        assert ck.lib().claim_attend(pool._h, s, a) == ck.OK


def test_plans_need_scratch_and_entries(torch, ck):
    pool, seqs, _ = world(torch, ck)
    L = ck.lib()
    with pool:
        s = ck.CSeqs.from_buffer_copy(seqs._seqs)
        at, ids = ctypes.addressof(s), torch.zeros(9, dtype=torch.int32, device="cuda")
        for n, work, want in ((5, s.work, ck.EINVAL), (1, None, ck.EINVAL), (0, s.work, ck.OK)):
            s.work = work
            assert L.claim_seqs_grow(pool._h, at, None, ids.data_ptr(), n, None) == want
            assert L.claim_seqs_fork(pool._h, at, ids.data_ptr(), ids.data_ptr(), n, None) == want
        assert L.claim_seqs_free(pool._h, at, None, 5) == ck.EINVAL
        assert L.claim_seqs_grow(pool._h, at, None, None, 1, None) == ck.EINVAL
        assert L.claim_seqs_fork(pool._h, at, None, ids.data_ptr(), 1, None) == ck.EINVAL
        assert L.claim_blocks_copy(pool._h, None, ids.data_ptr(), 1) == ck.EINVAL
        assert L.claim_blocks_copy(pool._h, ids.data_ptr(), ids.data_ptr(), 21) == ck.EINVAL


def test_binding_refuses_other_tensors(torch, ck):
    pool, seqs, _ = world(torch, ck)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pool:
        for bad in (q.float(), q.cpu(), q[0], q[..., :32], q.transpose(0, 2), q.repeat(1, 1, 2)[..., ::2]):
            with pytest.raises(ValueError):
                seqs.attend(0, bad)
        with pytest.raises(ck.ClaimError):
            seqs.attend(0, q[:, :3])  # heads that are no multiple of the pool's
        for kw in (dict(ids=ids[:1]), dict(ids=ids.long()), dict(offsets=ids.cpu()), dict(out=q[:1])):
            with pytest.raises(ValueError):
                seqs.attend(0, q, **kw)
        with pytest.raises(ValueError):
            seqs.attend(-1, q)
        with pytest.raises(ck.ClaimError):
            seqs.attend(2, q)
        with pytest.raises(ValueError):
            seqs.write(0, k, k[:1])
        with pytest.raises(ValueError):
            seqs.write(0, k, q)
        with pytest.raises(ValueError):
            seqs.grow(ids, ids[:1])
        with pytest.raises(ValueError):
            pool.copy_blocks(ids, ids[:1])
        with pytest.raises(ValueError):
            pool.copy_blocks(ids.long(), ids)


def test_sequences_want_matching_state(torch, ck):
    from paper_2606_01387_amd.sequences import Sequences

    pool, _, _ = world(torch, ck)
    t = torch.zeros(3, 4, dtype=torch.int32, device="cuda")
    with pool:
        for kw in (dict(), dict(max_seqs=3), dict(tables=t[0]), dict(tables=t.cpu()), dict(tables=t.long()),
                   dict(tables=t, lengths=t[0]), dict(tables=t, refs=t[0]), dict(tables=t[:, :2])):
            with pytest.raises(ValueError):
                Sequences(pool, **kw)


def test_nothing_to_do(torch, ck):
    """No rows, no sequences: accepted, and nothing happens."""
    pool, seqs, kv = world(torch, ck)
    q = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    with pool:
        assert seqs.attend(0, q).shape == (0, 4, 64)
        seqs.write(0, q[:, :2], q[:, :2])
        off = torch.zeros(4, dtype=torch.int32, device="cuda")
        assert seqs.attend(0, q, offsets=off).shape == (0, 4, 64)
        assert not kv.any()


@pytest.mark.parametrize("change, seqs_change", [
    ({"kv.num_rows": 2**25 + 1, "kv.offsets": 256}, {}),  # refused before anything is read
    ({"kv.num_rows": 2**31, "kv.offsets": 256}, {}),
    ({}, {"max_seqs": 2**22 + 1})], ids=str)
def test_counts_past_the_limits(torch, ck, change, seqs_change):
    pool, seqs, _ = world(torch, ck)
    with pool:
        assert call(ck, seqs, "attend", change, seqs_change) == ck.EINVAL
        assert call(ck, seqs, "write", change, seqs_change) == ck.EINVAL


@pytest.mark.parametrize("change, seqs_change", [
    ({"kv.num_rows": 2**24, "kv.offsets": 256}, {}),  # of 4 heads: 2^26 rows and heads
    ({"kv.num_seqs": 2**21 + 1, "kv.offsets": 256}, {"max_seqs": 2**22})], ids=str)  # of 2 KV heads
def test_attention_past_the_limits(torch, ck, change, seqs_change):
    pool, seqs, _ = world(torch, ck)
    with pool:
        assert call(ck, seqs, "attend", change, seqs_change) == ck.EINVAL
