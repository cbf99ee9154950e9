"""The sequence calls of the C ABI on the CPU: record layouts, and refusals
that come before any GPU work."""

import ctypes
import os
import subprocess

import pytest

from paper_2606_01387_amd import claimkv as ck
from paper_2606_01387_amd import sequences

STRUCTS = {"claim_seqs": ck.CSeqs, "claim_rows": ck.CRows, "claim_kv_desc": ck.CKvDesc,
           "claim_attend_desc": ck.CAttendDesc}


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(ck.LIBRARY):
        ck.build()
    return ck.lib()


def test_record_layouts_match_header(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "claimkv.h"', "int main(void){"]
    for name, cls in STRUCTS.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    lines.append('printf("work %llu\\n", (unsigned long long)CLAIM_SEQS_WORK(1000, 7));')
    src = tmp_path / "probe.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", f"-I{ck.INCLUDE}", str(src), "-o", str(tmp_path / "probe")], check=True)
    got = dict(ln.split() for ln in subprocess.run([str(tmp_path / "probe")], capture_output=True, text=True,
                                                   check=True).stdout.splitlines())
    for name, cls in STRUCTS.items():
        assert int(got[name]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)
    assert int(got["work"]) == 16 + 3 * 1000 + 4 * 7


def test_packed_records_are_the_structs():
    """The struct formats that fill a description in one step."""
    values = [1, 2, 3, 0, 5, 6, 0.5, 0.25, 7, 8, 16, 10, 24, 32, 4, 9, 11, 2.0, 0, 12, 13]
    buf = ctypes.create_string_buffer(sequences._ATTEND.pack(*values), sequences._ATTEND.size)
    d = ck.CAttendDesc.from_buffer(buf)
    assert (d.kv.layer, d.kv.num_seqs, d.kv.num_rows, d.kv.reserved, d.kv.ids, d.kv.offsets, d.kv.k_scale,
            d.kv.v_scale, d.q.data, d.q.row_stride, d.q.head_stride, d.out.data, d.out.row_stride,
            d.out.head_stride, d.num_heads, d.prefix_blocks, d.prefix, d.scale, d.reserved, d.work,
            d.work_bytes) == tuple(values)


def test_null_arguments_are_refused(L):
    seqs, rows, kv, attend = ck.CSeqs(), ck.CRows(), ck.CKvDesc(), ck.CAttendDesc()
    need = ctypes.c_uint64()
    s, r, k, a = (ctypes.addressof(x) for x in (seqs, rows, kv, attend))
    assert L.claim_seqs_grow(None, s, None, None, 0, None) == ck.EINVAL
    assert L.claim_seqs_fork(None, s, None, None, 0, None) == ck.EINVAL
    assert L.claim_seqs_free(None, s, None, 0) == ck.EINVAL
    assert L.claim_seqs_compact(None, s, None) == ck.EINVAL
    assert L.claim_blocks_copy(None, None, None, 0) == ck.EINVAL
    assert L.claim_kv_write(None, s, k, r, r) == ck.EINVAL
    assert L.claim_attend(None, s, a) == ck.EINVAL
    assert L.claim_attend_work(None, s, a, ctypes.byref(need)) == ck.EINVAL
