"""The calls that keep a cache bounded, on the CPU: record layouts, and
refusals that come before any GPU work."""

import ctypes
import os
import subprocess

import pytest

from paper_2606_01387_amd import claimkv as ck
from paper_2606_01387_amd import sequences

STRUCTS = {"claim_rotate_desc": ck.CRotateDesc, "claim_window_desc": ck.CWindowDesc,
           "claim_weigh_desc": ck.CWeighDesc, "claim_evict_desc": ck.CEvictDesc}
PACKED = {ck.CRotateDesc: sequences._ROTATE, ck.CWindowDesc: sequences._WINDOW,
          ck.CWeighDesc: sequences._WEIGH, ck.CEvictDesc: sequences._EVICT}


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
    src = tmp_path / "probe.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", f"-I{ck.INCLUDE}", str(src), "-o", str(tmp_path / "probe")], check=True)
    got = dict(ln.split() for ln in subprocess.run([str(tmp_path / "probe")], capture_output=True, text=True,
                                                   check=True).stdout.splitlines())
    for name, cls in STRUCTS.items():
        assert int(got[name]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)


def _leaves(cls, base=0):
    """Offsets and types of a record's plain fields, in order."""
    for f, t in cls._fields_:
        at = base + getattr(cls, f).offset
        if issubclass(t, ctypes.Structure):
            yield from _leaves(t, at)
        elif issubclass(t, ctypes.Array):
            for i in range(t._length_):
                yield at + i * ctypes.sizeof(t._type_), t._type_
        else:
            yield at, t


@pytest.mark.parametrize("cls", PACKED, ids=lambda c: c.__name__)
def test_packed_records_are_the_structs(cls):
    """The struct formats that fill a description in one step."""
    leaves = list(_leaves(cls))
    values = [i + 1 for i in range(len(leaves))]
    buf = PACKED[cls].pack(*values)
    assert len(buf) == ctypes.sizeof(cls)
    for (at, t), want in zip(leaves, values):
        assert t.from_buffer_copy(buf, at).value == want, at


def test_null_arguments_are_refused(L):
    s, need = ctypes.addressof(ck.CSeqs()), ctypes.c_uint64()
    w = ctypes.addressof(ck.CWindowDesc())
    assert L.claim_attend_window(None, s, w) == ck.EINVAL
    assert L.claim_attend_window_work(None, s, w, ctypes.byref(need)) == ck.EINVAL
    assert L.claim_kv_write_rotated(None, s, ctypes.addressof(ck.CRotateDesc())) == ck.EINVAL
    d = ctypes.addressof(ck.CWeighDesc())
    assert L.claim_weigh(None, s, d) == ck.EINVAL
    assert L.claim_weigh_work(None, s, d, ctypes.byref(need)) == ck.EINVAL
    d = ctypes.addressof(ck.CEvictDesc())
    assert L.claim_seqs_evict(None, s, d) == ck.EINVAL
    assert L.claim_seqs_evict_work(None, s, d, ctypes.byref(need)) == ck.EINVAL
