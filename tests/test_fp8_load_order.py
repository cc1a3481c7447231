"""Audit of the counted waits of the 8-bit products (gemm_fp8.hip), on the code the compiler
emits (CPU only: hipcc compiles the source to gfx950 assembly).

The kernels wait for all but a number of their youngest loads, a number that holds only
while each slab's loads stay between the slab's own marks (empty asm statements, which
the compiler's memory accesses do not cross).  This test counts the loads between marks."""
import collections
import os
import re
import subprocess
import tempfile

import pytest

from paper_2110_15456_amd import build as B
from tests.test_wave_lds_order import unordered

MARK = re.compile(r"^;;#ASMSTART")
TO_LDS = re.compile(r"^buffer_load_dword(x4)?\b.*\blds\b")
TO_REG = re.compile(r"^buffer_load_")


def segments(asm):
    """{kernel: [(16-byte loads to LDS, 4-byte ones, loads to registers) between marks]}"""
    found, name, now = {}, None, None
    for raw in asm.splitlines():
        s = raw.strip()
        m = re.match(r"^(_Z\w+):", raw)
        if m:
            name, now = m.group(1), [0, 0, 0]
            found[name] = [now]
        elif name is None:
            continue
        elif MARK.match(s):
            now = [0, 0, 0]
            found[name].append(now)
        elif TO_LDS.match(s):
            now[0 if "dwordx4" in s else 1] += 1
        elif TO_REG.match(s):
            now[2] += 1
        elif s.startswith("s_endpgm"):
            name = None
    return found


def assembly(source):
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "k.s")
        cmd = [os.path.join(B.ROCM, "bin", "hipcc"), *B.HIPFLAGS, "--cuda-device-only", "-S",
               os.path.join(B.CSRC, source), "-o", out]
        subprocess.run(cmd, check=True, capture_output=True)
        with open(out) as f:
            return f.read()


@pytest.fixture(scope="module")
def products():
    return assembly("gemm_fp8.hip")


@pytest.fixture(scope="module")
def kernels(products):
    return segments(products)


def test_few_rows(kernels):
    seen = 0
    for name, parts in kernels.items():
        m = re.search(r"k_gemm_fp8_fewILi(\d+)ELi(\d+)ELi\d+E", name)
        if not m:
            continue
        rm, rn = int(m.group(1)), int(m.group(2))
        loads, scales = 2 * (rm + rn), rm + rn
        seen += 1
        # in front of the loop four slabs and a run's scales; in it a slab's loads behind
        # each slab's second mark, the first one's with the next run's scales
        first, rest = parts[0], collections.Counter(tuple(p) for p in parts[1:])
        assert tuple(first) == (4 * loads, 0, scales), (name, first)
        assert rest[(loads, 0, scales)] == 1 and rest[(loads, 0, 0)] == 3, (name, rest)
        assert set(rest) == {(loads, 0, scales), (loads, 0, 0), (0, 0, 0)}, (name, rest)
    assert seen >= 24  # three tiles, four pairs of formats, two types


def test_tiles_of_64(kernels):
    seen = 0
    for name, parts in kernels.items():
        if not re.search(r"k_gemm_fp8ILi64ELi64E", name):
            continue
        seen += 1
        loads = 4  # of a wave: 64 + 64 rows of 128 bytes, 1 KB each, over four waves
        first, rest = parts[0], collections.Counter(tuple(p) for p in parts[1:])
        assert tuple(first) == (4 * loads, 1, 0), (name, first)
        assert rest[(loads, 1, 0)] == 1 and rest[(loads, 0, 0)] == 3, (name, rest)
        assert set(rest) == {(loads, 1, 0), (loads, 0, 0), (0, 0, 0)}, (name, rest)
    assert seen >= 8


def test_audit_sees_a_moved_load():
    asm = "_Zk:\n\tbuffer_load_dwordx4 v0, s[4:7], 0 offen lds\n\t;;#ASMSTART\n%s\t;;#ASMSTART\n\ts_endpgm\n"
    assert segments(asm % "")["_Zk"] == [[1, 0, 0], [0, 0, 0], [0, 0, 0]]
    assert segments(asm % "\tbuffer_load_dword v1, v2, s[4:7], 0 offen\n")["_Zk"][1] == [0, 0, 1]


def test_lanes_meet_between_lds_writes_and_reads(products):
    """Rows of a tile on their way out, and values that a norm converts to BFP, pass from
    lane to lane of a wave through LDS: every turn has its mark."""
    kernels, turns = unordered(products)
    assert kernels >= 48 and not turns, turns[:3]
    # (norms of one wave a row: in the others the waves' sums pass through LDS of their own)
    turns = [t for t in unordered(assembly("rms_norm.hip"))[1] if re.search(r"10k_rms_normILi64E", t[0])]
    assert not turns, turns[:3]
