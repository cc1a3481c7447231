"""Audit of the waits of the 8-bit products' loops (gemm_fp8.hip), on the code the compiler
emits (CPU only: hipcc compiles the source to gfx950 assembly).

The kernels count the loads that may still be on the way; the compiler adds waits of its
own wherever it cannot tell that what is read has landed.  One of those in a loop that
is stricter than the counted ones takes away what the counting is for."""
import re

import pytest

from tests.test_fp8_load_order import assembly

COUNT = re.compile(r"vmcnt\((\d+)\)")


def loops(asm):
    """{kernel: [the compiler's own vmcnt waits]} of the loops that multiply.  (A counted wait
    stands right in front of an empty asm statement, the mark of its slab.)"""
    found, name, lines = {}, None, []
    for raw in asm.splitlines():
        m = re.match(r"^(_Z\w+):", raw)
        if m:
            name, lines = m.group(1), []
        elif name and raw.strip().startswith("s_endpgm"):
            found.setdefault(name, []).extend(waits(lines))
            name = None
        elif name and raw.strip() and not re.match(r"^\s*(;[^;]|\.p2align)", raw):
            lines.append(raw.strip())
    return found


def waits(lines):
    at = {m.group(1): i for i, l in enumerate(lines) for m in [re.match(r"^(\.LBB\w+):", l)] if m}
    own = set()
    for i, l in enumerate(lines):
        m = re.match(r"^s_c?branch\w* (\.LBB\w+)", l)
        if not m or at.get(m.group(1), i) >= i:
            continue
        body = range(at[m.group(1)], i)  # back to a label further up: a loop
        if not any(lines[k].startswith("v_mfma") for k in body):
            continue
        own.update(k for k in body if lines[k].startswith("s_waitcnt") and COUNT.search(lines[k])
                   and not lines[k + 1].startswith(";;#ASMSTART"))
    return [int(COUNT.search(lines[k]).group(1)) for k in sorted(own)]


@pytest.fixture(scope="module")
def products():
    return loops(assembly("gemm_fp8.hip"))


@pytest.mark.parametrize("edge", [64, 128, 256])
def test_tiles_wait_for_what_they_count_alone(products, edge):
    mine = {n: w for n, w in products.items() if "k_gemm_fp8ILi%dE" % edge in n}
    assert len(mine) == 8  # four pairs of formats, two types
    for name, own in mine.items():
        assert own == [], (name, own)


def test_audit_sees_a_wait():
    asm = ("_Zk:\n.LBB0_1:\n\tv_mfma_scale_f32_32x32x64_f8f6f4 v0\n%s\ts_waitcnt vmcnt(8) lgkmcnt(0)\n\t;;#ASMSTART\n"
           "\ts_barrier\n\t;;#ASMSTART\n\ts_cbranch_vccnz .LBB0_1\n\ts_waitcnt vmcnt(0)\n\ts_endpgm\n")
    assert loops(asm % "") == {"_Zk": []}
    assert loops(asm % "\ts_waitcnt vmcnt(0)\n\tds_read_b128 v1, v2\n") == {"_Zk": [0]}
    assert loops(asm % "\ts_waitcnt lgkmcnt(0)\n") == {"_Zk": []}


def test_few_rows_keep_three_slabs_on_the_way(products):
    seen = 0
    for name, own in products.items():
        m = re.search(r"k_gemm_fp8_fewILi(\d+)ELi(\d+)ELi\d+E", name)
        if not m:
            continue
        seen += 1
        loads = 2 * (int(m.group(1)) + int(m.group(2)))  # of a slab
        assert all(n >= 3 * loads for n in own), (name, own)
    assert seen == 24  # three tiles, four pairs of formats, two types
