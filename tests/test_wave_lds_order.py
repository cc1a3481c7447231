"""Audit of data that the lanes of a wave pass to one another through LDS in the
few-token products of experts (gemm_direct.h), on the code the compiler emits (CPU
only: hipcc compiles the source to gfx950 assembly).

A lane's program order does not order its LDS accesses against another lane's, so
the source marks every turn from writes to reads and back.  The marks emit nothing but
the comment that is looked for here: in every kernel no LDS read may follow an LDS
write, nor a write a read, without a mark or a workgroup barrier between."""
import os
import re
import subprocess
import tempfile

from paper_2110_15456_amd import build as B

WRITE = re.compile(r"^ds_write")
READ = re.compile(r"^ds_read")
MARK = re.compile(r"^(; wave barrier|s_barrier)")


def unordered(asm):
    """(kernels seen, turns without a mark), in the order of the text."""
    kernels, turns, last, name = 0, [], None, None
    for raw in asm.splitlines():
        s = raw.strip()
        m = re.match(r"^(_Z\w+):", raw)
        if m:
            kernels, last, name = kernels + 1, None, m.group(1)
        elif MARK.match(s):
            last = None
        elif WRITE.match(s) or READ.match(s):
            kind = "write" if WRITE.match(s) else "read"
            if last not in (None, kind):
                turns.append((name, s))
            last = kind
    return kernels, turns


def test_turns_are_marked():
    src = os.path.join(B.CSRC, "gemm_direct_experts.hip")
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "k.s")
        cmd = [os.path.join(B.ROCM, "bin", "hipcc"), *B.HIPFLAGS, "--cuda-device-only", "-S", src, "-o", out]
        subprocess.run(cmd, check=True, capture_output=True)
        with open(out) as f:
            kernels, turns = unordered(f.read())
    assert kernels >= 24  # every operand format, on 16 rows and (one plane of A) 32
    assert not turns, "%d, first %s" % (len(turns), turns[0])


def test_audit_finds_a_missing_mark():
    asm = "_Zk:\n\tds_write_b128 v0, v[2:5]\n\t; wave barrier\n\tds_read_b128 v[2:5], v1\n%s\tds_write_b128 v0, v[2:5]\n"
    assert unordered(asm % "\t; wave barrier\n") == (1, [])
    assert unordered(asm % "\ts_barrier\n") == (1, [])
    assert unordered(asm % "") == (1, [("_Zk", "ds_write_b128 v0, v[2:5]")])
