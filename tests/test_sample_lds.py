"""The waves of a row's workgroup read what one of them has found (a border, the
counts behind it) at fixed places in LDS, and the next cut writes these again.  In
the sampled commit's intermediate code every path from a read of such a place to
the next write of it passes a workgroup barrier.  Compiles k_sample.hip for the
device (CPU only)."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2608_26140_amd import build as B
from tests.test_quant_lds import blocks_of, body_of

SIZE = {"i8": 1, "i16": 2, "i32": 4, "float": 4, "i64": 8, "double": 8}


def fixed(ins):
    """("read" or "write", offset, bytes) of an access of LDS at an offset that the code holds as a number."""
    m = re.search(r"(?:= |^)load (?:volatile )?(<[^>]*>|\w+), ptr addrspace\(3\) (.*)$", ins)
    kind = "read"
    if not m:
        m = re.match(r"store (?:volatile )?(<[^>]*>|\w+) .*?, ptr addrspace\(3\) (.*)$", ins)
        kind = "write"
    if not m:
        return None
    t, where = m.groups()
    at = re.match(r"getelementptr [^(]*\(i8, ptr addrspace\(3\) @[\w.$]+, i32 (\d+)\)", where)
    if not at and not re.match(r"@[\w.$]+,", where):
        return None
    v = re.match(r"<(\d+) x (\w+)>", t)
    return kind, int(at.group(1)) if at else 0, int(v.group(1)) * SIZE[v.group(2)] if v else SIZE[t]


def overwritten(lines):
    """Offsets written on a path on which they were read before and no barrier stands between."""
    blocks, first = blocks_of(lines)
    entry = {first: set()}
    work, bad = [first], set()
    while work:
        ins, succ = blocks[work[-1]]
        read = set(entry[work.pop()])
        for i in ins:
            if "llvm.amdgcn.s.barrier" in i:
                read = set()
            a = fixed(i)
            if a and a[0] == "read":
                read.add(a[1:])
            elif a:
                bad |= {a[1] for at, n in read if at < a[1] + a[2] and a[1] < at + n}
        for s in succ:
            if s in blocks and (s not in entry or not read <= entry[s]):
                entry[s] = entry.get(s, set()) | read
                work.append(s)
    return sorted(bad)


@pytest.mark.skipif(not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)), reason="hipcc not found")
def test_no_cut_overwrites_what_another_wave_may_still_read(tmp_path):
    out = str(tmp_path / "k.ll")
    subprocess.run([B.HIPCC, *B.FLAGS, "--offload-device-only", "-S", "-emit-llvm", os.path.join(B.CSRC, "k_sample.hip"),
                    "-o", out], check=True, capture_output=True)
    ir = open(out).read()
    for name in ("sample_f32_kernel", "sample_bf16_kernelILi1024", "sample_bf16_kernelILi512"):
        body = body_of(ir, name)
        kinds = [a[0] for a in map(fixed, (line.strip() for line in body)) if a]
        assert kinds.count("read") > 20 and kinds.count("write") > 20, name  # the accesses are seen
        assert overwritten(body) == [], name


def test_the_check_sees_a_missing_barrier():
    loop = """
  br label %3
3:
  store i32 %a, ptr addrspace(3) getelementptr inbounds nuw (i8, ptr addrspace(3) @sh, i32 8), align 4
  tail call void @llvm.amdgcn.s.barrier()
  %b = load i64, ptr addrspace(3) getelementptr inbounds nuw (i8, ptr addrspace(3) @sh, i32 8), align 8
  br i1 %c, label %3, label %9
9:
  store i32 %a, ptr addrspace(3) @sh, align 4
  ret void
""".splitlines()
    assert overwritten(loop) == [8]
    assert overwritten(loop[:3] + ["  tail call void @llvm.amdgcn.s.barrier()"] + loop[3:]) == []
