"""Lanes of a wave of the 32-query kernel over the 8-bit cache hand each other
offsets, scales and codes through LDS without a workgroup barrier.  The LDS
keeps a wave's order; the compiler, which sees one lane's addresses and the
types they are accessed with, has to be told to.  In the kernel's intermediate
code every path from an LDS write to an LDS read, or from a read to a write,
passes a fence.  Compiles k_quant_attention.hip for the device (CPU only)."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2608_26140_amd import build as B


def blocks_of(lines):
    """Basic blocks of a function's body: {label: (instructions, successors)}, the first label."""
    out, label, first = {}, "0", None
    cur = []
    for line in lines + ["end:"]:
        m = re.match(r"^([\w.$-]+):", line)
        if m:
            if cur:
                succ = re.findall(r"label %([\w.$-]+)", " ".join(cur))
                out[label] = (cur, succ)
                first = first or label
            label, cur = m.group(1), []
        else:
            cur.append(line.strip())
    return out, first


def kind_of(ins):
    if re.search(r"\bfence\b", ins):
        return "fence"
    if "ds.read" in ins and " call " in f" {ins}":
        return "read"
    if "addrspace(3)" in ins:
        if re.search(r"(= |^)load ", ins):
            return "read"
        if ins.startswith("store "):
            return "write"
    return None


def unordered(lines):
    """(read or write, instruction) pairs where the other kind came before and no fence between."""
    blocks, first = blocks_of(lines)
    entry = {b: set() for b in blocks}
    entry[first] = {None}
    work, bad = [first], set()
    while work:
        b = work.pop()
        ins, succ = blocks[b]
        state = set(entry[b])
        for i in ins:
            k = kind_of(i)
            if k == "fence":
                state = {None}
            elif k:
                if ("read" if k == "write" else "write") in state:
                    bad.add((k, i))
                state = {k}
        for s in succ:
            if s in entry and not state <= entry[s]:
                entry[s] |= state
                work.append(s)
    return sorted(bad)


def body_of(ir, name):
    m = re.search(r"^define [^\n]*%s[^\n]*\{\n(.*?)^\}" % name, ir, re.S | re.M)
    assert m, name
    return m.group(1).splitlines()


@pytest.mark.skipif(not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)), reason="hipcc not found")
def test_lds_accesses_of_a_wave_are_ordered(tmp_path):
    out = str(tmp_path / "k.ll")
    subprocess.run([B.HIPCC, *B.FLAGS, "--offload-device-only", "-S", "-emit-llvm",
                    os.path.join(B.CSRC, "k_quant_attention.hip"), "-o", out], check=True, capture_output=True)
    body = body_of(open(out).read(), "quant_attention_narrow_kernel")
    kinds = [kind_of(line.strip()) for line in body]
    assert kinds.count("read") > 20 and kinds.count("write") > 10  # the accesses are seen
    assert unordered(body) == []


def test_the_check_sees_missing_fences():
    loop = """
  br label %3
3:
  store i32 %a, ptr addrspace(3) %p, align 4
  fence syncscope("wavefront") acquire
  %b = load float, ptr addrspace(3) %q, align 4
  br i1 %c, label %3, label %9
9:
  ret void
""".splitlines()
    assert [k for k, _ in unordered(loop)] == ["write"]  # round the loop, read then write
    fenced = loop[:2] + ["3:", "  fence syncscope(\"wavefront\") acquire"] + loop[3:]
    assert unordered(fenced) == []
    assert [k for k, _ in unordered([line for line in fenced if "fence" not in line])] == ["read", "write"]
    read = "  %b = tail call <2 x i32> @llvm.amdgcn.ds.read.tr8.b64.v2i32(ptr addrspace(3) %q)"
    assert [k for k, _ in unordered(["  store i32 0, ptr addrspace(3) %p", read, "  ret void"])] == ["read"]
