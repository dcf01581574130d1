"""Loads from memory straight to LDS written as assembly in the cache's attention: what they declare, and their distances (CPU).

``global_load_lds_*`` writes LDS at an address in m0.  The statement has to say that it writes memory and m0, m0 has to be
written a wait state before, and a wait for the loads has to stand in one statement with the block's barrier: the compiler
knows of none of them.
"""

import os
import re
import shutil
import subprocess

import pytest

from test_inline_assembly import CSRC, _states, statements

TO_LDS = re.compile(r"\b(?:buffer|global)_load_lds_\w+")
M0_TO_LOAD = 1  # wait states


def distances(lines):
    """Lines that load to LDS less than M0_TO_LOAD wait states behind a write of m0 (a label leaves them as they are)."""
    out, m0 = [], 99
    for line in lines:
        line = line.split(";")[0].strip()
        if not line or line.startswith(".") or re.match(r"^\.?\w+:", line):
            continue
        if TO_LDS.match(line) and m0 < M0_TO_LOAD:
            out.append(line)
        m0 += _states(line)
        if re.match(r"(s_\w+|v_readfirstlane_b32|v_readlane_b32) m0\b", line):
            m0 = 0
    return out


def faults(source):
    """What is wrong with the statements of a source that load to LDS, or wait for it."""
    out = []
    for volatile, text, clobbers in statements(source):
        declared = volatile and "memory" in clobbers
        if TO_LDS.search(text):
            if not declared:
                out.append("memory: " + text)
            if re.search(r"\bs_\w+ m0\b", text):
                if "m0" not in clobbers:
                    out.append("m0: " + text)
                parts = re.split(r" (?=(?:s|v|global|buffer)_\w+ )", text)
                if distances(parts):
                    out.append("distance: " + text)
            else:
                out.append("m0 is not written in the statement: " + text)
        if "s_barrier" in text and not (declared and "vmcnt(0)" in text and "lgkmcnt(0)" in text):
            out.append("wait: " + text)
    return out


def attention():
    with open(os.path.join(CSRC, "tt_attention.hip")) as f:
        return f.read()


def test_the_statements():
    source = attention()
    assert sum(bool(TO_LDS.search(t)) for _, t, _ in statements(source)) == 1
    assert sum("s_barrier" in t for _, t, _ in statements(source)) == 1
    assert faults(source) == []


@pytest.mark.parametrize("old,new,kind", [
    (': "m0", "memory"', ': "m0"', "memory"), (': "m0", "memory"', ': "memory"', "m0"),
    (': "m0", "memory"', "", "memory"), ("asm volatile(\"s_mov_b32 m0", "asm(\"s_mov_b32 m0", "memory"),
    ("s_nop 3\\n\\t", "", "distance"), ("s_mov_b32 m0, %0\\n\\t", "", "m0 is not written"),
    ("vmcnt(0) lgkmcnt(0)", "lgkmcnt(0)", "wait"), ("vmcnt(0) lgkmcnt(0)", "vmcnt(0)", "wait"),
    ('s_barrier" ::: "memory"', 's_barrier" ::', "wait")])
def test_a_statement_that_is_wrong_is_found(old, new, kind):
    """Each part taken out of the source's text."""
    source = attention()
    at = source.index("global_load_lds_dwordx4 %1") if kind != "wait" else source.index("s_waitcnt vmcnt(0) lgkmcnt(0)")
    first, last = source.rindex("asm", 0, at), source.index(";", at)
    statement = source[first:last]
    assert statement.count(old) == 1
    found = faults(source[:first] + statement.replace(old, new) + source[last:])
    assert any(f.startswith(kind) for f in found), found


def test_the_distances():
    load = "\tglobal_load_lds_dwordx4 v[2:3], off\n"
    assert len(distances(("\ts_mov_b32 m0, s4\n" + load).split("\n"))) == 1
    assert len(distances(("\tv_readfirstlane_b32 m0, v4\n" + load).split("\n"))) == 1
    assert distances(("\ts_mov_b32 m0, s4\n\ts_nop 0\n" + load).split("\n")) == []
    assert distances(("\ts_mov_b32 m0, s4\n\tv_add_u32_e32 v0, v1, v2\n" + load).split("\n")) == []


@pytest.mark.timeout(600)
def test_the_generated_code_keeps_the_distances(tmp_path):
    cc = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)
    if cc is None:
        pytest.skip("hipcc not found")
    out = str(tmp_path / "attention.s")
    r = subprocess.run([cc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "--cuda-device-only", "-S", "-Xclang",
                        "-target-feature", "-Xclang", "-packed-fp32-ops", os.path.join(CSRC, "tt_attention.hip"), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        lines = f.read().split("\n")
    kernels = {}
    func = None
    for line in lines:
        m = re.match(r"^(_Z\w+):", line)
        func = m.group(1) if m else func
        if TO_LDS.match(line.split(";")[0].strip()):
            kernels[func] = kernels.get(func, 0) + 1
    # two types of four widths, two tiles for each of two places of a pass of loads
    assert len(kernels) == 8 and min(kernels.values()) >= 4, kernels
    assert distances(lines) == []
