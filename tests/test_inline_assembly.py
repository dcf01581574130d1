"""Assembly written into the kernels: what it tells the compiler, and the waits that the compiler does not add in it (CPU).

The source has to declare what an asm statement writes (m0, memory), and the generated code has to keep the distances that
the hardware asks for around the statements: a vector instruction's write of a scalar register to a load's use of it, a
write of m0 to its use, a matrix product to a read of its sums.
"""

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_29678_amd", "csrc")
STATEMENT = re.compile(r"\basm\s*(volatile)?\s*\(((?:\"(?:[^\"\\]|\\.)*\"|[^;])*)\)\s*;")


def statements(source: str):
    """(volatile, template, clobbers) of the asm statements of a source."""
    out = []
    for m in STATEMENT.finditer(re.sub(r"//[^\n]*", "", source)):
        body = m.group(2)
        template = re.match(r"\s*((?:\"(?:[^\"\\]|\\.)*\"\s*)+)", body).group(1)
        rest = body[len(template):]
        # sections behind the template start at colons outside of parentheses, strings and ?:
        parts, depth, quoted, part = [], 0, False, ""
        for ch in rest:
            quoted ^= ch == '"'
            if not quoted:
                depth += (ch in "([") - (ch in ")]")
                if ch == ":" and depth == 0:
                    parts.append(part)
                    part = ""
                    continue
            part += ch
        parts.append(part)
        text = " ".join(re.sub(r'\\[nt]|"', " ", template).split())
        out.append((m.group(1) is not None, text, re.findall(r'"([^"]*)"', parts[3]) if len(parts) > 3 else []))
    return out


def undeclared(source: str):
    """What the statements write without saying so."""
    out = []
    for volatile, text, clobbers in statements(source):
        if re.search(r"\bs_\w+ m0\b", text) and "m0" not in clobbers:
            out.append("m0: " + text)
        if re.search(r"\b(buffer|global)_load\w* .*\blds\b", text) and not (volatile and "memory" in clobbers):
            out.append("memory: " + text)
        if "s_barrier" in text and not (volatile and "memory" in clobbers):
            out.append("memory: " + text)
    return out


def test_the_parser():
    src = 'asm volatile("s_mov_b32 m0, %0\\n\\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(f(a, b)), "v"(c ? d[0] : e), "s"(g)CLOBBERS);'
    assert len(undeclared(src.replace("CLOBBERS", ""))) == 2
    assert len(undeclared(src.replace("CLOBBERS", ' : "m0"'))) == 1
    assert undeclared(src.replace("CLOBBERS", ' : "m0", "memory"')) == []
    assert statements('asm("v_x %0, %1" : "=v"(x) : "a"(y[1][2]));')[0] == (False, "v_x %0, %1", [])


def test_what_is_written_is_declared():
    bad = {}
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".hip", ".h")):
            with open(os.path.join(CSRC, name)) as f:
                found = undeclared(f.read())
            if found:
                bad[name] = found
    assert not bad, bad


def _registers(text, kind):
    """Numbers of the `kind` registers (s, v, a) that an operand text names."""
    out = set()
    for a, b in re.findall(r"\b%s\[(\d+):(\d+)\]" % kind, text):
        out.update(range(int(a), int(b) + 1))
    out.update(int(n) for n in re.findall(r"\b%s(\d+)\b" % kind, text))
    return out


def _states(line):
    m = re.match(r"s_nop (\d+)", line)
    return int(m.group(1)) + 1 if m else 1


SGPR_TO_LOAD, M0_TO_LOAD, PRODUCT_TO_READ = 5, 1, 19  # wait states; 19: the longest products


def too_near(asm: str):
    """Places where one of the distances is not kept, by the order of the text (a label starts anew)."""
    out, scalar, m0, product, func = [], {}, 99, 99, None
    for raw in asm.split("\n"):
        m = re.match(r"^(_Z\w+):", raw)
        if m:
            func = m.group(1)
        line = raw.split(";")[0].strip()
        if re.match(r"^\.?\w+:", line):
            # the text before a label is one of the ways to it
            continue
        if not line or line.startswith("."):
            continue
        op, _, args = line.partition(" ")
        operands = [a.strip() for a in args.split(",")]
        if op.startswith("buffer_load") and " lds" in args:
            for r in _registers(operands[1], "s") | _registers(operands[2] if len(operands) > 2 else "", "s"):
                if scalar.get(r, 99) < SGPR_TO_LOAD:
                    out.append((func, "s%d" % r, line))
            if m0 < M0_TO_LOAD:
                out.append((func, "m0", line))
        if op.startswith("v_accvgpr_read") and product < PRODUCT_TO_READ:
            out.append((func, "product", line))
        states = _states(line)
        scalar = {r: n + states for r, n in scalar.items() if n + states < 16}
        m0, product = m0 + states, product + states
        if op.startswith(("v_readfirstlane", "v_readlane")):
            for r in _registers(operands[0], "s"):
                scalar[r] = 0
        if op.startswith("s_") and operands[0] == "m0":
            m0 = 0
        if op.startswith("v_mfma"):
            product = 0
    return out


def test_the_distances():
    load = "\tbuffer_load_dwordx4 v1, s[4:7], 0 offen lds\n"
    near = "_Zk:\n\tv_readfirstlane_b32 s5, v2\n\ts_mov_b32 m0, s9\n\ts_nop 0\n" + load
    assert too_near(near) == [("_Zk", "s5", load.strip())]
    assert too_near(near.replace("s_nop 0", "s_nop 3")) == []
    assert too_near("_Zk:\n\ts_mov_b32 m0, s9\n" + load) == [("_Zk", "m0", load.strip())]
    read = "\tv_accvgpr_read_b32 v0, a3\n"
    assert len(too_near("_Zk:\n\tv_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]\n\ts_nop 15\n" + read)) == 1
    assert too_near("_Zk:\n\tv_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]\n\ts_nop 15\n\ts_nop 15\n" + read) == []


@pytest.mark.timeout(600)
def test_the_generated_code_keeps_the_distances(tmp_path):
    cc = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)
    if cc is None:
        pytest.skip("hipcc not found")
    out = str(tmp_path / "head.s")
    r = subprocess.run([cc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "--cuda-device-only", "-S", "-Xclang",
                        "-target-feature", "-Xclang", "-packed-fp32-ops", os.path.join(CSRC, "tt_head.hip"), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        asm = f.read()
    assert asm.count("offen lds") + asm.count("offen nt lds") > 100  # (what is looked at is there)
    found = too_near(asm)
    assert not found, found[:5]
