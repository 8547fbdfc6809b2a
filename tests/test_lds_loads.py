"""Loads straight to LDS, written in inline assembly, where the compiler puts in
no wait states: such a load needs one between it and a write of m0 (its place in
LDS), and five between it and a vector instruction that writes a scalar register
it reads.  Counted in the assembly that the build's own flags give."""
import os
import re
import subprocess

import pytest

from paper_2606_02955_amd import build

SOURCES = ["prompt_attn.hip", "lmhead.hip"]
LOAD = re.compile(r"buffer_load_\w+ (?:v\d+|off), s\[(\d+):(\d+)\], (\S+) .*\blds\b")


def _instructions(path):
    for line in open(path):
        line = line.split(";")[0].strip()
        if line and not line.startswith(".") and not line.endswith(":"):
            yield line


def _scalars(operand):
    """Numbers of the scalar registers of one operand."""
    m = re.fullmatch(r"s(\d+)", operand) or re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    return set(range(int(m.group(1)), int(m.groups()[-1]) + 1)) if m else set()


def _violations(lines):
    bad, loads = [], 0
    for at, line in enumerate(lines):
        m = LOAD.match(line)
        if not m:
            continue
        loads += 1
        reads = set(range(int(m.group(1)), int(m.group(2)) + 1)) | _scalars(m.group(3))
        states, i = 0, at - 1
        while states < 5 and i >= 0:
            before = lines[i]
            op, _, rest = before.partition(" ")
            written = rest.split(",")[0].strip()
            if states < 1 and op.startswith("s_") and written == "m0":
                bad.append((before, line))
            if op.startswith("v_") and _scalars(written) & reads:
                bad.append((before, line))
            states += int(rest.strip(), 0) + 1 if op == "s_nop" else 1
            i -= 1
    return bad, loads


def test_the_count_finds_both():
    load = "buffer_load_dwordx4 v1, s[8:11], 0 offen lds"
    assert len(_violations(["s_mov_b32 m0, s5", load])[0]) == 1
    assert _violations(["s_mov_b32 m0, s5", "s_nop 0", load]) == ([], 1)
    assert len(_violations(["v_readfirstlane_b32 s9, v3", "s_nop 1", "s_mov_b32 m0, s5", "s_nop 0", load])[0]) == 1
    assert _violations(["v_readfirstlane_b32 s9, v3", "s_nop 2", "s_mov_b32 m0, s5", "s_nop 0", load]) == ([], 1)


@pytest.mark.parametrize("src", SOURCES)
def test_wait_states(src, tmp_path):
    out = str(tmp_path / "a.s")
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    res = subprocess.run([build.hipcc(), *flags, "-I", build.INCLUDE, "--cuda-device-only", "-S",
                          os.path.join(build.PKG, "csrc", src), "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    bad, loads = _violations(list(_instructions(out)))
    assert loads > 0
    assert not bad, f"{len(bad)} of {loads}: {bad[0]}"
