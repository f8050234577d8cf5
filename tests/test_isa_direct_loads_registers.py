"""Static checks of loads that go straight to LDS, which are assembly blocks (no GPU needed): the compiler is told of everything that such a block writes (m0, and
memory: LDS), and no vector instruction of any kind writes one of its address registers within five wait states ahead of it."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2306_16699_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "paper_2306_16699_amd", "csrc", "rinr_nn.hip")
WAIT_STATES = 5

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")

LOAD = re.compile(r"buffer_load_dwordx4 v\d+, s\[(\d+):(\d+)\], .*\blds\b")
REGISTERS = r"s(?:\[(\d+):(\d+)\]|(\d+))(?=,|\s|$)"
# vector instructions whose first operand is a scalar register write it; these write their second
FIRST = re.compile(r"v_\S+ " + REGISTERS)
SECOND = re.compile(r"v_(?:add|sub|subrev|addc|subb|subbrev)_co_\S+ v\d+, " + REGISTERS + r"|v_(?:mad_[iu]64_[iu]32|div_scale_\S+) v(?:\d+|\[\d+:\d+\]), " + REGISTERS)
SCALAR = re.compile(r"s_\S+ " + REGISTERS)


def span(m):
    lo, hi, one = [g for g in (m.groups()[:3], m.groups()[3:]) if any(g)][0]
    return range(int(one), int(one) + 1) if one else range(int(lo), int(hi) + 1)


def nearest(lines):
    """(loads, wait states between the nearest vector instruction that writes a scalar register and a load that takes it, or None)."""
    writer, states, loads, worst = {}, 0, 0, None
    for ln in lines:
        m = re.match(r"s_nop (\d+)", ln)
        states += int(m.group(1)) + 1 if m else 1
        m = LOAD.match(ln)
        if m:
            loads += 1
            for r in range(int(m.group(1)), int(m.group(2)) + 1):
                if r in writer:
                    gap = states - writer[r] - 1
                    worst = gap if worst is None else min(worst, gap)
            continue
        m = FIRST.match(ln) or SECOND.match(ln)
        if m:
            writer.update((r, states) for r in span(m))
            continue
        m = SCALAR.match(ln)
        if m:
            for r in span(m):
                writer.pop(r, None)
    return loads, worst


def test_the_scan_sees_every_vector_writer():
    load = "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"
    for ln in ("v_readfirstlane_b32 s5, v0", "v_readlane_b32 s4, v9, 3", "v_cmp_lt_i32_e64 s[6:7], v1, v2", "v_add_co_u32 v3, s[4:5], v1, v2", "v_mad_u64_u32 v[2:3], s[4:5], v1, v2, v[6:7]",
               "v_div_scale_f32 v3, s[6:7], v1, v2, v1"):
        assert nearest([ln, load]) == (1, 0), ln
        assert nearest([ln, "s_nop 4", load]) == (1, 5), ln
    for ln in ("v_cmp_lt_i32_e32 vcc, v1, v2", "v_add_u32_e32 v3, s5, v1", "v_mov_b32_e32 v4, s4", "v_cmp_lt_i32_e64 s[8:9], s4, v2", "v_fma_f32 v3, s4, v1, v2"):
        assert nearest([ln, load]) == (1, None), ln
    assert nearest(["v_readfirstlane_b32 s5, v0", "s_mov_b64 s[4:5], s[8:9]", load]) == (1, None)


def test_direct_loads_are_clear_of_vector_writers(tmp_path):
    out = tmp_path / "rinr_nn.s"
    subprocess.run(["hipcc", *build.HIP_FLAGS, *build.SOURCES["rinr_nn.hip"], "--cuda-device-only", "-S", "-o", str(out), SRC], check=True, stdout=subprocess.DEVNULL,
                   stderr=subprocess.PIPE)
    total = 0
    for part in re.split(r"\n(?=_ZN\S+:)", out.read_text()):
        loads, worst = nearest([ln.strip() for ln in part.split("\n") if ln.startswith("\t") and not ln.strip().startswith((".", ";"))])
        total += loads
        assert worst is None or worst >= WAIT_STATES, (part.split(":")[0], worst)
    assert total >= 100, total


def test_direct_loads_name_what_they_write(tmp_path):
    """The constraints of every such assembly block in the compiler's own notation."""
    out = tmp_path / "rinr_nn.ll"
    subprocess.run(["hipcc", *build.HIP_FLAGS, *build.SOURCES["rinr_nn.hip"], "--cuda-device-only", "-Xclang", "-disable-llvm-passes", "-emit-llvm", "-S", "-o", str(out), SRC], check=True,
                   stdout=subprocess.DEVNULL, stderr=subprocess.PIPE)
    blocks = re.findall(r'asm sideeffect "([^"]*buffer_load[^"]*)", "([^"]*)"', out.read_text())
    assert blocks
    for text, constraints in blocks:
        named = set(re.findall(r"~\{(\w+)\}", constraints))
        assert " lds" in text and "m0" in text and {"m0", "memory"} <= named, (text, constraints)
