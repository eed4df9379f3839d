"""Loads from memory into LDS take their place in LDS from m0, and an instruction that writes m0 has to be one wait state before them;
a vector instruction that writes a scalar register has to be five wait states before a load that takes its address from there.  Where a
load is in an asm block the compiler does not see to that, so the built device code is looked over, instruction by instruction."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2604_05250_amd as dd

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")


def _scalars(text):
    found = set()
    for first, last, one in re.findall(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b", text):
        found |= {int(one)} if one else set(range(int(first), int(last) + 1))
    return found


def too_close(lines):
    """(loads into LDS; memory instructions right behind a write of m0 that they read, or of their address by a vector instruction)"""
    loads, bad = 0, []
    m0, written = 9, {}                                      # wait states since m0, and since a scalar register by a vector instruction
    for line in lines:
        if re.match(r"[0-9a-f]+ <", line):                   # the next kernel
            m0, written = 9, {}
        text = line.split("//")[0].strip()
        if not re.match(r"[a-z]+_", text):                   # a label, a heading
            continue
        op, _, rest = text.partition(" ")
        if op.startswith(("global_", "buffer_", "scratch_")):
            into_lds = "_load_lds_" in op or re.search(r"\blds\b", rest) is not None
            loads += into_lds
            if (into_lds and m0 < 1) or any(written.get(s, 9) < 5 for s in _scalars(rest)):
                bad.append(text)
        states = int(rest, 0) + 1 if op == "s_nop" else 1
        m0 += states
        written = {s: n + states for s, n in written.items() if n < 5}
        if op.startswith("s_") and re.match(r"m0\b", rest):
            m0 = 0
        if op.startswith(("v_readlane", "v_readfirstlane", "v_cmp")):
            written.update((s, 0) for s in _scalars(rest.split(",")[0]))
    return loads, bad


def test_what_is_too_close():
    mov, load, nop = "s_mov_b32 m0, s3  // 0: 1", "global_load_lds_dwordx4 v1, s[2:3]", "s_nop 0"
    assert too_close([mov, load]) == (1, [load]) and too_close([mov, "<L1>:", load])[1] and too_close([mov, "buffer_load_dword v1, s[0:3], 0 offen lds"])[1]
    assert too_close([mov, nop, load, mov, "s_add_u32 s1, s2, s3", load, load, "global_load_dwordx4 v[0:3], v1, s[2:3]"]) == (3, [])
    lane = "v_readlane_b32 s3, v9, 12"
    for between, close in (([mov, nop], True), ([mov, "s_nop 2"], True), ([mov, "s_nop 3"], False), ([nop] * 5, False), ([nop] * 4, True)):
        assert bool(too_close([lane, *between, load])[1]) == close
    assert too_close(["v_readlane_b32 s4, v9, 12", load]) == (1, []) and too_close(["v_cmp_gt_i32_e64 s[2:3], v1, v2", load])[1]


def test_wait_states_before_loads_into_lds(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    dd.lib()
    shutil.copy(dd.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL, timeout=60)
    parts = sorted(p.name for p in tmp_path.iterdir() if "gfx950" in p.name)
    assert parts
    loads, bad = 0, []
    for part in parts:
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", part], cwd=tmp_path, check=True, stdout=subprocess.PIPE, text=True, timeout=120).stdout
        n, b = too_close(text.splitlines())
        loads += n
        bad += b
    assert loads > 100
    assert not bad, f"{len(bad)} instructions, such as {bad[0]}"
