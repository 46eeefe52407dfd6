"""The large form of as_linear reads its fragments from LDS by hand, a slice ahead of the products, so the compiler takes their
registers as filled when they are only on their way.  In the library as it was built, nothing may touch such a register before a
wait, on any path, and no read may be in flight when a wave ends."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2210_15458_amd import binding

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def registers(text):
    out = set()
    for kind, first, last, kind1, one in re.findall(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        out |= {kind + str(r) for r in range(int(first), int(last) + 1)} if kind else {kind1 + one}
    return out


def kernels(folder, name):
    """{mangled name: [(address, instruction, address of the branch's target or None)]} of the kernels whose name has `name` in it."""
    shutil.copy(binding.LIB_PATH, folder / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=folder, check=True, capture_output=True)
    found = {}
    for f in sorted(os.listdir(folder)):
        if not f.endswith("gfx950") or name.encode() not in (folder / f).read_bytes():
            continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", f], cwd=folder, check=True, capture_output=True, text=True).stdout
        start, here = 0, None
        for line in text.splitlines():
            head = re.match(r"^([0-9a-f]+) <(\S+)>:$", line)
            if head:
                here = found.setdefault(head.group(2), []) if name in head.group(2) else None
                start = int(head.group(1), 16)
                continue
            m = re.match(r"^\s+(\S.*?)\s*// ([0-9A-F]+):.*?(?:<\S+?(?:\+0x([0-9a-f]+))?>)?$", line)
            if here is None or not m:
                continue
            to = start + int(m.group(3) or "0", 16) if m.group(1).startswith(("s_cbranch", "s_branch")) else None
            here.append((int(m.group(2), 16), m.group(1), to))
    return found


def faults(code):
    """Instructions that touch a register in flight, and how many registers are in flight at the end of some path."""
    at = {a: i for i, (a, _, _) in enumerate(code)}
    state, work, bad, left = {0: frozenset()}, [0], set(), 0
    while work:
        i = work.pop()
        flying = set(state[i])
        while True:
            _, text, to = code[i]
            if text.startswith("s_waitcnt") and "lgkmcnt(0)" in text:
                flying = set()
            elif text.startswith("ds_read_b128"):
                if registers(text) & flying:
                    bad.add(text)
                flying |= registers(text.split(",")[0])
            elif registers(text) & flying:
                bad.add(text)
            if text.startswith("s_endpgm"):
                left = max(left, len(flying))
                break
            after = ([] if text.startswith("s_branch") else [i + 1]) + ([at[to]] if to is not None else [])
            if len(after) == 1 and to is None and (i + 1) not in state:
                i += 1
                continue
            for j in after:
                new = frozenset(flying) | state.get(j, frozenset())
                if j not in state or new != state[j]:
                    state[j] = new
                    work.append(j)
            break
    return bad, left


def test_the_reading_of_the_code():
    code = [(0, "ds_read_b128 v[0:3], v9", None), (8, "s_cbranch_scc1 2", 24), (12, "v_add_f32_e32 v5, v2, v6", None),
            (16, "s_waitcnt vmcnt(0) lgkmcnt(0)", None), (20, "s_endpgm", None), (24, "v_mov_b32_e32 v8, v9", None), (28, "s_endpgm", None)]
    bad, left = faults(code)
    assert bad == {"v_add_f32_e32 v5, v2, v6"} and left == 4


@pytest.mark.skipif(not os.path.exists(OBJDUMP) or not os.path.exists(binding.LIB_PATH), reason="no disassembler, or nothing built")
def test_large_form(tmp_path):
    found = kernels(tmp_path, "linear_big")
    assert len(found) == 6
    for name, code in found.items():
        assert sum(text.startswith("ds_read_b128") for _, text, _ in code) > 30
        bad, left = faults(code)
        assert not bad and not left, f"{name}: touched in flight {sorted(bad)[:4]}, in flight at the end {left}"
