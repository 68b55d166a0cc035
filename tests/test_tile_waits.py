"""The tiled FP8 kernels' waits, in the compiled code: the wait in front of a barrier covers by itself the loads to LDS that the barrier hands over.

Such a wait lets as many loads be under way as were issued behind those to LDS.  A load whose result nothing reads is removed by the compiler, and the count is then too high: on every
way to a barrier, at least as many loads have to stand behind the last one to LDS as the wait allows."""
import re
import shutil
import subprocess
from pathlib import Path

import pytest

from paper_2411_00288_amd import build

OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
LINE = re.compile(r"\t(\S+)(.*?)\s*// 0*([0-9A-F]+):.*?(?:<\S+?\+0x([0-9a-f]+)>)?$")
MEMORY = re.compile(r"(buffer|global|flat|scratch)_(load|store|atomic)")
NOTHING_STAGED = 1 << 20                                  # no load to LDS is on the way


def _kernels(listing, name):
    """{symbol: [(mnemonic, operands, address, branch target or None)]} of the kernels whose symbol has `name` in it."""
    found, code = {}, None
    for line in listing.splitlines():
        if line.endswith(">:"):
            code = found.setdefault(line.split("<")[1][:-2], []) if name in line else None
        m = LINE.match(line) if code is not None else None
        if m:
            code.append((m[1], m[2], int(m[3], 16), int(m[4], 16) if m[4] else None))
    return found


def _behind(code):
    """For each instruction, the least number of memory instructions behind the last load to LDS, over all ways to it."""
    start = code[0][2]
    at = {address - start: i for i, (_, _, address, _) in enumerate(code)}
    least, todo = [None] * len(code), [(0, NOTHING_STAGED)]
    while todo:
        i, n = todo.pop()
        while i < len(code) and (least[i] is None or n < least[i]):
            least[i] = n
            op, operands, _, target = code[i]
            if MEMORY.match(op):
                n = 0 if operands.split("//")[0].rstrip().endswith(" lds") else n + 1
            if op.startswith("s_cbranch"):
                todo.append((at[target], n))
            if op == "s_endpgm":
                break
            i = at[target] if op == "s_branch" else i + 1
    return least


def _too_early(code):
    """(barriers, those whose own wait leaves a load to LDS under way)"""
    least, wait, bad, barriers = _behind(code), None, [], 0
    for i, (op, operands, address, _) in enumerate(code):
        if op == "s_waitcnt":
            m = re.search(r"vmcnt\((\d+)\)", operands)
            wait = int(m[1]) if m else wait
        elif MEMORY.match(op) or "branch" in op:
            wait = None
        elif op == "s_barrier":
            barriers += 1
            # (nothing was counted down: all that is under way may be a load to LDS)
            if least[i] is not None and least[i] != NOTHING_STAGED and least[i] < (wait if wait is not None else NOTHING_STAGED):
                bad.append((hex(address), wait, least[i]))
    return barriers, bad


@pytest.mark.skipif(not Path(OBJDUMP).exists(), reason="no llvm-objdump")
def test_staged_pieces_are_waited_for(tmp_path):
    if not build.LIB.exists():
        pytest.skip("the library is not built")
    shutil.copy(build.LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    seen = 0
    for part in sorted(tmp_path.glob("lib.so.*gfx950")):
        if b"pw_f8_tile_kernel" not in part.read_bytes():
            continue
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", part.name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        for name, code in _kernels(listing, "pw_f8_tile_kernel").items():
            barriers, bad = _too_early(code)
            assert barriers >= 5, name                    # (the listing was understood: a loop of four chunks and what stands before it)
            assert not bad, (name, bad)
            seen += 1
    assert seen == 12                                     # two types, three tiles, two ways of storing
