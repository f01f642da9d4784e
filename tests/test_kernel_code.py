"""The assembly of the library's kernels as they were built: no register is copied or spilled at the head
of a block where lanes come together, ahead of the instruction that brings the waiting lanes back. Such a
copy leaves theirs out. The compiler has made them where registers are scarce and some lanes branch."""
import os
import re
from concurrent.futures import ProcessPoolExecutor

import pytest

from conftest import ROOT

OBJECTS = os.path.join(ROOT, "_build", "kvx")
RESTORE = ("s_or_b64 exec, exec,", "s_or_saveexec", "s_andn2_saveexec")
# what ends a block, or takes lanes away
LEAVE = re.compile(r"s_cbranch|s_branch|s_endpgm|s_barrier|s_setpc|s_\w+_saveexec|s_(mov|xor|and|andn2)_b64 exec")
SCALAR = re.compile(r"v_(readlane|readfirstlane|writelane)")
COPY = re.compile(r"v_accvgpr_|v_mov_b|scratch_(load|store)|v_bfrev_b32_e32 v\d+, -?\d")  # and constants made again
JOIN = re.compile(r"s_cbranch_execz (\.LBB\S+)")


def misplaced(lines):
    """(kernel, block, instructions): at a block's head only copies stand before the lanes come back, or,
    where a branch leads there past some lanes' code, any vector instruction."""
    found, kernel, heads, joins = [], None, [], set()
    block = None  # (name, vector instructions so far) while at a block's head

    def close():
        found.extend((kernel, name, code) for name, code in heads
                     if name in joins or all(COPY.match(t) for t in code))

    for line in lines:
        c = line[0] if line else ""
        if c == "\t":
            t = line.split(";")[0].strip()
            j = JOIN.match(t) if t.startswith("s_cbranch_execz") else None
            if j:
                joins.add(j.group(1))
            if block is None or not t:
                continue
            if t.startswith(RESTORE):
                if block[1]:
                    heads.append(block)
                block = None
            elif LEAVE.match(t):
                block = None
            elif t[:2] in ("v_", "ds") or t.startswith(("scratch_", "global_", "flat_", "buffer_")):
                if not SCALAR.match(t):
                    block[1].append(t)
        elif c == "." and line.startswith(".LBB"):
            block = (line.split(":")[0], [])
        elif line.startswith("; %bb"):
            block = (line.split(":")[0], [])
        elif c == "_" and ":" in line:
            close()
            kernel, heads, joins, block = line.split(":")[0], [], set(), None
    close()
    return found


PLANTED = """_Zkernel:                             ; @_Zkernel
; %bb.0:
	s_and_saveexec_b64 s[0:1], vcc
{}	v_add_u32_e32 v1, v2, v3
{}
{}
	s_or_b64 exec, exec, s[0:1]
	s_endpgm
.Lfunc_end0:
"""


@pytest.mark.parametrize("skipped", [True, False])  # whether the branch past the lanes' code was kept
@pytest.mark.parametrize("code,bad", [
    ("	s_nop 0", False), ("	v_readlane_b32 s4, v254, 2", False), ("	v_accvgpr_write_b32 a152, v10", True),
    ("	scratch_store_dword off, v174, off offset:56 ; 4-byte Folded Spill", True),
    ("	s_mov_b32 s1, s2\n	v_mov_b32_e32 v9, v8", True), ("	v_mov_b32_e32 v9, 0", True),
    ("	s_and_saveexec_b64 s[2:3], vcc\n	v_mov_b32_e32 v9, v8", False)])
def test_what_is_looked_for(code, bad, skipped):
    jump, label = ("	s_cbranch_execz .LBB0_2\n", ".LBB0_2:") if skipped else ("", "; %bb.2:    ;   in Loop")
    assert bool(misplaced(PLANTED.format(jump, label, code).split("\n"))) == bad


def _look(path):
    with open(path) as f:
        lines = f.read().split("\n")
    return sum(x.startswith("\ts_endpgm") for x in lines), misplaced(lines)


def test_kernels_of_the_library():
    built = [os.path.join(OBJECTS, f) for f in sorted(os.listdir(OBJECTS))
             if f.endswith("gfx950.s")] if os.path.isdir(OBJECTS) else []
    if not built:
        pytest.skip("the build's assembly is not here")
    with ProcessPoolExecutor(4) as pool:
        looked = list(pool.map(_look, built))
    assert sum(n for n, _ in looked) > 400
    assert not [x for _, bad in looked for x in bad]
