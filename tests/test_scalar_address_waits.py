"""Wait states between a vector instruction that writes scalar registers and a memory instruction that takes its address
from them: five, which the hardware does not hold back for.  The compiler counts them up to its own memory instructions
and not into assembly statements, such as the load-to-LDS copies.  Every way through the built library is counted, and
the counting is checked on listings with a known answer."""
import collections
import os
import re
import shutil
import subprocess

import pytest

from paper_2504_06419_amd import spire
from tests.test_matrix_waits import LLVM, _listing, parse

NEED = 5
MEMORY = ("global_", "buffer_", "flat_", "scratch_")
# their second operand is a scalar result too
CARRY = ("v_add_co", "v_addc_co", "v_sub_co", "v_subb_co", "v_subrev_co", "v_mad_u64", "v_mad_i64", "v_div_scale")


def scalars(operand):
    m = re.match(r"^s(\d+)\b", operand)
    if m:
        return {int(m.group(1))}
    m = re.match(r"^s\[(\d+):(\d+)\]", operand)  # modifiers may follow
    return set(range(int(m.group(1)), int(m.group(2)) + 1)) if m else set()


def shortfalls(code):
    """[(writer, memory instruction, wait states between them)] of one function."""
    at = {ins[3]: i for i, ins in enumerate(code)}
    found = []
    for i, (name, _, ops, addr, _) in enumerate(code):
        if not name.startswith("v_") or not ops:
            continue
        written = scalars(ops[0]) | (scalars(ops[1]) if name.startswith(CARRY) and len(ops) > 1 else set())
        todo, best = collections.deque([(i + 1, 0, frozenset(written))]), {}
        while todo:
            j, waits, live = todo.popleft()
            if j >= len(code) or waits >= NEED or not live or best.get((j, live), NEED) <= waits:
                continue
            best[(j, live)] = waits
            op, _, o, where, target = code[j]
            if op.startswith(MEMORY) and any(scalars(x) & live for x in o):
                found.append((f"{name} {hex(addr)}", f"{op} {hex(where)}", waits))
            if op == "s_endpgm":
                continue
            if op.startswith("s_") and o and not op.startswith(("s_cmp", "s_bitcmp", "s_nop", "s_waitcnt", "s_cbranch")):
                live = live - scalars(o[0])      # written anew by the scalar unit, which memory instructions wait for
            waits += int(o[0], 0) + 1 if op == "s_nop" else 1
            if target is not None:
                todo.append((at[target], waits, live))
            if op != "s_branch":
                todo.append((j + 1, waits, live))
    return found


WRITE = ("v_readlane_b32 s5, v1, s9", "")
LOAD = ("global_load_lds_dwordx4 v2, s[4:5]", "")
OTHER = ("v_mov_b32_e32 v12, v13", "")


@pytest.mark.parametrize("body,short", [
    ([WRITE, LOAD], 1), ([WRITE, (LOAD[0] + " offset:16 nt", "")], 1), ([WRITE, ("s_mov_b32 m0, s7", ""), ("s_nop 0", ""), LOAD], 1), ([WRITE, ("s_nop 3", ""), LOAD], 1),
    ([WRITE, ("s_nop 4", ""), LOAD], 0), ([WRITE] + [OTHER] * 4 + [LOAD], 1), ([WRITE] + [OTHER] * 5 + [LOAD], 0),
    ([WRITE, ("s_mov_b32 s5, s8", ""), LOAD], 0), ([WRITE, ("global_load_dword v3, v4, s[6:7]", "")], 0),
    ([("v_cmp_eq_u32_e64 s[4:5], v1, v2", ""), LOAD], 1), ([("v_add_co_u32 v3, s[4:5], v1, v2", ""), LOAD], 1),
    # a branch around ten other instructions: the direct way has one wait state
    ([WRITE, ("s_cbranch_scc1 11", " <f+0x30>")] + [OTHER] * 10 + [LOAD], 1)])
def test_counting(body, short):
    code = parse(_listing(body))["f"]
    assert len(code) == len(body) and len(shortfalls(code)) == short


def test_library(tmp_path):
    objdump = os.path.join(LLVM, "llvm-objdump")
    if not os.path.exists(objdump) or not os.path.exists(spire.LIB_PATH):
        pytest.skip("needs llvm-objdump and the built library")
    lib = shutil.copy(spire.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([objdump, "--offloading", str(lib)], cwd=tmp_path, check=True, capture_output=True)
    objects = sorted(p for p in os.listdir(tmp_path) if "gfx950" in p)
    assert objects
    copies, bad = 0, []
    for obj in objects:
        text = subprocess.run([objdump, "-d", "--mcpu=gfx950", str(tmp_path / obj)], check=True, capture_output=True,
                              text=True).stdout
        for name, code in parse(text).items():
            copies += sum(ins[0].startswith("global_load_lds") for ins in code)
            bad += [(name,) + b for b in shortfalls(code)]
    assert copies > 100
    assert not bad, f"{len(bad)} short, first {bad[:3]}"
