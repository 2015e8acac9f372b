"""What the compiler cannot check of tile loads written out in assembly, on the built library's code.

Linear attention's bf16 kernels load tiles from memory straight into LDS by instructions that the
compiler neither counts nor schedules (la_landed waits for them, LaLoad writes m0 before them).  Every
path through every such kernel is walked here:
  * a wave meets a barrier only with its loads into LDS landed: the waves behind it read the tile.
    vmcnt(n) leaves the n youngest memory instructions in flight, so a load has landed if at least n
    were issued behind it;
  * a scalar write of m0, the loads' LDS address, is one wait state ahead of the load;
  * scalar registers of the load's buffer come from vector instructions five wait states before.
"""

import os
import re
import shutil
import subprocess

import pytest

import paper_2605_22791_amd as g2

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
LANDED = 1 << 20  # no load under way

pytestmark = pytest.mark.skipif(not os.path.exists(g2.lib_path()) or not os.path.exists(OBJDUMP),
                                reason="libgdr2.so not built, or no llvm-objdump")


def _parse(text):
    """Kernel name -> list of (address, mnemonic, operands, branch target or None)."""
    out, code = {}, None
    for line in text.splitlines():
        head = re.match(r"^([0-9a-f]+) <(\S+)>:", line)
        if head:
            base, code = int(head[1], 16), out.setdefault(head[2], [])
            continue
        ins = re.match(r"^\t(\S+)\s*(.*?)\s*// ([0-9A-F]{12}):(.*)$", line)
        if ins is None or code is None:
            continue
        to = re.search(r"<[^>+]+(?:\+0x([0-9a-f]+))?>", ins[4]) if "branch" in ins[1] else None
        code.append((int(ins[3], 16), ins[1], ins[2], base + int(to[1] or "0", 16) if to else None))
    return out


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """The kernels that load into LDS."""
    at = tmp_path_factory.mktemp("isa")
    shutil.copy(g2.lib_path(), at / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, check=True, capture_output=True)
    found = {}
    for f in sorted(os.listdir(at)):
        if "amdgcn" in f:
            text = subprocess.run([OBJDUMP, "-d", f], cwd=at, check=True, capture_output=True, text=True).stdout
            found.update({n: c for n, c in _parse(text).items() if any(_to_lds(i) for i in c)})
    return found


def _to_lds(ins):
    return ins[1].startswith(("buffer_load", "global_load")) and ins[2].split()[-1] == "lds"


def _memory(ins):
    return re.match(r"(buffer|global|flat|scratch)_(load|store|atomic)", ins[1]) is not None


def _barriers_with_loads_under_way(code):
    """Addresses of the barriers that a wave can meet with a load into LDS under way."""
    index = {ins[0]: i for i, ins in enumerate(code)}
    # memory instructions issued behind the youngest load that may not have landed; the fewest of all ways there
    state, work = {0: LANDED}, [0]
    bad = set()
    while work:
        i = work.pop()
        s, ins = state[i], code[i]
        name, operands = ins[1], ins[2]
        if name == "s_barrier" and s != LANDED:
            bad.add(ins[0])
        wait = re.search(r"vmcnt\((\d+)\)", operands) if name == "s_waitcnt" else None
        if _to_lds(ins):
            s = 0
        elif s != LANDED and _memory(ins):
            s = min(s + 1, 63)
        elif wait and s >= int(wait[1]):
            s = LANDED
        assert name not in ("s_setpc_b64", "s_swappc_b64"), "a call: its instructions are not followed"
        nexts = [] if name in ("s_endpgm", "s_branch") else [i + 1]
        if ins[3] is not None:
            nexts.append(index[ins[3]])
        for j in nexts:
            if j < len(code) and s < state.get(j, LANDED + 1):
                state[j] = s
                work.append(j)
    return bad


def _scalars(operands):
    regs = set()
    for a, b, c in re.findall(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b", operands):
        regs |= set(range(int(a), int(b) + 1)) if a else {int(c)}
    return regs


def _states(ins):
    return int(ins[2], 0) + 1 if ins[1] == "s_nop" else 1


def test_kernels_that_load_into_lds_are_found(kernels):
    names = " ".join(kernels)
    assert all(n in names for n in ("la_segstate_kernel", "la_scan_fwd_kernel", "la_scan_bwd_kernel"))


def test_loads_into_lds_have_landed_at_barriers(kernels):
    bad = {n: [hex(a) for a in sorted(b)] for n, b in ((n, _barriers_with_loads_under_way(c)) for n, c in kernels.items()) if b}
    assert not bad, bad


def test_m0_is_written_a_wait_state_before_a_load_into_lds(kernels):
    bad = [(n, hex(ins[0])) for n, code in kernels.items() for before, ins in zip(code, code[1:])
           if _to_lds(ins) and before[1].startswith("s_") and before[2].split(",")[0] == "m0"]
    assert not bad, (len(bad), bad[:4])


def test_buffers_of_loads_into_lds_are_not_fresh_from_vector_instructions(kernels):
    bad = []
    for n, code in kernels.items():
        for i, ins in enumerate(code):
            if not _to_lds(ins):
                continue
            need, ahead, j = _scalars(ins[2]), 0, i - 1
            while j >= 0 and ahead < 5:
                if code[j][1].startswith("v_") and need & _scalars(code[j][2].split(",")[0]):
                    bad.append((n, hex(ins[0])))
                    break
                ahead += _states(code[j])
                j -= 1
    assert not bad, (len(bad), bad[:4])


# ---- the walk itself, on a few lines -----------------------------------------
LOAD = "buffer_load_dwordx4 v1, s[0:3], 0 offen lds"
STORE = "buffer_store_dwordx4 v[0:3], v4, s[4:7], 0 offen"


@pytest.mark.parametrize("lines,bad", [
    ([LOAD, "s_barrier", "s_endpgm"], True),
    ([LOAD, "s_waitcnt vmcnt(0)", "s_barrier", "s_endpgm"], False),
    ([LOAD, LOAD, STORE, STORE, "s_waitcnt vmcnt(2)", "s_barrier", "s_endpgm"], False),
    ([LOAD, LOAD, STORE, STORE, "s_waitcnt vmcnt(3)", "s_barrier", "s_endpgm"], True),
    ([LOAD, "s_waitcnt lgkmcnt(0)", "s_barrier", "s_endpgm"], True),
    # a way round the store leaves fewer instructions behind the load than the wait counts on
    ([LOAD, ("s_cbranch_scc1", 3), STORE, "s_waitcnt vmcnt(1)", "s_barrier", "s_endpgm"], True),
    # around a loop: the load of one turn, the barrier of the next
    (["s_barrier", LOAD, STORE, ("s_cbranch_scc1", 0), "s_endpgm"], True),
    (["s_barrier", LOAD, STORE, "s_waitcnt vmcnt(1)", ("s_cbranch_scc1", 0), "s_endpgm"], False)])
def test_the_walk(lines, bad):
    code = []
    for i, line in enumerate(lines):
        name, _, operands = (line if isinstance(line, str) else line[0]).partition(" ")
        code.append((4 * i, name, operands, None if isinstance(line, str) else 4 * line[1]))
    assert bool(_barriers_with_loads_under_way(code)) is bad
