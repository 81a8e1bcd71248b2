"""Registers written to scratch memory, copied or read back while lanes are switched off.

Behind a conditional block all lanes are switched on again before anything else happens.  Where copies of scalar registers stood in
between, the compiler has put stores of vector registers to scratch memory before that instruction: lanes, and whole waves, that
skipped the block did not store, and later read back what scratch memory held from before.  (The sums of the delta rule's gradients,
spilled behind the staging of its gates, which the first six of eight waves do: wrong in the other two.)  This looks for it in the
assembly of all kernels."""
import concurrent.futures as cf
import os
import re

import pytest

from paper_2512_08061_amd import build
from test_matrix_waits import assembly, registers

VECTOR = ("v_", "ds_", "buffer_", "global_", "flat_", "scratch_")
WHATEVER_LANES = ("v_readlane", "v_writelane", "v_readfirstlane")  # (these do not ask which lanes are on)
SPILL, RELOAD = "Folded Spill", "Folded Reload"


def code_of(text):
    """Kernel -> its instructions (name, operands, comment), labels among them."""
    name, code = None, []
    for line in text.splitlines():
        if m := re.match(r"^(_Z\S+):", line):
            name, code = m.group(1), []
        elif name is None:
            continue
        elif line.startswith(".Lfunc_end"):
            yield name, code
            name = None
        elif m := re.match(r"^(\.LBB\S+):", line):
            code.append(("label", m.group(1), ""))
        elif (m := re.match(r"^\t([a-z]\S*)\s*(.*?)(;.*)?$", line)) and not line.startswith("\t."):
            code.append((m.group(1), m.group(2).strip(), m.group(3) or ""))


def switches(op, args):
    return op.startswith("s_") and (re.match(r"exec\b", args) is not None or "saveexec" in op)


def behind_blocks(code):
    """What stands between the place that lanes jump to around a block and the instruction that switches them on again."""
    at = {args: i for i, (op, args, _) in enumerate(code) if op == "label"}
    for label in {args for op, args, _ in code if op == "s_cbranch_execz"}:
        found = []
        for op, args, _ in code[at[label] + 1:]:
            if op == "label" or op.startswith(("s_cbranch", "s_branch", "s_endpgm")):
                break
            if switches(op, args):
                if op not in ("s_and_saveexec_b64", "s_mov_b64"):  # (these open a block: no lanes were off)
                    yield from found
                break
            if op.startswith(VECTOR) and not op.startswith(WHATEVER_LANES):
                found.append((label, op, args))


def within_blocks(code):
    """The same where the jump around a short block was left out: a register that the block has not written, stored within it, and
    anything read back within it."""
    written = None
    for op, args, comment in code:
        if op == "s_and_saveexec_b64":
            written = set()
        elif op == "label" or op.startswith(("s_cbranch", "s_branch")) or switches(op, args):
            written = None
        elif written is not None:
            if (SPILL in comment and not registers(args) & written) or RELOAD in comment:
                yield op, args
            if op.startswith("v_") or "load" in op or "read" in op:
                written |= registers(args.split(",")[0])


def lost(text):
    return [(name, *x) for name, code in code_of(text) for rule in (behind_blocks, within_blocks) for x in rule(code)]


def test_the_walk_finds_what_it_looks_for():
    around = ["_Zk:", "\ts_and_saveexec_b64 s[0:1], vcc", "\ts_cbranch_execz .LBB0_2", "\tds_write_b32 v1, v2", ".LBB0_2:",
              "\ts_mov_b32 s4, s5", "\tscratch_store_dwordx4 off, v[4:7], off ; 16-byte Folded Spill", "\ts_or_b64 exec, exec, s[0:1]",
              "\tv_mov_b32_e32 v4, 0", "\ts_endpgm", ".Lfunc_end0:"]
    assert len(lost("\n".join(around))) == 1
    around[6], around[7] = around[7], around[6]
    assert not lost("\n".join(around))
    straight = ["_Zk:", "\ts_and_saveexec_b64 s[0:1], vcc", "\tv_add_u32_e32 v1, v2, v3", "\tds_write_b32 v1, v2",
                "\tscratch_store_dword off, v9, off ; 4-byte Folded Spill", "\ts_or_b64 exec, exec, s[0:1]", "\ts_endpgm", ".Lfunc_end0:"]
    assert len(lost("\n".join(straight))) == 1
    assert not lost("\n".join(straight).replace("v9", "v1"))


SOURCES = [s for s in build.SOURCES if s.endswith(".hip")]


@pytest.fixture(scope="module")
def texts(tmp_path_factory):
    folder = tmp_path_factory.mktemp("assembly")
    with cf.ThreadPoolExecutor(8) as pool:
        return dict(zip(SOURCES, pool.map(lambda s: assembly(s, str(folder / (s + ".s"))), SOURCES)))


@pytest.mark.parametrize("source", SOURCES)
def test_no_register_is_spilled_with_lanes_off(source, texts):
    found = lost(texts[source])
    assert not found, "\n".join(map(str, found))
