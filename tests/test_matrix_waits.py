"""Wait states behind matrix products in the compiled kernels.

The result of a matrix instruction lies in its registers some wait states after it was issued, and the compiler fills these
with s_nop where need be.  Behind a short conditional block it has left out some of them on the path around the block.  This
walks all paths of the kernels' own assembly from every matrix instruction to the first other instruction that reads or
writes its result."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from paper_2512_08061_amd import build

# wait states until a result may be read or written: passes + 2 of fp32 products (8 passes), + 4 of bf16 ones (4, 8)
NEED = {"v_mfma_f32_16x16x4_f32": 10, "v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_32x32x16_bf16": 12}
STORES = ("ds_write", "buffer_store", "global_store", "flat_store", "scratch_store")


def registers(text):
    out = set()
    for m in re.finditer(r"\b([av])(\d+)\b|\b([av])\[(\d+):(\d+)\]", text):
        if m.group(1):
            out.add((m.group(1), int(m.group(2))))
        else:
            out.update((m.group(3), i) for i in range(int(m.group(4)), int(m.group(5)) + 1))
    return out


def kernels(text):
    """Kernel -> its basic blocks [(instructions, indices of the blocks that may follow)]."""
    found, name = {}, None
    for line in text.splitlines():
        if m := re.match(r"^(_Z\S+):", line):
            name = m.group(1)
            found[name] = [("", [])]
        elif name is None:
            continue
        elif line.startswith(".Lfunc_end"):
            name = None
        elif m := re.match(r"^(\.LBB\S+):", line):
            found[name].append((m.group(1), []))
        elif (m := re.match(r"^\t([a-z]\S*)\s*(.*?)(;.*)?$", line)) and not line.startswith("\t."):
            found[name][-1][1].append((m.group(1), m.group(2).strip()))
    for name, labelled in found.items():
        blocks, at = [], {}
        for label, code in labelled:
            at[label] = len(blocks)
            part = []
            for op in code:
                part.append(op)
                if op[0].startswith(("s_cbranch", "s_branch", "s_endpgm")):
                    blocks.append(part)
                    part = []
            blocks.append(part)
        follow = []
        for i, code in enumerate(blocks):
            last = code[-1] if code else ("", "")
            to = [at[last[1]]] if last[0].startswith(("s_cbranch", "s_branch")) else []
            if not last[0].startswith(("s_branch", "s_endpgm")) and i + 1 < len(blocks):
                to.append(i + 1)
            follow.append(to)
        yield name, list(zip(blocks, follow))


def early(blocks):
    """(matrix instruction, the instruction that touches its result too early, wait states between them)."""
    for b, (code, _) in enumerate(blocks):
        for i, (op, args) in enumerate(code):
            if not op.startswith("v_mfma"):
                continue
            need, result = NEED[op], registers(args.split(",")[0])
            work, least = [(b, i + 1, 0)], {}
            while work:
                at, k, waited = work.pop()
                code_at, follow = blocks[at]
                for name, text in code_at[k:]:
                    if waited >= need:
                        break
                    if name.startswith("v_mfma"):  # (as the sum that it adds to, a result needs no wait)
                        to, *operands = text.split(",")
                        if registers(",".join(operands[:2])) & result:
                            yield f"{op} {args}", f"{name} {text}", waited
                            break
                        if registers(to) & result:
                            break
                    elif name.startswith(("v_", "ds_", "buffer_", "global_", "flat_", "scratch_")) and registers(text) & result:
                        yield f"{op} {args}", f"{name} {text}", waited
                        break
                    waited += int(text, 0) + 1 if name == "s_nop" else 1
                else:
                    for to in follow:
                        if waited < need and waited < least.get(to, need):
                            least[to] = waited
                            work.append((to, 0, waited))


def assembly(source, to):
    cmd = [build.HIPCC, "-x", "hip", *build.FLAGS, "-S", "--offload-device-only", os.path.join(build.CSRC, source), "-o", to]
    subprocess.run(cmd, check=True, capture_output=True)
    with open(to) as f:
        return f.read()


def test_the_walk_finds_what_it_looks_for():
    text = "\n".join(["_Zk:", "\tv_mfma_f32_16x16x4_f32 v[0:3], v4, v5, v[0:3]", "\ts_cbranch_execz .LBB0_2", "\ts_nop 9", "\tv_mov_b32_e32 v9, v8",
                      ".LBB0_2:", "\tv_add_f32_e32 v6, v1, v7", "\ts_endpgm", ".Lfunc_end0:"])
    (name, blocks), = kernels(text)
    assert [x[2] for x in early(blocks)] == [1]  # around the block, not through it
    (name, blocks), = kernels(text.replace("s_cbranch_execz .LBB0_2", "s_nop 8"))
    assert not list(early(blocks))


SOURCES = ["luna_chunk_query.hip", "luna_chunk_key.hip", "luna_map_backward.hip", "luna_softmax.hip", "luna_softmax_split.hip",
           "luna_softmax_bwd.hip"] + [f"luna_decay_{t}_{m}.hip" for t in ("bf16", "f32") for m in ("plain", "norm", "aug")]


@pytest.fixture(scope="module")
def texts(tmp_path_factory):
    folder = tmp_path_factory.mktemp("assembly")
    with cf.ThreadPoolExecutor(8) as pool:
        return dict(zip(SOURCES, pool.map(lambda s: assembly(s, str(folder / (s + ".s"))), SOURCES)))


@pytest.mark.parametrize("source", SOURCES)
def test_results_of_matrix_products_are_waited_for(source, texts):
    found = [f"{name}: {a} -> {b}: {n}" for name, blocks in kernels(texts[source]) for a, b, n in early(blocks)]
    assert not found, "\n".join(found)
