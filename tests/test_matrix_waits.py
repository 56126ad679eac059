"""How long after a matrix instruction its result is read in the compiled kernels of the gated delta rule, over all paths of their code (hipcc cross-compiles, so no GPU is needed).

A wave has to leave some wait states (instructions, and what s_nop adds) between a matrix instruction and an instruction of another kind that reads its result: the compiler
leaves 8 after v_mfma_f32_16x16x32_bf16 and 10 after v_mfma_f32_16x16x4_f32 where both stand in one line of code.  Products behind uniform branches once gave wrong results in a
kernel that is no longer there, and no cause was found; so the waits are checked across branches too, and the preparation of chunks, which that was seen in, reads its products before it branches."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_11681_amd", "csrc")
WAIT = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}
FAR = 24
NO_RESULT = re.compile(r"global_store|ds_write|buffer_store|scratch_store|s_|v_cmp|v_readfirst")


def registers(operands):
    found = set()
    for kind, first, last, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", operands):
        found |= {(kind, r) for r in range(int(first or one), int(last or one) + 1)}
    return found


def read_and_written(op, operands):
    """Registers that an instruction writes, and reads; of a matrix instruction the accumulator that it goes on from counts as written alone."""
    parts = [p.strip() for p in re.findall(r"(?:\[[^\]]*\]|[^,\[])+", operands)]
    if op.startswith("v_mfma"):
        return registers(",".join(parts[:1] + parts[3:4])), registers(",".join(parts[1:3]))
    if NO_RESULT.match(op):
        return set(), registers(operands)
    return registers(parts[0]) if parts else set(), registers(",".join(parts[1:]))


def blocks_of(text):
    """Basic blocks of a kernel's listing: their instructions (name, operands, registers written, registers read), and the blocks that may follow."""
    blocks, labels = [[]], {}
    for line in text.split("\n"):
        line = line.split(";")[0].rstrip()
        if m := re.match(r"^(\.L\w+):", line):
            blocks.append([])
            labels[m.group(1)] = len(blocks) - 1
        elif (m := re.match(r"^\s+([a-z]\w+)\s*(.*)$", line)):
            op, operands = m.groups()
            blocks[-1].append((op, operands, *read_and_written(op, operands)))
            if op.startswith("s_cbranch") or op in ("s_branch", "s_endpgm"):
                blocks.append([])
    follow = []
    for i, block in enumerate(blocks):
        op, operands = block[-1][:2] if block else ("", "")
        after = [] if op in ("s_branch", "s_endpgm") else [i + 1]
        if op.startswith("s_cbranch") or op == "s_branch":
            after.append(labels.get(operands.strip(), len(blocks)))
        follow.append([a for a in after if a < len(blocks)])
    return blocks, follow


def waits(text):
    """(matrix instruction, whether a branch lies between) -> fewest wait states before another instruction reads its result, up to FAR."""
    blocks, follow = blocks_of(text)
    fewest = {}
    for i, block in enumerate(blocks):
        for k, (op, operands, written, _) in enumerate(block):
            if not op.startswith("v_mfma"):
                continue
            result = registers(operands.split("]")[0] + "]")
            paths, seen = [(i, k + 1, 0, False, frozenset(result))], {}
            while paths:
                at, j, states, branched, live = paths.pop()
                while live and states <= FAR:
                    if j == len(blocks[at]):
                        jumps = bool(blocks[at]) and blocks[at][-1][0].startswith(("s_cbranch", "s_branch"))
                        for b in follow[at]:
                            if seen.get((b, live), FAR + 1) > states:
                                seen[b, live] = states
                                paths.append((b, 0, states, branched or jumps, live))
                        break
                    name, args, writes, reads = blocks[at][j]
                    if live & reads:
                        if not name.startswith("v_mfma"):
                            key = (op, branched)
                            fewest[key] = min(states, fewest.get(key, FAR))
                        live = live - reads
                    live = live - writes
                    states += int(args, 0) + 1 if name == "s_nop" else 1
                    j += 1
    return fewest


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("listing") / "deltarule.s"
    subprocess.run(["hipcc", "--cuda-device-only", "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-S", "-o", str(out), os.path.join(CSRC, "deltarule.hip")], check=True, capture_output=True, timeout=600)
    found = {m.group(1): m.group(2) for m in re.finditer(r"^(_Z\w+):[^\n]*\n(.*?)^\.Lfunc_end", out.read_text(), flags=re.S | re.M)}
    assert len([n for n in found if "k_delta" in n]) > 40
    return found


def test_the_reader_of_listings():
    text = """
\tv_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], 0
\tv_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]
\ts_nop 3
\ts_cbranch_scc0 .LBB0_2
\tv_mov_b32_e32 v9, v8
\tv_accvgpr_read_b32 v8, a2
.LBB0_2:
\tv_accvgpr_read_b32 v8, a3
\ts_endpgm
"""
    assert waits(text) == {("v_mfma_f32_16x16x32_bf16", True): 5}
    assert waits(text.replace("\ts_cbranch_scc0 .LBB0_2\n", "")) == {("v_mfma_f32_16x16x32_bf16", False): 5}


def test_results_of_products_are_read_late_enough_on_every_path(kernels):
    for name, text in kernels.items():
        for (op, branched), states in waits(text).items():
            assert states >= WAIT[op], (name, op, branched, states)


def test_preparation_reads_its_products_before_it_branches(kernels):
    names = [n for n in kernels if "k_delta_prepare" in n]
    assert len(names) == 12
    for name in names:
        found = waits(kernels[name])
        assert ("v_mfma_f32_16x16x32_bf16", False) in found and ("v_mfma_f32_16x16x32_bf16", True) not in found, (name, found)


def test_no_assembly_writes_registers_that_it_does_not_declare():
    """m0 is the compiler's own: it may hold a value there across an assembly statement, which cannot declare that it changes it."""
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            for statement in re.findall(r"\basm\b[^;]*;", f.read()):
                assert not re.search(r"\bm0\b", statement), (name, statement)
