"""Matrix instructions' results are not read too early, checked on the built library's gfx950 code (no GPU needed).

The hardware does not hold a vector instruction back whose source a matrix instruction has still to write. The compiler
counts wait states for its own instructions and none for inline assembly, so code is checked as it was built: on every
path from a matrix instruction the first vector instruction, LDS or memory write that reads its result comes after
WAITS states at least (an instruction is one, s_nop n is n + 1), the number that the compiler keeps."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2608_20530_amd as L

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
WAITS = {"v_mfma_f32_16x16x4_f32": 10, "v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_32x32x16_bf16": 12,
         "v_mfma_f32_32x32x16_f16": 12}


def registers(operand):
    m = re.match(r"-?\|?([va])(?:(\d+)|\[(\d+):(\d+)\])", operand)
    if not m:
        return set()
    first, last = (int(m[2]),) * 2 if m[2] else (int(m[3]), int(m[4]))
    return {(m[1], i) for i in range(first, last + 1)}


def parse(lines):
    """Instructions of a function as (name, operands, number of the instruction that a branch goes to)."""
    at, code = {}, []
    for line in lines:
        text, _, note = line.strip().partition("//")
        address, _, rest = note.strip().partition(":")
        target = re.search(r"\+0x([0-9a-f]+)>", rest)
        at[int(address, 16)] = len(code)
        name, _, operands = text.strip().partition(" ")
        code.append((name, [o.strip() for o in operands.split(",")], target and int(target[1], 16)))
    start = min(at)
    return [(n, o, t if t is None else at[start + t]) for n, o, t in code]


def reads(name, operands):
    """Registers that a vector instruction, an LDS or a memory write reads."""
    if name.startswith("v_"):
        return set().union(*map(registers, operands[1:]))
    if re.match(r"ds_write|(global|buffer|flat|scratch)_(store|atomic)", name):
        return set().union(*(registers(o.split(" ")[0]) for o in operands))
    return set()


def too_early(code):
    """(matrix instruction, reader, wait states between them) of every pair that is too near."""
    found = []
    for i, (name, operands, _) in enumerate(code):
        if not name.startswith("v_mfma"):
            continue
        need, todo, seen = WAITS[name], [(i + 1, 0, frozenset(registers(operands[0])))], set()
        while todo:
            j, waited, live = todo.pop()
            while j < len(code) and waited < need and live and (j, waited) not in seen:
                seen.add((j, waited))
                op, args, target = code[j]
                if op.startswith("s_endpgm"):
                    break
                # a matrix instruction that takes the result as its own operand is held back by what the compiler puts there
                if not op.startswith("v_mfma") and reads(op, args) & live:
                    found.append((f"{name} {', '.join(operands)}", f"{op} {', '.join(args)}", waited))
                    break
                if op.startswith("v_"):
                    live -= registers(args[0])
                waited += int(args[0]) + 1 if op == "s_nop" else 1
                if op == "s_branch":
                    j = target
                    continue
                if op.startswith("s_cbranch"):
                    todo.append((target, waited, live))
                j += 1
    return found


@pytest.fixture(scope="module")
def functions(tmp_path_factory):
    assert os.path.exists(L.LIB_PATH), "the library is not built"
    d = tmp_path_factory.mktemp("code")
    lib = shutil.copy(L.LIB_PATH, d)
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=d, check=True, stdout=subprocess.DEVNULL)
    out = {}
    for obj in sorted(d.glob("*gfx950")):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(obj)], cwd=d, check=True, capture_output=True,
                              text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]+ <)", text):
            head, _, body = part.partition("\n")
            if "v_mfma" in body:
                out[head] = parse([x for x in body.splitlines() if x.startswith("\t") and "//" in x])
    return out


@pytest.mark.parametrize("kernel,least", [("attention4_kernel", 50), ("key_weights", 20), ("attention_kernel", 42), ("", 150)])
def test_results_are_waited_for(functions, kernel, least):
    some = {k: v for k, v in functions.items() if kernel in k}
    assert len(some) >= least
    for name, code in some.items():
        early = too_early(code)
        assert not early, (name, len(early), early[0])


def test_an_early_reader_is_noticed():
    def code(*lines):
        return parse([f"\t{x} // {4 * i:012X}: 00000000 {'<f+0x' + x.split('@')[1] + '>' if '@' in x else ''}"
                      for i, x in enumerate(lines)])
    product = "v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0"
    late = code(product, "s_nop 5", "v_add_f32 v20, v21, v22", "s_nop 0", "v_max3_f32 v9, v9, v3, v8", "s_endpgm")
    assert too_early(late) == []
    near = code(product, "s_nop 5", "v_max3_f32 v9, v9, v3, v8", "s_endpgm")
    assert [x[2] for x in too_early(near)] == [6]
    behind = code(product, "s_cbranch_scc0 1 @10", "s_nop 7", "s_branch 1 @14", "ds_write_b32 v30, v2", "s_endpgm")
    assert [x[2] for x in too_early(behind)] == [1]
    written = code(product, "v_mov_b32 v3, 0", "v_max3_f32 v9, v9, v3, v8", "s_endpgm")
    assert too_early(written) == []
