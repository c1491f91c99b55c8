"""64-bit vector shifts whose amount lies in the last register that a wave has, checked on the built library's gfx950 code
(no GPU needed).

Registers are given out eight at a time. Where the amount is in the last of them and nothing is behind it, such a shift
disturbs the first registers of the wave that comes next in the register file: with nothing but two register names
exchanged a kernel whose results were wrong in one launch of three was right in all. The compiler knows of no such rule for this
processor, so code is checked as it was built."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2608_20530_amd as L

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
SHIFT = re.compile(r"\s(?:v_(?:lshlrev|lshrrev)_b64|v_ashrrev_i64)\S* v\[\d+:\d+\], v(\d+),")


def last_register(text):
    """Number of the highest vector register that a function names."""
    return max((int(a or b) for a, b in re.findall(r"\bv(?:(\d+)\b|\[\d+:(\d+)\])", text)), default=-1)


def hits(text):
    """Shifts of a function whose amount is its last register, and the last of eight."""
    last = last_register(text)
    return [m[0].strip() for m in SHIFT.finditer(text) if int(m[1]) == last and last % 8 == 7]


def test_no_shift_amount_lies_in_the_last_register(tmp_path):
    assert os.path.exists(L.LIB_PATH), "the library is not built"
    lib = shutil.copy(L.LIB_PATH, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    functions = 0
    for obj in sorted(tmp_path.glob("*gfx950")):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(obj)], cwd=tmp_path, check=True,
                              capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=(?:[0-9a-f]+ )?<)", text):
            head, _, body = part.partition("\n")
            functions += "s_endpgm" in body
            code = "\n".join(line.split("//")[0] for line in body.splitlines())
            assert not hits(code), (head, hits(code))
    assert functions > 200


@pytest.mark.parametrize("amount,more,found", [(71, "", 1), (70, "v_mov_b32_e32 v71, 0", 0), (71, "v_mov_b32_e32 v72, 0", 0),
                                               (71, "global_load_dwordx4 v[72:75], v[0:1], off", 0), (69, "", 0)])
def test_one_is_noticed(amount, more, found):
    code = f"\tv_add_u32_e32 v{amount}, 28, v57\n\tv_lshlrev_b64 v[46:47], v{amount}, 1\n\t{more}\n\ts_endpgm"
    assert len(hits(code)) == found
