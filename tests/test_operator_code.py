"""What the compiler made of the operators' kernels (no GPU: the gfx950 code objects of the built library), where code
of some kinds has given wrong results on the GPU now and then."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2502_00922_amd", "libhufflm.so")
LLVM = "/opt/rocm/llvm/bin"
KERNELS = ("norm_kernel", "parts_kernel", "solo_kernel", "join_kernel", "weights_kernel", "select_kernel", "move_kernel")
VECTOR = r"([va])(?:\[(\d+):(\d+)\]|(\d+))"


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    """(kernel, instructions, vector registers) of each of the operators' kernels."""
    if not os.path.exists(LIB):
        pytest.skip("library not built")
    tmp = tmp_path_factory.mktemp("code")
    fat = str(tmp / "fat")
    subprocess.run([f"{LLVM}/llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", LIB, str(tmp / "copy")], check=True)
    data, found = open(fat, "rb").read(), []
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)]
    for i, at in enumerate(starts):
        part, obj = str(tmp / f"part{i}"), str(tmp / f"obj{i}")
        with open(part, "wb") as f:
            f.write(data[at:starts[i + 1] if i + 1 < len(starts) else len(data)])
        subprocess.run([f"{LLVM}/clang-offload-bundler", "--unbundle", "--type=o", f"--input={part}", f"--output={obj}",
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
        notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", obj], check=True, capture_output=True, text=True).stdout
        counts = {n: int(c) for n, c in re.findall(r"\.name:\s+(\S+).*?\.vgpr_count:\s+(\d+)", notes, re.S)}
        if not any(k in n for n in counts for k in KERNELS):
            continue
        text = subprocess.run([f"{LLVM}/llvm-objdump", "-d", "--no-show-raw-insn", obj], check=True, capture_output=True,
                              text=True).stdout
        for block in re.split(r"\n(?=[0-9a-f]+ <)", text):
            name = re.match(r"[0-9a-f]+ <(\S+)>:", block)
            if name and name.group(1) in counts and any(k in name.group(1) for k in KERNELS):
                lines = [line.split("//")[0].strip() for line in block.splitlines()[1:] if line.startswith("\t")]
                found.append((name.group(1), lines, counts[name.group(1)]))
    return found


def span(m):
    """(file, first, last) of a matched register operand."""
    return (m.group(1), int(m.group(2)), int(m.group(3))) if m.group(2) else (m.group(1), int(m.group(4)), int(m.group(4)))


def test_matrix_operands_are_not_overwritten_at_once(listing):
    # within five wait states of a matrix instruction no vector instruction writes its left or right operand
    products, bad = 0, []
    for kernel, lines, _ in listing:
        recent = []  # (wait states since, operands)
        for line in lines:
            nop = re.match(r"s_nop (\d+)", line)
            states = int(nop.group(1)) + 1 if nop else 1
            operands = [span(m) for m in re.finditer(VECTOR, line)]
            matrix = line.startswith("v_mfma")
            if line.startswith("v_") and not matrix and not line.startswith("v_cmp") and operands:
                f, a, b = operands[0]
                bad += [(kernel, line) for _, ops in recent for g, c, d in ops if f == g and a <= d and c <= b]
            recent = [(n + states, ops) for n, ops in recent if n + states < 5]
            if matrix:
                products += 1
                recent.append((0, operands[1:3]))
    assert products > 1000, products
    assert not bad, bad[:5]


def test_no_shift_count_in_the_last_register(listing):
    bad = []
    for kernel, lines, registers in listing:
        for line in lines:
            m = re.match(r"v_(?:lshlrev_b64|lshrrev_b64|ashrrev_i64)\S*\s+v\[\d+:\d+\], v(\d+),", line)
            if m and int(m.group(1)) == (registers + 7) // 8 * 8 - 1:
                bad.append((kernel, line))
    assert listing and not bad, bad


def test_no_packed_float32(listing):
    # some forms of v_pk_add_f32, v_pk_mul_f32 and v_pk_fma_f32 have given wrong results
    bad = [(kernel, line) for kernel, lines, _ in listing for line in lines if re.match(r"v_pk_(add|mul|fma)_f32", line)]
    assert not bad, bad[:5]
