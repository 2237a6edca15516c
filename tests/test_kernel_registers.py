"""No kernel of the built library keeps vector registers in memory, in any of its code objects (one for each source), and
every kernel of the sources is there (no GPU: the resource counts in the code objects' metadata). A spill costs trips to
memory in a loop that was made to have none."""
import glob
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2502_00922_amd", "libhufflm.so")
LLVM = "/opt/rocm/llvm/bin"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: (vector registers spilled, bytes of private memory a lane)} of every code object."""
    if not os.path.exists(LIB):
        pytest.skip("library not built")
    tmp = tmp_path_factory.mktemp("code")
    run = lambda *a: subprocess.run(a, check=True, capture_output=True, text=True).stdout  # noqa: E731
    fat, part, obj = (str(tmp / name) for name in ("fat", "part", "obj"))
    run(f"{LLVM}/llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", LIB, str(tmp / "copy"))
    data, found = open(fat, "rb").read(), {}
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)]
    for begin, end in zip(starts, [*starts[1:], len(data)]):
        with open(part, "wb") as f:
            f.write(data[begin:end])
        run(f"{LLVM}/clang-offload-bundler", "--unbundle", "--type=o", f"--input={part}", f"--output={obj}",
            "--targets=hipv4-amdgcn-amd-amdhsa--gfx950")
        notes = run(f"{LLVM}/llvm-readelf", "--notes", obj)
        for kernel in notes.split("- .agpr_count")[1:]:
            value = lambda key: re.search(rf"\.{key}:\s+(\S+)", kernel).group(1)  # noqa: E731
            found[value("name")] = int(value("vgpr_spill_count")), int(value("private_segment_fixed_size"))
    return found


def test_every_kernel_is_looked_at(kernels):
    named = set()
    for source in glob.glob(os.path.join(ROOT, "paper_2502_00922_amd", "csrc", "*.hip")):
        named |= set(re.findall(r"__global__[^;{]*?(\w+_kernel)\(", open(source).read()))
    assert {"gemv_stream_kernel", "norm_kernel", "parts_kernel", "solo_kernel", "join_kernel", "weights_kernel",
            "select_kernel", "move_kernel"} <= named
    missing = [name for name in named if not any(f"{len(name)}{name}" in kernel for kernel in kernels)]
    assert not missing, missing


def test_no_vector_register_in_memory(kernels):
    spilled = {name: counts for name, counts in kernels.items() if counts != (0, 0)}
    assert not spilled, spilled
