"""The kernels of the microscaled products as the compiler made them from this library's sources: what it does not see to inside of an asm block."""
import os
import re
import subprocess

import pytest

import paper_2508_00806_amd as adacc
from test_kernel_resources import BUNDLE, LLVM


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: its instructions} of the code object that holds the products"""
    if not os.path.exists(adacc.LIB_PATH) or not os.path.exists(LLVM + "llvm-objdump"):
        pytest.skip("needs the built library and the compiler's tools")
    d = tmp_path_factory.mktemp("instructions")
    whole, part, code = d / "bundles", d / "bundle", d / "co"
    subprocess.run([LLVM + "llvm-objcopy", "--dump-section", f".hip_fatbin={whole}", adacc.LIB_PATH, os.devnull], check=True)
    data = whole.read_bytes()
    starts = [m.start() for m in re.finditer(BUNDLE, data)] + [len(data)]
    (ours,) = [data[a:b] for a, b in zip(starts, starts[1:]) if b"mx4_product_kernel" in data[a:b]]
    part.write_bytes(ours)
    subprocess.run([LLVM + "clang-offload-bundler", "--type=o", "--unbundle", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                    f"--input={part}", f"--output={code}"], check=True)
    text = subprocess.run([LLVM + "llvm-objdump", "-d", "--no-show-raw-insn", str(code)], check=True, capture_output=True, text=True).stdout
    found = {}
    parts = re.split(r"^[0-9a-f]+ <(\S+)>:\n", text, flags=re.M)
    for name, body in zip(parts[1::2], parts[2::2]):
        found[name] = [line.split("//")[0].strip() for line in body.splitlines() if line.strip()]
    assert any("mx4_product_kernel" in n for n in found) and any("mx4_gradient_kernel" in n for n in found)
    return found


def test_loads_to_lds_wait_for_the_registers_of_their_address(kernels):
    """Five wait states between a vector instruction's write of an SGPR and a vector load that reads it: right before each of these loads, whatever the compiler
    puts ahead of them (s_nop n is n + 1 wait states)."""
    loads = 0
    for name, lines in kernels.items():
        for i, line in enumerate(lines):
            if line.startswith("global_load_lds"):
                loads += 1
                wait = re.match(r"s_nop (\d+)", lines[i - 1])
                assert wait and int(wait.group(1)) + 1 >= 5, (name, lines[i - 2:i + 1])
    assert loads >= 6 * 10  # two kernels in three tile sizes, each with the first loads of a tile and those of its steps
