"""The kernels of the microscaled products as the compiler made them from this library's sources: what it does not see to around an asm block."""
import os
import re
import subprocess

import pytest

import paper_2508_00806_amd as adacc
from test_kernel_resources import BUNDLE, LLVM

NEEDED = 5  # wait states between a vector instruction's write of an SGPR and a vector load that reads it


class Kernel:
    def __init__(self, text):
        """The lines of a disassembled function: instruction // address: ... <function+offset of a branch's target>"""
        self.lines, self.before = [], []
        address, targets = {}, []
        for line in text.splitlines():
            m = re.match(r"\s+(\S.*?)\s*// ([0-9A-F]+):(.*)", line)
            if m:
                address[int(m.group(2), 16)] = len(self.lines)
                to = re.search(r"<\S+\+0x([0-9a-f]+)>", m.group(3))
                if to:
                    targets.append((len(self.lines), int(to.group(1), 16)))
                self.lines.append(m.group(1))
        first = min(address)
        # what may have come right before each instruction
        ends = re.compile(r"s_branch|s_endpgm|s_setpc")
        self.before = [[i - 1] if i and not ends.match(self.lines[i - 1]) else [] for i in range(len(self.lines))]
        for at, to in targets:
            assert self.lines[at].startswith(("s_branch", "s_cbranch")), self.lines[at]
            self.before[address[first + to]].append(at)

    def vector_writes_before(self, at, states):
        """[(scalar registers that a vector instruction writes, the instruction)] within so many wait states before instruction `at`"""
        found, seen, todo = [], {}, [(i, 0) for i in self.before[at]]
        while todo:
            i, passed = todo.pop()
            if seen.get(i, states) <= passed:
                continue
            seen[i] = passed
            line = self.lines[i]
            if line.startswith("v_"):
                registers = scalar_results(line)
                if registers:
                    found.append((registers, line))
            wait = re.match(r"s_nop (\d+)", line)
            passed += int(wait.group(1)) + 1 if wait else 1
            if passed < states:
                todo += [(j, passed) for j in self.before[i]]
        return found


def scalars(operand):
    m = re.match(r"s\[(\d+):(\d+)\]$|s(\d+)$", operand)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1)) if m.group(1) else {int(m.group(3))}
    return {operand} if operand in ("m0", "vcc", "vcc_lo", "vcc_hi") else set()


def scalar_results(line):
    """The scalar registers that a vector instruction writes: its first operand, or of those with a carry the second too."""
    name, _, rest = line.partition(" ")
    operands = [o.strip() for o in rest.split(",")]
    written = scalars(operands[0])
    if "_co_" in name or name.startswith(("v_mad_u64", "v_mad_i64", "v_div_scale")):
        written |= scalars(operands[1])
    return written


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: Kernel} of the code object that holds the products"""
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
    text = subprocess.run([LLVM + "llvm-objdump", "-d", str(code)], check=True, capture_output=True, text=True).stdout
    parts = re.split(r"^[0-9a-f]+ <(\S+)>:\n", text, flags=re.M)
    return {name: Kernel(body) for name, body in zip(parts[1::2], parts[2::2]) if "mx4_" in name}


def loads_to_lds(kernels):
    found = [(name, k, i) for name, k in kernels.items() for i, line in enumerate(k.lines) if line.startswith("global_load_lds")]
    assert len({name for name, _, _ in found}) == 6  # products and gradients in three tile sizes
    assert len(found) >= 6 * 10
    return found


def test_loads_to_lds_find_the_registers_of_their_address_ready(kernels):
    for name, k, i in loads_to_lds(kernels):
        reads = scalars(k.lines[i].split(",")[-1].strip().split(" ")[0]) | {"m0"}
        assert len(reads) == 3, k.lines[i]
        for written, line in k.vector_writes_before(i, NEEDED):
            assert not written & reads, (name, line, k.lines[i])


def test_m0_belongs_to_the_loads_to_lds(kernels):
    """m0 is written for such loads alone, by scalar instructions, and every block waits the state between the write and its load."""
    for name, k, i in loads_to_lds(kernels):
        assert k.lines[i - 1] == "s_nop 0", (name, k.lines[i - 3:i + 1])
    for name, k in kernels.items():
        users = [line for line in k.lines if re.search(r"\bm0\b", line)]
        assert all(re.match(r"s_\w+ m0, (?!.*\bm0\b)", line) for line in users), name
        assert len(users) <= sum(line.startswith("global_load_lds") for line in k.lines), name


def test_no_asm_block_writes_m0_without_the_compilers_knowing():
    """(m0 is reserved: a block can not name it as overwritten.  As an operand the compiler writes it itself.)"""
    folder = os.path.join(os.path.dirname(os.path.abspath(adacc.__file__)), "csrc")
    for f in os.listdir(folder):
        with open(os.path.join(folder, f)) as source:
            for block in re.findall(r"asm(?:\s+volatile)?\s*\((.*?)\);", source.read(), re.S):
                assert not re.search(r"\bm0\s*,", block.split(":")[0]), (f, block)


def test_the_search_finds_what_it_looks_for():
    """Planted in the text: a write four states before a load, one on the way of a branch to it, one far enough off."""
    def kernel(*lines):
        return Kernel("\n".join(f"\t{line:40s} // {16 * i:012X}: 00 {rest}" for i, (line, _, rest) in enumerate(l.partition(" @") for l in lines)))
    load = "global_load_lds_dwordx4 v1, s[4:5]"
    near = kernel("v_readlane_b32 s5, v9, 3", "s_nop 2", load)
    assert near.vector_writes_before(2, NEEDED) == [({5}, "v_readlane_b32 s5, v9, 3")]
    assert kernel("v_readlane_b32 s5, v9, 3", "s_nop 3", "s_nop 0", load).vector_writes_before(3, NEEDED) == []
    round_ = kernel("s_nop 7", load, "s_nop 0", "v_add_co_u32_e64 v1, s[4:5], v2, v3", "s_cbranch_scc1 65533 @<kernel+0x10>", "s_endpgm")
    assert round_.vector_writes_before(1, NEEDED) == [({4, 5}, "v_add_co_u32_e64 v1, s[4:5], v2, v3")]
    assert kernel("v_readfirstlane_b32 s4, v1", "s_branch 2 @<kernel+0x30>", "s_nop 0", load).vector_writes_before(3, NEEDED) != []
