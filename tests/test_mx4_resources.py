"""The kernels of the microscaled matrices keep no vector registers in scratch memory."""
import re

from test_kernel_resources import spills  # noqa: F401  (the fixture)


def test_no_vector_register_is_spilled(spills):  # noqa: F811
    ours = {n: s for n, s in spills.items() if re.search(r"\d+mx4_\w+_kernel", n)}
    for kernel in ("along", "across", "restore", "product", "gradient", "few"):
        assert any(f"mx4_{kernel}_kernel" in n for n in ours), kernel
    assert {n: s for n, s in ours.items() if s} == {}
