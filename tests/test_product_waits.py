"""No instruction of the built point-wise product kernels reads a matrix instruction's result before it is there, along every path of the built code
(what may go wrong, and how it is found, stands in tests/test_window_waits.py)."""
import re

import pytest

from tests.test_abi_host import code_objects, kernel_notes, lib  # noqa: F401
from tests.test_window_waits import functions, too_early


@pytest.mark.parametrize("kernel", [b"product_kernel", b"product_thin_kernel", b"product_weights_kernel", b"strip_kernel", b"strip_back_kernel"])
def test_products_are_there_before_they_are_read(kernel):
    products = 0
    for text in code_objects(("llvm-objdump", "-d", "--no-show-raw-insn"), kernel):
        for name, code, jumps in functions(text):
            if kernel.decode() in name:
                products += sum(op.startswith("v_mfma") for op, _ in code)
                assert not too_early(code, jumps), (name, too_early(code, jumps)[:3])
    assert products > 10


def test_kernels_use_no_scratch(lib):  # noqa: F811
    found = [k for k in kernel_notes() if re.search("product_(thin_|weights_)?kernel|strip_(back_)?kernel|norm_(back_|weights_)?(any_)?kernel|dropout_kernel|parts_kernel", k[0])]
    assert len(found) > 200
    for name, scratch, vgprs, lds in found:
        assert scratch == 0 and vgprs <= 256 and lds <= 80 * 1024, (name, scratch, vgprs, lds)
