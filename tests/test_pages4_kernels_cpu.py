"""Which attention kernels over pages of 4 bits the library holds: those that some call reaches, and no other."""
import re

from test_pages_cpu import lib  # noqa: F401


def test_no_kernel_that_no_call_reaches(lib):  # noqa: F811
    with open(lib.load_library()._name, "rb") as f:
        names = set(re.findall(rb"attend_(?:thin|pair|tile|few)_kernel(?:ILb[01]E|ILi\d+E|Lb[01]E|Li\d+E)+E", f.read()))
    assert len(names) > 20
    four = {n.decode() for n in names if b"Li%dE" % lib.LRQK_PAGE_E2M1 in n or b"few" in n}
    assert four == {
        "attend_few_kernelILi1ELb1EE", "attend_few_kernelILi2ELb1EE", "attend_few_kernelILi1ELb0EE",   # <sets of 16 rows, bf16>
        "attend_tile_kernelILb1ELi8EE",                                                                # <bf16, pages>: prompts
        "attend_thin_kernelILb1ELi8ELb1EE", "attend_thin_kernelILb0ELi8ELb1EE"}                        # pages of less than 16 positions
