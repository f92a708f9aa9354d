"""The same properties of the 4-bit cache's kernels as tests/test_kernel_isa.py checks of the others (no GPU needed): no
scalar load with a register offset, and no scratch memory."""
import pytest

from tests.test_kernel_isa import FORM, assembly, scratch_bytes

KERNELS = {"lychee_q4.hip": 2 + 3 * 4, "lychee_topk.hip": 1, "lychee_pages.hip": 2}


@pytest.mark.parametrize("source", sorted(KERNELS))
def test_no_register_offset_and_no_scratch(source):
    text = assembly(source)
    hits = [line.strip() for line in text.splitlines() if FORM.match(line)]
    assert not hits, "scalar loads with a register offset: %s" % hits[:5]
    sizes = scratch_bytes(text)
    assert len(sizes) == KERNELS[source] and all(v == 0 for v in sizes.values()), sizes
