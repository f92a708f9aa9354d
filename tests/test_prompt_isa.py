"""The same properties of the kernels of attention over prompts as tests/test_kernel_isa.py checks of the others (no GPU needed):
no scalar load with a register offset; no scratch memory, but for one register at a tile's beginning in the kernel that shares
out tiles over the 4-bit cache."""
import pytest

from tests.test_kernel_isa import FORM, assembly, scratch_bytes

KERNELS = {"lychee_prompt.hip": 5, "lychee_prompt_grad.hip": 5}


@pytest.mark.parametrize("source", sorted(KERNELS))
def test_no_register_offset_and_no_scratch(source):
    text = assembly(source)
    hits = [line.strip() for line in text.splitlines() if FORM.match(line)]
    assert not hits, "scalar loads with a register offset: %s" % hits[:5]
    sizes = scratch_bytes(text)
    assert len(sizes) == KERNELS[source]
    for name, size in sizes.items():
        assert size <= (8 if "prompt_kernelILb1ELb1E" in name else 0), sizes
