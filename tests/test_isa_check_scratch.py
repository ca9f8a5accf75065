"""The build's check that the 4-bit and the grouped products keep their sums and loads in registers."""
import pytest

from paper_2510_25590_amd import isa_check as ic

KERNEL = "_Z19gemm_mx_tile_kernelILi1EEvv"


def asm(name, scratch):
    return f"{name}:\n\tv_mfma_f32_32x32x16_bf16 v[4:19], v[20:23], v[24:27], v[4:19]\n\ts_endpgm\n.Lfunc_end0:\n" + (f"; ScratchSize: {scratch}\n" if scratch is not None else "")


def test_registers_only():
    ic.check_asm(asm(KERNEL, 0))


@pytest.mark.parametrize("scratch", [4, 512, None])
def test_scratch_is_found(scratch):
    with pytest.raises(RuntimeError, match="scratch memory"):
        ic.check_asm(asm(KERNEL, scratch))


def test_the_second_kernel_of_a_file_is_looked_at():
    with pytest.raises(RuntimeError, match="128 bytes"):
        ic.check_asm(asm(KERNEL, 0) + asm(KERNEL.replace("ILi1E", "ILi0E"), 128))


def test_other_products_may_spill_where_nothing_is_counted():
    ic.check_asm(asm("_Z12gemm_f32_kernv", 16))
