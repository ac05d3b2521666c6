"""Properties of the compiled kernels of the operators on packed samples."""
import pytest

from tests import kernel_code

KERNELS = ["packed_fwd_kernelILi", "packed_dq_kernelILi", "packed_dkv_kernelILi", "packed_dkv_narrow_kernelILi", "packed_bwd_kernelILi", "packed_join_kernelILi", "packed_f32_", "rotary_axes_kernelI", "dropout_kernelI"]


@pytest.mark.parametrize("kernel", KERNELS)
def test_no_register_is_spilled_to_memory(kernel):
    for name, k in kernel_code.kernels(kernel).items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name


@pytest.mark.parametrize("kernel", ["packed_fwd_kernelILi", "packed_dq_kernelILi", "packed_dkv_narrow_kernelILi", "packed_bwd_kernelILi"])
def test_staged_tiles_begin_at_the_start_of_lds(kernel):
    """These kernels turn from one buffer to the other by an XOR of the address, so their dynamic LDS has to begin at 0."""
    for name, k in kernel_code.kernels(kernel).items():
        assert k[".group_segment_fixed_size"] == 0, name
