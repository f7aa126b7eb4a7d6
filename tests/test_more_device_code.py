"""CPU-only checks of the compiled kernels of pages in blocks, of attention over another sequence's states and of pages dealt on
the device: what a compute unit can hold of them."""
import pytest

from tests.test_device_code import kernels  # noqa: F401


@pytest.mark.parametrize("kernel,waves,variants", [("blocks_few_kernel", 1, 10), ("blocks_many_kernel", 1, 16), ("blocks_wide_kernel", 2, 4),
                                                   ("blocks_scalar_kernel", 4, 4), ("blocks_write_kernel", 4, 12), ("blocks_read_kernel", 4, 4),
                                                   ("cross_few_kernel", 1, 25), ("cross_many_kernel", 1, 40), ("cross_wide_kernel", 2, 10),
                                                   ("cross_scalar_kernel", 4, 10), ("assign_kernel", 4, 8), ("assign_rows_kernel", 8, 1)])
def test_kernels_spill_nothing(kernels, kernel, waves, variants):  # noqa: F811
    """Every variant keeps its values in registers, and leaves so many waves room on a SIMD (vector and accumulation registers together)."""
    some = {name: k for name, k in kernels.items() if kernel in name}
    assert len(some) == variants
    for name, k in some.items():
        assert int(k["vgpr_count"]) <= 512 // waves // 8 * 8, (name, k["vgpr_count"])
        assert int(k["vgpr_spill_count"]) == 0 and int(k["private_segment_fixed_size"]) == 0, name
