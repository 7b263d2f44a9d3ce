"""Registers of the cross-attention kernels, read from the metadata of the built library.  The bf16 ones read LDS in ways the
compiler does not track, so a spilled register could be one that a read in flight still writes: none may spill.  The fp32 ones
read through the compiler; only dK / dV at head dim 64 keeps a few addresses in scratch, for a second wavefront on its SIMD."""
import pytest

from test_kernel_registers import kernels  # noqa: F401  (the fixture)


@pytest.mark.parametrize("kind,count", [("cross_fwd_kernel", 10), ("cross_dq_kernel", 6), ("cross_dkv_kernel", 2), ("cross_fwd_f32_kernel", 6),
                                        ("cross_dq_f32_kernel", 6), ("cross_dkv_f32_kernel", 6)])
def test_cross_attention_kernels_do_not_spill(kernels, kind, count):  # noqa: F811
    found = {n: k for n, k in kernels.items() if kind in n}
    assert len(found) == count, sorted(found)
    for n, k in found.items():
        few = 8 if "cross_dkv_f32_kernelILi64E" in n else 0
        assert k[".vgpr_spill_count"] <= few and k[".private_segment_fixed_size"] <= 4 * (few + 1), n
