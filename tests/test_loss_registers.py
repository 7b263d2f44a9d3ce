"""Registers of the kernels of the losses, read from the metadata of the built library: a row stays in registers, so that none of
them may spill, and those of 1024 threads have to leave room for all of their wavefronts (128 a thread)."""
import pytest

from test_kernel_registers import kernels  # noqa: F401  (the fixture)


@pytest.mark.parametrize("kind", ["loss_row_kernel", "loss_grad_kernel", "top_kernel", "pairs_kernel"])
def test_loss_kernels_do_not_spill(kernels, kind):  # noqa: F811
    found = {n: k for n, k in kernels.items() if kind in n}
    assert found
    for n, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
        assert k[".vgpr_count"] <= 512 // (k[".max_flat_workgroup_size"] // 256 or 1), n
