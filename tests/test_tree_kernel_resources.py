"""Registers and LDS of the kernels of a drafted step: what the shares and runs of its attention are cut for."""
import re

from test_kernel_resources import kernels, workgroups_per_unit  # noqa: F401


def test_residency_that_attention_by_masks_is_cut_for(kernels):  # noqa: F811
    """Two workgroups to a compute unit in every form."""
    cut = {n: k for n, k in kernels.items() if re.match(r"tree_(16|many_16|f32)_kernel<", n)}
    assert len(cut) == 2 * 2 * (3 + 2) + 2 * 2
    for name, k in cut.items():
        assert workgroups_per_unit(k) >= 2, name


def test_a_wave_has_its_registers(kernels):  # noqa: F811
    """Verification: eight workgroups of four waves to a compute unit would need 64 registers, four have 128."""
    found = [k for n, k in kernels.items() if "tree_verify_kernel" in n]
    assert len(found) == 6, found
    for k in found:
        assert workgroups_per_unit(k) >= 4
