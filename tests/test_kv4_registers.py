"""No kernel of the 4-bit cache keeps anything in scratch memory: the attention's inner loops are
register-bound, and their tile shapes were chosen so that they fit."""
import pytest

from tests.test_kernel_registers import kernels  # noqa: F401


@pytest.mark.parametrize("name,least", [("kv4_prefill", 4), ("kv4_decode", 12), ("kv4_write", 2), ("kv4_stats", 3), ("kv4_select", 1),
                                        ("kv4_move", 3)])
def test_no_scratch(kernels, name, least):   # noqa: F811
    found = {n: k for n, k in kernels.items() if name in n}
    assert len(found) >= least, sorted(kernels)
    for n, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n


def test_waves_per_simd(kernels):   # noqa: F811
    """512 vector registers of a SIMD: two waves of a prefill workgroup, three of a 16-column decode."""
    for n, k in kernels.items():
        if "kv4_prefill_plan" in n or "kv4_prefill_kernel" in n or "kv4_decode_kernelILi32" in n:
            assert k[".vgpr_count"] <= 256, n
        if "kv4_decode_kernelILi16" in n:
            assert k[".vgpr_count"] <= 168, n
