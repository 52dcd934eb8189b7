"""No kernel of linear attention or of the norm keeps anything in scratch memory: a prefill workgroup's loads of the next
chunk lie in registers beside the state, and one that spills waits for them."""
import pytest

from tests.test_kernel_registers import kernels  # noqa: F401


@pytest.mark.parametrize("name,least", [("linear_sums", 1), ("linear_join", 1), ("linear_outputs", 1), ("linear_decode", 1), ("norm_rows", 4), ("norm_row_", 2)])
def test_no_scratch(kernels, name, least):   # noqa: F811
    found = {n: k for n, k in kernels.items() if name in n}
    assert len(found) >= least, sorted(kernels)
    for n, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n


def test_waves_per_simd(kernels):   # noqa: F811
    """512 vector registers of a SIMD: two waves of a prefill workgroup, six of a join."""
    for n, k in kernels.items():
        if "linear_sums" in n or "linear_outputs" in n:
            assert k[".vgpr_count"] <= 256, n
        if "linear_join" in n:
            assert k[".vgpr_count"] <= 84, n
