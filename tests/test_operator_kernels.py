"""What the compiler gave the kernels of the operators around the decode step: no scratch memory, no spilled registers, and the registers
that their workgroups a compute unit count on."""
import pytest

from test_kernel_resources import _group, kernels      # noqa: F401  (a fixture)


@pytest.mark.parametrize("name", ["k_rotate", "k_rotate_any", "k_cache_slots", "k_cache_append", "k_cache_gather", "k_logprobs_part", "k_logprobs_join"])
def test_no_scratch(kernels, name):      # noqa: F811
    for n, k in _group(kernels, name).items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n


def test_log_probabilities_hold_their_columns_packed(kernels):      # noqa: F811
    """Six waves a SIMD for 64 columns of 16 bits a lane (512 registers a lane and SIMD), four for 128, four for 64 of 32 bits."""
    for n, k in _group(kernels, "k_logprobs_part").items():
        if n.endswith(", 64>"):
            assert k[".vgpr_count"] <= (128 if "<0u" in n else 80), n
        if n.endswith(", 128>") and "<0u" not in n:
            assert k[".vgpr_count"] <= 128, n
