"""Registers and scratch of the 4-bit decode kernels, from the code objects' metadata in libspts.so (no GPU needed)."""
import pytest

from tests.test_kernel_resources import _named, kernels  # noqa: F401  (the fixture)


@pytest.mark.parametrize("part", ["q4_pack_kernel", "q4_matvec_kernel", "kv4_append_kernel", "kv4_read_kernel", "kv4_rope_append_kernel", "kv4_attn_kernel",
                                  "kv4_merge_kernel", "kv4_merge_few_kernel", "process_logits_kernel", "pick_token_kernel"])
def test_nothing_in_scratch(kernels, part):  # noqa: F811
    for name, k in _named(kernels, part).items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, name


def test_products_leave_room_for_two_workgroups(kernels):  # noqa: F811
    """Two workgroups of four wavefronts (fp32) or eight (bf16) to a CU: 256 or 128 of a SIMD's 512 registers each."""
    for name, k in _named(kernels, "q4_matvec_kernel").items():
        assert k[".vgpr_count"] <= (128 if "q4_matvec_kernelINS" in name else 256), name
