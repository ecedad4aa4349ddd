"""The paged-cache kernels keep what they compute in registers: no scratch memory, and as many wavefronts a SIMD as they are
built for (built library, no GPU)."""
import re

import pytest

from test_kernel_resources import kernels  # noqa: F401  (a fixture)


@pytest.mark.parametrize("name,least", [("paged_attn_kernel", 24), ("paged_few_kernel", 24), ("paged_merge_kernel", 4), ("paged_append", 4), ("paged_plan", 1)])
def test_no_kernel_uses_scratch(kernels, name, least):  # noqa: F811
    found = {n: k for n, k in kernels.items() if name in n}
    assert len(found) >= least
    for n, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n


def test_two_workgroups_of_the_attention_share_a_cu(kernels):  # noqa: F811
    for n, k in kernels.items():
        if "paged_attn_kernel" in n or re.search(r"paged_few_kernelI.*ELi4ELi1E", n):
            assert 512 // (-(-k[".vgpr_count"] // 8) * 8) >= 2, n
            assert k[".group_segment_fixed_size"] <= 80 * 1024, n
