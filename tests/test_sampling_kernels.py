"""What the compiler made of the kernels of sampled decoding."""
import os

import pytest

from paper_2502_17421_amd import build as ls_build


@pytest.mark.parametrize("name,least", [("tree_sample_kernel", 9), ("page_copy_kernel", 1), ("fork_one_kernel", 1), ("fork_list_kernel", 1),
                                        ("fork_write_kernel", 1), ("compact_one_kernel", 1), ("compact_parts_kernel", 1), ("compact_rank_kernel", 1)])
def test_they_use_no_scratch_memory(name, least):
    if not os.path.exists(ls_build.RESOURCE_REPORT) or ls_build.is_stale():
        ls_build.build_library()
    kernels = {k: v for k, v in ls_build.kernel_resources().items() if name in k}
    assert len(kernels) >= least
    for full, r in kernels.items():
        assert r["ScratchSize"] == 0 and r["VGPRs Spill"] == 0, (full, r)
        if name == "tree_sample_kernel":  # the slices are chosen for four workgroups of four waves on a compute unit
            assert r["VGPRs"] + r["AGPRs"] <= 128, (full, r)
