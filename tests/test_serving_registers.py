"""The built library's kernel metadata: the attention kernels, whose loops hold their operands and
sums in registers, spill none of them, nor do the kernels that choose tokens."""
import paper_2607_09686_amd.moecache as moecache
from test_kernel_registers import kernels


def test_attention_kernels_use_no_scratch():
    found = {n: k for n, k in kernels(moecache.LIB_PATH).items() if "attend_" in n}
    # few rows (32, 64), many rows, joined (of tiles of 32, 64, 128): three head sizes, two types
    assert len(found) == 6 * 3 * 2
    for name, k in found.items():
        assert (k[".vgpr_spill_count"], k[".private_segment_fixed_size"]) == (0, 0), name


def test_sampling_kernels_use_no_scratch():
    steps = ("row_kernel", "largest_kernel", "bins_kernel", "collect_kernel", "draw_kernel")
    found = {n: k for n, k in kernels(moecache.LIB_PATH).items() if "SampleArgs" in n and any(s in n for s in steps)}
    assert len(found) == len(steps) * 3  # types of logits
    for name, k in found.items():
        assert (k[".vgpr_spill_count"], k[".private_segment_fixed_size"]) == (0, 0), name
