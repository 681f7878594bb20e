"""Registers and scratch memory of the operators' kernels as built.  A choice between two places of the kernel's arguments, or an
array of which a part is filled under a condition, ends in scratch memory or in a load for every lane, without a word."""
import re

from test_kernel_resources import resources, waves_per_simd


def test_no_kernel_spills_and_copies_keep_their_waves(tmp_path):
    seen = {}
    for name, (registers, scratch) in resources(tmp_path).items():
        m = re.search(r"\d(rotary_kernel|rotary_uneven_kernel|page_copy_kernel|reorder_kernel|beam_rows_kernel|beam_merge_kernel)", name)
        if m:
            assert scratch == 0, name
            seen.setdefault(m.group(1), []).append(registers)
    # two types, three head sizes, two layouts, two sizes of call; halves of other sizes; rows and sizes of copy; units; types; one
    assert {k: len(v) for k, v in seen.items()} == {"rotary_kernel": 24, "rotary_uneven_kernel": 6, "page_copy_kernel": 8, "reorder_kernel": 20,
                                                    "beam_rows_kernel": 6, "beam_merge_kernel": 1}
    for kernel, least in (("rotary_kernel", 8), ("rotary_uneven_kernel", 6), ("page_copy_kernel", 8), ("reorder_kernel", 8), ("beam_rows_kernel", 4)):
        assert min(waves_per_simd(r) for r in seen[kernel]) >= least, (kernel, seen[kernel])
