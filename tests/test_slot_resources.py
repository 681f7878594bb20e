"""How many instances of the kernels of tables, slots, axes and two maps are built, and the waves of a call's usual slot kernel."""
import re

from test_kernel_resources import resources, waves_per_simd

# tables whose rows are aligned, and others; the rest of this line one form; rows by axes as without axes: two types, three head sizes, two
# layouts, two sizes of call; two types, three head sizes; two types, three sizes, and three forms of tasks or of lists
INSTANCES = {"block_table_kernel": 2, "slot_map_kernel": 1, "slot_sums_kernel": 1, "slot_find_kernel": 1, "rotary_axes_kernel": 24,
             "rotary_axes_uneven_kernel": 6, "pair_kernel": 18, "differential_reduction_kernel": 18}


def test_instances_and_waves(tmp_path):
    seen = {}
    for name, (registers, scratch) in resources(tmp_path).items():
        m = re.search(r"\d(" + "|".join(INSTANCES) + ")", name)
        if m:
            assert scratch == 0, name
            seen.setdefault(m.group(1), []).append(registers)
    assert {k: len(v) for k, v in seen.items()} == INSTANCES
    assert min(waves_per_simd(r) for r in seen["slot_map_kernel"]) >= 8, seen["slot_map_kernel"]
