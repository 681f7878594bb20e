"""The kernels of differential attention: which one a plan runs, their registers, and results of each on the GPU."""
import re

import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C
from differential_choice import pair_launches
from helpers import GOING_ROUND, GOING_ROUND_OPTS, ROTATING, ROTATING_OPTS, going_round_forest, rotating_forest
from kernel_choice import case
from test_differential import DEV, head_of, make, run
from test_kernel_resources import resources, waves_per_simd
from workloads import Forest, build_paged_kv, concat_forests, two_level_forest, unshared_forest, DTYPE_BF16, DTYPE_FP16

NARROW, WIDE, FINISH = 0, 1, 2


def _case(f, heads, hkv, d, dtype=DTYPE_BF16, layout="thd", **opts):
    head = head_of(heads, hkv, d, dtype)
    return case(f, build_paged_kv(f, head, 1, layout=layout), head, **opts)


# one KV head has `group` rows a request, two for each head of the result
FORMS = [(unshared_forest([100, 40]), 4, 2, 64, {}, FINISH), (unshared_forest([33] * 9), 8, 1, 128, {}, FINISH),
         (unshared_forest([2000]), 4, 2, 64, dict(fixed_slices=4, num_slots=4), NARROW), (two_level_forest(300, [30, 40]), 4, 2, 64, {}, NARROW),
         (two_level_forest(300, [30, 40, 50]), 8, 1, 32, {}, NARROW),           # 48 rows: two row tiles of 64 channels, one task each
         (two_level_forest(300, [30] * 9), 4, 2, 64, {}, WIDE), (two_level_forest(700, [30] * 64), 32, 8, 32, {}, WIDE),
         (two_level_forest(1500, [30] * 64), 16, 8, 128, {}, WIDE), (two_level_forest(300, [30] * 3), 4, 2, 128, {}, NARROW)]


def test_forms():
    """Finished rows where every request has one partial result; tasks of up to sixteen rows alone; all shapes of tasks."""
    cases = [_case(f, heads, hkv, d, **opts) for f, heads, hkv, d, opts, _ in FORMS]
    for (f, heads, hkv, d, _, form), got in zip(FORMS, pair_launches(cases)):
        kernels = ["pair_kernel"] + ["differential_reduction_kernel"] * (form != FINISH)
        assert [k for k, _, _ in got] == kernels and got[0][1] == (DTYPE_BF16, form, 2 * d), (f.num_requests, heads, d, got)


@pytest.mark.parametrize("d", [32, 64, 128])
def test_reductions(d):
    """A wave a list, or four or eight for long lists of few requests, as in ordinary decode attention."""
    lists = [2, 15, 16, 23, 24, 39, 40, 72]
    few = [_case(Forest(np.array([-1]), np.array([32 * n]), np.zeros(2, np.int64)), 4, 2, d, DTYPE_FP16, split_align=32, fixed_slices=n, num_slots=4)
           for n in lists]
    for n, got in zip(lists, pair_launches(few)):
        waves = 1 if n < 24 else 4 if n <= 39 else 8
        units = 2 * (4 // 2)                                    # heads of a KV head, of both requests
        assert got[1] == ("differential_reduction_kernel", (DTYPE_FP16, 2 * d, waves),
                          (2, units // (2 if waves == 1 else 1), 1, 128 if waves == 1 else 64 * waves)), (n, got[1])


def test_registers(tmp_path):
    """None spills; two workgroups of a form share a CU up to 128 channels, and the reductions keep the waves of the ordinary ones."""
    seen = {}
    for name, (registers, scratch) in resources(tmp_path).items():
        m = re.search(r"\d(pair_kernel|differential_reduction_kernel|rotary_axes_kernel|rotary_axes_uneven_kernel|block_table_kernel|"
                      r"slot_map_kernel|slot_sums_kernel|slot_find_kernel)", name)
        if m:
            assert scratch == 0, name
            seen.setdefault(m.group(1), []).append((tuple(int(x) for x in re.findall(r"L[ib](\d+)E", name)), registers))
    assert {k: len(v) for k, v in seen.items() if "rotary" not in k} == {
        "pair_kernel": 18, "differential_reduction_kernel": 18, "block_table_kernel": len(seen["block_table_kernel"]),
        "slot_map_kernel": len(seen["slot_map_kernel"]), "slot_sums_kernel": len(seen["slot_sums_kernel"]), "slot_find_kernel": len(seen["slot_find_kernel"])}
    assert seen["rotary_axes_kernel"] and seen["rotary_axes_uneven_kernel"]
    for args, registers in seen["pair_kernel"]:
        assert registers <= (512 if args[2] > 128 else 256), (args, registers)
    for kernel, least in (("differential_reduction_kernel", 4), ("rotary_axes_kernel", 8), ("rotary_axes_uneven_kernel", 6), ("block_table_kernel", 8),
                          ("slot_sums_kernel", 8), ("slot_find_kernel", 8)):
        assert min(waves_per_simd(r) for _, r in seen[kernel]) >= least, (kernel, seen[kernel])


# ---- on the GPU ------------------------------------------------------------------------------------------


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [DTYPE_BF16, DTYPE_FP16])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_forms_on_the_gpu(form, dtype):
    f, heads, hkv, d, opts, _ = FORMS[form]
    run(f, heads, hkv, d, kind="token", norm=True, dtype=dtype, layout="htd" if dtype else "thd", opts=opts)


@pytest.mark.gpu
@pytest.mark.parametrize("opts", GOING_ROUND_OPTS)
@pytest.mark.parametrize("channels,hq,hkv,leaves", [c for c in GOING_ROUND if c[1] // c[2] % 2 == 0])
def test_stream_tasks_go_round_the_heads(channels, hq, hkv, leaves, opts):
    """Long plans whose contexts are read by one request each, [token][head] pools: every (task, head) is run once."""
    f = going_round_forest(leaves)
    run(f, hq // 2, hkv, channels // 2, kind="head", norm=True, only=range(0, f.num_requests, 9), opts=opts)


@pytest.mark.gpu
@pytest.mark.parametrize("opts", ROTATING_OPTS)
@pytest.mark.parametrize("channels,hq,hkv,dtype,nodes,requests,below,form", [c for c in ROTATING if c[1] // c[2] % 2 == 0])
def test_tasks_of_all_shapes_go_round_the_heads(channels, hq, hkv, dtype, nodes, requests, below, form, opts):
    f = rotating_forest(nodes, requests, below)
    run(f, hq // 2, hkv, channels // 2, kind="token", dtype=dtype, only=range(0, f.num_requests, 13), opts=opts)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [32, 64, 128])
def test_many_heads_beside_contexts_of_one_token(d):
    """Rows of all kinds in one plan: dense tasks, contexts of one token, requests that share a leaf."""
    f = concat_forests(concat_forests(two_level_forest(257, [1 + i % 3 for i in range(70)]), unshared_forest([1, 2, 1])),
                       Forest(np.array([-1]), np.array([65]), np.zeros(5, np.int64)))
    run(f, 6, 3, d, kind="token", norm=True, only=range(0, f.num_requests, 5))


@pytest.mark.gpu
@pytest.mark.parametrize("length", [2047, 2048, 2049, 2079, 2304, 2305, 2337, 4100])
@pytest.mark.parametrize("requests,dtype", [(24, DTYPE_BF16), (75, DTYPE_FP16)])
def test_tasks_that_share_a_long_slice(length, requests, dtype):
    """Packs of a node's rows with 256 channels, which take their blocks in orders of their own, in slices that end inside one."""
    f = two_level_forest(length, [1 + i % 40 for i in range(requests)])
    run(f, 8, 2, 128, kind="token", norm=True, dtype=dtype, only=range(0, requests, 7), opts=dict(fixed_slices=1, num_slots=8))


@pytest.mark.gpu
def test_numbers_that_are_negated_when_they_are_read():
    """Views that carry their sign beside them are refused: the kernels read memory as it is."""
    w = make(two_level_forest(40, [20, 3]), 4, 2, 64).to(DEV)
    pa = C.PlannedAttention(w.forest, w.paged, w.head, device=DEV)
    lam = torch.view_as_complex(torch.rand(4, 2, device=DEV)).conj().imag
    weight = torch._neg_view(torch.rand(128, device=DEV))
    good = dict(lam=lam.resolve_neg(), weight=weight.resolve_neg(), eps=1e-5)
    pa.decode_differential(w.q, w.k_pool, w.v_pool, **good)
    for bad in (dict(lam=lam), dict(weight=weight)):
        with pytest.raises(ValueError):
            pa.decode_differential(w.q, w.k_pool, w.v_pool, **dict(good, **bad))
    pa.close()
