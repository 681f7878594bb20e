"""Differential attention over keys that are infinite in one of the two maps: the definition holds, in every form of the kernels."""
import math

import pytest
import torch

import paper_2505_17694_amd as C
from test_differential import DEV, compare, make
from test_differential_kernels import FORMS, FINISH, NARROW, WIDE
from workloads import draft_masked_forest, two_level_forest, unshared_forest, DTYPE_BF16, DTYPE_FP16

# beside the forms: teams of a wave (short contexts in one slot), the run-time queue, masked tasks, slices of one block
MORE = [(unshared_forest([5, 40, 33, 7, 64, 1, 90]), 4, 2, 64, dict(num_slots=1), NARROW), (unshared_forest([5, 40, 33, 7, 64, 1, 90]), 2, 2, 128, dict(num_slots=1), NARROW),
        (two_level_forest(300, [30, 40, 50]), 8, 1, 32, dict(schedule=1, num_slots=2, fixed_slices=3), NARROW),
        (draft_masked_forest(50, [100, 33, 1], 5, seed=5), 4, 2, 64, {}, NARROW), (two_level_forest(700, [30] * 40), 8, 2, 128, dict(fixed_slices=20, split_align=32), WIDE)]
CASES = FORMS + MORE


def token_of(w, node, t):
    p = w.paged
    return int(p.page_ids[p.node_page_off[node] + t // p.page_size]), t % p.page_size


def nodes_with_company(f):
    """A node every token of which somebody sees beside other tokens: the longest; and the last node of request 0."""
    longest = int(max(range(len(f.node_len)), key=lambda n: f.node_len[n]))
    return {longest, int(f.req_node[0])}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [DTYPE_BF16, DTYPE_FP16])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("map_", [0, 1])
def test_a_key_that_one_map_never_takes(case, map_, dtype):
    """-inf times the queries' positive channel is the score -inf: weight zero in that map, bit for bit what a score far below the
    others gives, and nothing at all in the other map.  The same with +inf times a negative channel."""
    f, heads, hkv, d, opts, form = CASES[case]
    print(f"[case] {case} form={form} requests={f.num_requests} heads={heads}/{hkv} d={d} map={map_} dtype={dtype} {opts}", flush=True)
    w = make(f, heads, hkv, d, dtype=dtype, seed=case + 1, poison=False)
    channel = 3 * d // 4 + 1
    q = w.q.view(f.num_requests, heads, 2, d)
    q[:, 0::2, map_, channel], q[:, 1::2, map_, channel] = 2.0, 1.0
    pa = C.PlannedAttention(f, w.paged, w.head, device=DEV, **opts)
    lam, weight = torch.rand(f.num_requests, heads, generator=torch.Generator().manual_seed(2)), torch.ones(2 * d, device=DEV)

    def results(key, sign):
        x = w.to(DEV)
        x.q.view(f.num_requests, heads, 2, d)[:, :, map_, channel] *= sign
        for node in nodes_with_company(f):
            for t in {0, int(f.node_len[node]) - 1} if f.node_len[node] > 2 else ():
                page, place = token_of(w, node, t)
                x.k_pool[page, place, :, map_ * d + channel] = key * sign
        return x, [pa.decode_differential(x.q, x.k_pool, x.v_pool, lam.to(DEV), weight=weight if eps else None, eps=eps) for eps in (None, 1e-5)]

    for sign in (1.0, -1.0):
        x, want = results(-30000.0, sign)
        _, got = results(-math.inf, sign)
        for a, b in zip(got, want):
            assert not torch.isnan(a).any(), (sign, int(torch.isnan(a).any(-1).sum()))
            assert torch.equal(a, b)
    low = x.to("cpu")
    low.forest, low.paged, low.head = w.forest, w.paged, w.head
    compare(low, got[0], lam, only=range(0, f.num_requests, 7))
    pa.close()


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_a_key_that_is_no_weight(case, value):
    """A score of +inf or NaN is NaN in the softmax of its map, and so is the result of the heads and requests that see the token;
    all others keep their bits."""
    f, heads, hkv, d, opts, form = CASES[case]
    print(f"[case] {case} form={form} requests={f.num_requests} heads={heads}/{hkv} d={d} value={value} {opts}", flush=True)
    w = make(f, heads, hkv, d, seed=case + 1, poison=False)
    channel, kv = d // 2, hkv - 1
    w.q.view(f.num_requests, heads, 2, d)[..., channel] = 1.0
    pa = C.PlannedAttention(f, w.paged, w.head, device=DEV, **opts)
    lam, node = torch.full((), 0.5, device=DEV), int(f.req_node[0])
    page, place = token_of(w, node, 0)
    clean = w.to(DEV)
    want = pa.decode_differential(clean.q, clean.k_pool, clean.v_pool, lam)
    first = kv * (heads // hkv)
    for map_ in (0, 1):
        x = w.to(DEV)
        x.k_pool[page, place, kv, map_ * d + channel] = value
        got = pa.decode_differential(x.q, x.k_pool, x.v_pool, lam)
        for r in range(f.num_requests):
            sees = node in f.path(r)
            if sees and node == f.req_node[r] and f.req_mask_off is not None and f.req_mask_off[r + 1] > f.req_mask_off[r]:
                sees = bool(int(f.req_mask[f.req_mask_off[r]]) & 1)
            assert torch.equal(got[r, :first], want[r, :first]), (r, map_)
            if sees:
                assert torch.isnan(got[r, first:]).all(), (r, map_)
            else:
                assert torch.equal(got[r, first:], want[r, first:]), (r, map_)
    pa.close()
