"""Differential attention over the prefix-shared cache: refusals on the CPU, results against a plain 64-bit one on the GPU."""
import math

import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C
from oracle import operators as O
from workloads import (Forest, HeadConfig, build_paged_kv, concat_forests, degenerate_forest, draft_masked_forest, make_workload, random_forest,
                       three_level_forest, two_level_forest, unshared_forest, DTYPE_BF16, DTYPE_FP16)

DEV = "cuda:0"


def head_of(heads, hkv, d, dtype=DTYPE_BF16, page=16):
    return HeadConfig(2 * heads, hkv, 2 * d, dtype, page, float(np.float32(1.0 / math.sqrt(d))))


# ---- on the CPU ------------------------------------------------------------------------------------------


def plan_of(f=None, head=None):
    f, head = f or two_level_forest(100, [20, 30]), head or head_of(4, 2, 64)
    paged = build_paged_kv(f, head, seed=1)
    st, plan = C.codec_plan_create(f.parent, f.node_len, f.req_node, paged.node_page_off, paged.page_ids, head.num_q_heads, head.num_kv_heads,
                                   head.head_dim, head.dtype, head.page_size, head.scale, num_slots=4, split_align=32, max_rows=64, share=1,
                                   cost_table=None)
    assert st == C.CODEC_OK
    return plan


def test_refusals():
    """Argument errors that are caught before any HIP call; a plan that was never uploaded refuses what is left."""
    plan = plan_of()
    need = C.codec_plan_workspace_bytes(plan)
    layout = C.codec_kv_layout(1000, 16 * 2 * 128, 2 * 128, 128)
    at = dict(q=1 << 20, k=1 << 24, v=1 << 26, out=1 << 21, ws=1 << 22, lam=4096, weight=8192)

    def status(of=plan, request=4, head=1, norm=1, dtype=C.CODEC_DTYPE_FP32, eps=1e-5, gain=0.5, config=True, lay=layout, nbytes=need, **kw):
        p = dict(at, **kw)
        c = C.codec_differential(p["lam"], request, head, norm, dtype, p["weight"], eps, gain) if config else None
        return C.codec_differential_attention(of, c, p["q"], p["k"], p["v"], lay, p["out"], p["ws"], nbytes)

    assert status() == status(weight=None) == status(norm=0, weight=None, eps=-1.0) == status(request=0, head=0) == C.CODEC_ERR_NOT_UPLOADED
    assert status(dtype=C.CODEC_DTYPE_BF16, weight=8194) == C.CODEC_ERR_NOT_UPLOADED
    nan, inf = math.nan, math.inf
    for bad in (dict(of=None), dict(config=False), dict(lay=None), dict(lam=None), dict(lam=4098), dict(request=-1), dict(head=-1), dict(head=1 << 37),
                dict(norm=2), dict(norm=-1), dict(norm=0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(gain=nan), dict(gain=-inf), dict(q=0),
                dict(out=0), dict(ws=0), dict(q=(1 << 20) + 8), dict(out=(1 << 21) + 2), dict(ws=(1 << 22) + 64), dict(weight=8194),
                dict(out=1 << 20), dict(out=(1 << 20) + 512), dict(out=1 << 22), dict(lam=(1 << 21) + 64), dict(weight=(1 << 22) + need - 4),
                dict(q=1 << 22), dict(out=4096 + 16)):
        assert status(**bad) == C.CODEC_ERR_INVALID_ARGUMENT, bad
    for dtype in (C.CODEC_DTYPE_FP16, 3, -1):
        assert status(dtype=dtype) == C.CODEC_ERR_UNSUPPORTED
    assert status(nbytes=need - 1) == C.CODEC_ERR_WORKSPACE_TOO_SMALL
    C.codec_plan_destroy(plan)
    odd = plan_of(head=HeadConfig(6, 2, 128))
    assert status(of=odd) == C.CODEC_ERR_UNSUPPORTED                            # three query heads do not pair up
    C.codec_plan_destroy(odd)
    empty = C.codec_plan_create(np.zeros(0), np.zeros(0), np.zeros(0), np.zeros(1, np.int32), np.zeros(0, np.int32), 8, 2, 128, 1, 16, 0.1, 4, 32, 64, 1, None)[1]
    assert status(of=empty, lam=None, q=0, out=0) == C.CODEC_OK
    C.codec_plan_destroy(empty)
    w = make_workload("cpu", two_level_forest(40, [20]), head_of(2, 1, 32), seed=1)
    pa = C.PlannedAttention(w.forest, w.paged, w.head, device="cpu")
    with pytest.raises(ValueError):
        pa.decode_differential(w.q[..., :32].contiguous(), w.k_pool, w.v_pool, torch.ones(()))
    pa.close()


# ---- on the GPU ------------------------------------------------------------------------------------------


def context(w, r):
    """K and V [n, heads, channels] (64 bits) that request r sees, root first."""
    f, p, rows = w.forest, w.paged, []
    path = f.path(r)
    for node in path:
        t = np.arange(int(f.node_len[node]))
        if node == path[-1] and f.req_mask_off is not None and f.req_mask_off[r + 1] > f.req_mask_off[r]:
            words = f.req_mask[f.req_mask_off[r]:f.req_mask_off[r + 1]].astype(np.int64)
            t = t[(words[t // 32] >> (t % 32)) & 1 == 1]
        rows.append((p.page_ids[p.node_page_off[node] + t // p.page_size], t % p.page_size))
    page, place = (torch.from_numpy(np.concatenate(x).astype(np.int64)) for x in zip(*rows))
    return tuple((pool[page, place] if p.layout == "thd" else pool[page, :, place]).double().numpy() for pool in (w.k_pool, w.v_pool))


def make(f, heads, hkv, d, dtype=DTYPE_BF16, page=16, layout="thd", seed=1, q_scale=2.0, poison=True):
    w = make_workload("differential", f, head_of(heads, hkv, d, dtype, page), seed=seed, layout=layout, poison=poison)
    gen = torch.Generator().manual_seed(seed)
    w.q = (torch.randn(f.num_requests, 2 * heads, d, generator=gen) * q_scale).to(w.q.dtype)
    return w


def lambdas(kind, requests, heads, gen):
    x = torch.rand(requests, heads, generator=gen) * 1.4 - 0.2
    if kind == "one":
        return x[0, 0].to(DEV), x[:1, :1].expand(requests, heads)
    if kind == "head":
        return x[0].to(DEV), x[:1].expand(requests, heads)
    if kind == "strided":                                       # a column of a projection's output, heads far apart
        big = torch.full((heads, requests, 3), math.nan, device=DEV)
        big[..., 1] = x.T.to(DEV)
        return big[..., 1].T, x
    return x.to(DEV), x


def bound(dtype):
    """Half a step of the type; what is left of a rounding below its smallest normal number."""
    info = torch.finfo((torch.float16, torch.bfloat16)[dtype])
    return info.eps / 2, info.tiny * info.eps / 2


def compare(w, got, lam, norm=None, gain=1.0, only=None):
    half, least = bound(w.head.dtype)
    got = got.double().cpu().numpy()
    heads, d, worst = w.q.shape[1] // 2, w.q.shape[2], 0.0
    for r in range(w.forest.num_requests) if only is None else only:
        k, v = context(w, r)
        want, off = O.differential(w.q[r].double().numpy().reshape(heads, 2, d), k, v, float(w.head.scale), lam[r].double().numpy(), norm, gain, half, least)
        err = np.abs(got[r] - want)
        worst = max(worst, float((err / off).max()))
        assert np.all(err <= off), (r, float(err.max()), float((err / off).max()))
    return worst


def run(f, heads, hkv, d, kind="head", norm=False, weight="float32", gain=1.0, only=None, opts=None, **kw):
    print(f"[case] requests={f.num_requests} heads={heads}/{hkv} d={d} lam={kind} norm={norm} {weight} {kw} {opts}", flush=True)
    w = make(f, heads, hkv, d, **kw)
    wd, gen = w.to(DEV), torch.Generator().manual_seed(5)
    lam, lam_of = lambdas(kind, f.num_requests, heads, gen)
    of = None
    if norm and weight:
        of = (torch.randn(2 * d, generator=gen) * 0.3 + 1.0).to(torch.float32 if weight == "float32" else w.q.dtype)
    pa = C.PlannedAttention(w.forest, w.paged, w.head, device=DEV, **(opts or {}))
    got = pa.decode_differential(wd.q, wd.k_pool, wd.v_pool, lam, weight=None if of is None else of.to(DEV), eps=1e-5 if norm else None, gain=gain)
    torch.cuda.synchronize()
    assert got.shape == (f.num_requests, heads, 2 * d) and got.dtype == w.q.dtype
    worst = compare(w, got, lam_of, (float(np.float32(1e-5)), np.ones(2 * d) if of is None else of.double().numpy()) if norm else None, gain, only)
    print(f"[case] worst error {worst:.3f} of what may be", flush=True)
    pa.close()
    return w, got


FORESTS = {"one token": unshared_forest([1]), "few": unshared_forest([1, 2, 15, 16, 17, 31, 33, 100]), "long": unshared_forest([2049, 5, 700]),
           "shared": two_level_forest(513, [1, 40, 33, 64, 7]), "many rows": two_level_forest(300, [3 + i % 29 for i in range(45)]),
           "three levels": three_level_forest(100, [333, 64, 1], 5, [(7 * i) % 60 + 1 for i in range(15)]), "spine": degenerate_forest(20, 19, 5),
           "irregular": random_forest(24, 4, 2.0, 60, 1.0, 16, 900, seed=3)}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(FORESTS))
@pytest.mark.parametrize("heads,hkv,d,dtype,page,layout", [(4, 4, 64, DTYPE_BF16, 16, "thd"), (8, 2, 64, DTYPE_FP16, 32, "htd"), (6, 2, 32, DTYPE_BF16, 16, "htd"),
                                                           (4, 1, 128, DTYPE_BF16, 16, "thd"), (3, 3, 128, DTYPE_FP16, 64, "htd"), (8, 1, 32, DTYPE_FP16, 16, "thd")])
def test_forests_and_heads(name, heads, hkv, d, dtype, page, layout):
    run(FORESTS[name], heads, hkv, d, kind="token", norm=heads % 2 == 0, dtype=dtype, page=page, layout=layout, gain=0.7)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("kind", ["one", "head", "token", "strided"])
@pytest.mark.parametrize("norm,weight", [(False, None), (True, None), (True, "float32"), (True, "own type")])
def test_weights(d, kind, norm, weight):
    run(two_level_forest(130, [9, 1, 70]), 6, 2, d, kind=kind, norm=norm, weight=weight, gain=-0.3, dtype=DTYPE_FP16 if kind == "head" else DTYPE_BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("group,d", [(1, 64), (3, 64), (5, 64), (7, 64), (8, 64), (16, 64), (32, 64), (1, 32), (5, 32), (8, 32), (3, 128), (8, 128)])
def test_groups(group, d):
    """Up to 64 rows of a request and KV head (16 with other than 128 channels a row)."""
    run(two_level_forest(200, [30, 5, 64]), 2 * group, 2, d, norm=True)


@pytest.mark.gpu
@pytest.mark.parametrize("opts", [dict(schedule=1), dict(schedule=2, extensions=3, share=2), dict(share=0), dict(fused=1), dict(fused=2), dict(max_rows=16),
                                  dict(num_slots=3, split_align=32, fixed_slices=7), dict(num_slots=1)])
@pytest.mark.parametrize("d,hkv", [(64, 2), (32, 2), (128, 3)])
def test_plan_options(opts, d, hkv):
    f = concat_forests(two_level_forest(700, [20 + i for i in range(20)]), unshared_forest([300, 1000, 17]))
    run(f, 4 * hkv, hkv, d, kind="token", norm=True, opts=opts)


@pytest.mark.gpu
@pytest.mark.parametrize("slices", [8, 9, 15, 16, 23, 24, 39, 40, 80])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_long_lists_of_partials(slices, d):
    """Every form of the reduction: a wave a list, lists behind fifteen rows, lists that four and eight waves share."""
    run(Forest(np.array([-1, 0]), np.array([32 * slices, 3]), np.array([0, 1, 0])), 4, 2, d, norm=True,
        opts=dict(num_slots=4, split_align=32, fixed_slices=slices))


@pytest.mark.gpu
@pytest.mark.parametrize("drafted", [1, 5, 31, 40])
@pytest.mark.parametrize("heads,hkv,d", [(4, 2, 64), (8, 1, 32), (8, 2, 128)])
def test_drafted_tokens(drafted, heads, hkv, d):
    run(draft_masked_forest(50, [100, 33, 1], drafted, seed=drafted), heads, hkv, d, kind="token", norm=drafted % 2 == 1)


@pytest.mark.gpu
def test_dense_tasks_and_large_reductions():
    """Hundreds of rows below one node, workgroups of all sizes; some of the requests are compared."""
    for heads, hkv, d in ((16, 2, 64), (16, 4, 32), (8, 2, 128)):
        run(two_level_forest(2100, [1 + i % 50 for i in range(300)]), heads, hkv, d, kind="token", norm=True, only=range(0, 300, 17), opts=dict(extensions=3))


@pytest.mark.gpu
@pytest.mark.parametrize("q_scale", [0.0, 0.1, 8.0, 60.0])
def test_flat_and_peaked_maps(q_scale):
    """Maps that average everything, and maps on one token, in either type."""
    for dtype in (DTYPE_BF16, DTYPE_FP16):
        run(two_level_forest(400, [30, 1]), 4, 2, 64, q_scale=q_scale, dtype=dtype, kind="token", norm=True)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [32, 64, 128])
def test_maps_that_are_the_same_cancel(d):
    """Equal queries, equal halves of the keys and lambda 1: exactly zero, normalised or not; lambda 0: the first map alone."""
    w = make(two_level_forest(300, [40, 17]), 4, 2, d, seed=3, poison=False)
    w.k_pool[..., d:] = w.k_pool[..., :d]
    w.q = w.q.view(-1, 4, 2, d)[:, :, :1].expand(-1, 4, 2, d).reshape(-1, 8, d).contiguous()
    wd = w.to(DEV)
    pa = C.PlannedAttention(w.forest, w.paged, w.head, device=DEV)
    for eps in (None, 1e-6):
        assert not pa.decode_differential(wd.q, wd.k_pool, wd.v_pool, torch.ones((), device=DEV), eps=eps).any()
    first = pa.decode_differential(wd.q, wd.k_pool, wd.v_pool, torch.zeros((), device=DEV))
    rows = torch.zeros(2, 8, 2 * d, dtype=wd.q.dtype, device=DEV)
    rows[:, 0::2, :d] = wd.q[:, 0::2]
    rows[:, 1::2, d:] = wd.q[:, 1::2]
    plain = pa.decode(rows, wd.k_pool, wd.v_pool)
    half = bound(DTYPE_BF16)[0]
    assert bool(((first - plain[:, 0::2]).abs() <= 2 * half * first.abs()).all())           # the same sums, rounded by other reductions
    pa.close()


@pytest.mark.gpu
def test_values_that_are_not_numbers_stay_where_they_are():
    """NaN and infinite keys reach the heads and requests that see them, hidden ones nobody; such values reach their channel, whether a
    request of their node sees them or not (they are multiplied by zero), and no other head, channel or node."""
    f = draft_masked_forest(64, [32, 40], 6, seed=2)
    w = make(f, 4, 2, 64, poison=True)
    clean = w.to(DEV)
    pa = C.PlannedAttention(f, w.paged, w.head, device=DEV)
    lam = torch.full((), 0.5, device=DEV)
    want = pa.decode_differential(clean.q, clean.k_pool, clean.v_pool, lam)
    for pool, value in (("k_pool", math.nan), ("v_pool", math.nan), ("v_pool", math.inf), ("v_pool", -math.inf), ("k_pool", math.inf)):
        dirty = w.to(DEV)
        node = int(f.req_node[1])                               # the drafted tokens of the first sequence; the third of them, head 1
        page = int(w.paged.page_ids[w.paged.node_page_off[node]])
        getattr(dirty, pool)[page, 2, 1, 5] = value
        got = pa.decode_differential(dirty.q, dirty.k_pool, dirty.v_pool, lam)
        for r in range(f.num_requests):
            sees = int(f.req_node[r]) == node and bool(int(f.req_mask[f.req_mask_off[r]]) >> 2 & 1)
            assert torch.equal(got[r, :2], want[r, :2])
            if int(f.req_node[r]) != node or (pool == "k_pool" and not sees):
                assert torch.equal(got[r, 2:], want[r, 2:]), r
            elif pool == "v_pool":
                others = [c for c in range(128) if c != 5]
                assert torch.equal(got[r, 2:][:, others], want[r, 2:][:, others]) and not (sees and torch.isfinite(got[r, 2:, 5]).any())
            elif math.isnan(value):
                assert torch.isnan(got[r, 2:]).all()
    pa.close()


@pytest.mark.gpu
def test_refreshed_lengths_side_by_side_pools_and_given_outputs():
    """The plan carried over to grown lengths; K and V in one pool; out in a larger tensor; q unchanged."""
    f = two_level_forest(200, [30, 64])
    w = make(f, 4, 2, 64, layout="hktd", seed=8)
    wd = w.to(DEV)
    lam = torch.rand(4, generator=torch.Generator().manual_seed(1))
    pa = C.PlannedAttention(f, w.paged, w.head, device=DEV)
    big = torch.full((4, 4, 128), 9.0, dtype=wd.q.dtype, device=DEV)
    q = wd.q.clone()
    got = pa.decode_differential(wd.q, wd.k_pool, wd.v_pool, lam.to(DEV), out=big[1:3])
    assert got.data_ptr() == big[1:3].data_ptr() and bool((big[0] == 9).all()) and bool((big[3] == 9).all()) and torch.equal(q, wd.q)
    w.paged.layout = "htd"                                      # views of the pool, addressed like it
    compare(w, got, lam.expand(2, 4))
    grown = f.node_len.copy()
    grown[1:] -= [7, 33]                                        # shorter than planned: a slice that ends earlier
    pa.refresh(grown)
    f.node_len = grown
    compare(w, pa.decode_differential(wd.q, wd.k_pool, wd.v_pool, lam.to(DEV)), lam.expand(2, 4))
    pa.close()


@pytest.mark.gpu
def test_tensors_are_checked():
    w = make(two_level_forest(40, [20, 3]), 4, 2, 64)
    wd = w.to(DEV)
    pa = C.PlannedAttention(w.forest, w.paged, w.head, device=DEV)
    lam, weight = torch.ones(4, device=DEV), torch.ones(128, device=DEV)
    good = dict(q=wd.q, k_pool=wd.k_pool, v_pool=wd.v_pool, lam=lam, weight=weight, eps=1e-5)
    pa.decode_differential(**good)
    gone = torch.ones(4, device=DEV)
    gone.untyped_storage().resize_(12)
    for bad in (dict(q=wd.q[:1]), dict(q=wd.q.float()), dict(q=w.q), dict(q=wd.q.transpose(0, 1)), dict(k_pool=wd.k_pool[:3].clone()), dict(v_pool=w.v_pool),
                dict(lam=lam[:3]), dict(lam=lam.double()), dict(lam=lam.cpu()), dict(lam=torch.ones(3, 4, device=DEV)), dict(lam=gone),
                dict(weight=weight[:64]), dict(weight=weight.half()), dict(weight=torch.ones(256, device=DEV)[::2]), dict(weight=weight.cpu()),
                dict(out=torch.zeros(2, 8, 64, dtype=wd.q.dtype, device=DEV)), dict(out=torch.zeros(2, 4, 128, device=DEV))):
        with pytest.raises(ValueError):
            pa.decode_differential(**dict(good, **bad))
    for bad in (dict(eps=None), dict(eps=-1.0), dict(eps=math.nan), dict(gain=math.inf), dict(out=wd.q.view(2, 4, 128))):
        with pytest.raises(C.CodecError):
            pa.decode_differential(**dict(good, **bad))
    odd = C.PlannedAttention(w.forest, w.paged, HeadConfig(6, 2, 128), device=DEV)
    with pytest.raises(C.CodecError):
        odd.decode_differential(torch.zeros(2, 6, 64, dtype=wd.q.dtype, device=DEV), wd.k_pool, wd.v_pool, torch.ones((), device=DEV))
    odd.close()
    pa.close()


@pytest.mark.gpu
@pytest.mark.parametrize("schedule", [0, 1])
def test_another_stream_and_replayed_graphs(schedule):
    """Two captured steps of one plan, replayed in turn with eager calls in between; the plain decode of the plan beside them."""
    w = make(concat_forests(two_level_forest(600, [9 + 5 * i for i in range(12)]), unshared_forest([700])), 8, 2, 64, poison=False)
    wd = w.to(DEV)
    pa = C.PlannedAttention(w.forest, w.paged, w.head, device=DEV, schedule=schedule, extensions=3)
    lam, weight = torch.rand(13, 8, device=DEV), torch.rand(128, device=DEV)
    call = lambda **kw: pa.decode_differential(wd.q, wd.k_pool, wd.v_pool, lam, weight=weight, eps=1e-5, **kw)
    want = call()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = call(stream=other)
    torch.cuda.current_stream().wait_stream(other)
    assert torch.equal(got, want)                               # and the same bits from call to call
    graphs, outs = [], []
    for _ in range(2):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call())
        graphs.append(graph)
    gen = torch.Generator().manual_seed(3)
    for k in range(4):
        wd.q.copy_(torch.randn(wd.q.shape, generator=gen))
        lam.copy_(torch.rand(lam.shape, generator=gen))
        graphs[k % 2].replay()
        pa.decode(torch.zeros(13, 16, 128, dtype=wd.q.dtype, device=DEV), wd.k_pool, wd.v_pool)
        assert torch.equal(outs[k % 2], call())
    pa.close()


@pytest.mark.gpu
def test_beyond_four_gigabytes():
    """Pages far behind the first 4 GB of their pools: offsets pass 32 bits."""
    head = head_of(2, 1, 64, DTYPE_BF16, 16)
    f = two_level_forest(70, [40, 5])
    paged = build_paged_kv(f, head, seed=3, layout="htd")
    small = make_workload("small", f, head, seed=3, layout="htd", paged=paged)
    pages = (1 << 20) + 200000                                  # of 4 KB: 5 GB
    moved = build_paged_kv(f, head, seed=3, layout="htd")
    moved.page_ids = (pages - 1 - paged.page_ids * 31).astype(np.int32)
    moved.num_pages = pages
    k, v = (torch.zeros((pages, 1, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    ids = torch.from_numpy(moved.page_ids.astype(np.int64)).to(DEV)
    for big, pool in ((k, small.k_pool), (v, small.v_pool)):
        big[ids] = pool[torch.from_numpy(paged.page_ids.astype(np.int64))].to(DEV)
    q = (torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(0)) * 2).bfloat16()
    small.q, lam = q, torch.full((2, 2), 0.5)
    pa = C.PlannedAttention(f, moved, head, device=DEV)
    compare(small, pa.decode_differential(q.to(DEV), k, v, lam.to(DEV)), lam)
    pa.close()
    del k, v
    torch.cuda.empty_cache()
