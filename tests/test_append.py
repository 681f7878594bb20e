"""Rotary positions and appending to the cache: frequencies and refusals on the CPU, results on the GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C
from oracle import operators as O
from workloads import HeadConfig, DTYPE_BF16, DTYPE_FP16

DEV = "cuda:0"
TORCH = {DTYPE_FP16: torch.float16, DTYPE_BF16: torch.bfloat16}
SCALINGS = [None, dict(kind="linear", factor=4.0), dict(kind="ntk", factor=8.0),
            dict(kind="wavelength", factor=8.0, original_length=8192, low=1.0, high=4.0),
            dict(kind="yarn", factor=4.0, original_length=4096, fast=32.0, slow=1.0),
            dict(kind="yarn", factor=0.5, original_length=64, fast=32.0, slow=1.0)]


def frequencies(r, theta, scaling):
    return O.rotary_frequencies(r, theta, **(scaling or {}))


# ---- on the CPU ------------------------------------------------------------------------------------------


@pytest.mark.parametrize("r", [2, 4, 20, 64, 128, 256])
@pytest.mark.parametrize("theta", [10000.0, 500000.0])
@pytest.mark.parametrize("scaling", SCALINGS)
def test_turns_of_a_position(r, theta, scaling):
    rot = C.Rotary(r, theta=theta, scaling=scaling, device="cpu")
    want, magnitude = frequencies(r, theta, scaling)
    # a handful of 64-bit operations, among them a power with an exponent of up to log(theta) = 13
    assert np.all(np.abs(rot.turns.numpy() * 2 * math.pi - want) <= 2.0 ** -47 * np.abs(want))
    assert abs(rot.magnitude - magnitude) <= 2.0 ** -24 * magnitude


def test_turns_refusals():
    def status(r=64, theta=1e4, **s):
        kind = s.pop("kind", 0)
        v = dict(original_length=4096, factor=2.0, low=1.0, high=4.0, fast=32.0, slow=1.0)
        v.update(s)
        return C.codec_rotary_turns(r, theta, C.codec_rotary_scaling(kind, v["original_length"], v["factor"], v["low"], v["high"],
                                                                    v["fast"], v["slow"]))[0]
    assert all(status(kind=k) == C.CODEC_OK for k in range(5))
    nan, inf = float("nan"), float("inf")
    bad = [dict(r=r) for r in (0, -2, 1, 63, 258)] + [dict(theta=t) for t in (1.0, 0.0, -5.0, nan, inf)] + [dict(kind=k) for k in (-1, 5)]
    bad += [dict(kind=k, factor=f) for k in (1, 2, 3, 4) for f in (0.0, -1.0, nan, inf)]
    bad += [dict(kind=k, original_length=n) for k in (3, 4) for n in (0, -1)]
    bad += [dict(kind=3, low=4.0), dict(kind=3, low=nan), dict(kind=3, high=inf)]
    bad += [dict(kind=4, slow=0.0), dict(kind=4, slow=32.0), dict(kind=4, fast=nan), dict(kind=4, fast=inf)]
    for b in bad:
        assert status(**b) == C.CODEC_ERR_INVALID_ARGUMENT, b
    assert C.codec_rotary_turns(64, 1e4, None)[0] == C.CODEC_OK
    lib = ctypes.CDLL(C.LIB_PATH)
    assert lib.codec_rotary_turns(64, ctypes.c_double(1e4), None, None, None) == C.CODEC_ERR_INVALID_ARGUMENT
    for s in (dict(kind="other", factor=2.0), dict(factor=2.0), dict(kind="linear", factor=2.0, length=3)):
        with pytest.raises(ValueError):
            C.Rotary(64, scaling=s, device="cpu")
    with pytest.raises(C.CodecError):
        C.Rotary(64, scaling=dict(kind="linear"), device="cpu")


def test_rotary_refusals():
    """Argument errors that are caught before any HIP call."""
    def status(tokens=4, heads=2, d=64, dtype=1, positions=4096, x=(1 << 20, 128, 64), out=(1 << 21, 128, 64), r=64, layout=0,
               magnitude=1.0, turns=4096, config=True):
        cfg = C.codec_rotary_config(r, layout, 0, magnitude, turns) if config else None
        return C.codec_rotary(cfg, heads, d, dtype, C.codec_rows(*x) if x else None, C.codec_rows(*out) if out else None,
                              positions, tokens)
    assert status(tokens=0) == C.CODEC_OK                              # nothing to do, nothing launched
    assert status(tokens=0, x=None, out=None, positions=0) == C.CODEC_OK
    at = 1 << 20
    for bad in (dict(config=False), dict(tokens=-1), dict(heads=0), dict(heads=1 << 17), dict(positions=0), dict(x=None), dict(out=None),
                dict(x=(0, 128, 64)), dict(x=(at + 8, 128, 64)), dict(x=(at, 132, 64)), dict(x=(at, 128, 68)), dict(x=(at, -128, 64)),
                dict(x=(at, 1 << 57, 64)), dict(out=(1 << 21, 64, 64)), dict(out=(1 << 21, 128, 0)), dict(out=(1 << 21, 0, 64)),
                dict(out=(at + 256, 128, 64)), dict(out=(at, 256, 64)), dict(out=(at + 128, 128, 64)),
                dict(r=0), dict(r=3), dict(r=66), dict(r=-2), dict(layout=2), dict(layout=-1), dict(magnitude=float("nan")),
                dict(magnitude=float("inf")), dict(turns=0)):
        assert status(**bad) == C.CODEC_ERR_INVALID_ARGUMENT, bad
    for bad in (dict(d=96), dict(d=32), dict(dtype=2), dict(dtype=-1)):
        assert status(**bad) == C.CODEC_ERR_UNSUPPORTED, bad


def test_append_refusals():
    base = 1 << 30
    good = dict(head=(8, 2, 128, 1, 16), q=(base, 1024, 128), q_out=(base, 1024, 128), k=(base + (1 << 20), 256, 128),
                v=(base + (1 << 21), 256, 128), positions=4096, slots=4096, tokens=3, kp=base * 2, vp=base * 3,
                layout=(8, 4096, 128, 2048), rotary=(128, 0, 0, 1.0, 4096))

    def status(**kw):
        a = dict(good, **kw)
        row = lambda r: C.codec_rows(*r) if r else None
        head = C.codec_head_config(*a["head"], 0.0) if a["head"] else None
        return C.codec_append(head, C.codec_rotary_config(*a["rotary"]) if a["rotary"] else None, row(a["q"]), row(a["q_out"]),
                              row(a["k"]), row(a["v"]), a["positions"], a["slots"], a["tokens"], a["kp"], a["vp"],
                              C.codec_kv_layout(*a["layout"]) if a["layout"] else None)
    assert status(tokens=0) == C.CODEC_OK
    at = base + (1 << 20)
    for bad in (dict(head=None), dict(layout=None), dict(tokens=-1), dict(q=None), dict(q_out=None), dict(k=None), dict(v=None),
                dict(slots=0), dict(positions=0), dict(kp=0), dict(vp=0), dict(kp=base * 2 + 8), dict(vp=base * 2),
                dict(head=(8, 0, 128, 1, 16)), dict(head=(0, 2, 128, 1, 16)), dict(head=(8, 2, 128, 1, 16), rotary=(130, 0, 0, 1.0, 4096)),
                dict(layout=(0, 4096, 128, 2048)), dict(layout=(8, 4096, 64, 2048)), dict(layout=(8, 4096, 132, 2048)),
                dict(layout=(8, 2048, 128, 2048)), dict(layout=(8, 4096, 128, 128)), dict(layout=(1 << 32, 4096, 128, 2048)),
                dict(k=(at + 2, 256, 128)), dict(k=(at, 256, 100)), dict(k=(base * 2 + 4096, 256, 128)), dict(v=(base * 3, 256, 128)),
                dict(q=(base * 3, 1024, 128), q_out=(base * 3, 1024, 128)), dict(q_out=(at, 1024, 128)),
                dict(q_out=(base + 1024, 1024, 128)), dict(head=(8, 4097, 128, 1, 16)),
                dict(vp=base * 2 + 256), dict(vp=base * 2 + 16 * 128 * 2), dict(vp=base * 2 + 4096 * 2)):
        assert status(**bad) == C.CODEC_ERR_INVALID_ARGUMENT, bad
    for bad in (dict(head=(8, 2, 96, 1, 16)), dict(head=(8, 2, 128, 2, 16)), dict(head=(8, 2, 128, 1, 24)), dict(head=(8, 2, 128, 1, 8))):
        assert status(**bad) == C.CODEC_ERR_UNSUPPORTED, bad


def test_cache_refusals():
    head = HeadConfig(8, 2, 128, DTYPE_BF16)
    cache = C.KVCache(head, 4, layers=2, device="cpu")
    assert cache.pools[0][0].shape == (4, 2, 16, 128) and C.KVCache(head, 4, layout="thd", device="cpu").pools[0][0].shape == (4, 16, 2, 128)
    z = torch.zeros(1, 2, 128, dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int64)
    with pytest.raises(ValueError):                      # no CPU path
        cache.append(0, None, z, z, None, i)
    with pytest.raises(ValueError):
        C.Rotary(128, device="cpu").apply(z, i)
    for pools in ([], [(cache.pools[0][0],)], [(cache.pools[0][0], cache.pools[0][1][:3])], [(cache.pools[0][0], cache.pools[0][1].half())],
                  [(cache.pools[0][0], torch.zeros(4, 2, 16, 256, dtype=torch.bfloat16)[..., :128])],
                  [(cache.pools[0][0].transpose(2, 3).contiguous().transpose(2, 3),) * 2]):
        with pytest.raises(ValueError):
            C.KVCache(head, 4, pools=pools, device="cpu")
    with pytest.raises(ValueError):
        C.KVCache(head, 4, layout="dht", device="cpu")
    with pytest.raises(ValueError):
        C.KVCache(HeadConfig(8, 2, 128, 2), 4, device="cpu")


def other_pools(cache, device):
    """What may become of a pool after it was handed over, that no call can use: (what, how)."""
    like = dict(dtype=cache.dtype, device=device)
    shape = cache.pools[0][0].shape
    p_bytes = 2 * cache.pools[0][0].numel()

    def cut(t):
        t.untyped_storage().resize_(p_bytes)
        return t

    def data(make):
        def change(p):
            p.data = make()
        return change
    return [("smaller", data(lambda: torch.zeros(shape[0] - 1, *shape[1:], **like))),
            ("a view that ends early", data(lambda: torch.zeros(shape, **like)[:2])),
            ("spread", data(lambda: torch.zeros(shape[0], 2 * shape[1], *shape[2:], **like)[:, ::2])),
            ("turned", data(lambda: torch.zeros(shape, **like).transpose(1, 2).contiguous().transpose(1, 2))),
            ("of 32 bits", data(lambda: torch.zeros(shape, dtype=torch.float32, device=device))),
            ("broadcast", data(lambda: torch.zeros(1, *shape[1:], **like).expand(shape))),
            ("set, then cut", lambda p: (p.set_(torch.zeros(shape, **like)), p.untyped_storage().resize_(64))),
            ("16 bytes too far", data(lambda: cut(torch.zeros(p_bytes // 2 + 8, **like)[8:].view(shape)))),
            ("given back", lambda p: p.untyped_storage().resize_(0))]


@pytest.mark.parametrize("which", range(9))
@pytest.mark.parametrize("layout", ["thd", "htd"])
def test_pools_are_looked_at_as_they_are_now(which, layout):
    head = HeadConfig(8, 2, 128, DTYPE_BF16)
    for at in (0, 1):
        cache = C.KVCache(head, 4, layers=2, layout=layout, device="cpu")
        cache._check_storage(0)
        what, change = other_pools(cache, "cpu")[which]
        change(cache.pools[1][at])
        cache._check_storage(0)
        with pytest.raises(ValueError):
            cache._check_storage(1)
    cache = C.KVCache(head, 4, layout=layout, device="cpu")
    for p in cache.pools[0]:                            # other memory of the same kind
        p.data = torch.zeros(8, *p.shape[1:], dtype=p.dtype)[2:6]
    cache._check_storage(0)
    with pytest.raises(AttributeError):
        cache.pools = [tuple(torch.zeros_like(p) for p in cache.pools[0])]


def test_pools_that_moved_where_no_copy_can_write_are_refused_before_pages_change_hands():
    cache = C.KVCache(HeadConfig(8, 2, 128, DTYPE_BF16), 4, device="cpu")
    ids = cache.take(2)
    with pytest.raises(ValueError):                     # no GPU
        cache.copy([(0, 0, 1, 0, 1)])
    k, v = cache.pools[0]
    k.data = v.data                                     # onto each other, and not aligned
    for _ in range(2):
        for call in (lambda: cache.copy([(0, 0, 1, 0, 1)]), cache.compact, lambda: cache.fork([0, 1], ids[:1], [3], [0, 0])):
            with pytest.raises(C.CodecError):
                call()
            assert cache.free_pages == 2
        k.data = torch.zeros(v.numel() + 8, dtype=v.dtype)[4:-4].view(v.shape)


def test_the_table_of_turns_is_the_calls_own():
    """What is done to the tensor that a program gets leaves the memory the kernels read as it is."""
    rot = C.Rotary(64, device="cpu")
    want, at = rot.turns, rot._config[0].turns
    rot.turns.untyped_storage().resize_(0)
    rot.turns.data = torch.zeros(3)
    rot.turns.mul_(2)
    with pytest.raises(AttributeError):
        rot.turns = want * 2
    assert torch.equal(rot.turns, want) and rot._config[0].turns == rot._config[1].turns == at != want.data_ptr()


# ---- on the GPU ------------------------------------------------------------------------------------------


def half_step(dtype):
    """A rounding's relative error, and its absolute one where the type's steps no longer shrink."""
    f = torch.finfo(TORCH[dtype])
    return f.eps / 2, f.tiny * f.eps / 2


def close(got, want, size, dtype, what=""):
    """One rounding to 16 bits, behind 32-bit products: cosine and sine are off by at most 3 half steps of a 32-bit one (the
    reduced angle, the series, the magnitude), a product and a sum round once each: 5 half steps of the pair's |a| + |b|;
    6 are allowed."""
    rel, least = half_step(dtype)
    got = got.double().cpu().numpy()
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = np.abs(got - want) <= rel * np.abs(want) + (1 + rel) * 6 * 2.0 ** -24 * size + least
    assert np.all(same | ok), f"{what}: {np.count_nonzero(~(same | ok))} values, worst {np.nanmax(np.abs(got - want))}"


def rows(gen, dtype, *shape):
    return torch.randn(shape, generator=gen).to(TORCH[dtype])


def flat_pool(pool, layout):
    """[pages * page_size, heads, d]"""
    return (pool if layout == "thd" else pool.transpose(1, 2)).flatten(0, 1)


def run_append(tokens, hq, hkv, d, dtype, page, layout, r, interleaved=False, scaling=None, fused=False, seed=0, positions=None, slots=None,
               pool=None, in_place=False, theta=10000.0, queries=True, rotate=True, spare=5):
    """One call against the oracle, pools checked whole: slots that are not named keep their bits."""
    print(f"[case] append tokens={tokens} heads={hq}/{hkv} d={d} dtype={dtype} page={page} {layout} r={r} interleaved={interleaved} "
          f"scaling={scaling} fused={fused} in_place={in_place} queries={queries} rotate={rotate}", flush=True)
    gen = torch.Generator().manual_seed(seed + 17)
    rng = np.random.default_rng(seed)
    head = HeadConfig(hq, hkv, d, dtype, page)
    pages = -(-tokens // page) + spare
    x = rows(gen, dtype, tokens, hq + 2 * hkv, d)
    x_dev = x.to(DEV)
    q, k, v = x_dev.split([hq, hkv, hkv], 1) if fused else (p.contiguous() for p in x_dev.split([hq, hkv, hkv], 1))
    if pool is None:
        shape = (pages, page, hkv, d) if layout == "thd" else (pages, hkv, page, d)
        pool = tuple(rows(gen, dtype, *shape).to(DEV) for _ in "kv")
    before = [p.cpu().clone() for p in pool]
    cache = C.KVCache(head, pages, layout=layout, device=DEV, pools=[pool])
    if positions is None:
        positions = rng.integers(-1000, 200000, tokens)
    if slots is None:
        slots = rng.permutation(pages * page)[:tokens]
        slots[rng.random(tokens) < 0.2] = -1
    positions, slots = np.asarray(positions, np.int64), np.asarray(slots, np.int64)
    rot = C.Rotary(r, theta=theta, interleaved=interleaved, scaling=scaling, device=DEV) if rotate else None
    out = cache.append(0, q if queries else None, k, v, torch.from_numpy(positions).to(DEV) if rotate else None,
                       torch.from_numpy(slots).to(DEV), rot, q_out=q if in_place else None)
    torch.cuda.synchronize()
    turns, magnitude = (rot.turns.cpu().numpy(), rot.magnitude) if rotate else (np.zeros(0), 1.0)
    x64 = x.double().numpy()
    turn = lambda a: O.rotary(a, positions, turns, magnitude, interleaved)
    if queries:
        close(out, *turn(x64[:, :hq]), dtype, "queries")
        if in_place:
            assert out.data_ptr() == q.data_ptr()
        elif fused:
            assert torch.equal(x_dev[:, :hq].cpu().view(torch.int16), x[:, :hq].view(torch.int16))
    else:
        assert out is None
    kept = (slots >= 0) & (slots < pages * page)
    want_k, size = turn(x64[:, hq:hq + hkv])
    k_now, v_now = (flat_pool(p.cpu(), layout) for p in pool)
    close(k_now[slots[kept]], want_k[kept], size[kept], dtype, "keys")
    v_want = flat_pool(before[1], layout).clone()
    v_want[slots[kept]] = x[:, hq + hkv:][kept]
    assert torch.equal(v_now.contiguous().view(torch.int16), v_want.contiguous().view(torch.int16))
    others = np.setdiff1d(np.arange(pages * page), slots)
    assert torch.equal(k_now[others].contiguous().view(torch.int16), flat_pool(before[0], layout)[others].contiguous().view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,r", [(64, 64), (64, 32), (64, 2), (64, 20), (64, 62), (64, 48), (128, 128), (128, 64), (128, 16), (128, 24),
                                 (128, 126), (256, 256), (256, 64), (256, 144), (256, 250)])
@pytest.mark.parametrize("dtype", [DTYPE_FP16, DTYPE_BF16])
def test_append_channels(d, r, interleaved, dtype):
    run_append(37, 6, 3, d, dtype, 16, "htd", r, interleaved, seed=d + r)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 2, 3, 7, 16, 33, 64, 129, 500, 1023, 2048, 4099])
@pytest.mark.parametrize("hq,hkv,d,layout,fused", [(8, 8, 128, "htd", False), (32, 8, 128, "thd", True), (28, 4, 64, "htd", True), (16, 1, 256, "thd", False),
                                                   (1, 1, 64, "thd", True)])
def test_append_sizes(tokens, hq, hkv, d, layout, fused):
    run_append(tokens, hq, hkv, d, DTYPE_BF16, 32, layout, d, fused=fused, seed=tokens)


@pytest.mark.gpu
@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("positions", [[0, 1, -1], [131071, 1 << 20, (1 << 31) + 5], [-(1 << 33) - 7, 12345678901, 3]])
def test_append_positions(scaling, positions):
    """Near and far positions: the angle keeps its fraction of a turn."""
    for r, interleaved in ((128, False), (128, True), (36, False)):
        run_append(3, 4, 2, 128, DTYPE_FP16, 16, "htd", r, interleaved, scaling=scaling, positions=positions, theta=500000.0)


@pytest.mark.gpu
@pytest.mark.parametrize("variant", [dict(in_place=True), dict(in_place=True, fused=True), dict(queries=False), dict(rotate=False),
                                     dict(rotate=False, queries=False), dict(slots=[-1] * 21), dict(fused=True, rotate=False)])
def test_append_variants(variant):
    run_append(21, 10, 2, 128, DTYPE_BF16, 16, "thd", 96, **variant)


@pytest.mark.gpu
def test_append_slots_out_of_range_are_not_stored():
    last = 6 * 16
    run_append(9, 4, 2, 64, DTYPE_FP16, 16, "htd", 64, slots=[last, last - 1, -1, 0, last + 5, 1 << 40, -(1 << 62), (1 << 63) - 1, 17], spare=5)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["side by side", "padded tokens", "pages last"])
def test_append_pools_with_other_strides(kind):
    pages, page, hkv, d = 7, 16, 3, 64
    gen = torch.Generator().manual_seed(5)
    if kind == "side by side":                          # K and V of a page and head in one pool
        big = rows(gen, DTYPE_BF16, pages, hkv, 2, page, d).to(DEV)
        pool = (big[:, :, 0], big[:, :, 1])
    elif kind == "padded tokens":
        pool = tuple(rows(gen, DTYPE_BF16, pages, hkv, page, d + 24).to(DEV)[..., 8:8 + d] for _ in "kv")
    else:                                               # all pages of a head together
        pool = tuple(rows(gen, DTYPE_BF16, hkv, pages, page, d).to(DEV).transpose(0, 1) for _ in "kv")
    run_append(20, 6, hkv, d, DTYPE_BF16, page, "htd", 64, pool=pool, spare=5)


@pytest.mark.gpu
@pytest.mark.parametrize("r", [2, 6, 14, 18, 30, 34, 58, 60, 62, 122, 124, 126])
@pytest.mark.parametrize("d", [64, 128])
def test_append_halves_of_any_size_in_place(d, r):
    """Other halves before and behind a lane's channels, over both ends of the row; queries onto themselves."""
    if r > d:
        return
    run_append(19, 7, 2, d, DTYPE_FP16, 16, "thd", r, in_place=True, fused=True, seed=r)
    run_append(700, 3, 1, d, DTYPE_BF16, 64, "htd", r, seed=r)


@pytest.mark.gpu
def test_append_beyond_four_gigabytes():
    """Pools of 8.6 GB each: slots, pages and byte offsets pass 32 bits."""
    head = HeadConfig(2, 1, 64, DTYPE_BF16, 16)
    pages = 1 << 22
    cache = C.KVCache(head, pages, device=DEV)
    gen = torch.Generator().manual_seed(3)
    x = rows(gen, DTYPE_BF16, 5, 4, 64).to(DEV)
    slots = torch.tensor([pages * 16 - 1, 0, (1 << 31) // 64, pages * 8 + 3, pages * 16 - 17], device=DEV)
    rot = C.Rotary(64, device=DEV)
    positions = torch.arange(5, device=DEV)
    cache.append(0, x[:, :2], x[:, 2:3], x[:, 3:], positions, slots, rot)
    want = rot.apply(x[:, 2:3], positions)[:, 0]
    k, v = (p[slots // 16, 0, slots % 16] for p in cache.pools[0])
    assert torch.equal(k, want) and torch.equal(v, x[:, 3])
    cache.copy([(pages - 1, 15, 7, 2, 1), (pages // 2, 3, pages - 2, 4, 1)])
    k, v = cache.pools[0]
    assert torch.equal(k[7, 0, 2], want[0]) and torch.equal(v[pages - 2, 0, 4], x[3, 3])
    del cache, k, v
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_append_values_that_are_not_numbers():
    """Infinities and NaN stay in their pairs; channels that pass keep their bits."""
    for r, interleaved in ((32, False), (32, True), (20, False), (22, True)):
        x = torch.randn(5, 4, 64, generator=torch.Generator().manual_seed(1)).half()
        x[0, 0, 3], x[1, 1, 40], x[2, 2, 63], x[3, 3, r], x[4, 0, r - 1] = math.inf, math.nan, -math.inf, math.nan, math.nan
        rot = C.Rotary(r, interleaved=interleaved, device=DEV)
        positions = np.array([5, 0, 9, 100, 7])
        got = rot.apply(x.to(DEV), torch.from_numpy(positions).to(DEV))
        want, size = O.rotary(x.double().numpy(), positions, rot.turns.cpu().numpy(), 1.0, interleaved)
        size[~np.isfinite(size)] = 0.0
        close(got, want, size, DTYPE_FP16)
        assert torch.equal(got[..., r:].cpu().view(torch.int16), x[..., r:].contiguous().view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,d,r", [(1, 1, 64, 64), (5, 3, 128, 128), (100, 16, 256, 64), (3001, 32, 128, 128), (64, 7, 64, 30)])
def test_rotary_back(tokens, heads, d, r, interleaved):
    """The inverse is the transpose: the gradient of the turn.  In place and not, from a strided view too."""
    print(f"[case] rotary back {tokens} {heads} {d} {r} {interleaved}", flush=True)
    gen = torch.Generator().manual_seed(tokens)
    rng = np.random.default_rng(3)
    scaling = dict(kind="yarn", factor=4.0, original_length=4096)
    g = rows(gen, DTYPE_BF16, tokens, heads + 2, d)
    positions = rng.integers(0, 1 << 17, tokens)
    rot = C.Rotary(r, interleaved=interleaved, scaling=scaling, device=DEV)
    at = torch.from_numpy(positions).to(DEV)
    turns, magnitude = rot.turns.cpu().numpy(), rot.magnitude
    want, size = O.rotary(g[:, 1:-1].double().numpy(), positions, turns, magnitude, interleaved, inverse=True)
    big = g.to(DEV)
    got = rot.apply(big[:, 1:-1], at, inverse=True)
    close(got, want, size, DTYPE_BF16)
    assert torch.equal(rot.apply(big[:, 1:-1], at, inverse=True, out=big[:, 1:-1]), got)
    assert torch.equal(big[:, 1:-1], got) and torch.equal(big[:, 0].cpu(), g[:, 0]) and torch.equal(big[:, -1].cpu(), g[:, -1])
    # against differences: the turn is linear, so a step of any size gives the derivative along it
    x, dx = (rng.standard_normal((1, 1, d)) for _ in range(2))
    ahead, behind = (O.rotary(x + h * dx, positions[:1], turns, magnitude, interleaved)[0] for h in (0.5, -0.5))
    w = g[:1, 1:2].double().numpy()
    assert abs(np.sum(w * (ahead - behind)) - np.sum(dx * want[:1, :1])) <= 1e-9 * d


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("tokens,heads,d,r,dtype", [(1, 1, 64, 64, DTYPE_BF16), (37, 3, 128, 128, DTYPE_FP16), (200, 5, 256, 64, DTYPE_BF16), (9, 2, 64, 30, DTYPE_FP16)])
def test_rotary_gradient(tokens, heads, d, r, dtype, interleaved, inverse):
    """Against the formula (the transpose) and against differences; gradients of any strides, broadcast ones too; twice."""
    print(f"[case] gradient {tokens} {heads} {d} {r} {interleaved} {inverse}", flush=True)
    gen = torch.Generator().manual_seed(tokens)
    scaling = dict(kind="yarn", factor=4.0, original_length=4096)
    rot = C.Rotary(r, interleaved=interleaved, scaling=scaling, device=DEV)
    turns, magnitude = rot.turns.cpu().numpy(), rot.magnitude
    positions = np.random.default_rng(tokens).integers(0, 1 << 17, tokens)
    at = torch.from_numpy(positions).to(DEV)
    x, w, u = (torch.randn(tokens, heads, d, generator=gen).to(TORCH[dtype]) for _ in range(3))
    leaf = x.to(DEV).requires_grad_()
    y = rot.apply(leaf, at, inverse=inverse)
    with torch.no_grad():
        plain = rot.apply(leaf, at, inverse=inverse)
    assert y.requires_grad and not plain.requires_grad and torch.equal(y, plain)
    back, size = O.rotary(w.double().numpy(), positions, turns, magnitude, interleaved, inverse=not inverse)
    odd = torch.zeros(tokens, heads, d + 3, dtype=TORCH[dtype], device=DEV)[:, :, 3:]     # no multiple of 16 bytes
    wide = torch.zeros(tokens * heads * d + 3, dtype=TORCH[dtype], device=DEV)[3:].view(tokens, heads, d)
    turned = torch.zeros(d, heads, tokens, dtype=TORCH[dtype], device=DEV).permute(2, 1, 0)
    for g in (w.to(DEV), odd.copy_(w), wide.copy_(w), turned.copy_(w)):
        (got,) = torch.autograd.grad(y, leaf, g, retain_graph=True)
        close(got, back, size, dtype)
    (got,) = torch.autograd.grad(y.sum(), leaf, retain_graph=True)                        # a broadcast gradient
    ones, ones_size = O.rotary(np.ones((tokens, heads, d)), positions, turns, magnitude, interleaved, inverse=not inverse)
    close(got, ones, ones_size, dtype)
    # the turn is linear, so the difference along u is the turn of u; each side is rounded by half a step, of |w| |turned u| and |u| |back|
    step = torch.finfo(TORCH[dtype]).eps / 2
    u_turned = rot.apply(u.to(DEV), at, inverse=inverse).double().cpu().numpy()
    (g,) = torch.autograd.grad(y, leaf, w.to(DEV), retain_graph=True)
    g, w64, u64 = g.double().cpu().numpy(), w.double().numpy(), u.double().numpy()
    assert abs(np.sum(w64 * u_turned) - np.sum(u64 * g)) <= 1.01 * step * (np.sum(np.abs(w64 * u_turned)) + np.sum(np.abs(u64 * g)))
    # the gradient of the gradient by what it was taken of: the turn itself
    v = w.to(DEV).requires_grad_()
    (g,) = torch.autograd.grad(y, leaf, v, create_graph=True)
    (gg,) = torch.autograd.grad(g, v, u.to(DEV))
    assert torch.equal(gg, rot.apply(u.to(DEV), at, inverse=inverse))


@pytest.mark.gpu
def test_rotary_gradient_in_a_program():
    """Through a projection, on another stream, of a part of a projection's output; what does not pass a gradient says so."""
    gen = torch.Generator().manual_seed(31)
    rot = C.Rotary(64, device=DEV)
    at = torch.arange(6, device=DEV)
    weight = torch.randn(3 * 64 * 4, 32, generator=gen).to(torch.bfloat16).to(DEV).requires_grad_()
    x = torch.randn(6, 32, generator=gen).to(torch.bfloat16).to(DEV)
    w = torch.randn(6, 4, 64, generator=gen).to(torch.bfloat16).to(DEV)
    grads = []
    side = torch.cuda.Stream()
    for stream in (None, side):
        q = (x @ weight.t()).view(6, 12, 64)[:, 4:8]
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        y = rot.apply(q, at, stream=stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        y.backward(w)
        torch.cuda.synchronize()
        grads.append(weight.grad.clone())
        weight.grad = None
    back = rot.apply(w, at, inverse=True)
    want = torch.zeros(6, 12, 64, dtype=torch.bfloat16, device=DEV)
    want[:, 4:8] = back
    want = want.view(6, -1).float().t() @ x.float()
    size = want.new_zeros(6, 12, 64)
    size[:, 4:8] = back.float().abs()
    size = size.view(6, -1).t() @ x.float().abs()
    # half a step of the sum, and 32-bit sums of six
    for g in grads:
        assert bool(((g.float() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * size).all())
    leaf = w.clone().requires_grad_()
    for out in (torch.empty_like(w), leaf):
        with pytest.raises(ValueError):
            rot.apply(leaf, at, out=out)
    with torch.no_grad():
        assert torch.equal(rot.apply(leaf, at, out=torch.empty_like(w)), rot.apply(w, at))
    y = rot.apply(leaf, at)
    at.add_(1)                                          # other positions than those of the call
    with pytest.raises(RuntimeError):
        y.backward(w)
    assert not rot.apply(w, at).requires_grad


@pytest.mark.gpu
def test_append_on_another_stream_and_captured():
    """The call's stream is the one it is given; a captured call replays on what its tensors then hold."""
    head = HeadConfig(8, 2, 128, DTYPE_BF16)
    cache = C.KVCache(head, 8, device=DEV)
    for p in cache.pools[0]:
        p.zero_()
    rot = C.Rotary(128, device=DEV)
    gen = torch.Generator().manual_seed(2)
    batches = [[rows(gen, DTYPE_BF16, 5, n, 128).to(DEV) for n in (8, 2, 2)] for _ in range(4)]
    positions = [torch.arange(5, device=DEV) * (i + 1) for i in range(4)]
    slots = [torch.arange(5, device=DEV) * 3 + 20 * i for i in range(4)]
    want = [cache.append(0, *b, p, s, rot) for b, p, s in zip(batches, positions, slots)]
    pools = [p.clone() for p in cache.pools[0]]
    for p in cache.pools[0]:
        p.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = cache.append(0, *batches[0], positions[0], slots[0], rot, stream=side)
    side.synchronize()
    assert torch.equal(got, want[0])
    held, at, where = [t.clone() for t in batches[0]], positions[0].clone(), slots[0].clone()
    out = torch.empty_like(held[0])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cache.append(0, *held, at, where, rot, q_out=out)
    for i in (1, 2, 3, 1, 2):
        for t, new in zip(held, batches[i]):
            t.copy_(new)
        at.copy_(positions[i])
        where.copy_(slots[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
    for p, q in zip(cache.pools[0], pools):
        assert torch.equal(p, q)


@pytest.mark.gpu
def test_append_tensor_refusals():
    head = HeadConfig(8, 2, 128, DTYPE_BF16)
    cache = C.KVCache(head, 8, device=DEV)
    rot = C.Rotary(128, device=DEV)
    q, k = (torch.zeros(3, n, 128, dtype=torch.bfloat16, device=DEV) for n in (8, 2))
    i = torch.zeros(3, dtype=torch.int64, device=DEV)
    for bad in (dict(q=q[:2]), dict(q=q.half()), dict(q=q.cpu()), dict(k=k[:, :1]), dict(v=k[:2]), dict(v=torch.zeros(3, 2, 256, dtype=torch.bfloat16, device=DEV)[..., ::2]),
                dict(positions=i[:2]), dict(positions=i.int()), dict(slots=i.int()), dict(slots=i.cpu()), dict(q=None, q_out=q), dict(q_out=q[:2]),
                dict(slots=torch.zeros(6, dtype=torch.int64, device=DEV)[::2])):
        a = dict(dict(q=q, k=k, v=k.clone(), positions=i, slots=i, rotary=rot, q_out=None), **bad)
        with pytest.raises(ValueError):
            cache.append(0, a["q"], a["k"], a["v"], a["positions"], a["slots"], a["rotary"], q_out=a["q_out"])
    odd = torch.zeros(3, 2, 132, dtype=torch.bfloat16, device=DEV)[..., 4:]                # not 16-byte aligned
    with pytest.raises(C.CodecError):
        cache.append(0, q, odd, k, i, i, rot)
    with pytest.raises(ValueError):                                                        # a table on the CPU
        cache.append(0, q, k, k.clone(), i, i, C.Rotary(128, device="cpu"))
    gone = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device=DEV)
    gone.untyped_storage().resize_(16)
    with pytest.raises(ValueError):
        cache.append(0, q, gone, k, i, i, rot)
    assert cache.append(0, q[:0], k[:0], k[:0], i[:0], i[:0], rot).shape == (0, 8, 128)
    cache.pools[0][1].untyped_storage().resize_(16)
    with pytest.raises(ValueError):
        cache.append(0, q, k, k.clone(), i, i, rot)
    both = torch.zeros(8, 2, 2, 16, 128, dtype=torch.bfloat16, device=DEV)
    for pools, apart in (((both[:, :, 0], both[:, :, 1]), True), ((both[:, :, 0], both[:, :, 0]), False), ((both[:7, :, 0], both[1:, :, 0]), False)):
        side = C.KVCache(head, len(pools[0]), device=DEV, pools=[pools])
        if apart:
            side.append(0, None, k, k.clone(), i, torch.arange(3, device=DEV), rot)
            side.copy([(0, 0, 1, 0, 3)])
        else:
            with pytest.raises(C.CodecError):
                side.append(0, None, k, k.clone(), i, torch.arange(3, device=DEV), rot)
            with pytest.raises(C.CodecError):
                side.copy([(0, 0, 1, 0, 3)])


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(9))
def test_pools_that_became_something_else_are_refused(which):
    head = HeadConfig(8, 2, 128, DTYPE_BF16)
    q, k = (torch.zeros(3, n, 128, dtype=torch.bfloat16, device=DEV) for n in (8, 2))
    i = torch.arange(3, device=DEV)
    cache = C.KVCache(head, 8, layers=2, device=DEV)
    ids = cache.take(3)
    cache.release(ids[:1])
    what, change = other_pools(cache, DEV)[which]
    print(f"[case] pool {what}", flush=True)
    if which % 3:                                       # before or after they were looked at
        cache.copy([(1, 0, 2, 0, 1)])
    change(cache.pools[1][which % 2])
    cache.append(0, q, k, k.clone(), i, i, C.Rotary(128, device=DEV))
    for call in (lambda: cache.append(1, q, k, k.clone(), i, i, C.Rotary(128, device=DEV)), lambda: cache.copy([(1, 0, 2, 0, 1)]), cache.compact,
                 lambda: cache.fork([0, 1], ids[1:2], [3], [0, 0])):
        with pytest.raises(ValueError):
            call()
        assert cache.free_pages == 6 and cache.take(1)[0] == 0
        cache.release([0])
    cache.release(ids[1:])                              # they are held as they were
    assert cache.free_pages == 8
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_fork_into_pools_that_moved_onto_each_other():
    """What the fork would copy is refused when its pages are known: they go back."""
    head = HeadConfig(8, 2, 128, DTYPE_BF16)
    cache = C.KVCache(head, 8, device=DEV)
    ids = cache.take(5)
    cache.hold(ids[:2])
    cache.copy([(0, 0, 1, 0, 1)])
    k, v = cache.pools[0]
    k.data = v.data
    off = [0, 2, 3, 5, 7]                               # two sequences share a page and a half, one goes on twice, one ends
    lists = ids[[0, 1, 2, 0, 1, 3, 4]]
    for _ in range(2):
        with pytest.raises(C.CodecError):
            cache.fork(off, lists, [20, 3, 20, 32], [0, 1, 1, 2])
        assert cache.free_pages == 3 and cache.take(3).tolist() == [5, 6, 7]
        cache.release([7, 6, 5])
    k.data = torch.zeros_like(v)
    new_off, new = cache.fork(off, lists, [20, 3, 20, 32], [0, 1, 1, 2])
    assert new_off.tolist() == [0, 2, 3, 4, 6] and new.tolist() == [0, 5, 2, 6, 0, 7] and cache.free_pages == 3      # 1, 3, 4
    cache.release(new)
    assert cache.free_pages == 8


@pytest.mark.gpu
def test_pools_that_got_other_memory():
    """The calls write where the tensor is now; what it had before is free."""
    head = HeadConfig(8, 2, 128, DTYPE_BF16)
    gen = torch.Generator().manual_seed(12)
    k, v = (torch.randn(3, 2, 128, generator=gen).to(torch.bfloat16).to(DEV) for _ in "kv")
    cache = C.KVCache(head, 4096, device=DEV)
    before = torch.cuda.memory_allocated()
    big = [torch.zeros(8192, 2, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    for p, b in zip(cache.pools[0], big):
        p.data = b[100:100 + 4096]
    slots = torch.tensor([5, 65535, 17], device=DEV)
    cache.append(0, None, k, v, None, slots)
    cache.copy([(1, 1, 4000, 3, 1)])
    del slots
    assert torch.cuda.memory_allocated() - before == 4096 * 2 * 16 * 128 * 2 * 2         # twice as much as there was, which is free
    torch.cuda.synchronize()
    for x, b in zip((k, v), big):
        want = torch.zeros_like(b)
        for row, page, token in ((0, 0, 5), (1, 4095, 15), (2, 1, 1), (2, 4000, 3)):
            want[100 + page, :, token] = x[row]
        assert torch.equal(b, want)


@pytest.mark.gpu
def test_rows_beyond_32_bits_are_refused():
    """2^32 + 64 channels are not 64."""
    x = torch.empty(1, 1, (1 << 32) + 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        C.Rotary(64, device=DEV).apply(x, torch.zeros(1, dtype=torch.int64, device=DEV))
    del x
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_append_more_tokens_than_a_launch():
    """2^24 + 5 tokens: every row as by a call of few tokens, stored in reverse order."""
    n = (1 << 24) + 5
    head = HeadConfig(1, 1, 64, DTYPE_BF16, 16)
    cache = C.KVCache(head, (n + 15) // 16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(11)
    x = torch.randint(-30000, 30000, (1024, 3, 64), dtype=torch.int16, device=DEV, generator=gen) & 0xbfff       # (no NaN, no inf)
    x = x.view(torch.bfloat16).repeat((n + 1023) // 1024, 1, 1)[:n]
    positions = torch.arange(n, device=DEV)
    rot = C.Rotary(64, device=DEV)
    print("[case] more tokens than a launch", flush=True)
    q = cache.append(0, x[:, :1], x[:, 1:2], x[:, 2:], positions, n - 1 - positions, rot)
    k, v = (p[:, 0].reshape(-1, 64)[:n].flip(0) for p in cache.pools[0])
    assert torch.equal(v, x[:, 2])
    for at in (0, 12345, (1 << 23) - 100, (1 << 24) - 200, n - 300):
        part = slice(at, at + 300)
        assert torch.equal(q[part], rot.apply(x[part, :1], positions[part])) and torch.equal(k[part, None], rot.apply(x[part, 1:2], positions[part]))
    del cache, k, v, q, x
    torch.cuda.empty_cache()
