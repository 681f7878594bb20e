"""Rotary positions with several axes: tables and refusals on the CPU, turns, gradients and appends on the GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C
from oracle import operators as O
from test_append import DEV, TORCH, close, flat_pool, rows
from workloads import HeadConfig, DTYPE_BF16, DTYPE_FP16

SCALINGS = [None, dict(kind="linear", factor=4.0), dict(kind="ntk", factor=8.0),
            dict(kind="yarn", factor=4.0, original_length=4096, fast=32.0, slow=1.0)]


# ---- on the CPU ------------------------------------------------------------------------------------------


@pytest.mark.parametrize("axes", [(16, 24, 24), (24, 20, 20), (5, 9, 2), (64,), (32, 32), (1, 1, 1, 1), (10, 0, 4, 3), (0, 7)])
@pytest.mark.parametrize("alternating,restart,blocks", [(False, False, 1), (True, False, 1), (False, True, 1), (True, True, 2), (False, False, 2)])
@pytest.mark.parametrize("scaling", SCALINGS)
def test_tables(axes, alternating, restart, blocks, scaling):
    r = 2 * sum(axes) * blocks
    rot = C.Rotary(r, theta=500000.0, scaling=scaling, device="cpu", axes=axes, alternating=alternating, restart=restart, blocks=blocks)
    want, axis, magnitude = O.axes_frequencies(list(axes), 500000.0, alternating, restart, blocks, **(scaling or {}))
    assert np.all(np.abs(rot.turns.numpy() * 2 * math.pi - want) <= 2.0 ** -47 * np.abs(want))       # as for one axis
    assert rot._axes.tolist() == axis.tolist() and abs(rot.magnitude - magnitude) <= 2.0 ** -24 * magnitude
    assert [rot._axes.tolist().count(a) for a in range(len(axes))] == [n * blocks for n in axes]


def test_one_axis_in_one_block_is_the_plain_table():
    plain = C.Rotary(96, device="cpu")
    assert plain._axes is None
    for kw in (dict(axes=[48]), dict(restart=True), dict(alternating=True)):
        rot = C.Rotary(96, device="cpu", **kw)
        assert torch.equal(rot.turns, plain.turns) and rot._axes.tolist() == [0] * 48


@pytest.mark.parametrize("kw", [dict(axes=[16, 15]), dict(axes=[]), dict(axes=[33, -1]), dict(axes=[8, 8, 8, 4, 4]), dict(axes=[16, 16], blocks=2),
                                dict(blocks=0), dict(blocks=3), dict(blocks=-1), dict(blocks=256)])
def test_axes_that_do_not_fit_are_refused(kw):
    with pytest.raises(ValueError):
        C.Rotary(64, device="cpu", **kw)


def test_refusals():
    """Argument errors that are caught before any HIP call, of both calls."""
    at = 1 << 20

    def status(tokens=4, d=64, x=(at, 128, 64), positions=4096, r=64, layout=0, block=0, n=3, axes=4096, stride=4, config=True, magnitude=1.0):
        cfg = C.codec_rotary_axes(C.codec_rotary_config(r, layout, 0, magnitude, 4096), block, n, axes, stride) if config else None
        rows_of = C.codec_rows(*x) if x else None
        one = C.codec_rotary_by_axes(cfg, 2, d, 1, rows_of, C.codec_rows(1 << 21, 128, 64), positions, tokens)
        head = C.codec_head_config(2, 2, d, 1, 16, 0.0)
        other = C.codec_append_by_axes(head, cfg, rows_of, C.codec_rows(1 << 21, 128, 64), C.codec_rows(1 << 22, 128, 64), C.codec_rows(1 << 23, 128, 64),
                                       positions, 4096, tokens, 1 << 24, 1 << 25, C.codec_kv_layout(8, 16 * 2 * 64, 128, 64))
        assert one == other
        return one

    assert status(tokens=0) == C.CODEC_OK and status(tokens=0, positions=0, block=64, stride=0) == C.CODEC_OK
    for bad in (dict(config=False), dict(n=0), dict(n=5), dict(n=-1), dict(axes=0), dict(stride=-1), dict(stride=1 << 60), dict(block=-16),
                dict(block=24), dict(block=128), dict(positions=0), dict(x=None), dict(r=0), dict(r=66), dict(layout=2), dict(magnitude=math.nan)):
        assert status(**bad) == C.CODEC_ERR_INVALID_ARGUMENT, bad
    # blocks of halves that are no multiple of 16 channels; neighbouring pairs want whole pairs in a block
    for bad in (dict(r=48, block=24), dict(r=64, block=8), dict(r=60, block=30), dict(r=60, block=15, layout=1)):
        assert status(**bad) == C.CODEC_ERR_UNSUPPORTED, bad
    lib = ctypes.CDLL(C.LIB_PATH)
    assert lib.codec_append_by_axes(None, None, None, None, None, None, None, None, 0, None, None, None, None) == C.CODEC_ERR_INVALID_ARGUMENT


# ---- on the GPU ------------------------------------------------------------------------------------------


def some_positions(rng, axes, tokens):
    p = rng.integers(-1000, 200000, (axes, tokens))
    p[:, : tokens // 3] = p[0, : tokens // 3]                   # text: the same on every axis
    return p


def apply_case(tokens, heads, d, dtype, axes, interleaved=False, inverse=False, seed=0, positions=None, theta=10000.0, scaling=None, **order):
    print(f"[case] axes={axes} tokens={tokens} heads={heads} d={d} dtype={dtype} interleaved={interleaved} inverse={inverse} "
          f"scaling={scaling} {order}", flush=True)
    gen, rng = torch.Generator().manual_seed(seed + 3), np.random.default_rng(seed)
    blocks = order.get("blocks", 1)
    rot = C.Rotary(2 * sum(axes) * blocks, theta=theta, interleaved=interleaved, scaling=scaling, device=DEV, axes=axes, **order)
    if positions is None:
        positions = some_positions(rng, len(axes), tokens)
    x = rows(gen, dtype, tokens, heads, d)
    got = rot.apply(x.to(DEV), torch.from_numpy(np.asarray(positions, np.int64)).to(DEV), inverse=inverse)
    turns = rot.turns.cpu().numpy()
    want, size = O.rotary_by_axes(x.double().numpy(), positions, turns, rot._axes.cpu().numpy(), rot.magnitude, interleaved, blocks, inverse)
    close(got, want, size, dtype, "rows")
    r = 2 * len(turns)
    assert torch.equal(got[..., r:].cpu().contiguous().view(torch.int16), x[..., r:].contiguous().view(torch.int16))
    return rot, x, positions, want, size


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,axes,blocks", [(64, (8, 12, 12), 1), (64, (16, 16), 1), (64, (5, 9, 2), 1), (64, (10, 0, 4, 3), 1), (64, (31,), 1),
                                           (64, (4, 4), 2), (64, (8,), 4), (128, (16, 24, 24), 1), (128, (24, 20, 20), 1), (128, (1, 1, 1, 1), 1),
                                           (128, (13, 19), 2), (128, (32,), 2), (128, (63, 0), 1), (256, (64,), 2), (256, (16, 20, 20), 2),
                                           (256, (3, 2, 1, 2), 16), (256, (40, 41, 42), 1)])
@pytest.mark.parametrize("order", [dict(), dict(alternating=True, restart=True)])
def test_channels(d, axes, blocks, interleaved, order):
    dtype = DTYPE_FP16 if sum(axes) % 2 else DTYPE_BF16
    apply_case(23, 5, d, dtype, axes, interleaved, seed=sum(axes) + d, blocks=blocks, **order)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 2, 3, 16, 65, 500, 1023, 4099])
@pytest.mark.parametrize("heads,d,axes", [(1, 64, (8, 12, 12)), (28, 128, (16, 24, 24)), (7, 256, (30, 20, 13))])
def test_sizes(tokens, heads, d, axes):
    apply_case(tokens, heads, d, DTYPE_BF16, axes, seed=tokens)


@pytest.mark.gpu
@pytest.mark.parametrize("scaling", SCALINGS)
def test_positions_near_and_far(scaling):
    far = [[0, 1, -1, 131071, 1 << 20], [(1 << 31) + 5, -(1 << 33) - 7, 12345678901, 3, 0], [7, 0, 1 << 40, -5, 9]]
    for interleaved in (False, True):
        apply_case(5, 3, 128, DTYPE_FP16, (24, 20, 20), interleaved, positions=far, theta=500000.0, scaling=scaling, alternating=True)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_one_position_for_all_axes_is_the_plain_turn(interleaved):
    """Text tokens: bit for bit what a rotary without axes gives; positions as [tokens], as equal rows, as an expanded view."""
    gen = torch.Generator().manual_seed(1)
    x = rows(gen, DTYPE_BF16, 77, 6, 128).to(DEV)
    p = torch.randint(-100, 1 << 20, (77,), generator=gen).to(DEV)
    want = C.Rotary(128, interleaved=interleaved, device=DEV).apply(x, p)
    rot = C.Rotary(128, interleaved=interleaved, device=DEV, axes=(16, 24, 24))
    for positions in (p, p.repeat(3, 1), p.expand(3, 77), p[None].repeat(4, 1)[1:]):
        assert torch.equal(rot.apply(x, positions), want)
    padded = torch.full((3, 100), 1 << 50, device=DEV)
    padded[:, 11:88] = p
    assert torch.equal(rot.apply(x, padded[:, 11:88]), want)


@pytest.mark.gpu
def test_an_axis_that_does_not_exist_counts_as_the_first():
    x = rows(torch.Generator().manual_seed(2), DTYPE_FP16, 9, 2, 64).to(DEV)
    p = torch.arange(27, device=DEV).view(3, 9)
    rot = C.Rotary(64, device=DEV, axes=(16, 8, 8))
    rot._axes[16:24] = 255                                      # read as axis 0, not from behind the positions
    want = C.Rotary(64, device=DEV, axes=(16, 8, 8))
    want._axes[16:24] = 0
    assert torch.equal(rot.apply(x, p), want.apply(x, p))
    rot._axes[16:24] = 3                                        # an axis of another rotary: there are three here
    assert torch.equal(rot.apply(x, p), want.apply(x, p))


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes,d,order", [((16, 24, 24), 128, {}), ((16, 16), 64, dict(restart=True)), ((5, 9, 2), 64, dict(alternating=True)),
                                          ((32, 32), 256, dict(blocks=2))])
def test_back_and_gradient(axes, d, order, interleaved):
    """The gradient of the turn is the turn back: against the formula, against differences, in place, from strided views."""
    rot, g, positions, want, size = apply_case(41, 4, d, DTYPE_BF16, axes, interleaved, inverse=True, seed=9, **order)
    at = torch.from_numpy(positions).to(DEV)
    x = rows(torch.Generator().manual_seed(8), DTYPE_BF16, 41, 4, d).to(DEV).requires_grad_()
    y = rot.apply(x, at)
    got, = torch.autograd.grad(y, x, g.to(DEV))
    close(got, want, size, DTYPE_BF16, "gradient")
    assert torch.equal(y.detach(), rot.apply(x.detach(), at))
    # a broadcast head: its gradient is the sum over the heads it stands for
    one = x.detach()[:, :1].clone().requires_grad_()
    got, = torch.autograd.grad(rot.apply(one.expand(-1, 4, -1), at), one, g.to(DEV))
    total, room = want.sum(1, keepdims=True), np.abs(want).sum(1, keepdims=True)
    err = np.abs(got.double().cpu().numpy() - total)
    # each summand is rounded once (2^-8 and the 32-bit products, as in close()), so is the sum of four in 32 bits
    each = 2.0 ** -8 * room + (1 + 2.0 ** -8) * 6 * 2.0 ** -24 * size.sum(1, keepdims=True)
    assert np.all(err <= each + (2.0 ** -8 + 4 * 2.0 ** -24) * (np.abs(total) + each) + 1e-30)
    # differences: the turn is linear in x
    rng = np.random.default_rng(0)
    a, da = rng.standard_normal((2, 41, 1, d))
    forward = [O.rotary_by_axes(a + h * da, positions, rot.turns.cpu().numpy(), rot._axes.cpu().numpy(), rot.magnitude, interleaved,
                                order.get("blocks", 1))[0] for h in (0.5, -0.5)]
    w = g[:, :1].double().numpy()
    assert abs(np.sum(w * (forward[0] - forward[1])) - np.sum(da * want[:, :1])) <= 1e-9 * 41 * d
    big = torch.zeros(41, 6, d, dtype=g.dtype, device=DEV)
    big[:, 1:5] = g.to(DEV)
    close(rot.apply(big[:, 1:5], at, inverse=True, out=big[:, 1:5]), want, size, DTYPE_BF16, "in place")
    assert not big[:, 0].any() and not big[:, 5].any()


def run_append(tokens, hq, hkv, d, dtype, page, layout, axes, interleaved=False, fused=False, in_place=False, text=False, seed=0, **order):
    """One call against the oracle, pools checked whole: slots that are not named keep their bits."""
    print(f"[case] append axes={axes} tokens={tokens} heads={hq}/{hkv} d={d} dtype={dtype} page={page} {layout} interleaved={interleaved} "
          f"fused={fused} in_place={in_place} {order}", flush=True)
    gen, rng = torch.Generator().manual_seed(seed + 5), np.random.default_rng(seed)
    pages = -(-tokens // page) + 4
    x = rows(gen, dtype, tokens, hq + 2 * hkv, d)
    parts = x.to(DEV).split([hq, hkv, hkv], 1)
    q, k, v = parts if fused else (p.contiguous() for p in parts)
    cache = C.KVCache(HeadConfig(hq, hkv, d, dtype, page), pages, layout=layout, device=DEV)
    for p in cache.pools[0]:
        p.copy_(rows(gen, dtype, *p.shape))
    before = [p.cpu().clone() for p in cache.pools[0]]
    positions = rng.integers(0, 9999, tokens) if text else some_positions(rng, len(axes), tokens)
    slots = rng.permutation(pages * page)[:tokens]
    slots[rng.random(tokens) < 0.2] = -1
    blocks = order.get("blocks", 1)
    rot = C.Rotary(2 * sum(axes) * blocks, interleaved=interleaved, device=DEV, axes=axes, **order)
    out = cache.append(0, q, k, v, torch.from_numpy(positions).to(DEV), torch.from_numpy(slots).to(DEV), rot, q_out=q if in_place else None)
    by_axis = np.tile(positions, (len(axes), 1)) if text else positions
    turn = lambda a: O.rotary_by_axes(a, by_axis, rot.turns.cpu().numpy(), rot._axes.cpu().numpy(), 1.0, interleaved, blocks)
    x64 = x.double().numpy()
    close(out, *turn(x64[:, :hq]), dtype, "queries")
    kept = slots >= 0
    want, size = turn(x64[:, hq:hq + hkv])
    k_now, v_now = (flat_pool(p.cpu(), layout) for p in cache.pools[0])
    close(k_now[slots[kept]], want[kept], size[kept], dtype, "keys")
    v_want = flat_pool(before[1], layout).clone()
    v_want[slots[kept]] = x[:, hq + hkv:][kept]
    assert torch.equal(v_now.contiguous().view(torch.int16), v_want.contiguous().view(torch.int16))
    others = np.setdiff1d(np.arange(pages * page), slots)
    assert torch.equal(k_now[others].contiguous().view(torch.int16), flat_pool(before[0], layout)[others].contiguous().view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 5, 33, 700, 2049])
@pytest.mark.parametrize("variant", [dict(axes=(16, 24, 24), d=128), dict(axes=(24, 20, 20), d=128, alternating=True, fused=True, in_place=True),
                                     dict(axes=(16, 16), d=64, restart=True, interleaved=True), dict(axes=(32,), d=64, text=True),
                                     dict(axes=(64,), d=256, blocks=2), dict(axes=(9, 4, 1), d=64, in_place=True)])
def test_append(tokens, variant):
    v = dict(variant)
    run_append(tokens, 8, 2, v.pop("d"), DTYPE_BF16, 16, "thd" if tokens % 2 else "htd", v.pop("axes"), seed=tokens, **v)


@pytest.mark.gpu
def test_positions_are_checked():
    x = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device=DEV)
    rot = C.Rotary(64, device=DEV, axes=(16, 8, 8))
    good = torch.zeros(3, 5, dtype=torch.int64, device=DEV)
    rot.apply(x, good)
    empty = torch.zeros(3, 5, dtype=torch.int64, device=DEV)
    empty.untyped_storage().resize_(8 * 14)
    for bad in (good[:2], good[:, :4], good.int(), good.cpu(), torch.zeros(5, 3, dtype=torch.int64, device=DEV).T, good[0, :4], good[None], empty):
        with pytest.raises(ValueError):
            rot.apply(x, bad)
    with pytest.raises(ValueError):
        C.Rotary(64, device=DEV).apply(x, good)                 # a rotary without axes takes one position a token
    assert rot.apply(x[:0], good[:, :0]).shape == (0, 2, 64)


@pytest.mark.gpu
def test_another_stream_and_a_replayed_graph():
    gen = torch.Generator().manual_seed(4)
    x, g = (rows(gen, DTYPE_FP16, 64, 4, 128).to(DEV) for _ in range(2))
    p = torch.randint(0, 5000, (3, 64), generator=gen).to(DEV)
    rot = C.Rotary(128, device=DEV, axes=(24, 20, 20), alternating=True)
    want = rot.apply(x, p)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = rot.apply(x, p, stream=other)
    torch.cuda.current_stream().wait_stream(other)
    assert torch.equal(got, want)
    # forward and backward captured: replays follow the buffers' contents
    leaf = x.clone().requires_grad_()

    def step():
        y = rot.apply(leaf, p)
        return y.detach(), torch.autograd.grad(y, leaf, g)[0]

    with torch.cuda.stream(other):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = step()
    for k in range(3):
        p.copy_(torch.randint(0, 5000, (3, 64), generator=gen))
        with torch.no_grad():
            leaf.copy_(rows(gen, DTYPE_FP16, 64, 4, 128))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, rot.apply(leaf.detach(), p)) and torch.equal(dx, rot.apply(g, p, inverse=True))
