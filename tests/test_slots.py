"""Block tables, positions and slots from lengths on the GPU: refusals on the CPU, results against a token-by-token oracle on the GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C
from oracle import operators as O
from workloads import HeadConfig, DTYPE_BF16, DTYPE_FP16

DEV = "cuda:0"


# ---- on the CPU ------------------------------------------------------------------------------------------


def test_table_refusals():
    """Argument errors that are caught before any HIP call."""
    def status(page=16, n=4, off=4096, ids=8192, num_ids=100, tokens=12288, table=1 << 20, stride=8, width=8):
        return C.codec_block_table(page, n, off, ids, num_ids, tokens, table, stride, width)
    assert status(n=0) == status(width=0, stride=0) == status(n=0, off=0, ids=0, tokens=0, table=0) == C.CODEC_OK
    for bad in (dict(n=-1), dict(n=(1 << 22) + 1), dict(num_ids=-1), dict(width=-1), dict(stride=7), dict(stride=1 << 60), dict(off=0), dict(ids=0),
                dict(tokens=0), dict(table=0), dict(off=4098), dict(ids=8193), dict(tokens=12290), dict(table=(1 << 20) + 2), dict(table=4096 + 16),
                dict(table=8192 - 64), dict(table=12288 - 124)):
        assert status(**bad) == C.CODEC_ERR_INVALID_ARGUMENT, bad
    for page in (0, -16, 8, 24, 8192):
        assert status(page=page) == C.CODEC_ERR_UNSUPPORTED


def test_slot_map_refusals():
    places = dict(table=1 << 20, tokens=1 << 21, new=1 << 22, before=1 << 23, spare=1 << 24, positions=1 << 25, slots=1 << 26, sequences=1 << 27,
                  offsets=1 << 28, out=1 << 29, taken=1 << 30, ws=1 << 31)

    def status(n=4, page=16, width=8, num_tokens=100, num_spare=10, num_pages=1000, stride=8, ws_bytes=0, **kw):
        at = dict(places, **kw)
        cfg = C.codec_slot_config(n, page, width, num_tokens, num_spare, num_pages, stride)
        return C.codec_slot_map(cfg, at["table"], at["tokens"], at["new"], at["before"], at["spare"], at["positions"], at["slots"], at["sequences"],
                                at["offsets"], at["out"], at["taken"], at["ws"], ws_bytes)

    bad = [dict(n=-1), dict(n=(1 << 22) + 1), dict(width=-1), dict(width=9), dict(num_tokens=-1), dict(num_spare=-1), dict(num_pages=-1),
           dict(num_pages=(1 << 31) + 1), dict(stride=1 << 60)]
    bad += [{k: 0} for k in ("table", "tokens", "new", "positions", "slots", "offsets", "out", "taken")]
    bad += [{k: places[k] + 2} for k in places if k != "ws"] + [{k: places[k] + 4} for k in ("before", "positions", "slots")]
    # outputs on one another and on what is read; the table is read, and written if pages are taken for it
    outputs = ("positions", "slots", "sequences", "offsets", "out", "taken")
    bad += [{a: places[b]} for a in outputs for b in outputs if a < b]
    bad += [{a: places[b]} for a in outputs for b in ("table", "tokens", "new", "before", "spare")]
    bad += [dict(table=places[b]) for b in ("tokens", "new", "before", "spare")]
    for b in bad:
        assert status(**b) == C.CODEC_ERR_INVALID_ARGUMENT, b
    for page in (0, 8, 48, 8192):
        assert status(page=page) == C.CODEC_ERR_UNSUPPORTED
    many = dict(n=4097, stride=8)
    need = C.codec_slot_workspace_bytes(C.codec_slot_config(4097, 16, 8, 100, 10, 1000, 8))
    assert need >= 4 * (2 * 4097 + 1) and C.codec_slot_workspace_bytes(C.codec_slot_config(4096, 16, 8, 100, 10, 1000, 8)) == 0
    assert C.codec_slot_workspace_bytes(C.codec_slot_config((1 << 22) + 1, 16, 8, 100, 10, 1000, 8)) == 0
    assert status(**many, ws_bytes=need - 1) == C.CODEC_ERR_WORKSPACE_TOO_SMALL
    for b in (dict(ws=0), dict(ws=(1 << 31) + 8), dict(ws=places["slots"])):
        assert status(**many, ws_bytes=need, **b) == C.CODEC_ERR_INVALID_ARGUMENT, b
    lib = ctypes.CDLL(C.LIB_PATH)
    assert lib.codec_slot_map(None, *[None] * 12, 0, None) == C.CODEC_ERR_INVALID_ARGUMENT
    cache = C.KVCache(HeadConfig(1, 1, 64, DTYPE_BF16), 4, device="cpu")
    none = torch.zeros(0, dtype=torch.int32)
    with pytest.raises(ValueError):
        cache.slots(none.view(0, 4), none, none, 1)
    with pytest.raises(ValueError):
        cache.table([0], [], [], 4)


# ---- on the GPU ------------------------------------------------------------------------------------------


def gpu(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def cache_of(num_pages, page=16):
    return C.KVCache(HeadConfig(1, 1, 64, DTYPE_FP16, page), num_pages, device=DEV)


def lists_of(rng, n, longest, page, num_pages):
    tokens = rng.integers(0, longest + 1, n)
    pages = -(-tokens // page) + rng.integers(0, 3, n)              # some are ahead of their tokens
    off = np.concatenate([[0], np.cumsum(pages)])
    return tokens, off, rng.integers(0, num_pages, off[-1])


@pytest.mark.gpu
@pytest.mark.parametrize("n,longest,width,page", [(1, 1, 1, 16), (1, 0, 5, 16), (3, 100, 7, 16), (33, 1000, 64, 16), (64, 4000, 33, 32), (257, 500, 8, 64),
                                                  (5, 70000, 4501, 16), (5000, 40, 3, 16), (1000, 2000, 130, 16), (2, 60000, 20, 4096)])
@pytest.mark.parametrize("aligned", [True, False])
def test_table(n, longest, width, page, aligned):
    """Entries of wider rows around the table, and the lists themselves, stay as they were."""
    print(f"[case] table n={n} longest={longest} width={width} page={page} aligned={aligned}", flush=True)
    rng = np.random.default_rng(n + width)
    tokens, off, ids = lists_of(rng, n, longest, page, 1 << 20)
    cache = cache_of(1, page)
    want = O.block_table(page, off, ids, tokens, width)
    on_gpu = gpu(off), gpu(ids), gpu(tokens)
    assert np.array_equal(cache.table(*on_gpu, width).cpu().numpy(), want)
    assert np.array_equal(cache.table(off, ids.astype(np.int64), tokens.tolist(), width).cpu().numpy(), want)        # lists on the host
    big = torch.full((n, width + 9 if aligned else (width + 12) // 4 * 4), 77, dtype=torch.int32, device=DEV)
    first = 4 if aligned else 3
    got = cache.table(*on_gpu, width, out=big[:, first:first + width])
    assert got.data_ptr() == big.data_ptr() + 4 * first and np.array_equal(got.cpu().numpy(), want)
    assert bool((big[:, :first] == 77).all()) and bool((big[:, first + width:] == 77).all())
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(on_gpu, (off, ids, tokens)))


@pytest.mark.gpu
def test_tables_of_lists_that_are_none():
    """Offsets that do not lie in the list, that fall, negative lengths: nothing is read from outside, the entries are -1."""
    off = [5, 3, -7, 20, 1 << 30, 4, 8, 9]
    tokens = [40, 100, 100, 100, 16, -5, 2 ** 31 - 1]
    ids = np.arange(10) + 100
    want = O.block_table(16, off, ids, tokens, 6)
    assert np.array_equal(cache_of(1).table(gpu(off), gpu(ids), gpu(tokens), 6).cpu().numpy(), want)
    # ends so far before begins that their difference passes 32 bits
    off = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, -2 ** 31 + 5, 9, 2 ** 31 - 1]
    assert np.array_equal(cache_of(1).table(gpu(off), gpu(ids), gpu([100] * 5), 6).cpu().numpy(), O.block_table(16, off, ids, [100] * 5, 6))
    cache = cache_of(1)
    assert cache.table([0], [], [], 6).shape == (0, 6) and cache.table([0, 0], [], [5], 0).shape == (1, 0)
    assert cache.table([0, 0], [], [5], 3).tolist() == [[-1] * 3]


def check(cache, table, tokens, new, num_tokens, before=None, spare=None, on=None, stream=None):
    """One call against the oracle; the table in place, the other inputs as they were.  `on`: the table's tensor, if it has one."""
    want = O.slot_map(cache.head.page_size, cache.num_pages, table, tokens, new, num_tokens, before, spare)
    inputs = [gpu(tokens), gpu(new), None if before is None else gpu(before, torch.int64), None if spare is None else gpu(spare)]
    on = gpu(table) if on is None else on
    step = cache.slots(on, inputs[0], inputs[1], num_tokens, before=inputs[2], spare=inputs[3], stream=stream)
    torch.cuda.synchronize()
    for name, got, w in zip(("positions", "slots", "sequences", "offsets", "tokens", "taken", "table"), (*step, on), want):
        got = got.cpu().numpy()
        assert got.shape == w.shape and np.array_equal(got, w), (name, np.argwhere(got != w)[:5].tolist())
    for a, b in zip(inputs, (tokens, new, before, spare)):
        assert a is None or np.array_equal(a.cpu().numpy(), b)
    return step


def some_step(n, longest, most, page, seed, spare=True, ahead=0):
    rng = np.random.default_rng(seed)
    tokens = rng.integers(0, longest + 1, n)
    new = rng.integers(0, most + 1, n) * (rng.random(n) < 0.8)
    held, need = -(-tokens // page), -(-(tokens + new) // page)
    width = int(need.max(initial=0)) + ahead
    filled = held if spare else need
    num_pages = int(filled.sum() + (need - held).sum()) + 9
    ids = rng.permutation(num_pages)
    table = np.full((n, width), -1)
    table[np.arange(width) < filled[:, None]] = ids[:filled.sum()]
    return table, tokens, new, ids[filled.sum():] if spare else None, num_pages, rng.integers(-100, 10 ** 11, n)


@pytest.mark.gpu
@pytest.mark.parametrize("n,longest,most,page", [(1, 0, 1, 16), (1, 5000, 900, 16), (2, 31, 3, 16), (48, 3000, 1, 16), (63, 100, 40, 32), (64, 1, 17, 16),
                                                 (65, 700, 5, 64), (257, 300, 70, 16), (1000, 50, 2, 16), (4096, 40, 3, 16), (4097, 40, 3, 16),
                                                 (9001, 20, 2, 32), (300, 900, 0, 16), (3, 20000, 9000, 4096)])
@pytest.mark.parametrize("spare", [True, False])
def test_slots(n, longest, most, page, spare):
    print(f"[case] slots n={n} longest={longest} most={most} page={page} spare={spare}", flush=True)
    table, tokens, new, pages, num_pages, before = some_step(n, longest, most, page, n + most, spare, ahead=n % 3)
    total = int(new.sum())
    cache = cache_of(num_pages, page)
    check(cache, table, tokens, new, total, None, pages)
    check(cache, table, tokens, new, total + 300, before, pages)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 70, 4500])
@pytest.mark.parametrize("spare", [True, False])
def test_maps_that_are_too_short(n, spare):
    """New tokens beyond the map are left out everywhere, wherever it ends: in a page, between pages and sequences, before the first."""
    table, tokens, new, pages, num_pages, before = some_step(n, 60, 40, 16, n, spare)
    new[0] = max(new[0], 5)
    ends = np.concatenate([[0], np.cumsum(new)])
    if spare:
        pages = np.arange(num_pages)
    cache = cache_of(num_pages)
    width = int((-(-(tokens + new) // 16)).max())
    table = np.pad(table, ((0, 0), (0, width - table.shape[1])), constant_values=-1) if width > table.shape[1] else table
    for room in {0, 1, int(new[0]), int(ends[n // 2]), int(ends[n // 2]) + 1, int(ends[-1]) - 1, int(ends[-1]) // 2}:
        check(cache, table, tokens, new, room, before, pages)


@pytest.mark.gpu
def test_too_few_pages_and_entries_that_are_none():
    cache = cache_of(50)
    table = np.array([[3, -1, -1, -1], [50, 1 << 30, -7, -2], [7, 8, 9, 10], [11, 12, -1, -1], [0, 0, 0, 0]])
    tokens, new = [10, 0, 64, 20, -(2 ** 31)], [30, 64, 20, 50, -3]
    check(cache, table, tokens, new, 200)                                   # the table names them, or does not
    check(cache, table, tokens, new, 200, spare=[40, 41, 42])               # fewer pages than are taken
    check(cache, table, tokens, new, 200, spare=[])
    check(cache, table, tokens, new, 200, spare=[49, 50, -1, 48, 2 ** 31 - 1, 47, 46, 45, 44])     # ids that are none
    check(cache, table, [1000, 17, 64, 5, 2 ** 31 - 1], [3, 5, 1, 100, 9], 150, spare=np.arange(20))       # rows that end before their tokens do
    check(cache, table, [2 ** 31 - 3] * 5, [2 ** 31 - 1] * 5, 100)          # sums beyond 32 bits
    check(cache, table[:, :0], [3, 4, 5, 6, 7], [1, 2, 0, 1, 1], 9, spare=[1, 2])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1000, 70000])
def test_sums_beyond_32_bits(n):
    cache = cache_of(8)
    table = np.full((n, 3), 5)
    new = np.full(n, 2 ** 31 - 1)
    step = cache.slots(gpu(table), gpu(np.zeros(n)), gpu(new), 1000, spare=gpu(np.arange(8)))
    assert step.offsets[:2].tolist() == [0, 1000] and bool((step.offsets[1:] == 1000).all()) and int(step.taken) == 3
    assert step.slots.tolist() == [(t // 16) * 16 + t % 16 if t < 48 else -1 for t in range(1000)]
    assert step.tokens[0] == 1000 and not step.tokens[1:].any()


@pytest.mark.gpu
def test_no_sequences_and_no_tokens():
    cache = cache_of(8)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    for num_tokens in (0, 1, 300):
        step = cache.slots(none.view(0, 4), none, none, num_tokens, spare=none)
        assert step.slots.tolist() == [-1] * num_tokens and step.sequences.tolist() == [-1] * num_tokens and not step.positions.any()
        assert step.offsets.tolist() == [0] and step.tokens.shape == (0,) and step.taken.tolist() == [0]


@pytest.mark.gpu
def test_a_table_inside_a_larger_one():
    table, tokens, new, pages, num_pages, before = some_step(37, 200, 30, 16, 5)
    n, width = table.shape
    big = torch.full((n + 2, width + 5), 123, dtype=torch.int32, device=DEV)
    view = big[1:n + 1, 2:2 + width]
    view.copy_(gpu(table))
    check(cache_of(num_pages), table, tokens, new, int(new.sum()) + 3, before, pages, on=view)
    big[1:n + 1, 2:2 + width] = 123
    assert bool((big == 123).all())


@pytest.mark.gpu
def test_tensors_are_checked():
    cache = cache_of(100)
    table, tokens, new = torch.zeros(4, 3, dtype=torch.int32, device=DEV), *torch.zeros(2, 4, dtype=torch.int32, device=DEV).unbind(0)
    good = dict(table=table, tokens=tokens, new=new, num_tokens=5)
    cache.slots(**good)
    short = torch.zeros(4, dtype=torch.int32, device=DEV)
    short.untyped_storage().resize_(12)
    for bad in (dict(table=table.long()), dict(table=table[0]), dict(table=table.cpu()), dict(table=torch.zeros(3, 4, dtype=torch.int32, device=DEV).T),
                dict(tokens=tokens[:3]), dict(tokens=tokens.long()), dict(tokens=table[:, 0]), dict(new=new.cpu()), dict(new=short), dict(num_tokens=-1),
                dict(num_tokens=1 << 31), dict(before=tokens), dict(before=torch.zeros(3, dtype=torch.int64, device=DEV)), dict(spare=table),
                dict(spare=torch.zeros(3, device=DEV)), dict(table=table[:2])):
        with pytest.raises(ValueError):
            cache.slots(**dict(good, **bad))
    with pytest.raises(C.CodecError):
        cache.slots(table[:1].expand(4, 3), tokens, new, 5)             # rows that coincide
    with pytest.raises(C.CodecError):
        cache.slots(table, tokens, new, 5, spare=table[0])              # pages taken out of the table itself
    off, ids = torch.zeros(5, dtype=torch.int32, device=DEV), torch.zeros(9, dtype=torch.int32, device=DEV)
    for bad in ((off[:4], ids, tokens, 3), (off.long(), ids, tokens, 3), (off, ids.cpu(), tokens, 3), (off, ids, tokens, -1), (off, ids, table, 3),
                (off, [1.5], tokens, 3), (off, [1 << 40], tokens, 3)):
        with pytest.raises(ValueError):
            cache.table(*bad)
    for out in (table, table[:, :2], torch.zeros(4, 2, dtype=torch.int64, device=DEV)):
        with pytest.raises(ValueError):
            cache.table(off, ids, tokens, 4, out=out)


@pytest.mark.gpu
def test_another_stream_and_a_replayed_graph():
    """A captured step whose lengths go on from replay to replay on the GPU alone, between eager calls that share nothing with it."""
    n, page, num_pages = 21, 16, 4000
    cache = cache_of(num_pages, page)
    rng = np.random.default_rng(2)
    table, tokens, new, pages, _, before = some_step(n, 100, 20, page, 9)
    width = 40
    table = np.pad(table, ((0, 0), (0, width - table.shape[1])), constant_values=-1)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    check(cache, table, tokens, new, 500, before, np.arange(100, 400), stream=other)
    held, more, spare = gpu(tokens), gpu(new), gpu(np.arange(1000, 1400))
    on = gpu(table)
    cache.slots(on.clone(), held, more, 500, spare=spare)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step = cache.slots(on, held, more, 500, spare=spare)
        held.copy_(step.tokens)
    for k in range(4):
        new = rng.integers(0, 25, n)
        more.copy_(gpu(new))
        spare.copy_(gpu(np.arange(1000 + 400 * k, 1400 + 400 * k)))
        graph.replay()
        want = O.slot_map(page, num_pages, table, tokens, new, 500, None, np.arange(1000 + 400 * k, 1400 + 400 * k))
        check(cache, table, tokens, new, 300, None, np.arange(7))
        for got, w in zip((*step, on), want):
            assert np.array_equal(got.cpu().numpy(), w)
        tokens, table = want[4], want[6]
        assert np.array_equal(held.cpu().numpy(), tokens)


@pytest.mark.gpu
def test_from_forked_lists_to_the_pages():
    """Lists that a fork leaves, their table, new tokens' slots with pages of the cache, and the append that reads them."""
    head = HeadConfig(2, 1, 64, DTYPE_BF16)
    cache = C.KVCache(head, 64, device=DEV)
    for p in cache.pools[0]:
        p.zero_()
    ids = cache.take(5)
    off, ids = cache.fork([0, 3, 5], ids, [37, 32], [0, 0, 1])
    tokens, new = np.array([37, 37, 32]), np.array([2, 20, 1])
    spare = cache.take(6)
    table = cache.table(off, ids, tokens, 6)
    step = cache.slots(table, gpu(tokens), gpu(new), 30, spare=gpu(spare))
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(30, h, 64, generator=gen).bfloat16().to(DEV) for h in (2, 1, 1))
    rot = C.Rotary(64, device=DEV)
    cache.append(0, q, k, v, step.positions, step.slots, rot)
    taken = int(step.taken)
    cache.release(spare[taken:])                                            # what was not taken
    assert taken == 2 and cache.free_pages == 64 - len(set(ids.tolist())) - taken
    turned = rot.apply(k, step.positions)
    lists = table.cpu().numpy()
    for t in range(int(new.sum())):
        s = int(step.sequences[t])
        place = int(tokens[s]) + t - int(step.offsets[s])
        assert int(step.positions[t]) == place
        page = int(lists[s, place // 16])
        assert torch.equal(cache.pools[0][0][page, 0, place % 16], turned[t, 0]) and torch.equal(cache.pools[0][1][page, 0, place % 16], v[t, 0])
    assert int((cache.pools[0][1].abs().sum(-1) != 0).sum()) == int(new.sum())      # and nothing else was stored
