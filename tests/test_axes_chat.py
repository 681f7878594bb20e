"""The operators of a serving step as a program runs them together: page lists as a table, the new tokens' slots, keys of two maps turned
by positions on several axes into the cache, differential attention over the shared prefix; sequences are forked in between."""
import math

import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C
from oracle import operators as O
from test_differential import bound
from test_rotary_axes import close
from workloads import Forest, HeadConfig, DTYPE_BF16, DTYPE_FP16

DEV = "cuda:0"
PREFIX, PICTURE, PROMPTS = 45, (6, 5), [5, 16, 29]
STEPS = [[5, 16, 29], [1, 1, 1], [1, 4, 1], [1, 1, 2], [33, 1, 1], [1, 1, 1]]       # new tokens of a step: prompts, one, several, many
FORKS = {1: [0, 0, 2], 3: [1, 2, 1], 4: [2, 1, 0]}                                    # after which step who goes on


def gpu(a, dtype=torch.int32):
    return torch.from_numpy(np.asarray(a)).to(DEV, dtype)


def prefix_positions(axes):
    """Text, a picture of rows and columns behind it, text again: what stands behind the picture counts from its largest position."""
    lead, (rows, columns) = 7, PICTURE
    at = [np.arange(lead)] * axes
    for a in range(axes):
        i = np.arange(rows * columns)
        at[a] = np.concatenate([at[a], lead + (np.zeros_like(i), i // columns, i % columns)[(a + 3 - axes) % 3]])
    behind = lead + max(rows, columns)
    rest = PREFIX - lead - rows * columns
    return np.stack([np.concatenate([a, behind + np.arange(rest)]) for a in at]), behind + rest


@pytest.mark.gpu
@pytest.mark.parametrize("heads,hkv,d,dtype,page,layout,axes", [(4, 2, 64, DTYPE_BF16, 16, "htd", (16, 8, 8)), (4, 1, 32, DTYPE_FP16, 32, "thd", (6, 10)),
                                                                (6, 3, 128, DTYPE_BF16, 16, "thd", (24, 20, 20))])
def test_chats_over_a_picture(heads, hkv, d, dtype, page, layout, axes):
    print(f"[case] heads={heads}/{hkv} d={d} dtype={dtype} page={page} {layout} axes={axes}", flush=True)
    gen = torch.Generator().manual_seed(d)
    half, least = bound(dtype)
    stored = HeadConfig(heads, hkv, 2 * d, dtype, page)                     # rows of both maps side by side
    paired = HeadConfig(2 * heads, hkv, 2 * d, dtype, page, float(np.float32(1.0 / math.sqrt(d))))
    cache = C.KVCache(stored, 40, layout=layout, device=DEV)
    for p in cache.pools[0]:
        p.fill_(math.nan)                                                    # what is not written shows
    rot = C.Rotary(2 * d, device=DEV, axes=axes, alternating=len(axes) == 3, blocks=2)
    turns, axis = rot.turns.cpu().numpy(), rot._axes.cpu().numpy()
    model = torch.randn(59, heads + 2 * hkv, 2 * d, generator=gen).to(cache.dtype)      # a token's rows
    of_token, lam, weight = model.to(DEV), torch.rand(heads, generator=gen), torch.randn(2 * d, generator=gen) * 0.2 + 1
    rng = np.random.default_rng(heads)
    split = [heads, hkv, hkv]
    # the prefix, whose tokens are appended in one call
    root = cache.take(-(-PREFIX // page))
    where, base = prefix_positions(len(axes))
    tokens_of = rng.integers(0, 59, PREFIX)
    at = np.arange(PREFIX)
    slots = root[at // page].astype(np.int64) * page + at % page
    cache.append(0, *of_token[gpu(tokens_of, torch.long)].split(split, 1), gpu(where, torch.long), gpu(slots, torch.long), rot)
    # what a program keeps: page lists, lengths; and what the check keeps: tokens of a sequence
    n = len(PROMPTS)
    off, ids, lens = np.zeros(n + 1, np.int32), np.zeros(0, np.int32), np.zeros(n, np.int64)
    said = [np.zeros(0, np.int64) for _ in range(n)]
    before = gpu([base] * n, torch.long)
    for number, new in enumerate(STEPS):
        width, total = 8, sum(new)
        padded = total + (3 if number % 2 else 0)                            # a step's length is fixed in a captured program
        spare = cache.take(sum(-(-m // page) + 1 for m in new))
        table = cache.table(off, ids, lens.astype(np.int32), width)
        lists = O.block_table(page, off, ids, lens, width)
        assert np.array_equal(table.cpu().numpy(), lists)
        step = cache.slots(table, gpu(lens), gpu(new), padded, before=before, spare=gpu(spare))
        want = O.slot_map(page, cache.num_pages, lists, lens, new, padded, [base] * n, spare)
        for name, a, b in zip(step._fields, step, want):
            assert np.array_equal(a.cpu().numpy(), b), (number, name)
        taken, lists, lens = int(step.taken), want[6], want[4]
        cache.release(spare[taken:])
        fresh = rng.integers(0, 59, padded)
        q, k, v = of_token[gpu(fresh, torch.long)].split(split, 1)
        turned = cache.append(0, q, k, v, step.positions, step.slots, rot)  # text: one position for all axes
        said = [np.concatenate([s, fresh[a:b]]) for s, a, b in zip(said, want[3], want[3][1:])]
        held = [row[:-(-int(m) // page)] for row, m in zip(lists, lens)]
        off, ids = np.cumsum([0] + [len(x) for x in held]).astype(np.int32), np.concatenate(held).astype(np.int32)
        # the last tokens' queries over the prefix and the sequences
        forest = Forest(np.array([-1] + [0] * n), np.array([PREFIX, *lens]).astype(np.int32), 1 + np.arange(n))
        paged = cache.paged(np.cumsum([0, len(root)] + [len(x) for x in held]).astype(np.int32), np.concatenate([root, ids]).astype(np.int32))
        plan = C.PlannedAttention(forest, paged, paired, device=DEV, share=2, schedule=2)
        last = turned[step.offsets[1:].long() - 1]
        out = plan.decode_differential(last.view(n, 2 * heads, d), *cache.pools[0], lam.to(DEV), weight=weight.to(DEV), eps=1e-5, gain=0.2)
        torch.cuda.synchronize()
        plan.close()
        # the cache holds the sequences' rows, turned; the queries are turned; the answers follow from both
        kp, vp = (p.double().cpu().numpy() if layout == "thd" else p.transpose(1, 2).double().cpu().numpy() for p in cache.pools[0])
        for s in range(n):
            tokens = np.concatenate([tokens_of, said[s]])
            places = np.concatenate([where, np.tile(base + np.arange(lens[s]), (len(axes), 1))], 1)
            row = [*(root[at // page]), *(held[s][np.arange(lens[s]) // page])], [*(at % page), *(np.arange(lens[s]) % page)]
            x = model[torch.from_numpy(tokens)].double().numpy()
            keys, values = kp[row], vp[row]
            assert np.array_equal(values, x[:, heads + hkv:])
            turn, size = O.rotary_by_axes(x[:, :heads + hkv], places, turns, axis, 1.0, False, 2)
            close(torch.from_numpy(keys), turn[:, heads:], size[:, heads:], dtype, "keys")
            mine = last[s].cpu()
            close(mine, turn[-1, :heads], size[-1, :heads], dtype, "queries")
            answer, off_by = O.differential(mine.double().numpy().reshape(heads, 2, d), keys, values, float(paired.scale), lam.double().numpy(),
                                            (float(np.float32(1e-5)), weight.double().numpy()), float(np.float32(0.2)), half, least)
            err = np.abs(out[s].double().cpu().numpy() - answer)
            assert np.all(err <= off_by), (number, s, float((err / off_by).max()))
        if number in FORKS:
            off, ids = cache.fork(off, ids, lens.astype(np.int32), FORKS[number])
            lens, said = lens[FORKS[number]], [said[p] for p in FORKS[number]]
            before = before[gpu(FORKS[number], torch.long)]
    cache.release(ids)
    cache.release(root)
    assert cache.free_pages == cache.num_pages


@pytest.mark.gpu
def test_a_captured_step():
    """Slots, append and attention of one token a sequence as one graph: replays go on from the lengths and the table that the
    replay before left, while the plan's lengths stay (those of the prefix)."""
    head = HeadConfig(4, 2, 128, DTYPE_BF16, 16)
    paired = HeadConfig(8, 2, 128, DTYPE_BF16, 16, 0.125)
    gen = torch.Generator().manual_seed(2)
    cache = C.KVCache(head, 64, layout="htd", device=DEV)
    for p in cache.pools[0]:
        p.copy_(torch.randn(p.shape, generator=gen))
    forest = Forest(np.array([-1, 0, 0]), np.array([64, 47, 20]), np.array([1, 2]))
    pages = cache.take(4 + 3 + 2)
    plan = C.PlannedAttention(forest, cache.paged(np.array([0, 4, 7, 9], np.int32), pages), paired, device=DEV)
    rot = C.Rotary(128, device=DEV, axes=(16, 16), blocks=2)
    lam = torch.full((4,), 0.3, device=DEV)
    rows = torch.randn(2, 8, 128, generator=gen).bfloat16().to(DEV)
    new, before, spare = gpu([1, 1]), gpu([64, 64], torch.long), gpu(cache.take(8))

    def step(table, tokens):
        s = cache.slots(table, tokens, new, 2, before=before, spare=spare)
        q = cache.append(0, *rows.split([4, 2, 2], 1), s.positions, s.slots, rot)
        out = plan.decode_differential(q.view(2, 8, 64), *cache.pools[0], lam)
        tokens.copy_(s.tokens)
        return s.positions, s.slots, q, out

    def state():
        return cache.table([0, 3, 5], pages[4:], [47, 20], 8), gpu([47, 20])

    table, tokens = state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(table.clone(), tokens.clone())
    torch.cuda.synchronize()
    start = [p.clone() for p in cache.pools[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(table, tokens)
    replayed = []
    for _ in range(4):
        rows.copy_(torch.randn(2, 8, 128, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        replayed.append((rows.clone(), [x.clone() for x in captured], tokens.clone(), table.clone(), [p.clone() for p in cache.pools[0]]))
    for p, old in zip(cache.pools[0], start):
        p.copy_(old)
    again, held = state()
    for x, outs, lens, lists, pools in replayed:
        rows.copy_(x)
        eager = step(again, held)
        assert all(torch.equal(a, b) for a, b in zip(eager, outs)) and torch.equal(held, lens) and torch.equal(again, lists)
        assert all(torch.equal(a, b) for a, b in zip(cache.pools[0], pools))
    plan.close()
