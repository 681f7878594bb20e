"""The work around a decode step that users of this framework have it do, as a list of measurable cases.

A decode step reads a paged K/V cache that somebody fills, forks and tidies, and its output ends in a choice of
tokens.  The cases are those calls: ``KVCache.append`` and ``Rotary.apply`` (rotary positions of new queries and keys,
K and V into their pages), ``KVCache.fork`` and ``KVCache.copy`` (branches of a context, moved pages, packed nodes),
``beam_select`` (the best continuations over beams and vocabulary) and ``beam_reorder`` (the states of the beams that
go on).  With ``own`` false the same results come from elementary torch operations.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
FP16, BF16, FP32 = 0, 1, 2              # the framework's dtype codes
DTYPES = {FP16: torch.float16, BF16: torch.bfloat16, FP32: torch.float32}
SCALINGS = ("none", "linear", "ntk", "wavelength", "yarn")
ORIGINAL = 8192                         # context length before scaling
LOW, HIGH = 1.0, 4.0                    # "wavelength": periods in the original context between which factors blend
FAST, SLOW = 32.0, 1.0                  # "yarn": the same, as turns in the original context
POOL = 1 << 30                          # most bytes of the pools of a drawn fork or copy


# ---- the cases -------------------------------------------------------------------------------------------


def _append(tokens, hq, hkv, d, dtype, page, layout, turned, name=None, interleaved=False, scaling="none", factor=1.0,
            theta=10000.0, fused=False, prompts=0, context=32768, padded=0.0, shape=1):
    c = dict(op="append", tokens=tokens, hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, layout=layout, turned=turned,
             interleaved=interleaved, scaling=scaling, factor=factor, theta=theta, fused=fused, prompts=prompts,
             context=context, padded=padded, shape=shape)
    return dict(name=name, **c) if name else c


def _rotate(tokens, heads, d, dtype, turned, name=None, interleaved=False, inverse=False, scaling="none", factor=1.0,
            theta=10000.0, context=32768):
    c = dict(op="rotate", tokens=tokens, heads=heads, d=d, dtype=dtype, turned=turned, interleaved=interleaved,
             inverse=inverse, scaling=scaling, factor=factor, theta=theta, context=context)
    return dict(name=name, **c) if name else c


def _fork(sequences, children, shortest, longest, layers, hkv, d, dtype, page, layout, name=None, shape=1):
    c = dict(op="fork", sequences=sequences, children=children, shortest=shortest, longest=longest, layers=layers,
             hkv=hkv, d=d, dtype=dtype, page=page, layout=layout, shape=shape)
    return dict(name=name, **c) if name else c


def _copy(kind, pages, layers, hkv, d, dtype, page, layout, name=None, shape=1):
    c = dict(op="copy", kind=kind, pages=pages, layers=layers, hkv=hkv, d=d, dtype=dtype, page=page, layout=layout,
             shape=shape)
    return dict(name=name, **c) if name else c


def _select(batch, beams, vocab, k, dtype, name=None, masked=0.0, finished=False):
    c = dict(op="select", batch=batch, beams=beams, vocab=vocab, k=k, dtype=dtype, masked=masked, finished=finished)
    return dict(name=name, **c) if name else c


def _reorder(batch, beams, history, tensors, width, dtype, name=None):
    c = dict(op="reorder", batch=batch, beams=beams, history=history, tensors=tensors, width=width, dtype=dtype)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the next token of four short chats, a small MHA model: the latency of a call counts
        _append(4, 8, 8, 128, FP16, 16, "htd", 128, "append_four_chats", context=1088),
        # one token for each of 512 requests of an irregular forest, out of one projection of queries, keys and
        # values; a tenth of the rows is padding of a fixed batch
        _append(512, 32, 8, 128, BF16, 16, "htd", 128, "append_decode_batch", fused=True, theta=500000.0,
                scaling="wavelength", factor=8.0, padded=0.1, shape=2),
        # prompts of ragged length, behind a context stretched by four: the rate of a large call
        _append(16384, 64, 8, 128, BF16, 16, "thd", 128, "append_prompts", scaling="yarn", factor=4.0, prompts=9,
                context=16384, shape=3),
        # the gradient of rotated queries: turned back, neighbouring channels, a quarter of a wide head
        _rotate(4099, 16, 256, BF16, 64, "rotate_back_part_of_head", interleaved=True, inverse=True),
        # the answers of 64 searches, each behind a prompt in nodes of its own, go on in four branches and are pruned
        # again: shared pages are counted, the partly filled last pages copied in 16 layers
        _fork(64, 4, 17, 255, 16, 8, 128, BF16, 16, "htd", "fork_and_prune_beams", shape=4),
        # pages of a cache that has served for hours move together
        _copy("pages", 1000, 8, 8, 128, BF16, 16, "htd", "compact_pages", shape=5),
        # chains of nodes of one to five tokens become full pages, heads of 64 channels, tokens before heads
        _copy("chains", 96, 8, 8, 64, FP16, 16, "thd", "pack_short_nodes", shape=6),
        # the first token of one beam search: the latency of a call counts
        _select(1, 4, 32768, 8, FP32, "select_one_search"),
        # constrained decoding: an odd vocabulary, half of it ruled out, finished beams among the others
        _select(16, 5, 50021, 10, FP16, "select_constrained", masked=0.5, finished=True),
        # the largest: 64 searches of eight beams over a large vocabulary
        _select(64, 8, 131072, 16, BF16, "select_large_batch"),
        # token histories and a handful of small states of four searches
        _reorder(4, 4, 1000, 3, 129, FP16, "reorder_histories"),
        # states of a batch of searches: a few kilobytes a beam in each of 32 tensors
        _reorder(64, 8, 4096, 32, 8192, BF16, "reorder_states"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm, odd as often as not."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "append", "rotate", "fork", "copy", "copy", "select", "select", "select", "reorder"])
    hq, hkv, d = rng.choice([(8, 8, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (32, 1, 128), (64, 8, 64),
                             (9, 3, 64), (16, 8, 256)])
    dtype, page, layout = rng.choice([FP16, BF16]), rng.choice([16, 16, 32, 64]), rng.choice(["htd", "thd"])
    scaling = rng.choice(SCALINGS)
    rotary = dict(scaling=scaling, factor=1.0 if scaling == "none" else rng.uniform(1.5, 16.0),
                  theta=rng.choice([10000.0, 500000.0, 1000000.0]), interleaved=rng.random() < 0.4)
    turned = rng.choice([d, d, d, d // 2, d // 4, 2 * rng.randrange(1, d // 2)])
    shape = rng.randrange(1, 1 << 30)
    if op == "append":
        tokens = _spread(rng, 1, 16384)
        prompts = rng.randrange(1, 17) if tokens > 1000 else 0
        return _append(tokens, hq, hkv, d, dtype, page, layout, turned, fused=rng.random() < 0.5, prompts=prompts,
                       context=_spread(rng, 100, 1000000), padded=rng.choice([0.0, 0.0, 0.2]), shape=shape, **rotary)
    if op == "rotate":
        return _rotate(_spread(rng, 1, 8192), hq, d, dtype, turned, inverse=rng.random() < 0.7,
                       context=_spread(rng, 100, 1000000), **rotary)
    if op == "fork":
        layers, children, shortest = _spread(rng, 1, 16), rng.randrange(2, 9), _spread(rng, 1, 120)
        longest = _spread(rng, shortest, 4 * shortest)
        most = POOL // (layers * hkv * d * 4) // (longest + (children + 1) * page)
        return _fork(_spread(rng, 1, max(1, min(80, most))), children, shortest, longest, layers, hkv, d, dtype, page,
                     layout, shape=shape)
    if op == "copy":
        kind, layers = rng.choice(["pages", "chains"]), _spread(rng, 1, 8)
        most = POOL // (layers * hkv * d * 4) // (page * (2 if kind == "pages" else 1 + page // 2))
        return _copy(kind, _spread(rng, 1, max(1, min(1000, most))), layers, hkv, d, dtype, page, layout, shape=shape)
    if op == "select":
        beams = rng.randrange(1, 11)
        vocab = _spread(rng, 300, 131072)
        dtype = rng.choice([FP16, BF16, FP32])
        most = max(1, min(64, (1 << 27) // (beams * vocab * (4 if dtype == FP32 else 2))))
        return _select(_spread(rng, 1, most), beams, vocab, rng.choice([beams, 2 * beams, 2 * beams]), dtype,
                       masked=rng.choice([0.0, 0.0, 0.3, 0.95]),
                       finished=rng.random() < 0.4)
    dtype = rng.choice([FP16, BF16, FP32])
    return _reorder(_spread(rng, 1, 64), rng.randrange(1, 9), _spread(rng, 1, 4096), _spread(rng, 1, 32),
                    _spread(rng, 1, 4096 if dtype == FP32 else 8192), dtype)


# ---- inputs ----------------------------------------------------------------------------------------------


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return gen


def _pools(c, num_pages, gen):
    shape = (num_pages, c["page"], c["hkv"], c["d"]) if c["layout"] == "thd" else (num_pages, c["hkv"], c["page"], c["d"])
    return [tuple(torch.empty(shape, dtype=DTYPES[c["dtype"]], device=DEVICE).normal_(generator=gen) for _ in "kv")
            for _ in range(c.get("layers", 1))]


def _head(c):
    return SimpleNamespace(num_q_heads=c.get("hq", c["hkv"]), num_kv_heads=c["hkv"], head_dim=c["d"], dtype=c["dtype"],
                           page_size=c["page"], scale=float(np.float32(1.0 / math.sqrt(c["d"]))))


def _framework_cache(c, pools):
    from paper_2505_17694_amd import KVCache
    return KVCache(_head(c), pools[0][0].shape[0], layout=c["layout"], device=DEVICE, pools=pools)


def _framework_rotary(c):
    from paper_2505_17694_amd import Rotary
    scaling = None if c["scaling"] == "none" else dict(kind=c["scaling"], factor=c["factor"], original_length=ORIGINAL,
                                                       low=LOW, high=HIGH, fast=FAST, slow=SLOW)
    return Rotary(c["turned"], theta=c["theta"], interleaved=c["interleaved"], scaling=scaling, device=DEVICE)


def _prepare_append(c, seed):
    gen, rng = _generator(seed), np.random.Generator(np.random.PCG64(seed))
    t, ps = c["tokens"], c["page"]
    if c["prompts"]:                        # consecutive positions of some prompts behind cached contexts
        ends = np.sort(np.random.Generator(np.random.PCG64(c["shape"])).integers(0, t + 1, c["prompts"] - 1))
        lens = np.diff(np.concatenate([[0], ends, [t]]))
        starts = rng.integers(0, c["context"], len(lens))
    else:                                   # the next token of every sequence
        lens, starts = np.ones(t, np.int64), rng.integers(0, c["context"], t)
    need = (lens + ps - 1) // ps + 1        # wherever in a page a sequence goes on
    num_pages = int(sum(need)) + 64
    ids, positions, slots, at = rng.permutation(num_pages), [], [], 0
    for s, n, pages in zip(starts, lens, need):
        p = s + np.arange(n)
        positions.append(p)
        slots.append(ids[at + (s % ps + np.arange(n)) // ps] * ps + p % ps)
        at += pages
    positions, slots = np.concatenate(positions), np.concatenate(slots)
    slots[rng.random(t) < c["padded"]] = -1
    heads = c["hq"] + 2 * c["hkv"]
    if c["fused"]:
        x = torch.empty((t, heads, c["d"]), dtype=DTYPES[c["dtype"]], device=DEVICE).normal_(generator=gen)
        q, k, v = x.split([c["hq"], c["hkv"], c["hkv"]], 1)
    else:
        q, k, v = (torch.empty((t, h, c["d"]), dtype=DTYPES[c["dtype"]], device=DEVICE).normal_(generator=gen)
                   for h in (c["hq"], c["hkv"], c["hkv"]))
    pools = _pools(c, num_pages, gen)
    return SimpleNamespace(c=c, q=q, k=k, v=v, pools=pools, positions=torch.from_numpy(positions).to(DEVICE),
                           slots=torch.from_numpy(slots).to(DEVICE),
                           cache=_framework_cache(c, pools) if own else None,
                           rotary=_framework_rotary(c) if own else _plain_rotary(c))


def _prepare_rotate(c, seed):
    gen, rng = _generator(seed), np.random.Generator(np.random.PCG64(seed))
    x = torch.empty((c["tokens"], c["heads"], c["d"]), dtype=DTYPES[c["dtype"]], device=DEVICE).normal_(generator=gen)
    positions = torch.from_numpy(rng.integers(0, c["context"], c["tokens"])).to(DEVICE)
    return SimpleNamespace(c=c, x=x, positions=positions, rotary=_framework_rotary(c) if own else _plain_rotary(c))


def _sequences(c, seed):
    """Lengths of the case alone; pages of the sequences (offsets, ids) in a seeded order; pages of the pool."""
    rng = np.random.Generator(np.random.PCG64(c["shape"]))
    tokens = rng.integers(c["shortest"], c["longest"] + 1, c["sequences"]).astype(np.int32)
    pages = -(-tokens // c["page"])
    off = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    num_pages = int(off[-1]) + c["sequences"] * c["children"] + 64
    ids = np.random.Generator(np.random.PCG64(seed)).permutation(num_pages)[:off[-1]].astype(np.int32)
    return tokens, off, ids, num_pages


def _prepare_fork(c, seed):
    tokens, off, ids, num_pages = _sequences(c, seed)
    pools = _pools(c, num_pages, _generator(seed))
    parents = np.repeat(np.arange(c["sequences"], dtype=np.int32), c["children"])
    first = np.arange(c["sequences"], dtype=np.int32) * c["children"]
    s = SimpleNamespace(c=c, tokens=tokens, off=off, ids=ids, pools=pools, parents=parents, first=first, cache=None, holders=None)
    if own:
        s.cache = _framework_cache(c, pools)
        s.cache.hold(ids)
    else:
        s.holders = np.bincount(ids, minlength=num_pages)
    return s


def _runs(c, seed):
    """Copies (source page, source token, destination page, destination token, tokens) and the pool's pages."""
    rng, shape = np.random.Generator(np.random.PCG64(seed)), np.random.Generator(np.random.PCG64(c["shape"]))
    n, ps = c["pages"], c["page"]
    if c["kind"] == "pages":                # whole pages from anywhere above to anywhere below
        num_pages = 2 * n + 32
        src, dst = rng.permutation(np.arange(n, num_pages))[:n], rng.permutation(n)
        runs = [(int(a), 0, int(b), 0, ps) for a, b in zip(src, dst)]
    else:                                   # nodes of one to five tokens, a page each, into n full pages
        runs, sources = [], 0
        for page in range(n):
            at = 0
            while at < ps:
                take = min(int(shape.integers(1, 6)), ps - at)
                runs.append((sources, 0, page, at, take))
                at += take
                sources += 1
        num_pages = n + sources + 32
        order = rng.permutation(num_pages)
        runs = [(int(order[n + a]), b, int(order[p]), at, take) for a, b, p, at, take in runs]
    return np.array(runs, np.int32), num_pages


def _prepare_copy(c, seed):
    runs, num_pages = _runs(c, seed)
    pools = _pools(c, num_pages, _generator(seed))
    return SimpleNamespace(c=c, runs=runs, pools=pools, cache=_framework_cache(c, pools) if own else None)


def _prepare_select(c, seed):
    gen = _generator(seed)
    b, w, v = c["batch"], c["beams"], c["vocab"]
    logits = torch.empty((b, w, v), dtype=DTYPES[c["dtype"]], device=DEVICE).normal_(0.0, 3.0, generator=gen)
    if c["masked"]:
        out = torch.rand((b, w, v), generator=gen, device=DEVICE) < c["masked"]
        logits.masked_fill_(out, -math.inf)
    scores = torch.rand((b, w), generator=gen, device=DEVICE).mul_(-20.0).sort(1, descending=True).values
    finished = torch.rand((b, w), generator=gen, device=DEVICE) < 0.25 if c["finished"] else None
    return SimpleNamespace(c=c, logits=logits, scores=scores, finished=finished, eos=2)


def _prepare_reorder(c, seed):
    gen = _generator(seed)
    b, w = c["batch"], c["beams"]
    states = [torch.randint(0, 1 << 17, (b, w, c["history"]), dtype=torch.int32, generator=gen, device=DEVICE)]
    for _ in range(c["tensors"]):
        states.append(torch.empty((b, w, c["width"]), dtype=DTYPES[c["dtype"]], device=DEVICE).normal_(generator=gen))
    beams = torch.randint(0, w, (b, w), dtype=torch.int32, generator=gen, device=DEVICE)
    return SimpleNamespace(c=c, states=states, beams=beams)


_PREPARE = dict(append=_prepare_append, rotate=_prepare_rotate, fork=_prepare_fork, copy=_prepare_copy,
                select=_prepare_select, reorder=_prepare_reorder)


def prepare(case, seed):
    return _PREPARE[case["op"]](case, seed)


# ---- the calls -------------------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)[s.c["op"]](s)


def _own_append(s):
    q = s.cache.append(0, s.q, s.k, s.v, s.positions, s.slots, s.rotary)
    return [q, *s.pools[0]]


def _own_rotate(s):
    return s.rotary.apply(s.x, s.positions, inverse=s.c["inverse"])


def _own_fork(s):
    off, ids = s.cache.fork(s.off, s.ids, s.tokens, s.parents)
    kept = s.cache.fork(off, ids, s.tokens[s.parents], s.first)
    return [ids, kept[1], *(p for kv in s.pools for p in kv)]


def _own_copy(s):
    s.cache.copy(s.runs)
    return [p for kv in s.pools for p in kv]


def _own_select(s):
    from paper_2505_17694_amd import beam_select
    return beam_select(s.logits, s.scores, s.c["k"], finished=s.finished, eos=s.eos)


def _own_reorder(s):
    from paper_2505_17694_amd import beam_reorder
    return beam_reorder(s.states, s.beams)


_run_own = dict(append=_own_append, rotate=_own_rotate, fork=_own_fork, copy=_own_copy, select=_own_select,
                reorder=_own_reorder)


# ---- the plain forms -------------------------------------------------------------------------------------


def _plain_rotary(c):
    """Turns a position of every pair of channels (64 bits), and the factor on turned channels."""
    r, theta, f = c["turned"], c["theta"], c["factor"]
    i = np.arange(r // 2, dtype=np.float64)
    magnitude = 1.0
    if c["scaling"] == "ntk" and r > 2:
        theta *= f ** (r / (r - 2))
    freq = theta ** (-2.0 * i / r)
    if c["scaling"] == "linear":
        freq /= f
    elif c["scaling"] == "wavelength":
        periods = ORIGINAL * freq / (2 * math.pi)
        keep = np.clip((periods - LOW) / (HIGH - LOW), 0.0, 1.0)
        freq = keep * freq + (1 - keep) * freq / f
    elif c["scaling"] == "yarn":
        at = [r * math.log(ORIGINAL / (n * 2 * math.pi)) / (2 * math.log(theta)) for n in (FAST, SLOW)]
        low, high = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        ramp = np.clip((i - low) / max(high - low, 0.001), 0.0, 1.0)
        freq = (1 - ramp) * freq + ramp * freq / f
        magnitude = 0.1 * math.log(f) + 1.0 if f > 1 else 1.0
    return SimpleNamespace(turns=torch.from_numpy(freq / (2 * math.pi)).to(DEVICE), magnitude=magnitude)


def _turned(c, rotary, x, positions, inverse, dtype):
    u = positions.to(torch.float64)[:, None] * rotary.turns
    angle = (u - torch.round(u)) * (2 * math.pi)
    cos, sin = (rotary.magnitude * torch.cos(angle)).to(dtype), (rotary.magnitude * torch.sin(angle)).to(dtype)
    cos, sin = cos[:, None], (-sin if inverse else sin)[:, None]
    r, out = c["turned"], x.to(dtype).clone()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    first, second = x[..., a].to(dtype), x[..., b].to(dtype)
    out[..., a] = first * cos - second * sin
    out[..., b] = second * cos + first * sin
    return out


def _tokens_of(c, pool, pages, tokens, values=None):
    """Rows [n, heads, d] of the pool's tokens, or their new values."""
    at = (pages, tokens) if c["layout"] == "thd" else (pages, slice(None), tokens)
    if values is None:
        return pool[at]
    pool[at] = values


def _plain_append(s):
    c, (k_pool, v_pool) = s.c, s.pools[0]
    kind = s.q.dtype
    q = _turned(c, s.rotary, s.q, s.positions, False, torch.float32).to(kind)
    k = _turned(c, s.rotary, s.k, s.positions, False, torch.float32).to(kind)
    kept = (s.slots >= 0).nonzero()[:, 0]
    pages, tokens = s.slots[kept] // c["page"], s.slots[kept] % c["page"]
    _tokens_of(c, k_pool, pages, tokens, k[kept])
    _tokens_of(c, v_pool, pages, tokens, s.v[kept])
    return [q, k_pool, v_pool]


def _plain_rotate(s):
    return _turned(s.c, s.rotary, s.x, s.positions, s.c["inverse"], torch.float32).to(s.x.dtype)


def _copy_tokens(c, pools, runs):
    n = runs[:, 4]
    step = np.arange(int(n.sum())) - np.repeat(np.cumsum(n) - n, n)
    at = torch.from_numpy(np.stack([np.repeat(runs[:, 0], n), np.repeat(runs[:, 1], n) + step,
                                    np.repeat(runs[:, 2], n), np.repeat(runs[:, 3], n) + step]).astype(np.int64)).to(DEVICE)
    for kv in pools:
        for pool in kv:
            _tokens_of(c, pool, at[2], at[3], _tokens_of(c, pool, at[0], at[1]))


def _continued(holders, page, off, ids, tokens, parents):
    """Page lists of sequences that go on from `parents`: whole pages are shared, a partly filled last page goes to the
    first that goes on if nobody else holds it, and is copied for the others."""
    before, out, runs, taken = holders.copy(), [], [], set()
    free = iter(np.flatnonzero(before == 0).tolist())
    for parent in parents.tolist():
        own_pages = ids[off[parent]:off[parent + 1]].copy()
        if tokens[parent] % page:
            last = int(own_pages[-1])
            if before[last] > 1 or parent in taken:
                own_pages[-1] = next(free)
                runs.append((last, 0, int(own_pages[-1]), 0, int(tokens[parent]) % page))
            taken.add(parent)
        out.append(own_pages)
    joined = np.concatenate(out)
    np.add.at(holders, joined, 1)
    np.subtract.at(holders, ids, 1)
    offsets = np.concatenate([[0], np.cumsum([len(x) for x in out])]).astype(np.int32)
    return offsets, joined.astype(np.int32), np.array(runs, np.int64).reshape(-1, 5)


def _plain_fork(s):
    c = s.c
    off, ids, runs = _continued(s.holders, c["page"], s.off, s.ids, s.tokens, s.parents)
    _copy_tokens(c, s.pools, runs)
    _, kept, runs = _continued(s.holders, c["page"], off, ids, s.tokens[s.parents], s.first)
    _copy_tokens(c, s.pools, runs)
    return [ids, kept, *(p for kv in s.pools for p in kv)]


def _plain_copy(s):
    _copy_tokens(s.c, s.pools, s.runs)
    return [p for kv in s.pools for p in kv]


def _log_probabilities(s):
    """Scores of every continuation in 64 bits; a finished beam goes on with its last token alone."""
    x = s.logits.double()
    top = x.amax(-1, keepdim=True)
    x = x - torch.where(top == -math.inf, 0.0, top)
    x = x - torch.log(torch.exp(x).sum(-1, keepdim=True)).clamp_min(0.0)
    if s.finished is not None:
        last = torch.full((x.shape[-1],), -math.inf, dtype=torch.float64, device=DEVICE)
        last[s.eos] = 0.0
        x = torch.where(s.finished[..., None], last, x)
    return (x + s.scores.double()[..., None]).flatten(1)


def _plain_select(s):
    c = s.c
    x, k = _log_probabilities(s), c["k"]
    least = torch.topk(x, k, 1).values[:, -1:]
    above, equal = x > least, x == least
    wanted = k - above.sum(1, keepdim=True)
    kept = above | (equal & (torch.cumsum(equal, 1, dtype=torch.int32) <= wanted))
    at = kept.nonzero()[:, 1].view(-1, k)                       # lowest index first
    best = torch.sort(x.gather(1, at), dim=1, descending=True, stable=True)
    at = at.gather(1, best.indices)
    return best.values.float(), (at // c["vocab"]).int(), (at % c["vocab"]).int()


def _plain_reorder(s):
    rows = torch.arange(s.beams.shape[0], device=DEVICE)[:, None]
    return [x[rows, s.beams.long()] for x in s.states]


_run_plain = dict(append=_plain_append, rotate=_plain_rotate, fork=_plain_fork, copy=_plain_copy, select=_plain_select,
                  reorder=_plain_reorder)


# ---- what a pass cannot do without, and its result in 64 bits --------------------------------------------


def work(case):
    c, op = case, case["op"]
    size = {FP16: 2, BF16: 2, FP32: 4}[c["dtype"]]
    if op == "append":
        rows = 2 * c["hq"] + 4 * c["hkv"]
        return {"bytes": c["tokens"] * (rows * c["d"] * size + 16), "flops": c["tokens"] * (c["hq"] + c["hkv"]) * c["turned"] * 3}
    if op == "rotate":
        return {"bytes": c["tokens"] * (2 * c["heads"] * c["d"] * size + 8), "flops": c["tokens"] * c["heads"] * c["turned"] * 3}
    token = 2 * 2 * c["layers"] * c["hkv"] * c["d"] * size if op in ("fork", "copy") else 0      # K and V, read and written
    if op == "fork":
        tokens, off, *_ = _sequences(c, 0)                      # copied tokens, and the page lists
        return {"bytes": int((tokens % c["page"]).sum()) * (c["children"] - 1) * token + int(off[-1]) * 4 * (c["children"] + 1),
                "flops": 0}
    if op == "copy":
        return {"bytes": c["pages"] * c["page"] * token, "flops": 0}
    if op == "select":
        n = c["batch"] * c["beams"] * c["vocab"]
        return {"bytes": n * size + c["batch"] * (c["beams"] * 5 + c["k"] * 12), "flops": 4 * n}
    return {"bytes": 2 * c["batch"] * c["beams"] * (c["history"] * 4 + c["tensors"] * c["width"] * size), "flops": 0}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] in ("append", "rotate"):
        return _exact_rotary(c, s)
    if c["op"] in ("fork", "copy"):
        # what is copied is equal to its source, token by token; pages go by the lowest free one
        if c["op"] == "copy":
            runs, lists = s.runs.tolist(), []
        else:
            free = sorted(set(range(s.pools[0][0].shape[0])) - set(s.ids.tolist()))
            runs, forked = [], []
            for i, n in enumerate(s.tokens.tolist()):
                for child in range(c["children"]):
                    pages = s.ids[s.off[i]:s.off[i + 1]].tolist()
                    if n % c["page"] and child:
                        runs.append((pages[-1], 0, free[0], 0, n % c["page"]))
                        pages[-1] = free.pop(0)
                    forked += pages
            lists = [np.array(forked, np.int32), s.ids]
        by_size = {}
        for a, at, b, to, n in runs:
            by_size.setdefault((at, to, n), []).append((a, b))
        for (at, to, n), pairs in by_size.items():
            a, b = torch.tensor(pairs, device=DEVICE).T
            for kv in s.pools:
                for p in kv:
                    if c["layout"] == "thd":
                        p[b, to:to + n] = p[a, at:at + n]
                    else:
                        p[b, :, to:to + n] = p[a, :, at:at + n]
        return lists + [p.double() for kv in s.pools for p in kv]
    if c["op"] == "select":
        scores, beams, tokens = [], [], []
        for i in range(c["batch"]):
            x = s.logits[i].double()
            x = s.scores[i].double()[:, None] + torch.log_softmax(x, -1)
            if s.finished is not None:
                for w in range(c["beams"]):
                    if s.finished[i, w]:
                        x[w] = -math.inf
                        x[w, s.eos] = s.scores[i, w].double()
            best = torch.sort(torch.nan_to_num(x, nan=-math.inf, neginf=-math.inf).flatten(), descending=True, stable=True)
            scores.append(best.values[:c["k"]])
            beams.append((best.indices[:c["k"]] // c["vocab"]).int())
            tokens.append((best.indices[:c["k"]] % c["vocab"]).int())
        return torch.stack(scores), torch.stack(beams), torch.stack(tokens)
    source = (torch.arange(c["batch"], device=DEVICE)[:, None] * c["beams"] + s.beams).flatten()
    return [x.flatten(0, 1).index_select(0, source).view(x.shape) for x in s.states]


def _exact_rotary(c, s):
    """Every pair of channels as a complex number, times magnitude * exp(i * position * frequency)."""
    rotary = _plain_rotary(c)
    sign = -1.0 if c.get("inverse") else 1.0
    turn = torch.polar(torch.full((), rotary.magnitude, dtype=torch.float64, device=DEVICE).expand(c["tokens"], c["turned"] // 2).contiguous(),
                       sign * 2 * math.pi * torch.remainder(s.positions.double()[:, None] * rotary.turns, 1.0))

    def turned(x):
        x = x.double()
        r = c["turned"]
        pairs = x[..., :r].unflatten(-1, (r // 2, 2) if c["interleaved"] else (2, r // 2))
        if not c["interleaved"]:
            pairs = pairs.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        z = z if c["interleaved"] else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), x[..., r:]], -1)

    if c["op"] == "rotate":
        return turned(s.x)
    k_pool, v_pool = (p.double() for p in s.pools[0])
    k = turned(s.k)
    for pool, rows in ((k_pool, k), (v_pool, s.v.double())):
        flat = pool if c["layout"] == "thd" else pool.transpose(1, 2)
        for chunk in torch.split((s.slots >= 0).nonzero()[:, 0], 1 << 16):
            slot = s.slots[chunk]
            flat[slot // c["page"], slot % c["page"]] = rows[chunk]
    return [turned(s.q), k_pool, v_pool]
