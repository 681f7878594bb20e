"""From the lengths of a step's requests to their attention output: calls around and of a decode step, as measurable cases.

``KVCache.table`` and ``KVCache.slots`` (block tables, positions and slots of the new tokens, made on the GPU from the
requests' lengths), ``Rotary`` with several axes (``Rotary.apply`` with its gradient, ``KVCache.append``: images and video beside
text), ``PlannedAttention.decode_differential`` (the difference of two softmax maps over a prefix-shared cache).  With ``own``
false the same results come from elementary torch operations.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
FP16, BF16 = 0, 1                       # the framework's dtype codes
DTYPES = {FP16: torch.float16, BF16: torch.bfloat16}
SPARE_PAGES = 64
QUERY_SCALE = 2.0                       # logits spread with a standard deviation of two
EPS = 1e-5


# ---- the cases -------------------------------------------------------------------------------------------


def _case(name, **c):
    return dict(name=name, **c) if name else c


def _table(sequences, longest, page, width, name=None, shape=1):
    return _case(name, op="table", sequences=sequences, longest=longest, page=page, width=width, shape=shape)


def _slots(sequences, longest, new, page, name=None, before=False, spare=True, padded=0.0, shape=1):
    return _case(name, op="slots", sequences=sequences, longest=longest, new=new, page=page, before=before, spare=spare,
                 padded=padded, shape=shape)


def _turn(op, tokens, hq, hkv, d, dtype, axes, name=None, alternating=False, restart=False, blocks=1, interleaved=False, scaling="none",
          factor=1.0, theta=10000.0, images=1, page=16, layout="htd", fused=False, padded=0.0, shape=1):
    return _case(name, op=op, tokens=tokens, hq=hq, hkv=hkv, d=d, dtype=dtype, axes=axes, alternating=alternating, restart=restart,
                 blocks=blocks, interleaved=interleaved, scaling=scaling, factor=factor, theta=theta, images=images, page=page,
                 layout=layout, fused=fused, padded=padded, shape=shape)


def _differential(requests, heads, hkv, d, dtype, page, layout, shortest, longest, name=None, root=0, branches=0, branch=0, drafted=0,
                  weights="head", norm=True, shape=1):
    return _case(name, op="differential", requests=requests, heads=heads, hkv=hkv, d=d, dtype=dtype, page=page, layout=layout,
                 shortest=shortest, longest=longest, root=root, branches=branches, branch=branch, drafted=drafted, weights=weights,
                 norm=norm, shape=shape)


def listed():
    return [
        # block tables of a few dozen chats, after their page lists changed: the latency of a call counts
        _table(33, 1000, 16, 64, "table_few_chats", shape=1),
        # all requests of a large server, contexts of up to 64k tokens
        _table(4096, 65536, 16, 4096, "table_large_batch", shape=2),
        # one decoding step of 48 requests, a new page for those whose last one is full: latency
        _slots(48, 32768, 1, 16, "slots_decode_step", before=True, shape=3),
        # chunks of the prompts of 300 requests, some waiting with none, a padded batch
        _slots(300, 20000, 437, 16, "slots_prompt_chunks", padded=0.1, shape=4),
        # text tokens of a few chats about images, three axes in sections: latency
        _turn("append", 5, 8, 8, 128, FP16, "16,24,24", "append_axes_chats", images=0, theta=1000000.0),
        # prompts with video, axes in turn, queries, keys and values of one projection
        _turn("append", 16384, 64, 8, 128, BF16, "24,20,20", "append_axes_video_prompts", alternating=True, theta=5000000.0,
              layout="thd", fused=True, padded=0.05, shape=5),
        # training an image encoder: rows and columns with frequencies of their own, forward and backward
        _turn("train", 4099, 16, 16, 64, BF16, "16,16", "train_axes_image_encoder", restart=True),
        # the next tokens of a batch whose heads hold two maps each, as differential attention reads them
        _turn("append", 512, 32, 4, 256, BF16, "64", "append_two_maps", blocks=2, images=0, theta=500000.0, shape=6),
        # four short chats that share nothing, a small model: the latency of a call counts
        _differential(4, 8, 8, 64, FP16, 16, "htd", 100, 1100, "differential_four_chats", shape=7),
        # questions on one document
        _differential(32, 32, 8, 64, BF16, 16, "htd", 64, 600, "differential_document", root=8192, weights="one", shape=8),
        # verification of 24 drafted tokens on each of 16 sequences; weights from a projection of each token
        _differential(16, 16, 4, 64, BF16, 32, "thd", 2000, 4100, "differential_drafts", root=500, drafted=24, weights="token",
                      norm=False, shape=9),
        # the largest: an irregular forest of three levels, heads of two times 128 channels
        _differential(64, 32, 8, 128, BF16, 16, "htd", 500, 4000, "differential_forest", root=32768, branches=8, branch=8192, shape=10),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm, odd as often as not."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["table", "slots", "slots", "append", "append", "train", "differential", "differential", "differential"])
    shape, page = rng.randrange(1, 1 << 30), rng.choice([16, 16, 32, 64])
    if op == "table":
        n, width = _spread(rng, 1, 4096), _spread(rng, 1, 4096)
        return _table(n, max(1, width * page * rng.randrange(3, 13) // 12), page, width, shape=shape)
    if op == "slots":
        n = _spread(rng, 1, 20000)
        return _slots(n, _spread(rng, 1, min(60000, (1 << 25) // n)), _spread(rng, 1, max(2, 130000 // n)), page, before=rng.random() < 0.5,
                      spare=rng.random() < 0.7, padded=rng.choice([0.0, 0.0, 0.3]), shape=shape)
    dtype, layout = rng.choice([FP16, BF16]), rng.choice(["htd", "thd"])
    if op in ("append", "train"):
        hq, hkv, d = rng.choice([(8, 8, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (64, 8, 64), (9, 3, 64), (16, 8, 256)])
        blocks = rng.choice([1, 1, 1, 2])
        interleaved = rng.random() < 0.4
        most = d // (2 * blocks)                        # pairs of a block
        pairs = rng.choice([most, most, most // 2]) if blocks == 2 or rng.random() < 0.7 else rng.randrange(2, most + 1)
        n = rng.randrange(1, 5) if blocks == 2 else rng.randrange(2, 5)
        cuts = sorted(rng.randrange(0, pairs + 1) for _ in range(n - 1))
        axes = [b - a for a, b in zip([0] + cuts, cuts + [pairs])]
        scaling = rng.choice(["none", "none", "linear", "ntk"])
        return _turn(op, _spread(rng, 1, 16384 if op == "append" else 6000), hq, hkv, d, dtype, ",".join(map(str, axes)),
                     alternating=rng.random() < 0.4, restart=rng.random() < 0.4, blocks=blocks, interleaved=interleaved,
                     scaling=scaling, factor=1.0 if scaling == "none" else rng.uniform(1.5, 16.0),
                     theta=rng.choice([10000.0, 500000.0, 1000000.0]), images=rng.randrange(0, 2), page=page, layout=layout,
                     fused=rng.random() < 0.5, padded=rng.choice([0.0, 0.0, 0.2]), shape=shape)
    heads, hkv, d = rng.choice([(8, 8, 64), (32, 8, 64), (16, 4, 64), (14, 2, 64), (16, 1, 64), (16, 16, 32), (24, 8, 32),
                                (16, 8, 128), (32, 8, 128), (8, 2, 128)])
    shortest = _spread(rng, 1, 2000)
    longest = _spread(rng, shortest, 4 * shortest)
    drafted = rng.choice([0, 0, 0, 3, 17, 40])
    if heads // hkv > 8:                    # groups of 16 rows, two a head, have masks
        drafted = 0
    root, branches = rng.choice([0, _spread(rng, 30, 30000)]), rng.choice([0, 0, rng.randrange(2, 9)])
    branch = _spread(rng, 30, 8000) if branches else 0
    # no more tokens and no more work than the largest listed case
    room = (200000 * 8 * 128 // (hkv * d) - root - 3 * branches * branch // 2) // longest
    work = (1 << 33) // (heads * d * (1 + drafted) * (root + 3 * branch // 2 + longest))
    requests = _spread(rng, 1, max(1, min(16 if drafted else 80, room, work)))
    return _differential(requests, heads, hkv, d, dtype, page, layout, shortest, longest, root=root, branches=branches,
                         branch=branch, drafted=drafted, weights=rng.choice(["one", "head", "token"]),
                         norm=rng.random() < 0.6, shape=shape)


# ---- inputs ----------------------------------------------------------------------------------------------


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return gen


def _random(seed):
    return np.random.Generator(np.random.PCG64(seed))


def _gpu(array, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(array, dtype)).to(DEVICE)


def _normal(shape, c, gen, scale=1.0):
    return torch.empty(shape, dtype=DTYPES[c["dtype"]], device=DEVICE).normal_(0.0, scale, generator=gen)


def _pools(c, num_pages, gen):
    shape = (num_pages, c["page"], c["hkv"], c["dim"]) if c["layout"] == "thd" else (num_pages, c["hkv"], c["page"], c["dim"])
    return [_normal(shape, c, gen) for _ in "kv"]


def _framework_cache(c, pools=None, num_pages=1):
    from paper_2505_17694_amd import KVCache
    head = SimpleNamespace(num_q_heads=c.get("hq", 1), num_kv_heads=c.get("hkv", 1), head_dim=c.get("dim", 64),
                           dtype=c.get("dtype", BF16), page_size=c["page"])
    return KVCache(head, num_pages, layout=c.get("layout", "htd"), device=DEVICE, pools=None if pools is None else [pools])


def _lengths(c):
    """Of the case alone: tokens of the sequences; for slots also the new ones."""
    rng, n = _random(c["shape"]), c["sequences"]
    tokens = rng.integers(0, c["longest"] + 1, n)
    if c["op"] == "table":
        return tokens, None
    new = np.ones(n, np.int64) if c["new"] == 1 else rng.integers(0, c["new"] + 1, n) * (rng.random(n) < 0.9)
    return tokens, new


def _prepare_table(c, seed):
    tokens, _ = _lengths(c)
    rng, n = _random(seed), c["sequences"]
    pages = np.minimum(-(-tokens // c["page"]) + _random(c["shape"] + 1).integers(0, 3, n), c["width"])    # some pages ahead
    off = np.concatenate([[0], np.cumsum(pages)])
    ids = rng.permutation(int(off[-1]) + SPARE_PAGES)[:off[-1]]
    return SimpleNamespace(c=c, off=_gpu(off), ids=_gpu(ids), tokens=_gpu(tokens),
                           cache=_framework_cache(c) if own else None)


def _prepare_slots(c, seed):
    tokens, new = _lengths(c)
    rng, n, ps = _random(seed), c["sequences"], c["page"]
    held, needed = -(-tokens // ps), -(-(tokens + new) // ps)
    width = int(needed.max()) + 1
    filled = held if c["spare"] else needed             # without spare pages the new ones are in the table already
    num_pages = int(filled.sum() + (needed - held).sum()) + SPARE_PAGES
    ids = rng.permutation(num_pages)
    table = np.full((n, width), -1, np.int64)
    table[np.arange(width) < filled[:, None]] = ids[:filled.sum()]
    total = int(new.sum())
    return SimpleNamespace(c=c, table=_gpu(table), tokens=_gpu(tokens), new=_gpu(new), num_tokens=total + int(total * c["padded"]),
                           before=_gpu(rng.integers(-50, 5000, n), np.int64) if c["before"] else None,
                           spare=_gpu(ids[filled.sum():]) if c["spare"] else None, num_pages=num_pages,
                           cache=_framework_cache(c, num_pages=num_pages) if own else None)


def _axis_positions(c, rng):
    """[axes, tokens]: with images text runs and grids in turn, where an axis counts frames, rows or columns; else one place each."""
    axes, t = len(c["axes"].split(",")), c["tokens"]
    if not c["images"]:
        return np.tile(rng.integers(0, 100000, t), (axes, 1))
    out, have, p = [], 0, int(rng.integers(0, 2000))
    while have < t:
        n = int(rng.integers(5, 200))
        out.append(np.tile(p + np.arange(n), (axes, 1)))
        grid = rng.integers(1, 5), rng.integers(4, 25), rng.integers(4, 25)
        at = p + n + np.stack([x.ravel() for x in np.meshgrid(*(np.arange(g) for g in grid), indexing="ij")])
        out.append(at[{1: [0], 2: [1, 2], 3: [0, 1, 2], 4: [0, 1, 2, 0]}[axes]])
        have += n + at.shape[1]
        p += n + int(max(grid))
    return np.concatenate(out, 1)[:, :t]


def _framework_rotary(c):
    from paper_2505_17694_amd import Rotary
    axes = [int(n) for n in c["axes"].split(",")]
    scaling = None if c["scaling"] == "none" else dict(kind=c["scaling"], factor=c["factor"])
    return Rotary(2 * sum(axes) * c["blocks"], theta=c["theta"], interleaved=c["interleaved"], scaling=scaling, device=DEVICE,
                  axes=axes, alternating=c["alternating"], restart=c["restart"], blocks=c["blocks"])


def _prepare_turn(c, seed):
    gen, rng = _generator(seed), _random(seed)
    t, c = c["tokens"], dict(c, dim=c["d"])
    s = SimpleNamespace(c=c, positions=_gpu(_axis_positions(c, rng), np.int64), rotary=_framework_rotary(c) if own else _plain_rotary(c))
    if c["op"] == "train":
        s.x, s.grad = (_normal((t, c["hq"], c["d"]), c, gen) for _ in range(2))
        s.x.requires_grad_()
        return s
    if c["fused"]:
        s.q, s.k, s.v = _normal((t, c["hq"] + 2 * c["hkv"], c["d"]), c, gen).split([c["hq"], c["hkv"], c["hkv"]], 1)
    else:
        s.q, s.k, s.v = (_normal((t, h, c["d"]), c, gen) for h in (c["hq"], c["hkv"], c["hkv"]))
    num_pages = -(-t // c["page"]) + SPARE_PAGES
    slots = rng.permutation(num_pages)[np.arange(t) // c["page"]] * c["page"] + np.arange(t) % c["page"]
    slots[rng.random(t) < c["padded"]] = -1
    s.slots = _gpu(slots, np.int64)
    s.pools = _pools(c, num_pages, gen)
    s.cache = _framework_cache(c, s.pools, num_pages) if own else None
    return s


def _forest(c):
    """Of the case alone: parent, node_len, req_node, req_mask_off, req_mask (None without drafted tokens), and for every request
    which tokens of its last node it sees (None: all)."""
    rng = _random(c["shape"])
    parent, length, last, seen = [], [], [], []

    def node(above, tokens):
        parent.append(above)
        length.append(int(tokens))
        return len(parent) - 1

    root = node(-1, c["root"]) if c["root"] else -1
    above = [node(root, rng.integers(c["branch"] // 2 + 1, c["branch"] + c["branch"] // 2 + 1)) for _ in range(c["branches"])] or [root]
    for i in range(c["requests"]):
        leaf = node(above[int(rng.integers(len(above)))], rng.integers(c["shortest"], c["longest"] + 1))
        last.append(leaf)
        seen.append(None)
        if c["drafted"]:                    # a token is drafted after the last one or any other, the context being one of them
            drafts, after = node(leaf, c["drafted"]), []
            for k in range(c["drafted"]):
                before = k - 1 if rng.random() < 0.5 else int(rng.integers(-1, k)) if k else -1
                after.append([k] + (after[before] if before >= 0 else []))
                last.append(drafts)
                seen.append(sorted(after[k]))
    off = words = None
    if c["drafted"]:
        per = (c["drafted"] + 31) // 32
        off = np.concatenate([[0], np.cumsum([0 if x is None else per for x in seen])]).astype(np.int32)
        words = np.zeros(off[-1], np.uint32)
        for r, x in enumerate(seen):
            for t in x or ():
                words[off[r] + t // 32] |= np.uint32(1 << (t % 32))
    return np.array(parent), np.array(length), np.array(last), off, words, seen


def _prepare_differential(c, seed):
    gen, rng = _generator(seed), _random(seed)
    parent, length, last, off, words, seen = _forest(c)
    c = dict(c, dim=2 * c["d"], hq=2 * c["heads"])
    pages = -(-length // c["page"])
    page_off = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    num_pages = int(page_off[-1]) + SPARE_PAGES
    ids = rng.permutation(num_pages)[:page_off[-1]].astype(np.int32)
    n = len(last)
    s = SimpleNamespace(c=c, pools=_pools(c, num_pages, gen), parent=parent, length=length, last=last, seen=seen, page_off=page_off, ids=ids)
    s.q = _normal((n, 2 * c["heads"], c["d"]), c, gen, QUERY_SCALE)
    shape = {"one": (), "head": (c["heads"],), "token": (n, c["heads"])}[c["weights"]]
    s.weights = torch.rand(shape, generator=gen, device=DEVICE).mul_(0.6).add_(0.2)
    s.norm = torch.empty(2 * c["d"], device=DEVICE).normal_(1.0, 0.1, generator=gen) if c["norm"] else None
    s.gain = 0.3 if c["norm"] else 1.0
    s.plan = None
    if own:
        from paper_2505_17694_amd import PlannedAttention
        head = SimpleNamespace(num_q_heads=2 * c["heads"], num_kv_heads=c["hkv"], head_dim=2 * c["d"], dtype=c["dtype"],
                               page_size=c["page"], scale=float(np.float32(1.0 / math.sqrt(c["d"]))))
        forest = SimpleNamespace(parent=parent, node_len=length, req_node=last, req_mask_off=off, req_mask=words)
        cache = _framework_cache(c, s.pools, num_pages)
        s.plan = PlannedAttention(forest, cache.paged(page_off, ids), head, device=DEVICE, share=2, schedule=2, extensions=3)
    else:                                   # pages and places in them of the tokens a request sees
        s.path = [tuple(_gpu(x, np.int64) for x in _path(s, r)) for r in range(n)]
    return s


def _path(s, r):
    """Pages and places in them of the tokens that request r sees, root first."""
    ps, nodes, n = s.c["page"], [], int(s.last[r])
    while n >= 0:
        nodes.insert(0, n)
        n = int(s.parent[n])
    at = [np.arange(s.length[n]) for n in nodes]
    if s.seen[r] is not None:
        at[-1] = np.array(s.seen[r])
    return (np.concatenate([s.ids[s.page_off[n] + t // ps] for n, t in zip(nodes, at)]), np.concatenate([t % ps for t in at]))


_PREPARE = dict(table=_prepare_table, slots=_prepare_slots, append=_prepare_turn, train=_prepare_turn, differential=_prepare_differential)


def prepare(case, seed):
    return _PREPARE[case["op"]](case, seed)


# ---- the calls -------------------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)[s.c["op"]](s)


def _own_table(s):
    return s.cache.table(s.off, s.ids, s.tokens, s.c["width"])


def _own_slots(s):
    step = s.cache.slots(s.table, s.tokens, s.new, s.num_tokens, before=s.before, spare=s.spare)
    return [step.positions, step.slots, step.sequences, step.offsets, step.tokens, step.taken, s.table]


def _own_append(s):
    q = s.cache.append(0, s.q, s.k, s.v, s.positions, s.slots, s.rotary)
    return [q, *s.pools]


def _own_train(s):
    y = s.rotary.apply(s.x, s.positions)
    return [y.detach(), *torch.autograd.grad(y, s.x, s.grad)]


def _own_differential(s):
    return s.plan.decode_differential(s.q, *s.pools, s.weights, weight=s.norm, eps=EPS if s.c["norm"] else None, gain=s.gain)


_run_own = dict(table=_own_table, slots=_own_slots, append=_own_append, train=_own_train, differential=_own_differential)


# ---- the plain forms -------------------------------------------------------------------------------------


def _plain_table(s):
    c = s.c
    entry = torch.arange(c["width"], device=DEVICE)
    held = torch.minimum((s.tokens + c["page"] - 1) // c["page"], s.off[1:] - s.off[:-1])
    at = torch.where(entry < held[:, None], s.off[:-1, None] + entry, 0)
    return torch.where(entry < held[:, None], s.ids[at] if s.ids.numel() else -1, -1)


def _plain_slots(s):
    ps = s.c["page"]
    tokens, new = s.tokens.long(), s.new.long()
    held, needed = (tokens + ps - 1) // ps, (tokens + new + ps - 1) // ps
    ends, taken = torch.cumsum(new, 0), torch.cumsum(needed - held, 0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    if s.spare is not None:
        entry = torch.arange(s.table.shape[1], device=DEVICE)
        new_page = (entry >= held[:, None]) & (entry < needed[:, None])
        at = torch.where(new_page, (taken - needed)[:, None] + entry, 0)        # exclusive sums + entry - held
        s.table.copy_(torch.where(new_page, s.spare[at], s.table))
    t = torch.arange(s.num_tokens, device=DEVICE)
    q = torch.searchsorted(ends, t, right=True)                                  # first sequence that ends behind t
    live = q < len(new)
    q = torch.where(live, q, 0)
    place = tokens[q] + t - offsets[q]
    page = s.table[q, torch.where(live, place // ps, 0)].long()
    slots = torch.where(live & (page >= 0), page * ps + place % ps, -1)
    positions = place if s.before is None else place + s.before[q]
    return [torch.where(live, positions, 0), slots, torch.where(live, q, -1).int(), offsets.int(), (tokens + new).int(),
            (taken[-1:] if s.spare is not None else taken.new_zeros(1)).int(), s.table]


def _plain_rotary(c):
    """Of every pair: its channels, its axis and its turns a position (64 bits)."""
    sizes = np.array([int(n) for n in c["axes"].split(",")])
    pairs = int(sizes.sum())
    if c["alternating"]:
        axis = np.concatenate([np.flatnonzero(sizes > i) for i in range(sizes.max(initial=0))])
    else:
        axis = np.repeat(np.arange(len(sizes)), sizes)
    if c["restart"]:
        place = np.array([np.count_nonzero(axis[:i] == a) for i, a in enumerate(axis)], np.float64)
        r = 2.0 * sizes[axis]
    else:
        place, r = np.arange(pairs, dtype=np.float64), np.full(pairs, 2.0 * pairs)
    theta = np.full(pairs, c["theta"])
    if c["scaling"] == "ntk":
        theta = np.where(r > 2, theta * c["factor"] ** (r / np.maximum(r - 2, 1.0)), theta)
    freq = theta ** (-2.0 * place / r)
    if c["scaling"] == "linear":
        freq = freq / c["factor"]
    first = 2 * np.arange(pairs) if c["interleaved"] else np.arange(pairs)
    first = np.concatenate([first + 2 * pairs * b for b in range(c["blocks"])])
    second = first + (1 if c["interleaved"] else pairs)
    return SimpleNamespace(first=_gpu(first, np.int64), second=_gpu(second, np.int64), axis=_gpu(np.tile(axis, c["blocks"]), np.int64),
                           turns=torch.from_numpy(np.tile(freq / (2 * math.pi), c["blocks"])).to(DEVICE))


def _turned(rotary, x, positions, back=False):
    u = positions[rotary.axis].T.to(torch.float64) * rotary.turns
    angle = (u - torch.round(u)) * (2 * math.pi)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if back:
        sin = -sin
    out = x.float()
    a, b = out[..., rotary.first], out[..., rotary.second]
    out = out.index_copy(-1, rotary.first, a * cos - b * sin)
    return out.index_copy(-1, rotary.second, b * cos + a * sin).to(x.dtype)


def _stored(c, pool, slots, rows):
    kept = (slots >= 0).nonzero()[:, 0]
    page, place = slots[kept] // c["page"], slots[kept] % c["page"]
    pool[(page, place) if c["layout"] == "thd" else (page, slice(None), place)] = rows[kept]


def _plain_append(s):
    _stored(s.c, s.pools[0], s.slots, _turned(s.rotary, s.k, s.positions))
    _stored(s.c, s.pools[1], s.slots, s.v)
    return [_turned(s.rotary, s.q, s.positions), *s.pools]


def _plain_train(s):
    return [_turned(s.rotary, s.x.detach(), s.positions), _turned(s.rotary, s.grad, s.positions, True)]


def _plain_differential(s):
    c = s.c
    heads, hkv, d = c["heads"], c["hkv"], c["d"]
    group, n = heads // hkv, len(s.last)
    weights = s.weights.expand(n, heads)
    out = []
    for r in range(n):
        pages, places = s.path[r]
        at = (pages, places) if c["layout"] == "thd" else (pages, slice(None), places)
        k, v = (pool[at].float().transpose(0, 1) for pool in s.pools)                      # [hkv, tokens, 2 d]
        q = s.q[r].float().view(hkv, group, 2, d)
        maps = []
        for m in range(2):
            x = torch.matmul(q[:, :, m], k[..., m * d:(m + 1) * d].transpose(1, 2).contiguous()) / math.sqrt(d)
            p = torch.exp(x - x.amax(-1, keepdim=True))
            maps.append(torch.matmul(p / p.sum(-1, keepdim=True), v.contiguous()).view(heads, 2 * d))
        x = maps[0] - weights[r][:, None] * maps[1]
        if s.norm is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * s.norm
        out.append(x * s.gain)
    return torch.stack(out).to(s.q.dtype)


_run_plain = dict(table=_plain_table, slots=_plain_slots, append=_plain_append, train=_plain_train, differential=_plain_differential)


# ---- what a pass cannot do without, and its result in 64 bits --------------------------------------------


def work(case):
    c, op = case, case["op"]
    if op == "table":
        tokens, _ = _lengths(c)
        held = int(np.minimum(-(-tokens // c["page"]), c["width"]).sum())
        return {"bytes": 4 * (held + 2 * c["sequences"] + 1 + c["sequences"] * c["width"]), "flops": 0}
    if op == "slots":
        tokens, new = _lengths(c)
        held, needed, total = -(-tokens // c["page"]), -(-(tokens + new) // c["page"]), int(new.sum())
        pages = int(((new > 0) * (needed - tokens // c["page"])).sum())                    # that new tokens lie in
        return {"bytes": 20 * (total + int(total * c["padded"])) + (16 + 8 * c["before"]) * c["sequences"] + 4 * pages
                + 4 * int((needed - held).sum()) * c["spare"], "flops": 0}
    if op in ("append", "train"):
        axes = [int(n) for n in c["axes"].split(",")]
        turned, rows = 2 * sum(axes) * c["blocks"], 4 * c["hq"] if op == "train" else 2 * c["hq"] + 4 * c["hkv"]
        heads = 2 * c["hq"] if op == "train" else c["hq"] + c["hkv"]
        return {"bytes": c["tokens"] * (2 * rows * c["d"] + 8 * len(axes) + (8 if op == "append" else 0)),
                "flops": 3 * c["tokens"] * heads * turned}
    parent, length, last, _, _, seen = _forest(c)
    n, d = len(last), c["d"]
    context = 0
    for r in range(n):
        node = int(last[r])
        context += len(seen[r]) if seen[r] is not None else int(length[node])
        while int(parent[node]) >= 0:
            node = int(parent[node])
            context += int(length[node])
    return {"bytes": 8 * d * c["hkv"] * int(length.sum()) + n * c["heads"] * d * 8, "flops": 12 * d * c["heads"] * context}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "table":
        off, ids, tokens = (x.cpu().numpy() for x in (s.off, s.ids, s.tokens))
        out = np.full((c["sequences"], c["width"]), -1)
        for i in range(c["sequences"]):
            pages = ids[off[i]:off[i + 1]][:-(-int(tokens[i]) // c["page"])]
            out[i, :len(pages)] = pages
        return _gpu(out)
    if c["op"] == "slots":
        return _exact_slots(s)
    if c["op"] == "append":
        return _exact_append(s)
    if c["op"] == "train":
        return [_exact_turned(s, s.x.detach(), 1), _exact_turned(s, s.grad, -1)]
    return _exact_differential(s)


def _exact_slots(s):
    """Sequence by sequence."""
    ps, table = s.c["page"], s.table.cpu().numpy().copy()
    tokens, new = s.tokens.cpu().numpy().astype(np.int64), s.new.cpu().numpy().astype(np.int64)
    spare = None if s.spare is None else s.spare.cpu().numpy()
    before = np.zeros(len(new), np.int64) if s.before is None else s.before.cpu().numpy()
    positions, slots, sequences = np.zeros(s.num_tokens, np.int64), np.full(s.num_tokens, -1, np.int64), np.full(s.num_tokens, -1)
    at, used = [0], 0
    for i, (have, more) in enumerate(zip(tokens, new)):
        if spare is not None:
            lo, hi = -(-have // ps), -(-(have + more) // ps)
            table[i, lo:hi] = spare[used:used + hi - lo]
            used += hi - lo
        place, here = np.arange(have, have + more), slice(at[-1], at[-1] + more)
        positions[here], slots[here], sequences[here] = place + before[i], table[i, place // ps].astype(np.int64) * ps + place % ps, i
        at.append(at[-1] + int(more))
    return [_gpu(positions, np.int64), _gpu(slots, np.int64), _gpu(sequences), _gpu(at), _gpu(tokens + new), _gpu([used]), _gpu(table)]


def _exact_turned(s, x, sign):
    """Every pair of channels as a complex number times exp(i * position on its axis * frequency), pair by pair."""
    c, out = s.c, x.double()
    sizes = [int(n) for n in c["axes"].split(",")]
    pairs, left, order = sum(sizes), list(sizes), []
    while any(left):
        for a in range(len(sizes)):
            take = min(left[a], 1) if c["alternating"] else left[a]
            order += [(a, sizes[a] - left[a] + j) for j in range(take)]
            left[a] -= take
    for b in range(c["blocks"]):
        for i, (axis, nth) in enumerate(order):
            r, j = (2 * sizes[axis], nth) if c["restart"] else (2 * pairs, i)
            theta = c["theta"] * c["factor"] ** (r / (r - 2)) if c["scaling"] == "ntk" and r > 2 else c["theta"]
            turns = theta ** (-2 * j / r) / (2 * math.pi) / (c["factor"] if c["scaling"] == "linear" else 1.0)
            lo = 2 * pairs * b + (2 * i if c["interleaved"] else i)
            hi = lo + (1 if c["interleaved"] else pairs)
            turn = torch.remainder(s.positions[axis].double() * turns, 1.0) * (sign * 2 * math.pi)
            z = torch.complex(out[..., lo], out[..., hi]) * torch.polar(torch.ones_like(turn), turn)[:, None]
            out[..., lo], out[..., hi] = z.real, z.imag
    return out


def _exact_append(s):
    c, pools = s.c, [p.double() for p in s.pools]
    for pool, rows in zip(pools, (_exact_turned(s, s.k, 1), s.v.double())):
        by_token = pool.flatten(0, 1) if c["layout"] == "thd" else None
        for lo in range(0, c["tokens"], 1 << 14):
            slots, part = s.slots[lo:lo + (1 << 14)], rows[lo:lo + (1 << 14)]
            part, slots = part[slots >= 0], slots[slots >= 0]
            if by_token is not None:
                by_token.index_copy_(0, slots, part)
            else:
                pool[slots // c["page"], :, slots % c["page"]] = part
    return [_exact_turned(s, s.q, 1), *pools]


def _exact_differential(s):
    """Node by node: every node's scores for all requests below it, joined by their running maxima and sums."""
    c = s.c
    heads, hkv, d, ps = c["heads"], c["hkv"], c["d"], c["page"]
    n, group = len(s.last), heads // hkv
    below = [[] for _ in s.length]
    for r in range(n):
        node = int(s.last[r])
        while node >= 0:
            below[node].append(r)
            node = int(s.parent[node])
    q = s.q.double().view(n, hkv, group, 2, d).permute(1, 3, 0, 2, 4).contiguous()              # [hkv, map, request, group, d]
    top = torch.full((hkv, 2, n, group), -math.inf, dtype=torch.float64, device=DEVICE)
    total, acc = torch.zeros_like(top), torch.zeros((hkv, 2, n, group, 2 * d), dtype=torch.float64, device=DEVICE)
    for node, requests in enumerate(below):
        if not requests:
            continue
        which = torch.tensor(requests, device=DEVICE)
        for lo in range(0, int(s.length[node]), 4096):
            t = np.arange(lo, min(int(s.length[node]), lo + 4096))
            pages, places = _gpu(s.ids[s.page_off[node] + t // ps], np.int64), _gpu(t % ps, np.int64)
            k, v = ((p[pages, places] if c["layout"] == "thd" else p[pages, :, places]).double() for p in s.pools)      # [t, hkv, 2 d]
            visible = torch.ones((len(requests), len(t)), dtype=torch.bool, device=DEVICE)
            for i, r in enumerate(requests):
                if s.seen[r] is not None and int(s.last[r]) == node:
                    visible[i] = torch.isin(torch.from_numpy(t).to(DEVICE), torch.tensor(s.seen[r], device=DEVICE))
            for h in range(hkv):
                for m in range(2):
                    x = q[h, m, which].flatten(0, 1) @ k[:, h, m * d:(m + 1) * d].T.contiguous() * d ** -0.5
                    x = x.view(len(requests), group, -1).masked_fill(~visible[:, None], -math.inf)
                    new = torch.maximum(top[h, m, which], x.amax(-1))
                    shift = torch.where(new == -math.inf, 0.0, new)
                    old = torch.exp(top[h, m, which] - shift)
                    e = torch.exp(x - shift[..., None])
                    total[h, m, which] = total[h, m, which] * old + e.sum(-1)
                    acc[h, m, which] = acc[h, m, which] * old[..., None] + (e.flatten(0, 1) @ v[:, h].contiguous()).view(len(requests), group, -1)
                    top[h, m, which] = new
    o = (acc / total[..., None]).permute(1, 2, 0, 3, 4).reshape(2, n, heads, 2 * d)
    x = o[0] - s.weights.double().expand(n, heads)[..., None] * o[1]
    if s.norm is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * s.norm.double()
    return x * s.gain
