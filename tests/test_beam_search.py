"""A beam search by the framework's own calls, step by step against a plain 64-bit implementation: new tokens into the
cache, attention over the prefix forest, selection, states and pages of the beams that go on."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C
from oracle import operators as O
from workloads import Forest, HeadConfig, DTYPE_BF16, DTYPE_FP16

DEV = "cuda:0"
PREFIX, PROMPTS = 37, [5, 16, 29]


class Model:
    """Two layers side by side: a token's queries, keys and values in each are rows of a table; the logits are a product of
    both layers' attention."""

    def __init__(self, head, vocab, seed):
        gen = torch.Generator().manual_seed(seed)
        dt, d = head.torch_dtype, head.head_dim
        self.head, self.vocab = head, vocab
        self.table = torch.randn((2, vocab, head.num_q_heads + 2 * head.num_kv_heads, d), generator=gen).to(dt)
        self.out = torch.randn((2 * head.num_q_heads * d, vocab), generator=gen) * 0.1
        self.dev = SimpleNamespace(table=self.table.to(DEV), out=self.out.to(DEV))

    def qkv(self, tokens):
        """[layer][q, k, v] of tokens [n] on the GPU"""
        h = self.head
        return [self.dev.table[l][tokens].split([h.num_q_heads, h.num_kv_heads, h.num_kv_heads], 1) for l in range(2)]

    def log_probabilities(self, context, rotary):
        """Of the token after `context`, in 64 bits from the rows as the cache keeps them; and how far off 32-bit logits from
        16-bit attention outputs may be."""
        h, d, n = self.head, self.head.head_dim, len(context)
        turns, magnitude, outs = rotary.turns.cpu().numpy(), rotary.magnitude, []
        for l in range(2):
            q, k, v = (x.double().numpy() for x in self.table[l][torch.tensor(context)].split([h.num_q_heads, h.num_kv_heads, h.num_kv_heads], 1))
            q, k = O.rotary(q[-1:], [n - 1], turns, magnitude, False)[0], O.rotary(k, np.arange(n), turns, magnitude, False)[0]
            q, k = (torch.from_numpy(x).to(h.torch_dtype).double().numpy() for x in (q, k))
            for i in range(h.num_q_heads):
                s = k[:, i // h.group] @ q[0, i] * h.scale
                p = np.exp(s - s.max())
                outs.append(p @ v[:, i // h.group] / p.sum())
        o = np.concatenate(outs)
        w = self.out.double().numpy()
        x = o @ w
        x = x - x.max()
        # the attention's outputs are within 2e-3 + 2^-7 |out| (the bound its tests hold it to); a key whose rounding went the
        # other way is another such error.  The logits' products are 32-bit: 2^-24 of the terms' sum for each of them
        off = 2 * ((2e-3 + 2.0 ** -7 * np.abs(o)) @ np.abs(w)).max() + len(o) * 2.0 ** -24 * (np.abs(o) @ np.abs(w)).max()
        return x - np.log(np.exp(x).sum()), off


class Search:
    """What a program keeps between steps."""

    def __init__(self, model, beams, layout, pages, seed):
        h = model.head
        self.model, self.beams, self.h, self.ps = model, beams, h, h.page_size
        self.cache = C.KVCache(h, pages, layers=2, layout=layout, device=DEV)
        for kv in self.cache.pools:
            for p in kv:
                p.fill_(float("nan"))                   # what is not written shows
        self.rotary = C.Rotary(h.head_dim, theta=10000.0, device=DEV)
        rng = np.random.default_rng(seed)
        self.prefix = rng.integers(0, model.vocab, PREFIX).tolist()
        self.prompts = [rng.integers(0, model.vocab, n).tolist() for n in PROMPTS]
        self.cache.take(3)                              # pages of somebody else
        self.node_pages = [self.cache.take(-(-PREFIX // self.ps))] + [self.cache.take(-(-n // self.ps)) for n in PROMPTS]
        self.append(self.prefix, np.arange(PREFIX), self.node_pages[0], np.arange(PREFIX))
        for pages, prompt in zip(self.node_pages[1:], self.prompts):
            self.append(prompt, PREFIX + np.arange(len(prompt)), pages, np.arange(len(prompt)))
        # the last token of a prompt is decoded again as the first step's query, as a leaf of its own
        n = len(PROMPTS)
        self.off, self.ids = np.zeros(n * beams + 1, np.int32), np.zeros(0, np.int32)
        self.tokens = np.zeros(n * beams, np.int32)     # generated tokens of a leaf
        self.scores = torch.full((n, beams), -np.inf, device=DEV)
        self.scores[:, 0] = 0.0
        self.finished = torch.zeros((n, beams), dtype=torch.bool, device=DEV)
        self.history = torch.full((n, beams, 64), -1, dtype=torch.int32, device=DEV)
        self.next = torch.tensor([[p[0]] * beams for p in self.prompts], dtype=torch.int32, device=DEV)

    def append(self, tokens, positions, pages, at):
        slots = pages[at // self.ps].astype(np.int64) * self.ps + at % self.ps
        return [self.cache.append(l, *qkv, torch.from_numpy(np.asarray(positions, np.int64)).to(DEV), torch.from_numpy(slots).to(DEV), self.rotary)
                for l, qkv in enumerate(self.model.qkv(torch.tensor(tokens, device=DEV)))]

    def step(self, eos):
        """Logits of all beams, and the beams that go on."""
        n, w, ps, cache = len(PROMPTS), self.beams, self.ps, self.cache
        # a page for the next token where a leaf's pages are full
        lists = [self.ids[a:b] for a, b in zip(self.off, self.off[1:])]
        lists = [np.concatenate([x, cache.take(1)]) if t == len(x) * ps else x for x, t in zip(lists, self.tokens)]
        at = self.tokens.astype(np.int64)
        slots = np.array([x[t // ps] * ps + t % ps for x, t in zip(lists, at)], np.int64)
        base = np.repeat([PREFIX + len(p) for p in self.prompts], w)
        q = [cache.append(l, *qkv, torch.from_numpy(base + at).to(DEV), torch.from_numpy(slots).to(DEV), self.rotary)
             for l, qkv in enumerate(self.model.qkv(self.next.flatten().long()))]
        self.tokens = self.tokens + 1
        self.off, self.ids = np.cumsum([0] + [len(x) for x in lists]).astype(np.int32), np.concatenate(lists).astype(np.int32)
        # prefix, prompts, leaves
        parent = [-1] + [0] * n + [1 + s for s in range(n) for _ in range(w)]
        lens = np.concatenate([[PREFIX], PROMPTS, self.tokens]).astype(np.int32)
        forest = Forest(np.array(parent), lens, 1 + n + np.arange(n * w))
        pages = [*self.node_pages, *lists]
        paged = cache.paged(np.cumsum([0] + [len(x) for x in pages]).astype(np.int32), np.concatenate(pages).astype(np.int32))
        plan = C.PlannedAttention(forest, paged, self.h, device=DEV, share=2, schedule=2, fused=2)
        outs = [plan.decode(x, *kv) for x, kv in zip(q, cache.pools)]
        logits = torch.cat([o.flatten(1) for o in outs], 1).float() @ self.model.dev.out
        scores, beams, tokens = C.beam_select(logits.view(n, w, -1), self.scores, w, finished=self.finished, eos=eos)
        torch.cuda.synchronize()
        plan.close()
        parents = (torch.arange(n, device=DEV)[:, None] * w + beams).flatten().cpu().numpy()
        self.off, self.ids = cache.fork(self.off, self.ids, self.tokens, parents)
        self.tokens = self.tokens[parents]
        self.history, done = C.beam_reorder([self.history, self.finished], beams)
        self.history[:, :, int(self.tokens.max()) - 1] = tokens
        self.finished = done | (tokens == eos)
        self.scores, self.next = scores, tokens
        return scores.double().cpu().numpy(), beams.cpu().numpy(), tokens.cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,dtype,page,layout,beams", [(8, 2, 64, DTYPE_BF16, 16, "htd", 4), (4, 4, 128, DTYPE_FP16, 16, "thd", 3), (4, 1, 64, DTYPE_BF16, 32, "thd", 6)])
def test_beam_search(hq, hkv, d, dtype, page, layout, beams):
    """Given the search's own choices so far, every choice is one of the best, and scores what the plain implementation
    says, within what its logits may be off, step after step."""
    head = HeadConfig(hq, hkv, d, dtype, page)
    model = Model(head, 53, seed=hq + d)
    eos = 7
    search = Search(model, beams, layout, 400, seed=beams)
    n, vocab = len(PROMPTS), model.vocab
    held = search.cache.free_pages
    contexts = [[search.prefix + p + [p[0]] for _ in range(beams)] for p in search.prompts]
    known = np.where(np.arange(beams) == 0, 0.0, -np.inf)[None].repeat(n, 0)        # the plain scores of the beams
    slack, done, chosen = np.zeros((n, beams)), np.zeros((n, beams), bool), [[[] for _ in range(beams)] for _ in range(n)]
    for step in range(36):
        print(f"[case] beam search step {step}", flush=True)
        scores, beam, token = search.step(eos)
        for s in range(n):
            plain, off = np.full((beams, vocab), -np.inf), np.zeros(beams)
            for b in range(beams):
                if known[s, b] == -np.inf:
                    continue
                if done[s, b]:
                    plain[b, eos] = known[s, b]
                else:
                    x, off[b] = model.log_probabilities(contexts[s][b], search.rotary)
                    plain[b] = known[s, b] + x
            tol = 2 * off + slack[s]                                                # a logit and the logarithm of the sum
            picked = plain[beam[s], token[s]]
            near = np.abs(scores[s] - picked) <= tol[beam[s]] + 2.0 ** -20 * np.abs(picked)
            assert np.all(near | (scores[s] == picked)), (step, s, scores[s], picked)
            best = np.sort(plain, axis=None)[::-1][:beams]
            assert np.all((picked >= best.min() - 2 * tol.max()) | (picked == best.min()))
            assert len({(b, t) for b, t in zip(beam[s], token[s])}) == beams
            known[s], slack[s] = picked, np.where(done[s, beam[s]], slack[s, beam[s]], tol[beam[s]])
            done[s] = done[s, beam[s]] | (token[s] == eos)
            contexts[s] = [contexts[s][b] + [int(t)] for b, t in zip(beam[s], token[s])]
            chosen[s] = [chosen[s][b] + [int(t)] for b, t in zip(beam[s], token[s])]
    assert np.array_equal(search.history[:, :, :36].cpu().numpy(), np.array(chosen))
    # nothing leaked: with the leaves gone the pages are those of prefix and prompts
    search.cache.fork(search.off, search.ids, search.tokens, [])
    assert search.cache.free_pages == held
