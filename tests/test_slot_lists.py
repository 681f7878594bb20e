"""KVCache.slots with lists on the host, as KVCache.take and a program's own bookkeeping hold them."""
import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C
from test_slots import DEV, cache_of, gpu, some_step


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 37, 5000])
@pytest.mark.parametrize("stream", [False, True])
def test_lists_on_the_host_are_those_on_the_gpu(n, stream):
    print(f"[case] host lists n={n} stream={stream}", flush=True)
    table, tokens, new, pages, num_pages, before = some_step(n, 200, 30, 16, n)
    cache, total, before = cache_of(num_pages), int(new.sum()) + 5, gpu(before, torch.int64)
    want_table = gpu(table)
    want = cache.slots(want_table, gpu(tokens), gpu(new), total, before=before, spare=gpu(pages))
    on = torch.cuda.Stream() if stream else None
    for kw in (dict(tokens=tokens, new=new, spare=pages), dict(tokens=tokens.tolist(), new=new.astype(np.int32), spare=gpu(pages)),
               dict(tokens=gpu(tokens), new=gpu(new), spare=pages.astype(np.int32)), dict(tokens=gpu(tokens), new=new.tolist(), spare=list(map(int, pages)))):
        t = gpu(table)
        torch.cuda.synchronize()
        got = cache.slots(t, num_tokens=total, before=before, stream=on, **kw)
        torch.cuda.synchronize()
        assert torch.equal(t, want_table) and all(torch.equal(a, b) for a, b in zip(got, want))
    none = cache.slots(want_table, [0] * n, [0] * n, 3, spare=[])
    assert none.slots.tolist() == [-1] * 3 and none.taken.tolist() == [0]


@pytest.mark.gpu
def test_pages_that_take_gave():
    """From take to the slots and back: what was not taken is released by the ids that take gave."""
    cache = cache_of(20)
    first = cache.take(3)
    table = cache.table([0, 2, 3], first, [20, 16], 6)
    spare = cache.take(8)
    step = cache.slots(table, [20, 16], [13, 40], 60, spare=spare)
    taken = int(step.taken)
    assert taken == 4 and table.tolist() == [[0, 1, 3, -1, -1, -1], [2, 4, 5, 6, -1, -1]] and step.tokens.tolist() == [33, 56]
    cache.release(spare[taken:])
    assert cache.free_pages == 20 - 3 - 4


@pytest.mark.gpu
def test_lists_that_are_none_are_refused():
    cache = cache_of(20)
    table, two = torch.full((2, 4), -1, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    good = dict(table=table, tokens=two, new=two, num_tokens=5)
    for bad in (dict(spare=[1.5]), dict(spare=[1 << 31]), dict(spare=np.zeros((2, 2), np.int64)), dict(spare=5), dict(tokens=[1]), dict(tokens=[1, 2, 3]),
                dict(tokens=[0.5, 1]), dict(new=[1 << 40, 0]), dict(new=None), dict(tokens=None), dict(new="ab"), dict(table=[[0] * 4] * 2),
                dict(table=np.zeros((2, 4), np.int32)), dict(table=None), dict(before=[0, 0]), dict(before=np.zeros(2, np.int64)),
                dict(spare=torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            cache.slots(**dict(good, **bad))
    assert cache.slots(**good).taken.tolist() == [0] and bool((table == -1).all())
