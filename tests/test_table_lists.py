"""Lists on the host that KVCache.table and KVCache.slots copy to the GPU."""
import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C
from workloads import HeadConfig, DTYPE_BF16

DEV = "cuda:0"


def test_a_number_is_no_list():
    cache = C.KVCache(HeadConfig(1, 1, 64, DTYPE_BF16), 4, device="cpu")
    for bad in (5, np.int32(5), np.array(5), None, "5", [[1, 2]], [1.0], [1 << 31]):
        with pytest.raises(ValueError):
            cache._to_device(bad, "tokens")
    for good in ([5], (5,), np.array([5], np.uint8), np.array([5])):
        got = cache._to_device(good, "tokens")
        assert got.dtype is torch.int32 and got.tolist() == [5]
    assert cache._to_device([], "tokens").shape == (0,)


@pytest.mark.gpu
def test_a_table_of_a_number_is_refused():
    cache = C.KVCache(HeadConfig(1, 1, 64, DTYPE_BF16), 4, device=DEV)
    assert cache.table([0, 1], [3], [5], 2).tolist() == [[3, -1]]
    for bad in (([0, 1], [3], 5, 2), ([0, 1], 3, [5], 2), (0, [], [], 2)):
        with pytest.raises(ValueError):
            cache.table(*bad)
