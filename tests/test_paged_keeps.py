"""A cache in pages keeps what it was made over: the pools and a table that nobody else holds (a converted one, say) are not freed under it."""
import weakref

import torch

from paper_2608_26140_b200 import binding as ab


def test_the_pools_and_the_table_live_as_long_as_the_cache():
    ctx = ab.Context.__new__(ab.Context)
    ctx.heads = (4, 2, 64)
    held = [torch.zeros((5, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((5, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((3, 4), dtype=torch.int64)]
    held[2] = held[2].to(torch.int32)
    at = [t.data_ptr() for t in held]
    there = [weakref.ref(t) for t in held]
    cache = ctx.paged_kv(*held)
    held.clear()
    assert all(r() is not None for r in there) and [cache.k, cache.v, cache.table] == at
    del cache
    assert all(r() is None for r in there)
