"""Calls of the 8-bit cache at the ends of what its arguments may be."""
import numpy as np
import pytest
import torch

from paper_2608_26140_b200 import binding as ab

from helpers import DEV
from test_gpu_kv8 import HEADS, Cache, check_attention, context, filled, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 40])
def test_rows_listed_for_a_context_of_no_tokens(n):
    """No position is inside it: every row is skipped and reported, nothing is written."""
    heads, B, cap = "gqa28", 2, 64
    H, hkv, d = HEADS[heads]
    ctx, cache = context(heads, B, cap), Cache(heads, B, cap, 16, "int8", garbage=True)
    rows = torch.ones((B, n, hkv, d), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros((B, n), dtype=torch.int32, device=DEV)
    ctx.kv8_write(cache.c, B, 0, rows, rows, pos=pos)
    cache.check()
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX
    out = torch.full_like(rows, 7.0)
    ctx.kv8_read(cache.c, B, 0, out, None, pos=pos)
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX and (out == 0).all()


ROWS_LIMIT = 65535 * 32          # of a request, per KV head


def test_rows_of_a_batch_have_no_limit_of_their_own():
    """64 requests of 1200 rows with 7 query heads per KV head, each with its cache; 64 of 4200 rows with 8, over one cache."""
    heads, B, n, T = "gqa28", 64, 1200, 48
    ctx = context(heads, B, T)
    cache, vals = filled(heads, B, T, 16, "int8", 1)
    check_attention(ctx, cache, vals, B, n, T, heads, queries(B, n, heads, 2))
    heads, n, T = "mqa8", 4200, 20
    assert B * n * 8 > ROWS_LIMIT
    ctx = context(heads, B, T)
    cache, vals = filled(heads, 1, T, 16, "int8", 1)
    check_attention(ctx, cache, vals, B, n, T, heads, queries(B, n, heads, 2), shared=True, c=ab.Context.kv8(*cache.dev, 16, ab.KV8_FORMATS["int8"], shared=True))
    assert ctx.poll_status() == 0


def test_the_most_rows_of_one_request():
    heads, T = "gqa4-64", 33
    H, hkv, d = HEADS[heads]
    n = ROWS_LIMIT // (H // hkv)
    ctx = context(heads, 1, T)
    cache, vals = filled(heads, 1, T, 16, "int8", 1)
    few = queries(1, 100, heads, 2)
    q = torch.zeros((1, n + 1, H, d), dtype=torch.bfloat16, device=DEV)
    q[:, n - 100:n] = few
    want, o = torch.empty_like(few), torch.full_like(q, 7.0)
    ctx.kv8_attention(cache.c, 1, T, few, want)
    ctx.kv8_attention(cache.c, 1, T, q[:, :n], o[:, :n])
    assert torch.equal(o[:, n - 100:n], want) and (o[:, n] == 7.0).all()
    assert torch.equal(o[:, :n - 100], o[:, :1].expand(1, n - 100, H, d)) and ctx.poll_status() == 0
    launched = ctx.launch_count()
    with pytest.raises(ab.AcacheError) as e:
        ctx.kv8_attention(cache.c, 1, T, q, o)
    assert e.value.status == ab.ERR_UNSUPPORTED_SHAPE and ctx.launch_count() == launched
