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


def test_single_rows_and_single_heads_have_no_stride_of_their_own():
    """One token's K and V inside a joint Q/K/V buffer; rows and codes of one KV head whose head dimension was moved: all are contiguous
    where there is more than one of something."""
    heads, B, T, block = "gqa28", 3, 40, 16
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, 48)
    qkv = torch.randn((B, 1, H + 2 * hkv, d), device=DEV).bfloat16()
    k, v = qkv[:, :, H:H + hkv], qkv[:, :, H + hkv:]
    results = []
    for rows in ((k, v), (k.clone(memory_format=torch.contiguous_format), v.clone(memory_format=torch.contiguous_format))):
        keep, c = ctx.new_kv8(B, 48, block, "int8")
        ctx.kv8_write(c, B, T, *rows, start=17)
        results.append(keep)
    assert all(torch.equal(a, b) for a, b in zip(*results)) and int(results[0][2].max()) > 0

    heads, n = "mqa8", 5
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, 48)
    rows = torch.randn((B, 1, n, d), device=DEV).bfloat16().transpose(1, 2)
    results = []
    for r, moved in ((rows, True), (rows.clone(memory_format=torch.contiguous_format), False)):
        t = [torch.zeros((B, 48, 1, d), dtype=torch.uint8, device=DEV).transpose(1, 2) if moved else torch.zeros((B, 1, 48, d), dtype=torch.uint8, device=DEV) for _ in range(2)]
        t += [torch.zeros((B, 1, 3), dtype=torch.uint8, device=DEV) for _ in range(2)]
        c = ab.Context.kv8(*t, block, 0)
        assert c.batch_stride == 48 * d
        ctx.kv8_write(c, B, T, r, r, start=3)
        results.append(t)
    assert all(torch.equal(a, b) for a, b in zip(*results)) and int(results[0][2].max()) > 0
    assert ctx.poll_status() == 0


def test_rows_that_do_lie_apart_are_refused():
    heads, B, T = "gqa28", 2, 40
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, 48)
    keep, c = ctx.new_kv8(B, 48, 16, "int8")
    for rows in (torch.zeros((B, 4, 2 * hkv, d), dtype=torch.bfloat16, device=DEV)[:, :, :hkv], torch.zeros((B, 1, hkv, 2 * d), dtype=torch.bfloat16, device=DEV)[..., :d],
                 torch.zeros((B, 1, hkv, d, 2), dtype=torch.bfloat16, device=DEV)[..., 0]):
        with pytest.raises(ValueError):
            ctx.kv8_write(c, B, T, rows, rows)
    codes, exps = torch.zeros((B, hkv, 96, d), dtype=torch.uint8, device=DEV)[:, :, :48], torch.zeros((B, hkv, 3), dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        ab.Context.kv8(codes, codes, exps, exps, 16, 0)
