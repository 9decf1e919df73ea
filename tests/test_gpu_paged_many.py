"""Attention over pages where its work is one line of units cut into equal pieces: items in many parts, requests whose lengths differ, each of the
row tiles; against 64 bits with the bounds of test_gpu_paged.py."""
import numpy as np
import pytest
import torch

from paper_2608_26140_b200 import binding as ab

from helpers import DEV
from test_gpu_paged import HEADS, check, context, pool_of, random, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,n,ctx_len,page", [("mqa8", 1, 100000, 16), ("mqa8", 4, 70001, 64), ("mqa8", 2, 65537, 4), ("gqa4-64", 3, 50000, 32), ("gqa4-64", 16, 33333, 128)])
def test_one_request_in_very_many_parts(heads, n, ctx_len, page):
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(ctx_len)
    k, v, table = pool_of(gen, heads, 1, ctx_len, page)
    q = random(gen, 1, n, H, d, std=1.5)
    o, lse = torch.empty_like(q), torch.empty((1, n, H), device=DEV)
    ctx = context(heads, 1)
    cache = ctx.paged_kv(k, v, table)
    for length in (ctx_len, ctx_len - 777, 63):
        lens = None if length == ctx_len else torch.tensor([length], dtype=torch.int32, device=DEV)
        ctx.paged_attention(cache, ctx_len, q, o, lse=lse, lens=lens)
        check(o, lse, reference(q, k, v, table, [np.arange(length)]))
        again = torch.empty_like(o)
        ctx.paged_attention(cache, ctx_len, q, again, lens=lens)
        assert torch.equal(o, again)
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("heads,batch,n,ctx_len,page", [("gqa28", 64, 1, 1500, 16), ("mqa8", 300, 2, 500, 32), ("gqa4-64", 90, 20, 700, 8), ("mha32", 7, 32, 900, 64), ("mha4-64", 150, 9, 400, 128)])
def test_requests_of_their_own_lengths(heads, batch, n, ctx_len, page):
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(batch)
    some = min(batch, 8)
    k, v, few = pool_of(gen, heads, some, ctx_len, page)
    table = few[torch.arange(batch, device=DEV) % some].contiguous()                     # (requests share pages)
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, ctx_len + 1, batch)
    lens[[0, 1, batch // 2, batch - 1]] = [ctx_len, 0, 1, 0]
    there = rng.random((batch, ctx_len)) < 0.7
    q = random(gen, batch, n, H, d)
    o, lse = torch.full_like(q, 7.0), torch.full((batch, n, H), 7.0, device=DEV)
    ctx = context(heads, batch)
    cache = ctx.paged_kv(k, v, table)
    on = torch.tensor(lens, dtype=torch.int32, device=DEV)
    looked_at = list(range(0, batch, max(1, batch // 12))) + [1, batch - 1]
    for drop in (False, True):
        ctx.paged_attention(cache, ctx_len, q, o, lse=lse, lens=on, key_drop=ctx.pack_key_drop(torch.as_tensor(~there, device=DEV)) if drop else None)
        keys = [np.flatnonzero(there[b, :lens[b]]) if drop else np.arange(lens[b]) for b in looked_at]
        at = torch.tensor(looked_at, device=DEV)
        check(o[at], lse[at], reference(q[at], k, v, table[at], keys))
    assert ctx.poll_status() == 0
    # what one request has does not depend on the others but for the order of sums
    alone_o, alone_lse = torch.empty_like(q[:1]), torch.empty_like(lse[:1])
    ctx.paged_attention(ctx.paged_kv(k, v, table[:1].contiguous()), ctx_len, q[:1].contiguous(), alone_o, lse=alone_lse, lens=on[:1].contiguous())
    check(alone_o, alone_lse, reference(q[:1], k, v, table[:1], [np.arange(lens[0])]))


def test_a_page_that_is_none_in_one_of_many_requests():
    heads, batch, ctx_len, page = "gqa28", 64, 1500, 16
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(3)
    k, v, few = pool_of(gen, heads, 4, ctx_len, page)
    table = few[torch.arange(batch, device=DEV) % 4].contiguous()
    table[9, 5], table[9, 6], table[30, 0] = -1, k.shape[0], 1 << 30
    lens = torch.full((batch,), ctx_len, dtype=torch.int32, device=DEV)
    lens[5], lens[6] = -4, ctx_len + 1
    q = random(gen, batch, 1, H, d)
    o, lse = torch.empty_like(q), torch.empty((batch, 1, H), device=DEV)
    ctx = context(heads, batch)
    ctx.paged_attention(ctx.paged_kv(k, v, table), ctx_len, q, o, lse=lse, lens=lens)
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX
    every = np.arange(ctx_len)
    at = torch.tensor([5, 6, 9, 30], device=DEV)
    good = few[at % 4]
    check(o[at], lse[at], reference(q[at], k, v, good, [[], every, every[(every < 80) | (every >= 112)], every[16:]]))


def test_more_work_than_a_call_takes_is_refused():
    heads = "gqa4-64"
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(4)
    k, v, _ = pool_of(gen, heads, 1, 1024, 1024)
    table = torch.zeros((64, 1 << 20), dtype=torch.int32, device=DEV)
    ctx = context(heads, 64)
    q = random(gen, 64, 17, H, d)
    launches = ctx.launch_count()
    with pytest.raises(ab.AcacheError) as e:                  # 2^24 units x 2 tiles x 2 KV heads x 64 requests
        ctx.paged_attention(ctx.paged_kv(k, v, table), 1 << 30, q, torch.empty_like(q))
    assert e.value.status == ab.ERR_UNSUPPORTED_SHAPE and ctx.launch_count() == launches


@pytest.mark.parametrize("heads,batch,n,ctx_len,page", [("mha32", 20, 1, 1500, 64), ("mha32", 12, 24, 1301, 16), ("mha4-64", 90, 20, 2001, 128), ("gqa4-64", 200, 12, 1100, 4), ("mha32", 9, 30, 640, 32)])
@pytest.mark.parametrize("how", ["two long", "one long, last", "all short", "all empty"])
def test_short_requests_between_long_ones(heads, batch, n, ctx_len, page, how):
    """Pieces that hold many items, and pieces that begin behind an item's last key; a request of none too."""
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(batch * 3 + n)
    k, v, few = pool_of(gen, heads, 4, ctx_len, page)
    table = few[torch.arange(batch, device=DEV) % 4].contiguous()
    lens = np.array([(1, 40, 64, 130, 0, 65)[b % 6] for b in range(batch)])
    if how == "two long":
        lens[[2, batch // 2]] = ctx_len, ctx_len - 3
    elif how == "one long, last":
        lens[-1] = ctx_len
    elif how == "all empty":
        lens[:] = 0
    q = random(gen, batch, n, H, d)
    o, lse = torch.full_like(q, 7.0), torch.full((batch, n, H), 7.0, device=DEV)
    ctx = context(heads, batch)
    ctx.paged_attention(ctx.paged_kv(k, v, table), ctx_len, q, o, lse=lse, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    looked_at = sorted({0, 1, 2, 3, 4, 5, batch // 2, batch - 2, batch - 1})
    at = torch.tensor(looked_at, device=DEV)
    check(o[at], lse[at], reference(q[at], k, v, table[at], [np.arange(lens[b]) for b in looked_at]))
    assert ctx.poll_status() == 0
    empty = torch.tensor(lens == 0, device=DEV)
    assert torch.equal(o[empty], torch.zeros_like(o[empty])) and torch.isneginf(lse[empty]).all()
    assert torch.isfinite(lse[~empty]).all() and torch.isfinite(o).all()
