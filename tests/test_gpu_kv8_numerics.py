"""Attention over the 8-bit cache where its arithmetic is stretched, against 64 bits and within the bound of test_gpu_kv8.py:
one key far ahead of thousands that matter, logits that keep rising, value scales at the ends of what is allowed."""
import math

import pytest
import torch

from paper_2608_26140_b200 import binding as ab

from helpers import DEV
from test_gpu_kv8 import HEADS, check_attention, context, filled, queries, ref_attention

pytestmark = pytest.mark.gpu

# one token, a decode block, many rows (tensor memory: one row tile, two); keys in splits and whole; head dimension 64
FORMS = [("mha32", 1, 1, 16384), ("mha32", 12, 1, 4096), ("mha32", 8, 32, 2560), ("gqa28", 1, 4, 8192),
         ("mha32", 5, 140, 8288), ("gqa28", 4, 18, 8200), ("mha4-64", 3, 40, 3000)]


def along(heads, B, T, seed):
    """Directions u [Hkv, d] of +-1, rows k [B, T, Hkv, d] = u (to be scaled), a generator."""
    H, hkv, d = HEADS[heads]
    g = torch.Generator(device=DEV).manual_seed(seed)
    u = torch.where(torch.rand((hkv, d), generator=g, device=DEV) < 0.5, -1.0, 1.0)
    return u, u.expand(B, T, hkv, d), g


def held(ctx, heads, B, T, k, v, block, fmt):
    """A cache with these rows, and the values it stands for."""
    keep, c = ctx.new_kv8(B, T, block, fmt)
    ctx.kv8_write(c, B, T, k.bfloat16().contiguous(), v.bfloat16().contiguous())
    out = [torch.empty_like(k, dtype=torch.bfloat16) for _ in range(2)]
    ctx.kv8_read(c, B, T, *out)
    return keep, c, [t.double().transpose(1, 2).contiguous() for t in out]


def queries_along(heads, B, n, u):
    """Rows along u, at full and at three quarters of its length."""
    H, hkv, d = HEADS[heads]
    size = torch.where(torch.arange(n, device=DEV) % 2 == 0, 1.0, 0.75).view(1, n, 1, 1)
    return (u.repeat_interleave(H // hkv, 0) * size).expand(B, n, H, d).bfloat16().contiguous()


@pytest.mark.parametrize("spread", [0.0, 1.0])
@pytest.mark.parametrize("nats", [8.0, 12.0, 14.6, 16.0])
@pytest.mark.parametrize("heads,B,n,T", FORMS)
def test_a_first_key_far_ahead_of_the_others(heads, B, n, T, nats, spread):
    """The first token is attended most and says little; what the others say has a common mean.  16 nats are 2^23.1: the others'
    probabilities are 2^-15.1 when the largest is 2^8, an f16 step there is 2^-24, so each is off by at most 2^-9.9 of itself; with the
    logits' share (X is about 20) 2^-9.5 A of the bound's 2^-9 A."""
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, T)
    for block, fmt in ((16, "int8"), (64, "e4m3")):
        u, k, g = along(heads, B, T, int(nats) + n)
        at = 0.25 + spread * torch.randn((B, T, hkv, 1), generator=g, device=DEV) / math.sqrt(d)
        at[:, 0] = 0.25 + nats / math.sqrt(d)
        v = 1.0 + 0.25 * torch.randn((B, T, hkv, d), generator=g, device=DEV)
        v[:, 0] = 0.05 * torch.randn((B, hkv, d), generator=g, device=DEV)
        keep, c, vals = held(ctx, heads, B, T, k * at, v, block, fmt)
        check_attention(ctx, None, vals, B, n, T, heads, queries_along(heads, B, n, u), c=c)
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("heads,B,n,T", FORMS)
def test_logits_that_keep_rising(heads, B, n, T):
    """From -30 to 30 nats along the keys, and in steps that pass the reference by a little: it moves all the time."""
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, T)
    for stairs in (1, 40):
        u, k, g = along(heads, B, T, n)
        at = torch.linspace(-30.0, 30.0, T, device=DEV).view(1, T, 1, 1) / math.sqrt(d)
        at = (at * stairs).round() / stairs if stairs > 1 else at
        at = at + 0.05 * torch.randn((B, T, hkv, 1), generator=g, device=DEV) / math.sqrt(d)
        v = 1.0 + 0.25 * torch.randn((B, T, hkv, d), generator=g, device=DEV)
        keep, c, vals = held(ctx, heads, B, T, k * at, v, 64, "int8")
        check_attention(ctx, None, vals, B, n, T, heads, queries_along(heads, B, n, u), c=c)
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("first,others,c_first", [
    (177, 77, -55), (177, 77, -67),              # the others' values 2^100 smaller, their weights 2^106 and 2^118 larger
    (77, 177, 55), (16, 16, 42), (16, 116, 49), (247, 247, 42), (247, 147, -55)])
@pytest.mark.parametrize("n,T", [(1, 65536), (32, 65536), (140, 24576)])
def test_scales_of_values_at_the_ends_of_what_is_allowed(n, T, first, others, c_first):
    """The first 128 keys (one step of every warp, one key tile) and all others, each kind with logits and a scale of its own: denominators run from the smallest to the largest
    that there can be, results from 2^-104 to 2^127.  As many items as leave the keys whole."""
    heads, B, block = "mha32", 9, 16
    H, hkv, d = HEADS[heads]
    ctx = ab.Context(128, H, hkv, d, 128, 1e-5, 0, B, T, 0, 1, 0, DEV)
    g = torch.Generator(device=DEV).manual_seed(n)
    u = torch.where(torch.rand((d,), generator=g, device=DEV) < 0.5, -1, 1)
    c = torch.full((T,), 49, device=DEV)
    c[:128] = c_first
    k = (c[:, None] * u).to(torch.int8).view(torch.uint8).expand(B, hkv, T, d).contiguous()
    v = torch.randint(64, 127, (1, hkv, T, d), generator=g, device=DEV, dtype=torch.uint8).expand(B, hkv, T, d).contiguous()
    ke = torch.full((B, hkv, T // block), 123, dtype=torch.uint8, device=DEV)      # a logit is c / sqrt(2)
    ve = torch.full((B, hkv, T // block), others, dtype=torch.uint8, device=DEV)
    ve[:, :, :128 // block] = first
    cache = ab.Context.kv8(k, v, ke, ve, block, ab.KV8_FORMATS["int8"])
    q = u.expand(B, n, H, d).bfloat16().contiguous()
    o, lse = torch.empty_like(q), torch.empty((B, n, H), dtype=torch.float32, device=DEV)
    ctx.kv8_attention(cache, B, T, q, o, lse=lse)
    for b, h in ((0, 0), (4, 17), (8, 31)):
        K, V = (t[b, h].view(torch.int8).double() * torch.exp2(e[b, h].double() - 127).repeat_interleave(block)[:, None] for t, e in ((k, ke), (v, ve)))
        ro, rl, A, X = ref_attention(q[b, :1, h:h + 1].double(), K[None], V[None], torch.ones(T, dtype=torch.bool, device=DEV))
        assert float(X.max()) < 64
        assert ((o[b, :, h].double() - ro[:, 0]).abs() <= 2.0 ** -8 * ro[:, 0].abs() + 2.0 ** -9 * A[:, 0]).all()
        assert ((lse[b, :, h].double() - rl[:, 0]).abs() <= 2.0 ** -16 * X[:, 0] + 2.0 ** -18 * (1 + rl[:, 0].abs())).all()
    assert ctx.poll_status() == 0


PLACES = [("mha32", 1, 4096, 64), ("mha32", 1, 300, 16), ("mha32", 32, 1000, 64), ("gqa28", 29, 1531, 32), ("mha32", 140, 1500, 128),
          ("mha4-64", 40, 700, 16)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads,n,T,block", PLACES)
def test_exponents_of_places_that_do_not_count(heads, n, T, block, fmt):
    """Blocks none of whose keys exists, and blocks past a request's length, with exponents of any kind: of no account."""
    B = 4
    ctx = context(heads, B, T)
    cache, vals = filled(heads, B, T, block, fmt, n + T)
    blocks = -(-T // block)
    g = torch.Generator(device=DEV).manual_seed(3)
    gone = torch.rand((B, blocks), generator=g, device=DEV) < 0.3
    gone[0, 0], gone[1, :blocks // 2], gone[2, -1], gone[3] = True, True, True, True
    gone[3, blocks // 3] = False
    drop = (torch.rand((B, T), generator=g, device=DEV) < 0.2) | gone.repeat_interleave(block, 1)[:, :T]
    lens = [T, T, T // 2 + 3, T]
    past = torch.arange(blocks, device=DEV)[None] * block >= torch.tensor(lens, device=DEV)[:, None]
    odd = torch.tensor([247, 16, 255, 1, 254, 0], dtype=torch.uint8, device=DEV)
    for e in cache.dev[2:]:
        e[:, :, :blocks] = torch.where((gone | past)[:, None], odd[torch.randint(0, 6, (B, e.shape[1], blocks), generator=g, device=DEV)], e[:, :, :blocks])
    q = queries(B, n, heads, 5)
    check_attention(ctx, cache, vals, B, n, T, heads, q, lens=lens, drop=drop)
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads,n,T,block", PLACES)
def test_blocks_that_hold_nothing_have_no_scale(heads, n, T, block, fmt):
    """Empty blocks in front, behind and between; the values of the others, up to 2^-95, lie near the lowest exponent."""
    B = 2
    ctx = context(heads, B, T)
    blocks = -(-T // block)
    holes = [i for i in range(blocks) if i < blocks // 3 or i % 5 == 4]
    cache, vals = filled(heads, B, T, block, fmt, n + T, holes=holes)
    e = cache.dev[3]
    e.copy_(torch.where(e > 0, e - 100, e))
    assert int(e[e > 0].min()) >= 16
    vals[1] *= 2.0 ** -100
    check_attention(ctx, cache, vals, B, n, T, heads, queries(B, n, heads, 5))
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("heads,n,T,block", PLACES)
def test_sharp_logits_over_scales_far_apart_to_the_bound_that_is_stated(heads, n, T, block):
    """Queries along one key, value blocks 2^30 and more apart: the key that softmax prefers may be small beside another's p times scale.
    To the usual bound come 2^-33 of the row's largest product of a probability and a scale, for every code of a column."""
    B = 2
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, T)
    cache, vals = filled(heads, B, T, block, "int8", n + T, v_spread=8.0)
    for at, nats in ((T // 2, 9.0), (T - 1, 25.0)):
        k = vals[0][:, :, at].repeat_interleave(H // hkv, 1)
        q = (k / (k ** 2).sum(-1, keepdim=True) * nats * math.sqrt(d))[:, None].expand(B, n, H, d).bfloat16().contiguous()
        o = torch.empty_like(q)
        ctx.kv8_attention(cache.c, B, T, q, o)
        for b in range(B):
            ro, _, A, X = ref_attention(q[b].double(), vals[0][b], vals[1][b], torch.ones(T, dtype=torch.bool, device=DEV))
            assert float(X.max()) < 64
            scale = torch.exp2(cache.dev[3][b].double() - 127).repeat_interleave(block, 1)[:, :T]
            codes = (vals[1][b].abs() / scale[..., None]).sum(1)
            for h in range(H):
                p = torch.softmax(q[b, :, h].double() @ vals[0][b, h // (H // hkv)].T / math.sqrt(d), 1)
                lost = 2.0 ** -33 * (p * scale[h // (H // hkv)]).amax(1)[:, None] * codes[h // (H // hkv)]
                assert ((o[b, :, h].double() - ro[:, h]).abs() <= 2.0 ** -8 * ro[:, h].abs() + 2.0 ** -9 * A[:, h] + lost).all()
    assert ctx.poll_status() == 0
