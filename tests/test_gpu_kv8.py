"""The 8-bit cache (acache_kv8_write, acache_kv8_read, acache_kv8_attention, acache_layer_step_kv8) against plain
implementations in 64 bits written from the definitions in the header.

Codes, exponents and read-back values are defined to the bit.  Attention is held to a bound per element:

    |o - ref| <= 2^-8 |ref| + 2^-9 A,   A = sum_j p_j |V_j|

(half a bf16 step of the result, 2^-9 |ref|, doubled for results at a step's edge; f16 probabilities, 2^-12 A; logits off by
up to 2^-16 X, X = max_j sum_i |q_i k_ij| / sqrt(d), which moves a probability by that share: X is kept below 64, so 2^-10 A)

    |lse - ref| <= 2^-16 X + 2^-18 (1 + |ref|)

(sums of 128 products in fp32, 128 * 2^-24 of the sum of their sizes at worst; the sums of exponentials and the logarithm.)
"""
import math

import numpy as np
import pytest
import torch

from oracle import acache_oracle as orc
from paper_2608_26140_b200 import binding as ab
from paper_2608_26140_b200 import workloads as wl

from helpers import DEV, DeviceCase, assert_close_bf16
from launched_kv8 import launched_kv8

pytestmark = pytest.mark.gpu

TOP = {"int8": 6, "e4m3": 7}
HEADS = {"mha4-64": (4, 4, 64), "gqa4-64": (4, 2, 64), "gqa28": (28, 4, 128), "mha32": (32, 32, 128), "mqa8": (8, 1, 128)}


def context(heads, batch, max_ctx):
    H, hkv, d = HEADS[heads]
    hidden = max(hkv * d, 128)
    return ab.Context(hidden, H, hkv, d, 128, 1e-5, 0, batch, max_ctx, 0, 1, 0, DEV)


# --------------------------------------------------------------------------
# the definitions, in 64 bits on the host
# --------------------------------------------------------------------------
def e4m3_table():
    t = np.zeros(256)
    for c in range(256):
        s, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        t[c] = s * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    t[0x7F] = t[0xFF] = np.nan
    return t


E4M3 = e4m3_table()


def values_of(codes, fmt):
    return E4M3[codes] if fmt == "e4m3" else codes.view(np.int8).astype(np.float64)


def scale_of(e):
    return np.where(e == 0, 0.0, np.exp2(e.astype(np.float64) - 127))


def round_codes(x, fmt, limit=448.0):
    """fp64 values in scales -> code bytes."""
    if fmt == "int8":
        return np.clip(np.rint(np.nan_to_num(x, nan=0.0, posinf=127, neginf=-127)), -127, 127).astype(np.int8).view(np.uint8)
    finite = np.isfinite(x)
    y = np.clip(np.where(finite, x, 0.0), -limit, limit)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    y = np.abs(np.rint(y / step) * step)
    codes = np.searchsorted(E4M3[:127], y).astype(np.uint8)
    assert np.array_equal(E4M3[codes], y)
    sign = np.signbit(x)
    return np.where(finite, codes | (sign.astype(np.uint8) << 7), np.uint8(0x7F)).astype(np.uint8)


def ref_write(codes, exps, rows, pos, ctx_len, block, fmt):
    """One request, K or V: codes [Hkv, cap, d], exps [Hkv, blocks] in place; rows [n, Hkv, d] fp64."""
    row_of = {}
    for i, p in enumerate(pos):
        if 0 <= p < ctx_len:
            row_of[int(p)] = i
    for blk in sorted({p // block for p in row_of}):
        here = np.arange(blk * block, (blk + 1) * block)
        new = [p for p in here if p in row_of]
        kept = [p for p in here if p not in row_of and p < ctx_len]
        for h in range(codes.shape[0]):
            x = rows[[row_of[p] for p in new], h]
            fin = np.abs(x[np.isfinite(x)])
            amax = fin.max() if fin.size else 0.0
            odd = fin.size < x.size
            field = 0 if amax < 2.0 ** -126 else int(np.floor(np.log2(amax))) + 127
            e = 0 if field == 0 and not odd else min(max(field - TOP[fmt], 16), 254)
            e_old = int(exps[h, blk]) if kept else 0
            e = max(e, e_old)
            if kept and e != e_old:
                old = values_of(codes[h, kept], fmt) * (2.0 ** (e_old - e) if e_old else 0.0)
                codes[h, kept] = round_codes(old, fmt) if e_old else 0
            if kept and e_old == 0:
                codes[h, kept] = 0
            limit = 240.0 if field == 254 else 448.0
            codes[h, new] = round_codes(x * 2.0 ** (127 - e), fmt, limit) if e else 0
            codes[h, [p for p in here if p >= ctx_len]] = 0
            exps[h, blk] = e


def ref_values(codes, exps, block, fmt):
    """codes [..., cap, d], exps [..., blocks] -> fp64 [..., cap, d]."""
    s = np.repeat(scale_of(exps), block, axis=-1)[..., None]
    return np.where(s == 0, 0.0, values_of(codes, fmt) * s)


class Cache:
    """An 8-bit cache on the device and its reference on the host."""

    def __init__(self, heads, batch, cap, block, fmt, garbage=False):
        H, hkv, d = HEADS[heads]
        self.block, self.fmt, self.cap = block, fmt, cap
        self.ref = [np.zeros((batch, hkv, cap, d), np.uint8) for _ in range(2)] + [np.zeros((batch, hkv, cap // block), np.uint8) for _ in range(2)]
        if garbage:                              # codes of blocks that hold nothing may be anything, NaN among it
            for c in self.ref[:2]:
                c[:] = np.random.default_rng(3).integers(0, 256, c.shape, dtype=np.uint8)
        self.dev = [torch.from_numpy(a.copy()).to(DEV) for a in self.ref]
        self.c = ab.Context.kv8(*self.dev, block, ab.KV8_FORMATS[fmt])

    def write_ref(self, k, v, pos, ctx_len):
        for b in range(k.shape[0]):
            ref_write(self.ref[0][b], self.ref[2][b], k[b], pos[b], ctx_len, self.block, self.fmt)
            ref_write(self.ref[1][b], self.ref[3][b], v[b], pos[b], ctx_len, self.block, self.fmt)

    def check(self):
        torch.cuda.synchronize()
        for name, a, b in zip(("k", "v", "k_exp", "v_exp"), self.ref, self.dev):
            got = b.cpu().numpy()
            if self.fmt == "e4m3" and name in "kv":       # a NaN is a NaN, 0 and -0 differ
                a, got = np.where((a & 127) == 127, 127, a), np.where((got & 127) == 127, 127, got)
            assert np.array_equal(a, got), (name, np.argwhere(a != got)[:4])

    def values(self):
        return [ref_values(self.ref[i], self.ref[i + 2], self.block, self.fmt) for i in range(2)]


def bf16(a):
    """fp64/fp32 array -> (device bf16 tensor, its exact fp64 values)."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)
    return t.to(DEV), t.double().numpy()


def draw_rows(rng, B, n, heads, spread=1.0):
    H, hkv, d = HEADS[heads]
    x = rng.standard_normal((B, n, hkv, d)) * np.exp(spread * rng.standard_normal((B, n, 1, 1)))
    return bf16(x)


# --------------------------------------------------------------------------
# writing and reading
# --------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads,block", [("mha4-64", 16), ("gqa4-64", 128), ("gqa28", 32), ("mha32", 64), ("mqa8", 128), ("gqa28", 16)])
def test_write_and_read_to_the_bit(heads, block, fmt):
    B, T = 2, 3 * block + 5
    cap = 5 * block
    ctx, cache = context(heads, B, cap), Cache(heads, B, cap, block, fmt, garbage=True)
    rng = np.random.default_rng(block)
    H, hkv, d = HEADS[heads]
    steps = [("span", 0, T, T, 1.0), ("span", T, 1, T + 1, 1.0),                  # all of it; one token more
             ("list", 0, 7, T + 1, 2.5), ("list", 0, block + 3, T + 1, 0.1),      # rows that make blocks grow; rows that do not
             ("span", block, block, T + 1, 0.0), ("span", block // 2, block, 2 * block, 1.0)]
    for how, start, n, ctx_len, spread in steps:
        (k, k64), (v, v64) = draw_rows(rng, B, n, heads, spread), draw_rows(rng, B, n, heads, spread)
        before = [a.copy() for a in cache.ref]
        if how == "span":
            pos = np.tile(np.arange(start, start + n), (B, 1))
            ctx.kv8_write(cache.c, B, ctx_len, k, v, start=start)
        else:
            pos = np.stack([rng.permutation(ctx_len)[:n] for _ in range(B)])
            ctx.kv8_write(cache.c, B, ctx_len, k, v, pos=torch.from_numpy(pos.astype(np.int32)).to(DEV))
        cache.write_ref(k64, v64, pos, ctx_len)
        cache.check()
        # rows that stay in blocks whose exponent stays keep their codes bit for bit
        for b in range(B):
            stay = np.setdiff1d(np.arange(ctx_len), pos[b])
            for i in range(2):
                same = np.repeat(before[2 + i][b] == cache.ref[2 + i][b], block, axis=-1)[:, stay] & (np.repeat(before[2 + i][b], block, axis=-1)[:, stay] > 0)
                assert np.array_equal(before[i][b][:, stay][same], cache.ref[i][b][:, stay][same])
        # read back: a span and a list, both and one
        kv = cache.values()
        ko, vo = (torch.full((B, ctx_len, hkv, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ctx.kv8_read(cache.c, B, ctx_len, ko, vo)
        for t, ref in zip((ko, vo), kv):
            assert np.array_equal(t.double().cpu().numpy(), ref[:, :, :ctx_len].transpose(0, 2, 1, 3))
        m = min(ctx_len, 9)
        p = np.stack([rng.integers(0, ctx_len, m) for _ in range(B)]).astype(np.int32)
        ko = torch.full((B, m, hkv, d), 7.0, dtype=torch.bfloat16, device=DEV)
        ctx.kv8_read(cache.c, B, ctx_len, ko, None, pos=torch.from_numpy(p).to(DEV))
        for b in range(B):
            assert np.array_equal(ko[b].double().cpu().numpy(), kv[0][b][:, p[b]].transpose(1, 0, 2))
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_write_of_odd_values(fmt):
    """Zeros, subnormal and huge numbers, the top of bf16's range, ties, infinities and NaN."""
    heads, block, B = "mha4-64", 16, 1
    H, hkv, d = HEADS[heads]
    cap = 12 * block
    ctx, cache = context(heads, B, cap), Cache(heads, B, cap, block, fmt)
    x = np.random.default_rng(0).standard_normal((B, cap, hkv, d))
    big = float(torch.finfo(torch.bfloat16).max)
    x[:, 0:16] = 0.0
    x[:, 16:32] *= 1e-39                         # below the normal numbers: the block is empty
    x[:, 32:48] *= 1e-36                         # at the lowest exponent
    x[:, 48:64] = np.clip(x[:, 48:64] * big, -big, big)
    x[:, 64:80] = 0.0
    x[:, 64, :, 0] = 1.0                         # ties: 1 is 64 (int8) or 128 (e4m3) steps of its block
    x[:, 65, :, :] = (np.arange(d) + 0.5) / 64
    x[:, 66, :, :] = -(np.arange(d) + 0.5) / 128
    x[:, 80:96] = big
    finite, finite64 = bf16(x)
    pos = np.arange(cap)[None]
    ctx.kv8_write(cache.c, B, cap, finite, finite)
    cache.write_ref(finite64, finite64, pos, cap)
    cache.check()
    assert ctx.poll_status() == 0
    out = torch.empty((B, cap, hkv, d), dtype=torch.bfloat16, device=DEV)
    ctx.kv8_read(cache.c, B, cap, out, None)
    back = out.double().cpu().numpy()
    assert np.isfinite(back).all()               # what was finite stays so
    assert np.array_equal(back, cache.values()[0].transpose(0, 2, 1, 3))
    x[:, 100] = np.inf
    x[:, 101, 1, 3] = -np.inf
    x[:, 117, 2, :] = np.nan
    x[:, 128:144] = np.nan                       # a block of nothing else
    x[:, 144:160] = 0.0
    x[:, 150, 0, 0] = np.inf
    odd, odd64 = bf16(x)
    ctx.kv8_write(cache.c, B, cap, odd, finite)
    cache.write_ref(odd64, finite64, pos, cap)
    cache.check()
    assert ctx.poll_status() == ab.FLAG_NONFINITE
    ctx.kv8_read(cache.c, B, cap, out, None)
    back = out.double().cpu().numpy()
    if fmt == "e4m3":
        assert np.array_equal(np.isnan(back), ~np.isfinite(odd64)) and not np.isinf(back).any()
    else:
        assert np.isfinite(back).all() and (back[0, 117, 2] == 0).all()


@pytest.mark.parametrize("n", [3, 40, 200])      # fewer rows than blocks, and more
def test_write_list_with_bad_and_double_positions(n):
    heads, block, B, fmt = "gqa28", 16, 3, "int8"
    H, hkv, d = HEADS[heads]
    T, cap = 187, 192
    ctx, cache = context(heads, B, cap), Cache(heads, B, cap, block, fmt)
    rng = np.random.default_rng(n)
    pos = rng.integers(0, T, (B, n))
    pos[0, n // 2], pos[1, 0], pos[2, n - 1], pos[2, 0] = -1, T, pos[2, 0], 2 ** 30
    (k, k64), (v, v64) = draw_rows(rng, B, n, heads), draw_rows(rng, B, n, heads)
    ctx.kv8_write(cache.c, B, T, k, v, pos=torch.from_numpy(pos.astype(np.int32)).to(DEV))
    cache.write_ref(k64, v64, pos, T)
    cache.check()
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX
    out = torch.full((B, n, hkv, d), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.kv8_read(cache.c, B, T, None, out, pos=torch.from_numpy(pos.astype(np.int32)).to(DEV))
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX
    bad = (pos < 0) | (pos >= T)
    got, ref = out.double().cpu().numpy(), cache.values()[1]
    for b in range(B):
        assert (got[b, bad[b]] == 0).all()
        assert np.array_equal(got[b, ~bad[b]], ref[b][:, pos[b][~bad[b]]].transpose(1, 0, 2))


def test_write_from_a_bf16_cache_and_of_shared_rows():
    """Rows of an ordinary cache (requests further apart than the rows), and the same rows for every request."""
    heads, block, B, fmt, T = "gqa28", 64, 3, "e4m3", 130
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, 256)
    rng = np.random.default_rng(5)
    (k, k64), (v, v64) = draw_rows(rng, B, 200, heads), draw_rows(rng, B, 200, heads)
    cache = Cache(heads, B, 256, block, fmt)
    ctx.kv8_write(cache.c, B, T, k[:, :T], v[:, :T])
    cache.write_ref(k64[:, :T], v64[:, :T], np.tile(np.arange(T), (B, 1)), T)
    cache.check()
    cache = Cache(heads, B, 256, block, fmt)
    ctx.kv8_write(cache.c, B, T, k[:1, :T].expand(B, T, hkv, d), v[1:2, :T].expand(B, T, hkv, d))
    cache.write_ref(np.repeat(k64[:1, :T], B, 0), np.repeat(v64[1:2, :T], B, 0), np.tile(np.arange(T), (B, 1)), T)
    cache.check()
    # nothing to do
    ctx.kv8_write(cache.c, B, T, k[:, :0], v[:, :0])
    ctx.kv8_write(cache.c, 0, T, k[:0, :T], v[:0, :T])
    cache.check()
    assert ctx.poll_status() == 0


# --------------------------------------------------------------------------
# attention
# --------------------------------------------------------------------------
def filled(heads, B, T, block, fmt, seed, k_scale=1.0, v_spread=0.5, holes=()):
    """A cache of T tokens and its values [B, Hkv, T, d]; holes: blocks that hold nothing, over garbage codes."""
    H, hkv, d = HEADS[heads]
    cap = -(-T // block) * block + block
    cache = Cache(heads, B, cap, block, fmt, garbage=True)
    g = torch.Generator(device=DEV).manual_seed(seed)
    spread = torch.exp(v_spread * torch.randn((B, hkv, cap // block, 1, 1), generator=g, device=DEV))
    for i in range(2):
        x = torch.randn((B, hkv, cap // block, block, d), generator=g, device=DEV) * (k_scale if i == 0 else spread)
        e = (torch.floor(torch.log2(x.abs().amax((3, 4)))) + 127 - TOP[fmt]).to(torch.int32)
        y = x * torch.exp2((127 - e).float())[..., None, None]
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8) if fmt == "e4m3" else y.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
        keep = torch.ones((cap // block,), dtype=torch.bool, device=DEV)
        for hole in holes:
            keep[hole] = False
        codes = torch.where(keep[None, None, :, None, None], codes, cache.dev[i].view(B, hkv, -1, block, d))
        cache.dev[i].copy_(codes.view(B, hkv, cap, d))
        cache.dev[2 + i].copy_(torch.where(keep, e, 0).to(torch.uint8))
    vals = []
    for i in range(2):
        c = cache.dev[i].view(torch.float8_e4m3fn if fmt == "e4m3" else torch.int8).double().view(B, hkv, -1, block, d)
        e = cache.dev[2 + i].double()[..., None, None]
        vals.append(torch.where(e == 0, 0.0, c * torch.exp2(e - 127)).view(B, hkv, cap, d)[:, :, :T])
    return cache, vals


def ref_attention(q, K, V, there):
    """q [n, H, d], K, V [Hkv, T, d] (fp64, device), there [T] bool -> o, lse, A, X (per row and head)."""
    n, H, d = q.shape
    G = H // K.shape[0]
    o = torch.zeros((n, H, d), dtype=torch.float64, device=DEV)
    A, lse, X = torch.zeros_like(o), torch.full((n, H), -math.inf, dtype=torch.float64, device=DEV), torch.zeros((n, H), dtype=torch.float64, device=DEV)
    if there.any():
        for h in range(H):
            k, v = K[h // G][there], V[h // G][there]
            x = q[:, h] @ k.T / math.sqrt(d)
            lse[:, h] = torch.logsumexp(x, 1)
            p = torch.softmax(x, 1)
            o[:, h], A[:, h] = p @ v, p @ v.abs()
            X[:, h] = (q[:, h].abs() @ k.abs().T / math.sqrt(d)).amax(1)
    return o, lse, A, X


def check_attention(ctx, cache, vals, B, n, T, heads, q, lens=None, drop=None, shared=False, c=None):
    H, hkv, d = HEADS[heads]
    o = torch.full((B, n, H, d), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((B, n, H), 7.0, dtype=torch.float32, device=DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV) if lens is not None else None
    dd = ab.Context.pack_key_drop(drop) if drop is not None else None
    ctx.kv8_attention(c or cache.c, B, T, q, o, lse=lse, lens=dl, key_drop=dd)
    torch.cuda.synchronize()
    for b in range(B):
        there = torch.arange(T, device=DEV) < (lens[b] if lens is not None else T)
        if drop is not None:
            there &= ~drop[b]
        kb = 0 if shared else b
        ro, rl, A, X = ref_attention(q[b].double(), vals[0][kb], vals[1][kb], there)
        assert float(X.max()) < 64 if there.any() else True
        if not there.any():
            assert (o[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        off = (o[b].double() - ro).abs() - (2.0 ** -8 * ro.abs() + 2.0 ** -9 * A)
        assert float(off.max()) <= 0, (b, float(off.max()))
        off = (lse[b].double() - rl).abs() - (2.0 ** -16 * X + 2.0 ** -18 * (1 + rl.abs()))
        assert float(off.max()) <= 0, (b, float(off.max()))
    return o, lse


def queries(B, n, heads, seed, scale=1.2):
    H, hkv, d = HEADS[heads]
    g = torch.Generator(device=DEV).manual_seed(seed)
    # rows of very different size: every row is brought to f16 over its own power of two
    size = torch.exp2(torch.randint(-12, 1, (B, n, H, 1), generator=g, device=DEV).float())
    return (torch.randn((B, n, H, d), generator=g, device=DEV) * scale * size).bfloat16()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads,n,T,block", [
    ("gqa28", 1, 1, 16), ("gqa28", 1, 17, 16), ("mha32", 1, 128, 128), ("mha32", 1, 4097, 64), ("mqa8", 1, 333, 32),
    ("mha4-64", 1, 31, 16), ("mha4-64", 58, 256, 16), ("gqa4-64", 9, 1000, 128), ("gqa4-64", 300, 129, 64),
    ("mha32", 8, 640, 64), ("mha32", 9, 640, 64), ("mha32", 16, 127, 16), ("mha32", 17, 129, 16), ("mha32", 32, 1000, 64),
    ("mha32", 33, 255, 32), ("gqa28", 5, 700, 16), ("gqa28", 29, 385, 32), ("mha32", 103, 1024, 64), ("mha32", 128, 383, 128),
    ("mha32", 129, 383, 128), ("gqa28", 37, 511, 64), ("mqa8", 65, 1153, 16), ("mha32", 300, 640, 64)])
def test_attention(heads, n, T, block, fmt):
    B = 2
    ctx = context(heads, B, T)
    cache, vals = filled(heads, B, T, block, fmt, n + T)
    q = queries(B, n, heads, T)
    check_attention(ctx, cache, vals, B, n, T, heads, q)
    assert ctx.poll_status() == 0


MANY_ROWS = [
    ("mha32", 1, 33, 300, 64, "kv8_attn_rows"), ("gqa28", 1, 18, 8192, 64, "kv8_attn_rows"), ("mha32", 4, 33, 300, 64, "kv8_attn_tc"),
    ("mha32", 1, 100, 1600, 16, "kv8_attn_tc"), ("gqa28", 4, 18, 8200, 128, "kv8_attn_tc"), ("gqa28", 1, 64, 3000, 32, "kv8_attn_tc"),
    ("mqa8", 16, 20, 2100, 64, "kv8_attn_tc"), ("mha32", 8, 200, 257, 32, "kv8_attn_tc")]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads,B,n,T,block,kernel", MANY_ROWS)
def test_attention_of_many_rows(heads, B, n, T, block, kernel, fmt):
    """Both kernels around the place where the one takes over from the other; keys split over two to eight CTAs of a cluster and
    over several clusters; a request whose length leaves splits without keys."""
    ctx = context(heads, B, T)
    cache, vals = filled(heads, B, T, block, fmt, n + T, holes=(3,))
    q = queries(B, n, heads, T)
    check_attention(ctx, cache, vals, B, n, T, heads, q)
    check_attention(ctx, cache, vals, B, n, T, heads, q, lens=[T // 3] + [T - 1] * (B - 1))
    assert ctx.poll_status() == 0


def test_which_kernel_takes_how_many_rows():
    names = launched_kv8([(*HEADS[heads], B, n, T, block, "int8") for heads, B, n, T, block, _ in MANY_ROWS])
    for case, name in zip(MANY_ROWS, names):
        assert name.count("kernel") == 1 and case[-1] in name, (case, name)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads,n,T,block", [("gqa28", 1, 999, 16), ("mha4-64", 40, 300, 16), ("mha32", 32, 600, 64),
                                             ("gqa28", 29, 1531, 32), ("mha32", 150, 900, 128), ("mha32", 20, 130, 64)])
def test_attention_lengths_drops_and_holes(heads, n, T, block, fmt):
    """Lengths 0, 1 and at tile edges; keys that do not exist, whole tiles among them and whole requests; blocks that hold
    nothing; NaN and garbage in every place that does not count."""
    lens = [T, 0, 1, 128, 127, min(T, 257), T - 1, T, T]
    B = len(lens)
    ctx = context(heads, B, T)
    cache, vals = filled(heads, B, T, block, fmt, n, holes=(1, 2))
    for b, m in enumerate(lens):
        for i in range(2):
            cache.dev[i][b, :, m:] = 0x7F            # e4m3: NaN
    g = torch.Generator(device=DEV).manual_seed(7)
    drop = torch.rand((B, T), generator=g, device=DEV) < 0.3
    drop[0, :140] = True
    drop[6, :] = True                                # nothing left
    drop[7, :-1] = True                              # the last key alone
    for i in range(2):
        d_ = cache.dev[i][:, :, :T]
        d_[drop[:, None, :].expand(-1, d_.shape[1], -1)] = 0x7F
        vals[i] = torch.where((drop | (torch.arange(T, device=DEV)[None] >= torch.tensor(lens, device=DEV)[:, None]))[:, None, :, None], 0.0, vals[i])
    q = queries(B, n, heads, 5)
    check_attention(ctx, cache, vals, B, n, T, heads, q, lens=lens, drop=drop)

    assert ctx.poll_status() == 0


def test_attention_lengths_outside_the_context():
    heads, n, T = "gqa28", 3, 300
    ctx = context(heads, 2, T)
    cache, vals = filled(heads, 2, T, 32, "int8", 1)
    q = queries(2, n, heads, 5)
    o = torch.empty_like(q)
    ctx.kv8_attention(cache.c, 2, T, q, o, lens=torch.tensor([T + 1, -5], dtype=torch.int32, device=DEV))
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX
    want = torch.empty_like(q)
    ctx.kv8_attention(cache.c, 2, T, q, want, lens=torch.tensor([T, 0], dtype=torch.int32, device=DEV))
    assert torch.equal(o, want) and ctx.poll_status() == 0
    o.fill_(7.0)
    ctx.kv8_attention(cache.c, 2, 0, q, o)           # a context of no tokens
    torch.cuda.synchronize()
    assert (o == 0).all()


@pytest.mark.parametrize("heads,n", [("mha32", 1), ("gqa28", 32), ("mha32", 130)])
def test_attention_over_one_cache_for_the_batch(heads, n):
    B, T = 5, 700
    ctx = context(heads, B, T)
    cache, vals = filled(heads, 1, T, 64, "e4m3", 3)
    c = ab.Context.kv8(*cache.dev, 64, ab.KV8_FORMATS["e4m3"], shared=True)
    q = queries(B, n, heads, 1)
    check_attention(ctx, cache, vals, B, n, T, heads, q, shared=True, c=c)
    check_attention(ctx, cache, vals, B, n, T, heads, q, lens=[T, 0, 5, 400, 129], shared=True, c=c)
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("n", [1, 32, 140])
def test_attention_of_far_apart_scales_and_sharp_logits(n, fmt):
    """Value blocks 2^60 apart, whatever the order; keys whose logits differ by thousands: the softmax is one key's."""
    heads, T, B = "mha32", 1200, 1
    ctx = context(heads, B, T)
    cache, vals = filled(heads, B, T, 64, fmt, 2, v_spread=12.0)
    q = queries(B, n, heads, 9)
    check_attention(ctx, cache, vals, B, n, T, heads, q)
    # sharp: queries along one key's direction, the largest key of all
    cache, vals = filled(heads, B, T, 64, fmt, 4, k_scale=40.0)
    H, hkv, d = HEADS[heads]
    q = (vals[0][:, :, 777] * 20).float()[:, None].expand(B, n, H, d).bfloat16().contiguous()
    o = torch.empty_like(q)
    ctx.kv8_attention(cache.c, B, T, q, o)
    x = torch.einsum("bnhd,bhtd->bnht", q.double(), vals[0]) / math.sqrt(d)
    top2 = x.topk(2, dim=-1).values
    sure = (top2[..., 0] - top2[..., 1]) > 200       # the second key weighs less than 2^-280
    assert bool(sure.any())
    want = torch.gather(vals[1][:, None].expand(B, n, H, T, d), 3, x.argmax(-1)[..., None, None].expand(B, n, H, 1, d))[..., 0, :]
    assert torch.equal(o.double()[sure], want.bfloat16().double()[sure])
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("n", [1, 32, 140])
def test_attention_lets_nan_through_where_it_counts(n):
    """A NaN among the keys that count, or in a query, makes exactly the results NaN that depend on it."""
    heads, T, B, fmt = "gqa28", 500, 2, "e4m3"
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, T)
    cache, vals = filled(heads, B, T, 64, fmt, 2)
    q = queries(B, n, heads, 9)
    clean = torch.empty_like(q)
    ctx.kv8_attention(cache.c, B, T, q, clean)
    cache.dev[0][0, 1, 300, 5] = 0x7F                # a key of request 0, head 1
    cache.dev[1][1, 2, 10, 9] = 0x7F                 # one element of a value of request 1, head 2
    q2 = q.clone()
    q2[1, n - 1, 0, 3] = math.nan
    o = torch.empty_like(q)
    lse = torch.empty((B, n, H), dtype=torch.float32, device=DEV)
    ctx.kv8_attention(cache.c, B, T, q2, o, lse=lse)
    torch.cuda.synchronize()
    G = H // hkv
    want = torch.zeros_like(o, dtype=torch.bool)
    want[0, :, G:2 * G] = True
    want[1, :, 2 * G:3 * G, 9] = True
    want[1, n - 1, 0] = True
    assert torch.equal(torch.isnan(o), want)
    assert torch.equal(o[~want], clean[~want])
    want_lse = torch.zeros_like(lse, dtype=torch.bool)
    want_lse[0, :, G:2 * G] = True
    want_lse[1, n - 1, 0] = True
    assert torch.equal(torch.isnan(lse), want_lse)


def test_attention_of_a_long_cache():
    """Offsets past 2^31 bytes: the last request of a batch of long contexts."""
    heads, T, B = "mha32", 131072 + 77, 5
    H, hkv, d = HEADS[heads]
    ctx = ab.Context(128, H, hkv, d, 128, 1e-5, 0, B, T, 0, 1, 0, DEV)
    block = 64
    cap = -(-T // block) * block
    g = torch.Generator(device=DEV).manual_seed(1)
    codes = [torch.randint(0, 256, (B, hkv, cap, d), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
    assert codes[0].numel() > 2 ** 31
    exps = [torch.randint(118, 121, (B, hkv, cap // block), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
    c = ab.Context.kv8(*codes, *exps, block, ab.KV8_FORMATS["int8"])
    lens = [100, 0, 5, 70000, T]
    for n in (1, 40):
        q = (torch.randn((B, n, H, d), generator=g, device=DEV) * 0.2).bfloat16()
        o = torch.empty_like(q)
        lse = torch.empty((B, n, H), dtype=torch.float32, device=DEV)
        ctx.kv8_attention(c, B, T, q, o, lse=lse, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
        for b, h in ((4, 31), (4, 0), (3, 17)):
            m = lens[b]
            K, V = (codes[i][b, h, :m].view(torch.int8).double() * torch.exp2(exps[i][b, h].double() - 127).repeat_interleave(block)[:m, None] for i in range(2))
            ro, rl, A, X = ref_attention(q[b, :, h:h + 1].double(), K[None], V[None], torch.ones(m, dtype=torch.bool, device=DEV))
            assert float(X.max()) < 64
            assert ((o[b, :, h].double() - ro[:, 0]).abs() <= 2.0 ** -8 * ro[:, 0].abs() + 2.0 ** -9 * A[:, 0]).all()
            assert ((lse[b, :, h].double() - rl[:, 0]).abs() <= 2.0 ** -16 * X[:, 0] + 2.0 ** -18 * (1 + rl[:, 0].abs())).all()
        assert (o[1] == 0).all()
    # the last rows of the last request: written and read back
    rows = torch.randn((B, 77, hkv, d), generator=g, device=DEV).bfloat16()
    out = torch.empty_like(rows)
    ctx.kv8_write(c, B, T, rows, rows, start=T - 77)
    ctx.kv8_read(c, B, T, out, None, start=T - 77)
    torch.cuda.synchronize()
    amax = rows.float().abs().amax()
    assert float((out.float() - rows.float()).abs().max()) <= float(amax) / 64
    assert ctx.poll_status() == 0


def test_calls_on_another_stream_and_repeated_give_the_same_bits():
    heads, B, T = "gqa28", 3, 1111
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, T)
    rng = np.random.default_rng(1)
    (k, _), (v, _) = draw_rows(rng, B, T, heads), draw_rows(rng, B, T, heads)
    for n in (1, 29, 50):
        q = queries(B, n, heads, 2)
        results = []
        for s in (torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                keep, c = ctx.new_kv8(B, T, 64, "int8")
                o, lse = torch.empty_like(q), torch.empty((B, n, H), dtype=torch.float32, device=DEV)
                ctx.kv8_write(c, B, T, k, v)
                ctx.kv8_attention(c, B, T, q, o, lse=lse)
                ctx.kv8_attention(c, B, T, q, o, lse=lse)
            torch.cuda.synchronize()
            results.append((o, lse, *keep))
        for r in results[1:]:
            assert all(torch.equal(a, b) for a, b in zip(results[0], r))


# --------------------------------------------------------------------------
# the layer-step
# --------------------------------------------------------------------------
@pytest.mark.parametrize("shape,B,pre,L,post,gen,extra,ratio,block,fmt,flags", [
    (wl.TINY, 2, 8, 128, 40, 32, "all", 0.2, 16, "int8", 0),
    (wl.TINY_GQA, 2, 0, 130, 30, 32, "masked", 0.3, 64, "e4m3", 0),
    (wl.LayerShape(512, 8, 2, 128, 768, 1e-6, True, 1e6, "mid-gqa"), 3, 5, 300, 33, 40, "all", 0.15, 32, "int8", ab.F_SCORE_NORM_FULL),
    (wl.LayerShape(512, 4, 4, 128, 768, 1e-5, False, 5e5, "mid"), 2, 0, 256, 64, 32, "none", 0.25, 128, "e4m3", ab.F_DROP_NON_ANCHOR),
])
def test_layer_step(shape, B, pre, L, post, gen, extra, ratio, block, fmt, flags):
    """Against the oracle: its scores on the cache's values; its K/V of the recomputed rows, quantised as the header says
    (within what the projection's own rounding moves); its layer over the cache as the call left it."""
    lay = wl.make_layout(B, pre, L, post, gen, 32, extra)
    T, l = lay.ctx_len, lay.affix_start
    case = wl.make_case(shape, lay, ratio, 0)
    dc = DeviceCase(case)
    ctx, hkv, d = dc.ctx, shape.n_kv_heads, shape.head_dim
    keep, c = ctx.new_kv8(B, T, block, fmt)
    ctx.kv8_write(c, B, T, dc.ck[:, :T], dc.cv[:, :T])

    def held():
        k, v = (torch.empty((B, T, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ctx.kv8_read(c, B, T, k, v)
        return ab.to_host_bits(k), ab.to_host_bits(v)

    k0, v0 = held()
    old_exps = [t.cpu().numpy() for t in keep[2:]]
    K = orc.k_from_ratio(L, ratio)
    n = K + lay.n_extra
    scores = torch.zeros((B, L), dtype=torch.float32, device=DEV)
    anchors = torch.zeros((B, K), dtype=torch.int32, device=DEV)
    y = torch.zeros((B, n, shape.hidden), dtype=torch.bfloat16, device=DEV)
    ctx.layer_step_kv8(dc.lw, dc.req, c, dc.x, 0, ratio, ab.F_SCORE | ab.F_SELECT | flags, scores, anchors, y)
    assert ctx.poll_status() == 0
    k1, v1 = held()
    for b in range(B):
        a = anchors[b].cpu().numpy()
        first = orc.layer_step(case.weights, shape, case.x[b], k0[b], v0[b], T, l, L, lay.masked_pos[b], lay.extra_rows[b],
                               case.rope_cos, case.rope_sin, ratio=ratio, norm_full=bool(flags & ab.F_SCORE_NORM_FULL))
        ref = first["scores64"]
        assert np.abs(scores[b].cpu().numpy() - ref).max() <= 1e-3 * ref.max()
        ok, why = orc.anchor_set_ok(a, K, L, first["must"], first["may"])
        assert ok, why
        rows = orc.recompute_set(a, l, lay.extra_rows[b])
        x = orc.bf16_bits_to_f64(case.x[b])[rows]
        fresh = orc.recompute_rows(case.weights, shape, x, rows, k0[b], v0[b], T, case.rope_cos, case.rope_sin)
        stay = np.setdiff1d(np.arange(T), rows)
        for i, (got, before, new) in enumerate(((k1[b], k0[b], fresh["k_new"]), (v1[b], v0[b], fresh["v_new"]))):
            got, before, new = (orc.bf16_bits_to_f64(t) for t in (got, before, new))
            e = np.repeat(keep[2 + i][b].cpu().numpy(), block, axis=-1)[:, :T].T[..., None]      # [T, Hkv, 1]
            e_before = np.repeat(old_exps[i][b], block, axis=-1)[:, :T].T[..., None]
            s = scale_of(e)
            onto = lambda x, at: values_of(round_codes(x / s[at], fmt), fmt) * s[at]              # noqa: E731
            # rows that stay: to the bit on the scale that their block has now
            assert np.array_equal(got[stay], onto(before[stay], stay))
            assert (e >= e_before)[stay].all()
            # fresh rows: rounding keeps the order, so they lie between the roundings of what the projection may give
            off = 2e-2 * np.maximum(np.abs(new), np.sqrt((new ** 2).mean()))
            assert (got[rows] >= onto(new - off, rows)).all() and (got[rows] <= onto(new + off, rows)).all()
        # the layer's output: the oracle's queries over the cache as it is now
        keep_keys = orc.dropna_key_keep(T, l, L, a) if flags & ab.F_DROP_NON_ANCHOR else np.ones(T, bool)
        Kc, Vc = orc.bf16_bits_to_f64(k1[b]), orc.bf16_bits_to_f64(v1[b])
        o = np.zeros((n, shape.n_heads, d))
        for h in range(shape.n_heads):
            z = fresh["q"][:, h] @ Kc[:, h // (shape.n_heads // hkv)].T / math.sqrt(d)
            z[:, ~keep_keys] = -np.inf
            o[:, h] = orc.softmax_rows(z) @ Vc[:, h // (shape.n_heads // hkv)]
        w = lambda name: orc._w(case.weights, name)                                            # noqa: E731
        o = orc.bf16_round(o.reshape(n, -1))
        h1 = orc.bf16_round(x + o @ w("wo").T)
        xn2 = orc.bf16_round(orc.rmsnorm(h1, w("mlp_norm_g"), shape.rms_eps))
        act = orc.bf16_round(orc.silu(xn2 @ w("w_gate").T) * (xn2 @ w("w_up").T))
        assert_close_bf16(ab.to_host_bits(y[b]), orc.bf16_round(h1 + act @ w("w_down").T), f"y of request {b}")
    # the same step with the anchors given: the same rows, the same bits
    keep2, c2 = ctx.new_kv8(B, T, block, fmt)
    ctx.kv8_write(c2, B, T, dc.ck[:, :T], dc.cv[:, :T])
    y2 = torch.zeros_like(y)
    ctx.layer_step_kv8(dc.lw, dc.req, c2, dc.x, 0, ratio, flags & ab.F_DROP_NON_ANCHOR, None, anchors, y2)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and all(torch.equal(s, t) for s, t in zip(keep, keep2))


# --------------------------------------------------------------------------
# refusals
# --------------------------------------------------------------------------
@pytest.mark.parametrize("heads,n", [("gqa28", 1), ("mha4-64", 70), ("mha32", 150)])
def test_tensors_that_begin_at_16_bytes(heads, n):
    """Every tensor at an address that is a multiple of 16 bytes but not of 32: the same bits as at rounder addresses."""
    B, T, block = 2, 640, 32
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, T)

    def at16(t):
        """a copy at an address of 16 mod 32"""
        raw = torch.zeros(t.numel() * t.element_size() + 64, dtype=torch.uint8, device=DEV)
        off = (16 - raw.data_ptr()) % 32
        view = raw[off:off + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
        view.copy_(t)
        assert view.data_ptr() % 32 == 16
        return view

    cache, _ = filled(heads, B, T, block, "int8", 3)
    q = queries(B, n, heads, 4)
    k, v = (torch.randn((B, 50, hkv, d), device=DEV).bfloat16() for _ in range(2))
    results = []
    for place in (torch.clone, at16):
        kc, vc, ke, ve = (place(t) for t in cache.dev)
        c = ab.Context.kv8(kc, vc, ke, ve, block, ab.KV8_FORMATS["int8"])
        o, ko, vo = place(torch.zeros_like(q)), place(torch.zeros_like(k)), place(torch.zeros_like(v))
        ctx.kv8_write(c, B, T, place(k), place(v), start=33)
        ctx.kv8_read(c, B, T, ko, vo, start=30)
        ctx.kv8_attention(c, B, T, place(q), o)
        torch.cuda.synchronize()
        results.append((kc, vc, ke, ve, ko, vo, o))
    assert all(torch.equal(x, y) for x, y in zip(*results))
    assert ctx.poll_status() == 0


def test_refusals():
    heads, B, T = "gqa28", 2, 256
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, T)
    keep, c = ctx.new_kv8(B, T, 64, "e4m3")
    rows = torch.zeros((B, 8, hkv, d), dtype=torch.bfloat16, device=DEV)
    q = torch.zeros((B, 8, H, d), dtype=torch.bfloat16, device=DEV)
    o = torch.zeros_like(q)
    launched = ctx.launch_count()

    def changed(**kw):
        t = ab.KV8(c.k, c.v, c.k_exp, c.v_exp, c.batch_stride, c.ctx_capacity, c.block, c.format)
        for name, v in kw.items():
            setattr(t, name, v)
        return t

    calls = [lambda t, b=B, T_=T: ctx.kv8_write(t, b, T_, rows, rows), lambda t, b=B, T_=T: ctx.kv8_read(t, b, T_, rows, rows),
             lambda t, b=B, T_=T: ctx.kv8_attention(t, b, T_, q, o)]
    for call in calls:
        for bad, status in [(dict(k=None), ab.ERR_INVALID_ARG), (dict(v=c.v + 8), ab.ERR_INVALID_ARG), (dict(v_exp=None), ab.ERR_INVALID_ARG),
                            (dict(format=2), ab.ERR_INVALID_ARG), (dict(block=48), ab.ERR_UNSUPPORTED_SHAPE), (dict(block=8), ab.ERR_UNSUPPORTED_SHAPE),
                            (dict(ctx_capacity=T - 64), ab.ERR_INVALID_ARG), (dict(ctx_capacity=T + 32), ab.ERR_INVALID_ARG),
                            (dict(batch_stride=c.batch_stride - 16), ab.ERR_INVALID_ARG), (dict(batch_stride=c.batch_stride + 8), ab.ERR_INVALID_ARG)]:
            with pytest.raises(ab.AcacheError) as e:
                call(changed(**bad))
            assert e.value.status == status, bad
        with pytest.raises(ab.AcacheError):
            call(c, T_=T + 1)                            # past the context's limit
    with pytest.raises(ab.AcacheError):                  # a shared cache is not written
        ctx.kv8_write(changed(batch_stride=0), B, T, rows, rows)
    for kw in (dict(start=T - 7), dict(start=-1)):
        with pytest.raises(ab.AcacheError):
            ctx.kv8_write(c, B, T, rows, rows, **kw)
        with pytest.raises(ab.AcacheError):
            ctx.kv8_read(c, B, T, rows, rows, **kw)
    with pytest.raises(ab.AcacheError):
        ctx.kv8_read(c, B, T, None, None)
    for bad in (rows.float(), rows[:, :, :2], rows.transpose(1, 2)):
        with pytest.raises(ValueError):
            ctx.kv8_write(c, B, T, bad, bad)
    for kw in (dict(lse=torch.zeros((B, 8, H), dtype=torch.bfloat16, device=DEV)), dict(lens=torch.zeros(B, device=DEV)),
               dict(key_drop=torch.zeros((B, 3), dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            ctx.kv8_attention(c, B, T, q, o, **kw)
    with pytest.raises(ValueError):
        ab.Context.kv8(keep[0], keep[1], keep[2], keep[3], 32, 0)
    with pytest.raises(ValueError):
        ab.Context.kv8(keep[0].transpose(1, 2), keep[1], keep[2], keep[3], 64, 0)
    assert ctx.launch_count() == launched and ctx.poll_status() == 0


def test_tensors_of_the_host_are_refused():
    heads, B, T, n = "gqa28", 1, 64, 2
    H, hkv, d = HEADS[heads]
    ctx = context(heads, B, T)
    keep, c = ctx.new_kv8(B, T, 16, "e4m3")
    launched = ctx.launch_count()
    rows, q = torch.zeros((B, n, hkv, d), dtype=torch.bfloat16, device=DEV), torch.zeros((B, n, H, d), dtype=torch.bfloat16, device=DEV)
    pos, lens = torch.zeros((B, n), dtype=torch.int32, device=DEV), torch.zeros((B,), dtype=torch.int32, device=DEV)
    for call in (lambda: ctx.kv8_write(c, B, T, rows.cpu(), rows), lambda: ctx.kv8_write(c, B, T, rows, rows.cpu()),
                 lambda: ctx.kv8_write(c, B, T, rows, rows, pos=pos.cpu()), lambda: ctx.kv8_read(c, B, T, rows, rows.cpu()),
                 lambda: ctx.kv8_read(c, B, T, rows.cpu(), None), lambda: ctx.kv8_read(c, B, T, None, rows, pos=pos.cpu()),
                 lambda: ctx.kv8_attention(c, B, T, q.cpu(), q), lambda: ctx.kv8_attention(c, B, T, q, q.cpu()),
                 lambda: ctx.kv8_attention(c, B, T, q, q, lens=lens.cpu())):
        with pytest.raises(ValueError):
            call()
    assert ctx.launch_count() == launched
