"""The operators of the 8-bit affix cache, as cases that can be timed and compared.

Three operators on a KV cache held in 8 bits with a power-of-two scale for each block of tokens and head: writing rows
into it (quantising them), reading rows back, and attention over it.  Codes are [B, Hkv, capacity, d], exponents
[B, Hkv, capacity / block] bytes, a value is code * 2^(exponent - 127).  Head layouts are those of the LLaDA-8B-,
Dream-7B-shaped and tiny layers of this repository; lengths, rows and batches those of its configurations and a
long cache.  The inputs behave as trained models' do where random ones would not: some channels of the keys are
several times larger than the others, token norms vary, the first tokens have small values.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
LAYOUTS = {"mha32": (32, 32, 128), "gqa28": (28, 4, 128), "mha4": (4, 4, 64), "gqa4": (4, 2, 64)}   # H, Hkv, d
FORMATS = ("e4m3", "int8")
E_MIN = 16                                    # lowest exponent of a block that holds something
TOP = {"e4m3": 7, "int8": 6}                  # a block's largest value lands in [2^TOP, 2^(TOP + 1)) times the scale


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _case(kind, heads, batch, ctx, rows, block, fmt, how, name=None):
    """how: of a write or read, "span" (`rows` consecutive positions from `ctx - rows` on) or "rows" (positions given one by
    one); of attention, "full" (every key), "lens" (a length per request, one of them 0) or "drop" (lengths, and three
    keys in ten do not exist)."""
    c = dict(kind=kind, heads=heads, batch=batch, ctx=ctx, rows=rows, block=block, fmt=fmt, how=how)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the 32 rows of the block being decoded, one request: latency
        _case("write", "mha32", 1, 1024, 32, 32, "e4m3", "span", "write-decode-block"),
        # a refresh of a batch: anchors and request rows scattered over the cache, most blocks keep some rows
        _case("write", "mha32", 16, 2560, 922, 64, "int8", "rows", "write-refresh-b16"),
        # the cache of a whole batch built from its bf16 form
        _case("write", "mha32", 16, 2560, 2560, 64, "e4m3", "span", "write-whole-b16"),
        # the affix keys of one request for scoring
        _case("read", "gqa28", 1, 1152, 1024, 16, "int8", "span", "read-affix-gqa"),
        # ragged gather of a batch's rows
        _case("read", "mha32", 5, 8288, 1639, 128, "e4m3", "rows", "read-rows-b5"),
        # one token of one request over a short and a long cache: latency, split over the keys
        _case("attention", "gqa28", 1, 1664, 1, 16, "e4m3", "full", "attn-token-gqa"),
        _case("attention", "mha32", 2, 65537, 1, 64, "int8", "full", "attn-token-long"),
        # the smallest layer's rows (head dimension 64)
        _case("attention", "mha4", 1, 256, 58, 16, "int8", "full", "attn-tiny"),
        # a decode pass over a batch: 32 rows of every request
        _case("attention", "mha32", 16, 2560, 32, 64, "e4m3", "full", "attn-decode-block-b16"),
        # grouped heads, lengths of their own, keys that do not exist, sizes that divide nothing
        _case("attention", "gqa28", 7, 1531, 29, 32, "int8", "drop", "attn-ragged-gqa"),
        # anchors of one request over a long affix
        _case("attention", "mha32", 1, 8288, 1639, 128, "e4m3", "full", "attn-anchors-long"),
        # the refresh of a batch with all its request rows: the largest
        _case("attention", "mha32", 16, 2560, 922, 64, "int8", "lens", "attn-refresh-b16"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top_flops = max(work(c)["flops"] for c in listed())
    top_bytes = max(work(c)["bytes"] for c in listed())
    while True:
        kind = rng.choice(["write", "read", "attention", "attention"])
        heads = rng.choice(list(LAYOUTS))
        ctx = _spread(rng, 1, 70000)
        rows = min(_spread(rng, 1, 2600), ctx) if kind != "attention" else _spread(rng, 1, 1700)
        how = rng.choice(["span", "rows"] if kind != "attention" else ["full", "lens", "drop"])
        c = _case(kind, heads, _spread(rng, 1, 64), ctx, rows, rng.choice([16, 32, 64, 128]), rng.choice(FORMATS), how)
        w = work(c)
        # the plain form holds the whole cache in 32 bits and every logit
        H, hkv, d = LAYOUTS[heads]
        held = 4 * c["batch"] * (4 * hkv * d * ctx + (3 * H * rows * ctx if kind == "attention" else 0))
        if w["flops"] <= top_flops and w["bytes"] <= top_bytes and held <= 24e9:
            return c


def _lens(case):
    """Keys each request has: a fixed spread, with a request of one key and one of none where there are enough."""
    B, T = case["batch"], case["ctx"]
    if case["how"] == "full":
        return [T] * B
    lens = [T - (b * T) // (2 * B) for b in range(B)]
    if B >= 3:
        lens[-1], lens[-2] = 0, 1
    return lens


def work(case):
    H, hkv, d = LAYOUTS[case["heads"]]
    B, n, T = case["batch"], case["rows"], case["ctx"]
    if case["kind"] in ("write", "read"):
        exps = 2 * B * hkv * -(-n // case["block"])
        pos = 4 * B * n if case["how"] == "rows" else 0
        return {"bytes": 2 * B * n * hkv * d * 3 + exps + pos, "flops": 2 * B * n * hkv * d}
    keys = sum(_lens(case))
    exps = 2 * hkv * -(-keys // case["block"])
    side = (4 * B if case["how"] != "full" else 0) + (keys // 8 if case["how"] == "drop" else 0)
    return {"bytes": 2 * keys * hkv * d + exps + side + B * n * H * (4 * d + 4), "flops": 4 * n * H * d * keys}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _rows(gen, B, n, hkv, d, values):
    """bf16 rows [B, n, Hkv, d] of keys or values."""
    t = torch.randn((B, n, hkv, d), generator=gen, device=DEV, dtype=torch.bfloat16)
    t *= (torch.randn((B, n, hkv, 1), generator=gen, device=DEV) * 0.3).exp().mul_(1.2).bfloat16()
    if values:
        t[:, :1] *= 0.05                        # the first token is attended much and says little
    else:
        loud = torch.rand((1, 1, hkv, d), generator=gen, device=DEV) < 0.03
        t = torch.where(loud, t * 4, t)
    return t


def _cache_of(rows, block, fmt):
    """The 8-bit cache that holds these rows from position 0 on: codes [B, Hkv, cap, d] (bytes), exponents [B, Hkv, cap / block]."""
    B, n, hkv, d = rows.shape
    cap = -(-n // block) * block
    codes = torch.empty((B, hkv, cap, d), dtype=torch.uint8, device=DEV)
    exps = torch.empty((B, hkv, cap // block), dtype=torch.uint8, device=DEV)
    for b in range(B):
        t = torch.zeros((hkv, cap, d), dtype=torch.float32, device=DEV)
        t[:, :n] = rows[b].permute(1, 0, 2)
        t = t.view(hkv, cap // block, block, d)
        exps[b] = _exponent(t, fmt)
        codes[b] = _round(t * _scale(254 - exps[b].int())[:, :, None, None], fmt).view(hkv, cap, d)
    return codes, exps


def _positions(gen, B, n, ctx):
    """n different positions of every request: the first half ascending (anchors), the others in any order."""
    pos = torch.rand((B, ctx), generator=gen, device=DEV).argsort(dim=1)[:, :n]
    return torch.cat([pos[:, :n // 2].sort(dim=1).values, pos[:, n // 2:]], dim=1).to(torch.int32).contiguous()


def prepare(case, seed):
    H, hkv, d = LAYOUTS[case["heads"]]
    B, n, T, block, fmt = case["batch"], case["rows"], case["ctx"], case["block"], case["fmt"]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case=case, B=B, n=n, T=T, H=H, hkv=hkv, d=d, block=block, fmt=fmt)
    whole = case["kind"] == "write" and case["how"] == "span" and n == T
    old = [_rows(gen, B, T, hkv, d, v) for v in (False, True)]
    (s["k"], s["ke"]), (s["v"], s["ve"]) = [_cache_of(r, block, fmt) for r in old]
    if whole:                                   # nothing in the cache yet
        for name in ("k", "ke", "v", "ve"):
            s[name].zero_()
    del old
    if case["kind"] != "attention":
        s["pos"] = _positions(gen, B, n, T) if case["how"] == "rows" else None
        s["start"] = 0 if case["how"] == "rows" else T - n
    if case["kind"] == "write":
        s["k_rows"], s["v_rows"] = _rows(gen, B, n, hkv, d, False), _rows(gen, B, n, hkv, d, True)
    elif case["kind"] == "read":
        s["k_out"], s["v_out"] = (torch.empty((B, n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    else:
        s["q"] = (torch.randn((B, n, H, d), generator=gen, device=DEV) * 1.2).bfloat16()
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((B, n, H), dtype=torch.float32, device=DEV)
        s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device=DEV) if case["how"] != "full" else None
        s["drop"] = None
        if case["how"] == "drop":               # bit t % 32 of word t / 32: position t does not exist as a key
            words = -(-T // 32)
            bits = torch.rand((B, words, 32), generator=gen, device=DEV) < 0.3
            weight = 2 ** torch.arange(32, device=DEV, dtype=torch.int64)
            s["drop"] = (bits.to(torch.int64) * weight).sum(-1).to(torch.uint32).view(torch.int32)
    if own:                                     # the handle a program keeps for a layer shape
        from paper_2608_26140_b200 import binding as ab
        s["ctx"] = ab.Context(hkv * d, H, hkv, d, 128, 1e-5, 0, B, T, 0, 1, 0, DEV)
        s["cache"] = ab.Context.kv8(s["k"], s["v"], s["ke"], s["ve"], block, ab.KV8_FORMATS[fmt])
    return s


# --------------------------------------------------------------------------
# the operators
# --------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        if kind == "write":
            s["ctx"].kv8_write(s["cache"], s["B"], s["T"], s["k_rows"], s["v_rows"], start=s["start"], pos=s["pos"])
            return _held(s, s["k"], s["v"], s["ke"], s["ve"])
        if kind == "read":
            s["ctx"].kv8_read(s["cache"], s["B"], s["T"], s["k_out"], s["v_out"], start=s["start"], pos=s["pos"])
            return dict(k=s["k_out"], v=s["v_out"])
        s["ctx"].kv8_attention(s["cache"], s["B"], s["T"], s["q"], s["o"], lse=s["lse"], lens=s["lens"], key_drop=s["drop"])
        return dict(o=s["o"], lse=s["lse"])
    if kind == "write":
        k, ke = _plain_write(s, s["k"], s["ke"], s["k_rows"])
        v, ve = _plain_write(s, s["v"], s["ve"], s["v_rows"])
        return _held(s, k, v, ke, ve)
    if kind == "read":
        return dict(k=_plain_read(s, s["k"], s["ke"]), v=_plain_read(s, s["v"], s["ve"]))
    return _plain_attention(s)


def _held(s, k, v, ke, ve):
    """The cache as the values its codes stand for, and the exponents."""
    as_values = torch.float8_e4m3fn if s["fmt"] == "e4m3" else torch.int8
    return dict(k=k.view(as_values), v=v.view(as_values), k_exp=ke, v_exp=ve)


def _scale(e):
    """2^(e - 127) for exponent bytes 1 .. 254 as int32, and 0 for 0 (a block that holds nothing)."""
    return (e << 23).view(torch.float32)


def _exponent(t, fmt):
    """Exponent bytes of blocks of fp32 values [..., block, d]: the largest finite one lands in [2^TOP, 2^(TOP + 1)) scales."""
    field = (t.abs().amax(dim=(-2, -1)).view(torch.int32) >> 23) & 255
    return (field - TOP[fmt]).clamp(E_MIN, 254).to(torch.uint8)


def _round(x, fmt):
    return (x.to(torch.float8_e4m3fn) if fmt == "e4m3" else x.round().clamp(-127, 127).to(torch.int8)).view(torch.uint8)


def _values(codes, fmt):
    return codes.view(torch.float8_e4m3fn if fmt == "e4m3" else torch.int8).float()


def _plain_write(s, codes, exps, rows):
    B, n, T, hkv, d, block, fmt = s["B"], s["n"], s["T"], s["hkv"], s["d"], s["block"], s["fmt"]
    # the blocks from the first to the last touched, as [B, Hkv, blocks, block, d]
    b0, b1 = (0, exps.shape[2]) if s["pos"] is not None else (s["start"] // block, -(-(s["start"] + n) // block))
    at = torch.arange(b0 * block, b1 * block, device=DEV)
    fresh = torch.zeros((B, (b1 - b0) * block, hkv, d), dtype=torch.float32, device=DEV)
    written = torch.zeros((B, (b1 - b0) * block), dtype=torch.bool, device=DEV)
    if s["pos"] is None:
        first = s["start"] - b0 * block
        fresh[:, first:first + n] = rows
        written[:, first:first + n] = True
    else:
        index = s["pos"].long()
        fresh.scatter_(1, index[:, :, None, None].expand(B, n, hkv, d), rows.float())
        written.scatter_(1, index, True)
    fresh = fresh.permute(0, 2, 1, 3).reshape(B, hkv, b1 - b0, block, d)
    written = written.view(B, 1, b1 - b0, block)
    kept = ~written & (at < T).view(1, 1, b1 - b0, block)
    touched = written.any(-1)
    e_old = exps[:, :, b0:b1].int()
    e_rows = _exponent(fresh, fmt).int()
    e_new = torch.where(kept.any(-1), torch.maximum(e_rows, e_old), e_rows)
    old = codes.view(B, hkv, -1, block, d)[:, :, b0:b1]
    # rows that stay are rounded to the new scale; a block that held nothing has none
    stay = torch.where((e_old > 0)[..., None, None], _values(old, fmt) * _scale(127 + e_old - e_new)[..., None, None], 0.0)
    new = torch.where(written[..., None], _round(fresh * _scale(254 - e_new)[..., None, None], fmt),
                      torch.where(kept[..., None], _round(stay, fmt), 0))
    out, out_e = codes.clone(), exps.clone()
    out.view(B, hkv, -1, block, d)[:, :, b0:b1] = torch.where(touched[..., None, None], new, old)
    out_e[:, :, b0:b1] = torch.where(touched, e_new, e_old).to(torch.uint8)
    return out, out_e


def _plain_read(s, codes, exps):
    B, n, hkv, d, block, fmt = s["B"], s["n"], s["hkv"], s["d"], s["block"], s["fmt"]
    if s["pos"] is None:
        at = torch.arange(s["start"], s["start"] + n, device=DEV).expand(B, n)
    else:
        at = s["pos"].long()
    c = codes.gather(2, at[:, None, :, None].expand(B, hkv, n, d))
    e = exps.int().gather(2, (at // block)[:, None, :].expand(B, hkv, n))
    return (_values(c, fmt) * _scale(e)[..., None]).transpose(1, 2).to(torch.bfloat16).contiguous()


def _plain_cache(s, codes, exps):
    """The cache in 32 bits, [B, Hkv, T, d]."""
    B, hkv, cap, d = codes.shape
    t = _values(codes, s["fmt"]).view(B, hkv, exps.shape[2], s["block"], d) * _scale(exps.int())[..., None, None]
    return t.view(B, hkv, cap, d)[:, :, :s["T"]]


def _plain_attention(s):
    B, n, T, H, hkv, d = s["B"], s["n"], s["T"], s["H"], s["hkv"], s["d"]
    k, v = _plain_cache(s, s["k"], s["ke"]), _plain_cache(s, s["v"], s["ve"])
    q = s["q"].float().view(B, n, hkv, H // hkv, d).transpose(1, 2).reshape(B, hkv, -1, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    if s["lens"] is not None:
        gone = torch.arange(T, device=DEV) >= s["lens"][:, None]
        if s["drop"] is not None:
            gone |= ((s["drop"][:, :, None] >> torch.arange(32, device=DEV)) & 1).view(B, -1)[:, :T].bool()
        x.masked_fill_(gone[:, None, None, :], -math.inf)
        v = v.masked_fill(gone[:, None, :, None], 0.0)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    lse = torch.where(total == 0, -math.inf, top + total.log()).view(B, hkv, n, H // hkv).transpose(1, 2).reshape(B, n, H)
    o = o.view(B, hkv, n, H // hkv, d).transpose(1, 2).reshape(B, n, H, d).to(torch.bfloat16)
    return dict(o=o, lse=lse)


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------
def _exact_codes(x, fmt):
    """x (in scales, fp64) rounded to the nearest value that the format has, ties to the even one."""
    if fmt == "int8":
        return torch.round(x).clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_write(s, codes, exps, rows):
    block, fmt = s["block"], s["fmt"]
    out, out_e = _values(codes, fmt).double(), exps.clone().long()
    for b in range(s["B"]):
        pos = s["pos"][b].tolist() if s["pos"] is not None else list(range(s["start"], s["start"] + s["n"]))
        row_of = dict(zip(pos, range(len(pos))))
        for blk in sorted({p // block for p in row_of}):
            here = range(blk * block, (blk + 1) * block)
            new = [p for p in here if p in row_of]
            kept = [p for p in here if p not in row_of and p < s["T"]]
            x = rows[b, [row_of[p] for p in new]].double().transpose(0, 1)          # [Hkv, rows, d]
            mantissa, exponent = torch.frexp(x.abs().amax(dim=(1, 2)))
            e = (exponent.long() - 1 + 127 - TOP[fmt]).clamp(min=E_MIN)
            before = out_e[b, :, blk].clone()
            if kept:
                e = torch.maximum(e, before)
                y = out[b, :, kept] * torch.exp2((before - e).double())[:, None, None]
                out[b, :, kept] = _exact_codes(torch.where((before > 0)[:, None, None], y, 0.0), fmt)
            out[b, :, new] = _exact_codes(x * torch.exp2((127 - e).double())[:, None, None], fmt)
            out[b, :, [p for p in here if p >= s["T"]]] = 0.0
            out_e[b, :, blk] = e
    return (out if fmt == "e4m3" else out.to(torch.int8)), out_e.to(torch.uint8)


def exact(case, seed):
    s = prepare(case, seed)
    B, n, T, H, hkv, d, block = s["B"], s["n"], s["T"], s["H"], s["hkv"], s["d"], s["block"]
    if case["kind"] == "write":
        if B * -(-n // block) > 4096:           # block by block, it would take too long
            return None
        (k, ke), (v, ve) = (_exact_write(s, s[a], s[a + "e"], s[a + "_rows"]) for a in "kv")
        return dict(k=k, v=v, k_exp=ke, v_exp=ve)
    if case["kind"] == "read":
        got = {}
        for a in "kv":
            out = torch.empty((B, n, hkv, d), dtype=torch.float64, device=DEV)
            for b in range(B):
                pos = s["pos"][b].long() if s["pos"] is not None else torch.arange(s["start"], s["start"] + n, device=DEV)
                scale = torch.exp2(s[a + "e"][b][:, pos // block].double() - 127)
                out[b] = (_values(s[a][b][:, pos], s["fmt"]).double() * scale[..., None]).transpose(0, 1)
            got[a] = out
        return got
    o = torch.zeros((B, n, H, d), dtype=torch.float64, device=DEV)
    lse = torch.full((B, n, H), -math.inf, dtype=torch.float64, device=DEV)
    for b, length in enumerate(_lens(case)):
        there = torch.arange(length, device=DEV)
        if s["drop"] is not None:
            there = there[((s["drop"][b, there // 32] >> (there % 32)) & 1) == 0]
        if there.numel() == 0:
            continue
        for g in range(hkv):
            k, v = (_values(s[a][b, g, there], s["fmt"]).double() *
                    torch.exp2(s[a + "e"][b, g, there // block].double() - 127)[:, None] for a in "kv")
            for h in range(g * (H // hkv), (g + 1) * (H // hkv)):
                x = s["q"][b, :, h].double() @ k.T / math.sqrt(d)
                lse[b, :, h] = torch.logsumexp(x, 1)
                o[b, :, h] = torch.softmax(x, 1) @ v
    return dict(o=o, lse=lse)
