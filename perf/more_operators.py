"""The operators of a decode pass over a paged cache, as cases that can be timed and compared.

Three operators: appending keys and values of new tokens to a cache that lies in pages, the rotary embedding applied on the
way (to the queries too), attention of few query rows over such a cache, and sampling tokens from logits with temperature,
top-k, top-p and min-p by given random numbers.  Pages are [n_pages, Hkv, page, d], a table names each request's pages in
order.  Head layouts are those of the LLaDA-8B-, Dream-7B-shaped and tiny layers of this repository; lengths, rows, batches
and the vocabulary those of its configurations, and long caches.  The inputs behave as trained models' do where random
ones would not: some channels of the keys are several times larger than the others, token norms vary, logits have a bulk and
a few tokens that stand out by a margin of the row's own, and some that are forbidden.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
LAYOUTS = {"mha32": (32, 32, 128), "gqa28": (28, 4, 128), "mha4": (4, 4, 64), "gqa4": (4, 2, 64)}   # H, Hkv, d
PAGES = (1, 8, 16, 32, 64, 128)
SETTINGS = ("temperature", "top", "nucleus", "min_p", "mixed")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _append(heads, batch, ctx, rows, page, how, name=None):
    """how: "next" (`rows` tokens behind those that each request has), "ragged" (as many as each has, up to `rows`, one request
    none) or "rows" (positions given one by one, in any order, without queries).  ctx: no request has a token from there on."""
    return dict(kind="append", heads=heads, batch=batch, ctx=ctx, rows=rows, page=page, how=how, **({"name": name} if name else {}))


def _attend(heads, batch, ctx, rows, page, how, shared=0, name=None):
    """how: "full" (every key), "lens" (a length per request, one of them 0) or "drop" (lengths, and three keys in ten do not
    exist).  The first `shared` tokens of all requests lie in the same pages."""
    return dict(kind="attention", heads=heads, batch=batch, ctx=ctx, rows=rows, page=page, how=how, shared=shared, **({"name": name} if name else {}))


def _sample(rows, vocab, dtype, settings, name=None):
    return dict(kind="sample", rows=rows, vocab=vocab, dtype=dtype, settings=settings, **({"name": name} if name else {}))


def listed():
    return [
        # the new token of every request of a batch: latency
        _append("gqa28", 32, 1664, 1, 16, "next", "append-token-gqa"),
        # anchors and request rows of a batch, refreshed in place
        _append("mha32", 16, 2560, 922, 64, "rows", "append-refresh-b16"),
        # prompts of their own lengths, from the rows of one fused projection: the largest
        _append("mha32", 16, 2560, 2560, 32, "ragged", "append-prompts-b16"),
        # one token of one request over a short and a long cache: latency, split over the keys
        _attend("gqa28", 1, 1664, 1, 16, "full", name="attn-token-gqa"),
        _attend("mha32", 2, 65537, 1, 64, "full", name="attn-token-long"),
        # one token of each request of a batch, lengths of their own
        _attend("gqa28", 64, 8191, 1, 16, "lens", name="attn-token-b64"),
        # the block being decoded by every request of a batch, over an affix that they share and tokens of their own
        _attend("mha32", 16, 2560, 32, 128, "full", shared=2048, name="attn-block-shared-affix"),
        # the smallest layer's rows (head dimension 64), keys that do not exist, sizes that divide nothing
        _attend("gqa4", 7, 251, 5, 8, "drop", name="attn-ragged-tiny"),
        # one request's token, the settings that chats use
        _sample(1, 126464, "bf16", "top", "sample-token"),
        # odd rows of a small vocabulary
        _sample(37, 1280, "f32", "min_p", "sample-small-vocab"),
        # the block of each request of a batch, from logits in 32 bits, each row with settings of its own
        _sample(512, 126464, "f32", "mixed", "sample-block-b16"),
        # a serving batch's tokens without a cut at a rank: every weight counts
        _sample(128, 126464, "bf16", "nucleus", "sample-nucleus-b128"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        top[c["kind"]] = [max(a, b) for a, b in zip(top.get(c["kind"], (0, 0)), (w["bytes"], w["flops"]))]
    while True:
        kind = rng.choice(["append", "attention", "attention", "sample"])
        heads, page = rng.choice(list(LAYOUTS)), rng.choice(PAGES)
        H, hkv, d = LAYOUTS[heads]
        batch, ctx = _spread(rng, 1, 64), _spread(rng, 1, 70000)
        if kind == "append":
            c = _append(heads, batch, ctx, min(ctx, _spread(rng, 1, 2600)), page, rng.choice(["next", "ragged", "rows"]))
            held = 4 * batch * ctx * hkv * d
        elif kind == "attention":
            rows = 1 if rng.random() < 0.5 else _spread(rng, 1, 32)
            shared = rng.choice([0, 0, ctx // 2 // page * page])
            c = _attend(heads, batch, ctx, rows, page, rng.choice(["full", "lens", "drop"]), shared)
            held = 4 * batch * ctx * (2 * hkv * d + 3 * H * rows)        # the plain form has keys, values and logits in 32 bits
        else:
            c = _sample(_spread(rng, 1, 600), _spread(rng, 256, 160000), rng.choice(list(TYPES)), rng.choice(SETTINGS))
            held = 0
        w = work(c)
        if w["bytes"] <= top[kind][0] and w["flops"] <= top[kind][1] and held <= 24e9:
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


def _counts(case):
    """New rows of each request."""
    B, n = case["batch"], case["rows"]
    counts = [n - (b * n) // (2 * B) for b in range(B)] if case["how"] == "ragged" else [n] * B
    if case["how"] == "ragged" and B >= 3:
        counts[-1] = 0
    return counts


def _held(case):
    """Tokens each request has before the new ones."""
    B, n, T = case["batch"], case["rows"], case["ctx"]
    return [T - n - (b * (T - n)) // (2 * B) for b in range(B)]


def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        # each logit becomes a weight (difference, scale, exponential) and is added up
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + 32 * case["rows"], "flops": 4 * n}
    H, hkv, d = LAYOUTS[case["heads"]]
    B, n, T = case["batch"], case["rows"], case["ctx"]
    if case["kind"] == "append":
        rows = sum(_counts(case))
        heads = 2 * hkv + (0 if case["how"] == "rows" else H)
        turned = heads - hkv
        at = 4 * rows if case["how"] == "rows" else 8 * B
        # rows in and out, the angles' table once, the pages' numbers
        return {"bytes": 4 * rows * heads * d + 4 * d * min(T, rows) + at + 4 * (rows // case["page"] + B), "flops": 3 * rows * turned * d}
    lens, shared = _lens(case), case["shared"]
    keys = sum(max(0, x - shared) for x in lens) + min(shared, max(lens))        # keys of shared pages are read once
    side = (4 * B if case["how"] != "full" else 0) + (sum(lens) // 8 if case["how"] == "drop" else 0) + 4 * sum(-(-x // case["page"]) for x in lens)
    return {"bytes": 4 * keys * hkv * d + side + B * n * H * (4 * d + 4), "flops": 4 * n * H * d * sum(lens)}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def _tokens(gen, shape, heads_at, token_at, values):
    """bf16 keys or values of this shape: token norms vary along dimension token_at, some channels of the heads are loud."""
    t = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    norms = [n if i in (0, token_at) else 1 for i, n in enumerate(shape)]
    t *= (torch.randn(norms, generator=gen, device=DEV) * 0.3).exp_().mul_(1.2).bfloat16()
    if not values:
        heads = [n if i in (heads_at, len(shape) - 1) else 1 for i, n in enumerate(shape)]
        t *= 1 + 3 * (torch.rand(heads, generator=gen, device=DEV) < 0.03)
    return t


def _pages(gen, case, hkv, d):
    """The pool's keys and values, and the table: pages in no order, those of the shared tokens named by every request."""
    B, page = case["batch"], case["page"]
    per, shared = -(-case["ctx"] // page), case.get("shared", 0) // page
    n_pages = B * (per - shared) + shared + 1                   # one that nobody names
    at = torch.randperm(n_pages - 1, generator=gen, device=DEV).to(torch.int32)
    table = at[shared:].view(B, per - shared)
    table = torch.cat([at[:shared].expand(B, shared), table], dim=1).contiguous()
    return [_tokens(gen, (n_pages, hkv, page, d), 1, 2, v) for v in (False, True)], table


def _angles(T, d):
    at = torch.arange(T, device=DEV, dtype=torch.float64)[:, None] * 5e5 ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)
    return at.cos().float(), at.sin().float()


def _settings(gen, case):
    """Temperature, top-k, top-p, min-p of each row; None: not asked for."""
    n = case["rows"]
    of = lambda v, dtype=torch.float32: torch.full((n,), v, dtype=dtype, device=DEV)  # noqa: E731
    kind = case["settings"]
    if kind == "temperature":
        return of(1.1), None, None, None
    if kind == "top":
        return of(0.7), of(50, torch.int32), of(0.95), None
    if kind == "nucleus":
        return of(0.8), None, of(0.9), None
    if kind == "min_p":
        return of(1.3), None, None, of(0.05)
    pick = lambda values, dtype: torch.tensor(values, dtype=dtype, device=DEV)[torch.randint(len(values), (n,), generator=gen, device=DEV)]  # noqa: E731
    return (pick([0.0, 0.3, 0.7, 1.0, 1.5], torch.float32), pick([0, 1, 20, 50, 1000], torch.int32),
            pick([0.5, 0.9, 0.95, 1.0], torch.float32), pick([0.0, 0.0, 0.02, 0.2], torch.float32))


def _logits(gen, n, vocab, dtype):
    t = torch.randn((n, vocab), generator=gen, device=DEV).mul_(2.3).sub_(2.0)
    # a few tokens stand out, in some rows by much
    m = min(40, vocab)
    at = torch.randint(vocab, (n, m), generator=gen, device=DEV)
    margin = torch.rand((n, 1), generator=gen, device=DEV) * 12
    t.scatter_add_(1, at, margin * torch.rand((n, m), generator=gen, device=DEV))
    t[:, torch.randint(vocab, (3,), generator=gen, device=DEV)] = -math.inf      # forbidden tokens
    return t.to(dtype)


def prepare(case, seed):
    gen = _generator(seed)
    s = dict(case=case)
    if case["kind"] == "sample":
        n = case["rows"]
        s["logits"] = _logits(gen, n, case["vocab"], TYPES[case["dtype"]])
        s["u"] = torch.rand((n,), generator=gen, device=DEV)
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = _settings(gen, case)
        s["token"] = torch.empty((n,), dtype=torch.int32, device=DEV)
        s["prob"], s["confidence"] = (torch.empty((n,), dtype=torch.float32, device=DEV) for _ in range(2))
        if own:                                 # the handle that a program keeps for its model
            from paper_2608_26140_b200 import binding as ab
            s["ctx"] = ab.Context(128, 1, 1, 128, 128, 1e-5, 0, 1, 1, 0, 1, 0, DEV)
        return s
    H, hkv, d = LAYOUTS[case["heads"]]
    B, n, T, page = case["batch"], case["rows"], case["ctx"], case["page"]
    s.update(B=B, n=n, T=T, H=H, hkv=hkv, d=d, page=page)
    (s["k_pages"], s["v_pages"]), s["table"] = _pages(gen, case, hkv, d)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    if case["kind"] == "append":
        s["q"] = s["q_out"] = s["lens"] = s["pos"] = s["counts"] = None
        s["rope"] = _angles(T, d)
        if case["how"] == "rows":               # as a layer that projects keys and values by themselves has them
            s["pos"] = torch.rand((B, T), generator=gen, device=DEV).argsort(dim=1)[:, :n].to(torch.int32).contiguous()
            s["k"], s["v"] = (_tokens(gen, (B, n, hkv, d), 2, 1, v) for v in (False, True))
        else:                                   # the rows of a fused projection
            rows = _tokens(gen, (B, n, H + 2 * hkv, d), 2, 1, False)
            s["q"], s["k"], s["v"] = rows.split((H, hkv, hkv), dim=2)
            s["q_out"] = torch.zeros((B, n, H, d), dtype=torch.bfloat16, device=DEV)
            s["lens"] = ints(_held(case))
            s["counts"] = ints(_counts(case)) if case["how"] == "ragged" else None
    else:
        s["q"] = (torch.randn((B, n, H, d), generator=gen, device=DEV) * 1.2).bfloat16()
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((B, n, H), dtype=torch.float32, device=DEV)
        s["lens"] = ints(_lens(case)) if case["how"] != "full" else None
        s["drop"] = None
        if case["how"] == "drop":               # bit t % 32 of word t / 32: position t does not exist as a key
            bits = torch.rand((B, -(-T // 32), 32), generator=gen, device=DEV) < 0.3
            weight = 2 ** torch.arange(32, device=DEV, dtype=torch.int64)
            s["drop"] = (bits.to(torch.int64) * weight).sum(-1).to(torch.uint32).view(torch.int32)
    if own:                                     # the handles that a program keeps for a layer shape and its cache
        from paper_2608_26140_b200 import binding as ab
        s["ctx"] = ab.Context(hkv * d, H, hkv, d, 128, 1e-5, 0, B, 1, 0, 1, 0, DEV)
        s["cache"] = s["ctx"].paged_kv(s["k_pages"], s["v_pages"], s["table"])
    return s


# --------------------------------------------------------------------------
# the operators
# --------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        if kind == "append":
            s["ctx"].paged_append(s["cache"], s["T"], s["k"], s["v"], lens=s["lens"], pos=s["pos"], counts=s["counts"],
                                  rope=s["rope"], q=s["q"], q_out=s["q_out"])
            return _appended(s)
        if kind == "attention":
            s["ctx"].paged_attention(s["cache"], s["T"], s["q"], s["o"], lse=s["lse"], lens=s["lens"], key_drop=s["drop"])
            return dict(o=s["o"], lse=s["lse"])
        s["ctx"].sample_tokens(s["logits"], s["u"], s["token"], prob=s["prob"], confidence=s["confidence"],
                               temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return dict(token=s["token"], prob=s["prob"], confidence=s["confidence"])
    if kind == "append":
        return _plain_append(s)
    return _plain_attention(s) if kind == "attention" else _plain_sample(s)


def _appended(s):
    out = dict(k=s["k_pages"], v=s["v_pages"])
    if s["q_out"] is not None:
        out["q"] = s["q_out"]
    return out


def _plain_turn(x, cos, sin):
    """x [B, n, heads, d] turned by cos, sin [B, n, d / 2]: the pairs are (i, i + d / 2)."""
    a, b = x.float().chunk(2, dim=-1)
    c, z = cos[:, :, None, :], sin[:, :, None, :]
    return torch.cat([a * c - b * z, b * c + a * z], dim=-1).to(torch.bfloat16)


def _plain_append(s):
    B, n, page = s["B"], s["n"], s["page"]
    row = torch.arange(n, device=DEV).expand(B, n)
    at = s["pos"].long() if s["pos"] is not None else s["lens"].long()[:, None] + row
    real = row < s["counts"][:, None] if s["counts"] is not None else torch.ones_like(row, dtype=torch.bool)
    at = torch.where(real, at, 0)
    cos, sin = (t[at] for t in s["rope"])
    # rows that are none go, as what is there already, to the page that nobody names
    where = torch.where(real, s["table"].long().gather(1, at // page), s["k_pages"].shape[0] - 1)
    slot = torch.where(real, at % page, 0)
    k, v = _plain_turn(s["k"], cos, sin), s["v"]
    for pages, new in ((s["k_pages"], k), (s["v_pages"], v)):
        pages[where, :, slot] = torch.where(real[:, :, None, None], new, pages[-1, :, 0])
    if s["q"] is not None:
        s["q_out"].copy_(torch.where(real[:, :, None, None], _plain_turn(s["q"], cos, sin), s["q_out"]))
    return _appended(s)


def _plain_attention(s):
    B, n, T, H, hkv, d = s["B"], s["n"], s["T"], s["H"], s["hkv"], s["d"]
    k, v = (p[s["table"].long()].transpose(1, 2).reshape(B, hkv, -1, d)[:, :, :T].float() for p in (s["k_pages"], s["v_pages"]))
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


def _plain_sample(s):
    """In 64 bits: sums over the whole vocabulary, compared with a random number's share of them."""
    n, vocab = s["logits"].shape
    values, order = s["logits"].double().sort(dim=1, descending=True, stable=True)     # equal ones by their index
    below = values - values[:, :1]                                                     # of the largest
    temperature = s["temperature"].double()[:, None]
    w = torch.where(temperature > 0, below / torch.where(temperature > 0, temperature, 1.0), torch.where(below == 0, 0.0, -math.inf)).exp_()
    cum = w.cumsum(1)
    kept = torch.full((n, 1), vocab, dtype=torch.int64, device=DEV)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        kept = torch.where(k > 0, k.clamp(max=vocab), kept)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        enough = (cum < p * cum.gather(1, kept - 1)).sum(1, keepdim=True) + 1
        kept = torch.where(p < 1, torch.minimum(kept, enough), kept)
    if s["min_p"] is not None:
        kept = torch.minimum(kept, (w >= s["min_p"].double()[:, None]).sum(1, keepdim=True))
    kept = torch.where(temperature > 0, kept, 1)
    total = cum.gather(1, kept - 1)
    rank = torch.minimum((cum <= s["u"].double()[:, None] * total).sum(1, keepdim=True), kept - 1)
    prob = w.gather(1, rank) / total
    confidence = below.gather(1, rank).exp() / below.exp_().sum(1, keepdim=True)
    return dict(token=order.gather(1, rank)[:, 0].int(), prob=prob[:, 0].float(), confidence=confidence[:, 0].float())


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "sample": _exact_sample}[case["kind"]](s)


def _exact_append(s):
    d, page = s["d"], s["page"]
    k, v = s["k_pages"].double(), s["v_pages"].double()
    q = s["q_out"].double() if s["q"] is not None else None
    counts = _counts(s["case"])
    for b in range(s["B"]):
        m = counts[b]
        if m == 0:
            continue
        at = s["pos"][b, :m].long() if s["pos"] is not None else int(s["lens"][b]) + torch.arange(m, device=DEV)
        angle = torch.complex(s["rope"][0][at].double(), s["rope"][1][at].double())[:, None, :]

        def turned(x):
            z = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double()) * angle
            return torch.cat([z.real, z.imag], dim=-1)
        where = s["table"][b].long()[at // page]
        k[where, :, at % page] = turned(s["k"][b, :m])
        v[where, :, at % page] = s["v"][b, :m].double()
        if q is not None:
            q[b, :m] = turned(s["q"][b, :m])
    return dict(k=k, v=v, q=q) if q is not None else dict(k=k, v=v)


def _exact_attention(s):
    B, n, H, hkv, d, page = s["B"], s["n"], s["H"], s["hkv"], s["d"], s["page"]
    o = torch.zeros((B, n, H, d), dtype=torch.float64, device=DEV)
    lse = torch.full((B, n, H), -math.inf, dtype=torch.float64, device=DEV)
    for b, length in enumerate(_lens(s["case"])):
        there = torch.arange(length, device=DEV)
        if s["drop"] is not None:
            there = there[((s["drop"][b, there // 32] >> (there % 32)) & 1) == 0]
        if there.numel() == 0:
            continue
        where = s["table"][b].long()[there // page]
        k, v = (p[where, :, there % page].double() for p in (s["k_pages"], s["v_pages"]))      # [keys, Hkv, d]
        for h in range(H):
            x = s["q"][b, :, h].double() @ k[:, h // (H // hkv)].T / math.sqrt(d)
            lse[b, :, h] = torch.logsumexp(x, 1)
            o[b, :, h] = torch.softmax(x, 1) @ v[:, h // (H // hkv)]
    return dict(o=o, lse=lse)


def _exact_sample(s):
    n, vocab = s["logits"].shape
    out = [[], [], []]
    for r in range(n):
        x = s["logits"][r].double()
        probs = torch.softmax(x, 0)
        T = float(s["temperature"][r])
        order = torch.argsort(x, descending=True, stable=True)
        if T == 0:
            kept, share = order[:1], torch.ones(1, dtype=torch.float64, device=DEV)
        else:
            share = torch.softmax(x[order] / T, 0)
            k = int(s["top_k"][r]) if s["top_k"] is not None else 0
            if 0 < k < vocab:
                share = share[:k] / share[:k].sum()
            least = float(s["min_p"][r]) if s["min_p"] is not None else 0.0
            few = int((share / share[0] >= least).sum())
            p = float(s["top_p"][r]) if s["top_p"] is not None else 1.0
            if p < 1:
                few = min(few, 1 + int(torch.searchsorted(share.cumsum(0), torch.tensor([p], dtype=torch.float64, device=DEV))))
            share = share[:max(1, few)]
            share = share / share.sum()
            kept = order[:share.numel()]
        i = min(int(torch.searchsorted(share.cumsum(0), s["u"][r:r + 1].double(), right=True)), share.numel() - 1)
        for to, value in zip(out, (kept[i], share[i], probs[kept[i]])):
            to.append(value)
    return dict(token=torch.stack(out[0]).int(), prob=torch.stack(out[1]), confidence=torch.stack(out[2]))
