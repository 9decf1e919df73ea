"""The cache in pages (acache_paged_append, acache_paged_attention) against plain implementations in 64 bits.

Values are copied, so compared to the bit; a turned key or query is held to one rounding of its value and the fp32 steps before it:

    |k' - ref| <= 2^-8 |ref| + 3 * 2^-24 (|a cos| + |b sin|)

Attention, A = sum_j p_j |V_j|, X = max_j sum_i |q_i k_ij| / sqrt(d) (kept below 64):

    |o - ref| <= 2^-8 |ref| + (2^-8 + 2^-9) A        |lse - ref| <= 2^-16 X + 2^-18 (1 + |ref|)

(half a bf16 step of the result; half a bf16 step of each probability, 2^-8 A; logits off by up to 128 * 2^-24 X in sums of 128 products, which with
the exponential's 2^-22 moves a probability and the sum of all by less than 2^-10 each; the logarithm of the sum.)
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_26140_b200 import binding as ab

from helpers import DEV

pytestmark = pytest.mark.gpu

HEADS = {"mha4-64": (4, 4, 64), "gqa4-64": (4, 2, 64), "gqa28": (28, 4, 128), "mha32": (32, 32, 128), "mqa8": (8, 1, 128)}


def context(heads, batch):
    H, hkv, d = HEADS[heads]
    return ab.Context(max(hkv * d, 128), H, hkv, d, 128, 1e-5, 0, batch, 1, 0, 1, 0, DEV)


def random(gen, *shape, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * std).bfloat16()


def pool_of(gen, heads, batch, ctx_len, page, spare=2, gap=0):
    """Pools, pages gap elements further apart than they take, and a table that names them in no order; spare pages and gaps hold NaN."""
    H, hkv, d = HEADS[heads]
    per = max(1, -(-ctx_len // page))
    n = batch * per + spare
    order = torch.randperm(n, generator=gen, device=DEV)[:batch * per].to(torch.int32)
    pools = []
    for _ in range(2):
        whole = torch.full((n, hkv * page * d + gap), float("nan"), dtype=torch.bfloat16, device=DEV)
        p = whole[:, :hkv * page * d].view(n, hkv, page, d) if gap == 0 else whole.as_strided((n, hkv, page, d), (hkv * page * d + gap, page * d, d, 1))
        p[order.long()] = random(gen, batch * per, hkv, page, d)
        pools.append(p)
    return pools[0], pools[1], order.view(batch, per).contiguous()


def tokens(pool, table, b, at):
    """Rows [len(at), Hkv, d] of request b."""
    page = pool.shape[2]
    return pool[table[b].long()[at // page], :, at % page]


def reference(q, k_pages, v_pages, table, keys):
    """q [B, n, H, d]; keys: a list of positions per request.  o, lse, A, X in 64 bits."""
    B, n, H, d = q.shape
    hkv = k_pages.shape[1]
    o = torch.zeros((B, n, H, d), dtype=torch.float64, device=DEV)
    A = torch.zeros_like(o)
    lse = torch.full((B, n, H), -math.inf, dtype=torch.float64, device=DEV)
    X = torch.zeros_like(lse)
    for b in range(B):
        if len(keys[b]) == 0:
            continue
        at = torch.as_tensor(keys[b], device=DEV)
        k, v = tokens(k_pages, table, b, at).double(), tokens(v_pages, table, b, at).double()
        for h in range(H):
            g = h // (H // hkv)
            x = q[b, :, h].double() @ k[:, g].T / math.sqrt(d)
            p = torch.softmax(x, 1)
            o[b, :, h], A[b, :, h] = p @ v[:, g], p @ v[:, g].abs()
            lse[b, :, h] = torch.logsumexp(x, 1)
            X[b, :, h] = (q[b, :, h].double().abs() @ k[:, g].abs().T).amax(1) / math.sqrt(d)
    return o, lse, A, X


def check(o, lse, ref):
    ro, rl, A, X = ref
    assert X.max() < 64
    assert not torch.isnan(o).any()
    assert ((o.double() - ro).abs() <= 2 ** -8 * ro.abs() + (2 ** -8 + 2 ** -9) * A).all(), ((o.double() - ro).abs() / A.clamp(min=1e-30)).max()
    if lse is not None:
        none = rl == -math.inf
        assert torch.equal(lse == -math.inf, none)
        assert ((lse.double() - rl).abs()[~none] <= (2 ** -16 * X + 2 ** -18 * (1 + rl.abs()))[~none]).all()


@pytest.mark.parametrize("heads,batch,n,ctx_len,page", [
    ("gqa28", 1, 1, 1, 16), ("gqa28", 3, 1, 1664, 16), ("mha32", 2, 1, 4099, 64), ("mqa8", 5, 1, 130, 128), ("mha4-64", 1, 1, 63, 1),
    ("gqa4-64", 4, 5, 251, 8), ("mha4-64", 2, 16, 257, 2), ("mha32", 2, 32, 1000, 32), ("gqa28", 2, 9, 777, 1024), ("gqa28", 1, 31, 200, 4),
    ("mqa8", 2, 3, 64, 16), ("gqa4-64", 1, 33, 1531, 32), ("mha32", 1, 17, 65, 256)])
@pytest.mark.parametrize("how", ["full", "lens", "drop"])
def test_attention(heads, batch, n, ctx_len, page, how):
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(ctx_len * 7 + n)
    k, v, table = pool_of(gen, heads, batch, ctx_len, page)
    q = random(gen, batch, n, H, d)
    lens = [ctx_len] * batch
    there = np.ones((batch, ctx_len), bool)
    if how != "full":
        lens = [max(0, ctx_len - 3 * b - b * ctx_len // 3) for b in range(batch)]
        lens[-1] = 0 if batch > 1 else ctx_len // 2
    if how == "drop":
        there = np.random.default_rng(n).random((batch, ctx_len)) < 0.6
        there[0] = False
    keys = [np.flatnonzero(there[b, :lens[b]]) for b in range(batch)]
    if how == "drop":                            # what does not count may be anything
        for b in range(batch):
            gone = torch.as_tensor(np.flatnonzero(~there[b]), device=DEV)
            for p in (k, v):
                p[table[b].long()[gone // page], :, gone % page] = float("nan")
    o, lse = torch.full_like(q, 7.0), torch.full((batch, n, H), 7.0, device=DEV)
    ctx = context(heads, batch)
    ctx.paged_attention(ctx.paged_kv(k, v, table), ctx_len, q, o, lse=lse,
                        lens=torch.tensor(lens, dtype=torch.int32, device=DEV) if how != "full" else None,
                        key_drop=ctx.pack_key_drop(torch.as_tensor(~there, device=DEV)) if how == "drop" else None)
    check(o, lse, reference(q, k, v, table, keys))
    assert ctx.poll_status() == 0
    again, again_lse = torch.empty_like(o), torch.empty_like(lse)
    ctx.paged_attention(ctx.paged_kv(k, v, table), ctx_len, q, again, lse=again_lse,
                        lens=torch.tensor(lens, dtype=torch.int32, device=DEV) if how != "full" else None,
                        key_drop=ctx.pack_key_drop(torch.as_tensor(~there, device=DEV)) if how == "drop" else None)
    assert torch.equal(o, again) and torch.equal(lse, again_lse)


def test_attention_of_requests_of_very_different_lengths():
    """Lengths on the device decide how the work is cut: one long request among short and empty ones, more requests than threads."""
    heads, batch, ctx_len, page = "gqa4-64", 300, 3001, 16
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(5)
    lens = [0, 1, 2, 64, 65][:5] * 60
    lens[137], lens[299], lens[298] = 3001, 0, 1999
    k, v, _ = pool_of(gen, heads, 1, 70 * page, page)
    table = torch.randint(70, (batch, -(-ctx_len // page)), generator=gen, device=DEV).to(torch.int32)      # requests share pages
    real = torch.nonzero(~torch.isnan(k[:, 0, 0, 0])).flatten().to(torch.int32)
    table = real[table.long() % real.numel()]
    q = random(gen, batch, 1, H, d)
    o, lse = torch.empty_like(q), torch.empty((batch, 1, H), device=DEV)
    ctx = context(heads, batch)
    ctx.paged_attention(ctx.paged_kv(k, v, table), ctx_len, q, o, lse=lse, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    check(o, lse, reference(q, k, v, table, [np.arange(x) for x in lens]))
    assert ctx.poll_status() == 0


def test_attention_when_logits_keep_rising_and_when_one_key_has_everything():
    heads, page, T = "mha32", 16, 1024
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(6)
    k, v, table = pool_of(gen, heads, 2, T, page)
    q = random(gen, 2, 1, H, d)
    direction = q[:, 0].double() / q[:, 0].double().norm(dim=-1, keepdim=True)           # [2, H, d]
    at = torch.arange(T, device=DEV)
    for b, rise in ((0, torch.linspace(-20, 20, T, device=DEV)), (1, torch.where(at == 777, 40.0, 0.0))):
        rows = (direction[b][None] * rise[:, None, None]).bfloat16()
        k[table[b].long()[at // page], :, at % page] = rows
    o, lse = torch.empty_like(q), torch.empty((2, 1, H), device=DEV)
    ctx = context(heads, 2)
    ctx.paged_attention(ctx.paged_kv(k, v, table), T, q, o, lse=lse)
    check(o, lse, reference(q, k, v, table, [np.arange(T)] * 2))


def test_rows_whose_logits_are_infinite():
    """-inf logits weigh nothing, wherever they come first; a NaN among the keys that count reaches the row."""
    heads, page, T = "mha4-64", 16, 200
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(7)
    k, v, table = pool_of(gen, heads, 3, T, page)
    q = torch.zeros((3, 1, H, d), dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 1.0
    at = torch.arange(T, device=DEV)
    for b in range(3):
        rows = torch.zeros((T, hkv, d), dtype=torch.bfloat16, device=DEV)
        rows[..., 0] = -600.0 + torch.rand((T, hkv), generator=gen, device=DEV).bfloat16()
        if b == 0:
            rows[:150, :, 0] = -math.inf
        if b == 1:
            rows[:, :, 0] = -math.inf
        if b == 2:
            rows[77, :, 0] = float("nan")
        k[table[b].long()[at // page], :, at % page] = rows
    o, lse = torch.empty_like(q), torch.empty((3, 1, H), device=DEV)
    ctx = context(heads, 3)
    ctx.paged_attention(ctx.paged_kv(k, v, table), T, q, o, lse=lse)
    ref = reference(q[:1], k, v, table, [np.arange(150, T)])
    assert ((o[:1].double() - ref[0]).abs() <= 2 ** -8 * ref[0].abs() + 2 ** -7 * ref[2]).all()
    assert ((lse[:1].double() - ref[1]).abs() <= 2 ** -18 * (1 + ref[1].abs())).all()
    assert (o[1] == 0).all() and (lse[1] == -math.inf).all()
    assert torch.isnan(o[2]).all() and torch.isnan(lse[2]).all()


def turned(x, pos, rope):
    """x [n, heads, d] (64 bits) turned to positions pos; and the sizes of the two products."""
    half = x.shape[-1] // 2
    c, s = (t[pos].double()[:, None, :] for t in rope)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1), torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1)


def angles(T, d):
    at = np.arange(T)[:, None] * 1e4 ** (-np.arange(0, d, 2) / d)
    return tuple(torch.tensor(f(at), dtype=torch.float32, device=DEV) for f in (np.cos, np.sin))


def near(got, ref, size):
    return ((got.double() - ref).abs() <= 2 ** -8 * ref.abs() + 3 * 2 ** -24 * size).all()


@pytest.mark.parametrize("heads,batch,n,ctx_len,page,gap", [("gqa28", 3, 1, 40, 16, 0), ("mha32", 2, 33, 100, 32, 64), ("mha4-64", 1, 7, 7, 1, 0),
                                                            ("gqa4-64", 4, 19, 70, 8, 8), ("mqa8", 2, 5, 3000, 1024, 0)])
@pytest.mark.parametrize("how", ["lens", "ragged", "pos", "fused", "plain"])
def test_append(heads, batch, n, ctx_len, page, gap, how):
    """Rows go where they belong, turned; everything else stays, queries behind a request's count too."""
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(n * 31 + page)
    k_pages, v_pages, table = pool_of(gen, heads, batch, ctx_len, page, gap=gap)
    before = k_pages.clone(), v_pages.clone()
    if how == "fused":
        rows = random(gen, batch, n, H + 2 * hkv, d)
        q, k, v = rows.split((H, hkv, hkv), dim=2)
    else:
        q, k, v = random(gen, batch, n, H, d), random(gen, batch, n, hkv, d), random(gen, batch, n, hkv, d)
    rope = None if how == "plain" else angles(ctx_len, d)
    counts = [n] * batch
    if how == "ragged":
        counts = [max(0, n - 2 * b) for b in range(batch)]
        counts[-1] = 0 if batch > 1 else n // 2
    lens, pos = [(ctx_len - n) // (b + 1) for b in range(batch)], None
    at = [lens[b] + np.arange(counts[b]) for b in range(batch)]
    if how == "pos":
        rng = np.random.default_rng(n)
        pos = np.stack([rng.permutation(ctx_len)[:n] for _ in range(batch)]).astype(np.int32)
        at = list(pos)
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)  # noqa: E731
    q_out = torch.full((batch, n, H, d), 3.0, dtype=torch.bfloat16, device=DEV)
    ctx = context(heads, batch)
    ctx.paged_append(ctx.paged_kv(k_pages, v_pages, table), ctx_len, k, v, lens=ints(lens) if pos is None else None,
                     pos=ints(pos) if pos is not None else None, counts=ints(counts) if how == "ragged" else None, rope=rope, q=q, q_out=q_out)
    assert ctx.poll_status() == 0
    touched = torch.zeros(k_pages.shape[0], page, dtype=torch.bool, device=DEV)
    for b in range(batch):
        m = counts[b]
        assert (q_out[b, m:] == 3.0).all()
        if m == 0:
            continue
        p = torch.as_tensor(at[b], device=DEV).long()
        touched[table[b].long()[p // page], p % page] = True
        got_k, got_v = tokens(k_pages, table, b, p), tokens(v_pages, table, b, p)
        assert torch.equal(got_v, v[b, :m])
        if rope is None:
            assert torch.equal(got_k, k[b, :m]) and torch.equal(q_out[b, :m], q[b, :m])
        else:
            assert near(got_k, *turned(k[b, :m].double(), p, rope))
            assert near(q_out[b, :m], *turned(q[b, :m].double(), p, rope))
    for now, then in zip((k_pages, v_pages), before):
        same = (now == then) | (torch.isnan(now) & torch.isnan(then))
        assert same.all(-1).all(1)[~touched].all()


def test_append_the_last_of_two_rows_of_one_token_stays():
    heads, n, T = "gqa28", 700, 300
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(11)
    k_pages, v_pages, table = pool_of(gen, heads, 2, T, 16)
    k, v = random(gen, 2, n, hkv, d), random(gen, 2, n, hkv, d)
    pos = torch.randint(T, (2, n), generator=gen, device=DEV).to(torch.int32)
    pos[:, 5] = pos[:, 699] = 17
    pos[:, 4] = 18
    counts = torch.tensor([700, 5], dtype=torch.int32, device=DEV)
    ctx = context(heads, 2)
    for _ in range(3):
        ctx.paged_append(ctx.paged_kv(k_pages, v_pages, table), T, k, v, pos=pos, counts=counts)
        for b, m in ((0, 700), (1, 5)):
            last = {int(p): i for i, p in enumerate(pos[b, :m].tolist())}
            at, rows = torch.tensor(list(last), device=DEV), torch.tensor(list(last.values()), device=DEV)
            assert torch.equal(tokens(k_pages, table, b, at), k[b, rows]) and torch.equal(tokens(v_pages, table, b, at), v[b, rows])
    assert ctx.poll_status() == 0


def test_append_queries_in_place_and_rows_shared_by_the_requests():
    heads, n, T = "gqa4-64", 6, 50
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(12)
    k_pages, v_pages, table = pool_of(gen, heads, 3, T, 8)
    q, one = random(gen, 3, n, H, d), random(gen, 1, n, 2 * hkv, d)
    k, v = one.expand(3, n, 2 * hkv, d).split((hkv, hkv), dim=2)
    rope, was = angles(T, d), q.clone()
    lens = torch.tensor([0, 44, 9], dtype=torch.int32, device=DEV)
    ctx = context(heads, 3)
    ctx.paged_append(ctx.paged_kv(k_pages, v_pages, table), T, k, v, lens=lens, rope=rope, q=q, q_out=q)
    for b in range(3):
        at = int(lens[b]) + torch.arange(n, device=DEV)
        assert near(q[b], *turned(was[b].double(), at, rope))
        assert near(tokens(k_pages, table, b, at), *turned(k[b].double(), at, rope))
        assert torch.equal(tokens(v_pages, table, b, at), v[b])


def test_what_is_out_of_range_is_skipped_and_reported():
    heads, T, page = "gqa4-64", 64, 8
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(13)
    k_pages, v_pages, table = pool_of(gen, heads, 2, T, page)
    before = k_pages.clone(), v_pages.clone()
    ctx = context(heads, 2)
    cache = ctx.paged_kv(k_pages, v_pages, table)
    k, v = random(gen, 2, 3, hkv, d), random(gen, 2, 3, hkv, d)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    unchanged = lambda: all(bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all()) for a, b in zip((k_pages, v_pages), before))  # noqa: E731
    for bad in (dict(pos=ints([-1, 64, 1 << 30], [-5, 100, 65])), dict(lens=ints(64, -3)), dict(lens=ints(2147483647, -2147483648))):
        ctx.paged_append(cache, T, k, v, **bad)
        assert ctx.poll_status() == ab.FLAG_BAD_INDEX
        assert unchanged()
    ctx.paged_append(cache, T, k, v, lens=ints(0, 0), counts=ints(0, -1))
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX and unchanged()
    was = table.clone()
    for entry in (-1, k_pages.shape[0], 2147483647, -2147483648):
        table[0, 1] = entry
        ctx.paged_append(cache, T, k[:, :1].contiguous(), v[:, :1].contiguous(), lens=ints(9, 0), counts=ints(1, 0))
        assert ctx.poll_status() == ab.FLAG_BAD_INDEX and unchanged()
        q = random(gen, 2, 1, H, d)
        o, lse = torch.empty_like(q), torch.empty((2, 1, H), device=DEV)
        ctx.paged_attention(cache, T, q, o, lse=lse, lens=ints(40, 64))
        assert ctx.poll_status() == ab.FLAG_BAD_INDEX
        table.copy_(was)
        check(o, lse, reference(q, k_pages, v_pages, table, [np.r_[0:8, 16:40], np.arange(64)]))
    q = random(gen, 2, 1, H, d)
    o, lse = torch.empty_like(q), torch.empty((2, 1, H), device=DEV)
    ctx.paged_attention(cache, T, q, o, lse=lse, lens=ints(-7, 1 << 30))
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX
    check(o, lse, reference(q, k_pages, v_pages, table, [[], np.arange(64)]))


def test_pages_beyond_two_to_the_31_elements():
    heads, page, T = "gqa28", 16, 100
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(14)
    stride = 300 * 1024 * 1024                                        # elements between pages: the eighth begins past 2^31
    big = torch.zeros(8 * stride, dtype=torch.bfloat16, device=DEV)
    k_pages = big.as_strided((8, hkv, page, d), (stride, page * d, d, 1))
    v_pages = big.as_strided((8, hkv, page, d), (stride, page * d, d, 1), hkv * page * d)
    table = torch.tensor([[7, 0, 6, 1, 5, 2, 3]], dtype=torch.int32, device=DEV)
    k, v, q = random(gen, 1, T, hkv, d), random(gen, 1, T, hkv, d), random(gen, 1, 1, H, d)
    ctx = context(heads, 1)
    cache = ctx.paged_kv(k_pages, v_pages, table)
    ctx.paged_append(cache, T, k, v, lens=torch.zeros(1, dtype=torch.int32, device=DEV))
    assert torch.equal(tokens(k_pages, table, 0, torch.arange(T, device=DEV)), k[0])
    assert torch.equal(tokens(v_pages, table, 0, torch.arange(T, device=DEV)), v[0])
    o, lse = torch.empty_like(q), torch.empty((1, 1, H), device=DEV)
    ctx.paged_attention(cache, T, q, o, lse=lse)
    check(o, lse, reference(q, k_pages, v_pages, table, [np.arange(T)]))


def test_token_by_token_on_another_stream_and_in_a_graph():
    """A cache filled token by token, a pass captured once and replayed with the lengths moved on."""
    heads, page, T, B = "gqa28", 16, 90, 3
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(15)
    k_pages, v_pages, table = pool_of(gen, heads, B, T, page)
    rows = random(gen, T, B, 1, H + 2 * hkv, d)
    rope, ctx = angles(T, d), context(heads, B)
    cache = ctx.paged_kv(k_pages, v_pages, table)
    lens = torch.tensor([0, 7, 30], dtype=torch.int32, device=DEV)
    begin = lens.tolist()
    now, q_out = rows[0].clone(), torch.empty((B, 1, H, d), dtype=torch.bfloat16, device=DEV)
    o, lse = torch.empty_like(q_out), torch.empty((B, 1, H), device=DEV)
    q, k, v = now.split((H, hkv, hkv), dim=2)

    def one():
        ctx.paged_append(cache, T, k, v, lens=lens, rope=rope, q=q, q_out=q_out)
        lens.add_(1)
        ctx.paged_attention(cache, T, q_out, o, lse=lse, lens=lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            one()
    torch.cuda.current_stream().wait_stream(side)
    for step in range(1, 60):
        now.copy_(rows[step])
        graph.replay()
        if step in (1, 20, 59):
            keys = [np.arange(x + step + 1) for x in begin]
            check(o, lse, reference(q_out, k_pages, v_pages, table, keys))
            for b in range(B):
                at = torch.tensor([begin[b] + step], device=DEV)
                assert near(tokens(k_pages, table, b, at), *turned(rows[step, b, :, H:H + hkv].double(), at, rope))
    assert ctx.poll_status() == 0


def test_refusals():
    heads, T, page = "gqa4-64", 64, 8
    H, hkv, d = HEADS[heads]
    gen = torch.Generator(device=DEV).manual_seed(16)
    k_pages, v_pages, table = pool_of(gen, heads, 2, T, page)
    ctx = context(heads, 2)
    cache = ctx.paged_kv(k_pages, v_pages, table)
    k, q = random(gen, 2, 3, hkv, d), random(gen, 2, 3, H, d)
    lens, o = torch.zeros(2, dtype=torch.int32, device=DEV), torch.empty_like(q)
    launches = ctx.launch_count()
    for call in (lambda: ctx.paged_append(cache, T, k, k), lambda: ctx.paged_append(cache, T, k, k, lens=lens, pos=torch.zeros((2, 3), dtype=torch.int32, device=DEV)),
                 lambda: ctx.paged_append(cache, T + 1, k, k, lens=lens), lambda: ctx.paged_append(cache, -1, k, k, lens=lens),
                 lambda: ctx.paged_attention(cache, T + 1, q, o)):
        with pytest.raises(ab.AcacheError) as e:
            call()
        assert e.value.status == ab.ERR_INVALID_ARG
    more = random(gen, 3, 3, hkv, d)
    for call in (lambda: ctx.paged_append(cache, T, more, more, lens=lens), lambda: ctx.paged_append(cache, T, k.float(), k, lens=lens),
                 lambda: ctx.paged_append(cache, T, k, k[:, :2], lens=lens), lambda: ctx.paged_append(cache, T, k, k, lens=lens.long()),
                 lambda: ctx.paged_append(cache, T, k, k, lens=lens, q=q), lambda: ctx.paged_append(cache, T, k, k, lens=lens[:1]),
                 lambda: ctx.paged_append(cache, T, k, k, lens=lens, rope=angles(T - 1, d)), lambda: ctx.paged_append(cache, T, k, k, lens=lens, rope=angles(T, 2 * d)),
                 lambda: ctx.paged_append(cache, T, k.transpose(1, 2).contiguous().transpose(1, 2)[..., ::2], k, lens=lens),
                 lambda: ctx.paged_attention(cache, T, q.float(), o), lambda: ctx.paged_attention(cache, T, q, o[:1]),
                 lambda: ctx.paged_attention(cache, T, q, o, lens=lens.cpu()), lambda: ctx.paged_attention(cache, T, q.transpose(1, 2), o),
                 lambda: ctx.paged_kv(k_pages, v_pages[:1], table), lambda: ctx.paged_kv(k_pages.float(), v_pages, table),
                 lambda: ctx.paged_kv(k_pages, v_pages, table.long()), lambda: ctx.paged_kv(k_pages[:, :1], v_pages[:, :1], table)):
        with pytest.raises(ValueError):
            call()
    assert ctx.launch_count() == launches
    empty = torch.empty((2, 0, hkv, d), dtype=torch.bfloat16, device=DEV)
    ctx.paged_append(cache, T, empty, empty, lens=lens)
    ctx.paged_attention(cache, T, q[:, :0].contiguous(), o[:, :0].contiguous())
    assert ctx.launch_count() == launches
    ctx.paged_attention(cache, 0, q, o)
    assert (o == 0).all()
