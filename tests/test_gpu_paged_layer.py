"""A layer over a cache in pages (acache_recompute_paged) against the same layer over a contiguous cache and the oracle, and a run of all of it:
tokens of several requests through the layers of a model, drawn and appended one by one."""
import numpy as np
import pytest
import torch

from oracle import acache_oracle as orc
from paper_2608_26140_b200 import binding as ab
from paper_2608_26140_b200 import workloads as wl

from helpers import DEV, DeviceCase, assert_close_bf16, oracle_step

pytestmark = pytest.mark.gpu

MID = wl.LayerShape(512, 8, 2, 128, 768, 1e-6, True, 1e6, "mid-gqa")


def pages_of(ctx, cache_k, cache_v, page, seed):
    """The contiguous caches [B, T, Hkv, d] in pages of their own, in no order."""
    B, T, hkv, d = cache_k.shape
    per = -(-T // page)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    table = torch.randperm(B * per, generator=gen, device=DEV).to(torch.int32).view(B, per)
    pools = []
    for c in (cache_k, cache_v):
        whole = torch.zeros((B, per * page, hkv, d), dtype=torch.bfloat16, device=DEV)
        whole[:, :T] = c
        pool = torch.empty((B * per, hkv, page, d), dtype=torch.bfloat16, device=DEV)
        pool[table.long().view(-1)] = whole.view(B * per, page, hkv, d).transpose(1, 2)
        pools.append(pool)
    return pools[0], pools[1], table, ctx.paged_kv(pools[0], pools[1], table)


def back(pool, table, T):
    """[B, T, Hkv, d]."""
    B, per = table.shape
    n, hkv, page, d = pool.shape
    return pool[table.long()].transpose(2, 3).reshape(B, per * page, hkv, d)[:, :T]


@pytest.mark.parametrize("shape,layout,page,ratio", [(wl.TINY, (2, 8, 131, 37, 32, 32, "all"), 16, 0.2), (MID, (3, 5, 300, 33, 40, 32, "all"), 64, 0.1),
                                                     (MID, (1, 0, 257, 9, 32, 20, "masked"), 8, 0.0), (wl.TINY, (1, 0, 64, 0, 32, 32, "masked"), 1, 1.0)])
def test_refresh(shape, layout, page, ratio):
    lay = wl.make_layout(*layout)
    case = wl.make_case(shape, lay, ratio, 0)
    dc = DeviceCase(case)
    ctx, B, T = dc.ctx, lay.batch, lay.ctx_len
    K = ab.k_from_ratio(lay.affix_len, ratio)
    rng = np.random.default_rng(1)
    anchors = np.stack([np.sort(rng.choice(lay.affix_len, K, replace=False)) for _ in range(B)]).astype(np.int32)
    d_anchors = torch.from_numpy(anchors).to(DEV) if K else None
    k_pool, v_pool, table, cache = pages_of(ctx, dc.ck[:, :T], dc.cv[:, :T], page, 3)
    y, want = (torch.full((B, K + lay.n_extra, shape.hidden), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.recompute_paged(dc.lw, dc.req, cache, dc.x, 0, d_anchors, K, y)
    ctx.layer_step(dc.lw, dc.req, ab.Context.kv(dc.ck, dc.cv), dc.x, 0, ratio, 0, None, d_anchors, want)
    assert ctx.poll_status() == 0
    # the projection is the same, and so are the caches, to the bit
    assert torch.equal(back(k_pool, table, T), dc.ck[:, :T]) and torch.equal(back(v_pool, table, T), dc.cv[:, :T])
    for b in range(B):
        ref = oracle_step(case, b, anchor_idx=anchors[b])
        assert_close_bf16(ab.to_host_bits(y[b]), ref["y"], f"y of request {b}")
    # compact input, lengths of their own: the keys behind them do not count
    x = torch.gather(dc.x, 1, torch.from_numpy(np.concatenate([anchors + lay.affix_start, lay.extra_rows], 1).astype(np.int64)).to(DEV)[..., None].expand(-1, -1, shape.hidden)).contiguous()
    ctx.recompute_paged(dc.lw, dc.req, cache, x, 1, d_anchors, K, want, lens=torch.full((B,), T, dtype=torch.int32, device=DEV))
    assert torch.equal(y, want)


def test_refused_without_weights_or_with_a_cache_that_does_not_fit():
    lay = wl.make_layout(2, 8, 64, 8, 32, 32, "masked")
    dc = DeviceCase(wl.make_case(wl.TINY, lay, 0.0, 0))
    ctx, T = dc.ctx, lay.ctx_len
    k, v, table, cache = pages_of(ctx, dc.ck[:, :T], dc.cv[:, :T], 16, 3)
    y = torch.empty((2, lay.n_extra, wl.TINY.hidden), dtype=torch.bfloat16, device=DEV)
    launches = ctx.launch_count()
    short = ctx.paged_kv(k, v, table[:, :2].contiguous())
    for call, code in ((lambda: ctx.recompute_paged(dc.lw, dc.req, short, dc.x, 0, None, 0, y), ab.ERR_INVALID_ARG),
                       (lambda: ctx.recompute_paged(ab.LayerWeights(), dc.req, cache, dc.x, 0, None, 0, y), ab.ERR_INVALID_ARG),
                       (lambda: ctx.recompute_paged(dc.lw, dc.req, cache, dc.x, 0, None, 5, y), ab.ERR_INVALID_ARG),
                       (lambda: ctx.recompute_paged(dc.lw, dc.req, cache, None, 0, None, 0, y), ab.ERR_INVALID_ARG)):
        with pytest.raises(ab.AcacheError) as e:
            call()
        assert e.value.status == code
    with pytest.raises(ValueError):
        ctx.recompute_paged(dc.lw, dc.req, ctx.paged_kv(k, v, table[:1].contiguous()), dc.x, 0, None, 0, y)
    with pytest.raises(ValueError):
        ctx.recompute_paged(dc.lw, dc.req, cache, dc.x, 0, None, 0, y, lens=torch.zeros(3, dtype=torch.int32, device=DEV))
    assert ctx.launch_count() == launches


def test_tokens_drawn_and_appended_one_by_one():
    """Prompts that share an affix, appended from their projections; then every request's tokens through two layers, drawn from the LM head's logits
    with settings of its own.  What a layer computes is compared with 64 bits on the values that went into it."""
    shape, B, V, page, L, steps = MID, 3, 1280, 8, 64, 5
    H, hkv, d, D = shape.n_heads, shape.n_kv_heads, shape.head_dim, shape.hidden
    T, n_layers = 128, 2
    gen = torch.Generator(device=DEV).manual_seed(2)
    weights = [wl.layer_weights(shape, 51, n) for n in range(n_layers)]
    on = [{k: ab.to_device_bf16(v, DEV) if v is not None else None for k, v in w.items()} for w in weights]
    lws = [ab.Context.weights(w) for w in on]
    embed = torch.randn((V, D), generator=gen, device=DEV).bfloat16()
    w_lm = (torch.randn((V, D), generator=gen, device=DEV) * 0.2).bfloat16()
    gain = torch.ones((D,), device=DEV).bfloat16()
    cos, sin = wl.rope_table(T, d, shape.rope_theta)
    rope = torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV)
    ctx = ab.Context.for_shape(shape, B, T, L, 8, 1, DEV, max_vocab=V, max_block=1)
    # the affix's pages first, then each request's own
    per, shared = T // page, L // page
    n_pages = shared + B * (per - shared)
    table = torch.cat([torch.arange(shared).expand(B, shared), shared + torch.arange(B * (per - shared)).view(B, -1)], 1).to(torch.int32).to(DEV).contiguous()
    pools = [[torch.zeros((n_pages, hkv, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)] for _ in range(n_layers)]
    caches = [ctx.paged_kv(k, v, table) for k, v in pools]
    counts = torch.tensor([7, 1, 20], dtype=torch.int32, device=DEV)
    for cache in caches:
        affix = torch.randn((1, L, 2 * hkv, d), generator=gen, device=DEV).bfloat16()
        one = ctx.paged_kv(*pools[caches.index(cache)], table[:1].contiguous())
        ctx.paged_append(one, T, affix[:, :, :hkv], affix[:, :, hkv:], lens=torch.zeros(1, dtype=torch.int32, device=DEV), rope=rope)
        own = torch.randn((B, 20, 2 * hkv, d), generator=gen, device=DEV).bfloat16()
        ctx.paged_append(cache, T, own[:, :, :hkv], own[:, :, hkv:], lens=torch.full((B,), L, dtype=torch.int32, device=DEV), counts=counts, rope=rope)
    lens = counts + L
    ids = torch.zeros((B, T), dtype=torch.int32, device=DEV)
    now = torch.tensor([5, 900, 33], dtype=torch.int32, device=DEV)
    rows, logits = torch.zeros((B, 1), dtype=torch.int32, device=DEV), torch.empty((B, V), device=DEV)
    token, conf, commit = torch.empty((B, 1), dtype=torch.int32, device=DEV), torch.empty((B, 1), device=DEV), torch.empty((B, 1), dtype=torch.int32, device=DEV)
    settings = dict(temperature=torch.tensor([0.0, 0.8, 1.5], device=DEV), top_k=torch.tensor([0, 40, 0], dtype=torch.int32, device=DEV),
                    top_p=torch.tensor([1.0, 0.9, 0.95], device=DEV))
    for step in range(steps):
        pos = lens[:, None].contiguous()
        ids.scatter_(1, pos.long(), now[:, None])
        lens = lens + 1
        req = ab.Context.request(B, T, 0, 0, None, pos, *rope, token_ids=ids, n_embed=V)
        x, ys = embed, []
        for n in range(n_layers):
            y = torch.empty((B, 1, D), dtype=torch.bfloat16, device=DEV)
            ctx.recompute_paged(lws[n], req, caches[n], x, int(n > 0), None, 0, y, lens=lens)
            ys.append(y)
            x = y
        u = torch.rand((B, 1), generator=gen, device=DEV)
        ctx.predict_sample(x, 1, rows, B, 1, gain, w_lm, V, logits, u, 0.5, token, conf, commit, **settings)
        assert ctx.poll_status() == 0
        for n in range(n_layers):
            for b in range(B):
                m = int(lens[b])
                k, v = (back(p, table, T)[b, :m] for p in pools[n])
                x_in = embed[now[b].long()][None] if n == 0 else ys[n - 1][b]
                full = torch.zeros((m, D), dtype=torch.bfloat16, device=DEV)
                full[m - 1] = x_in[0]
                ref = orc.layer_step(weights[n], shape, ab.to_host_bits(full), ab.to_host_bits(k), ab.to_host_bits(v), m, 0, 0, np.zeros(0, np.int32),
                                     np.array([m - 1], np.int32), cos, sin, anchor_idx=np.zeros(0, np.int32))
                assert_close_bf16(ab.to_host_bits(ys[n][b]), ref["y"], f"step {step}, layer {n}, request {b}")
                assert_close_bf16(ab.to_host_bits(k[m - 1:]), ref["k_new"], f"step {step}, layer {n}, request {b}: K")
        assert int(token[0]) == int(logits[0].argmax())
        now = token[:, 0].clone()
