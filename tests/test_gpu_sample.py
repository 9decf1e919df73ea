"""Sampling (acache_sample_tokens, acache_predict_sample) against the definition in 64 bits: tokens are the same, and

    |prob - ref| <= 2^-24 ref + (V 2^-45 ref + 2^-45) / S     |confidence - ref| <= 2^-17 ref

(prob: rounded once; weights are rounded to half of 2^-44 or less, the one of the token and V of them in the sum S >= 1.  confidence: weights in
fp32, an exponent y <= 40 off by 2^-23 y where the weight matters, 4e-6, sums of up to 64 of them a thread, 4e-6.)
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_26140_b200 import binding as ab
from paper_2608_26140_b200 import workloads as wl

from helpers import DEV

pytestmark = pytest.mark.gpu
INF = math.inf


@pytest.fixture(scope="module")
def ctx():
    return ab.Context(128, 1, 1, 128, 128, 1e-5, 0, 1, 1, 0, 1, 0, DEV)


def reference(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """One row (numpy, fp64): token, prob, confidence, S."""
    l = np.where(np.isnan(logits), -INF, logits.astype(np.float64))
    top = l.max()
    if top == -INF:
        return -1, 0.0, 0.0, 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        below = np.where(l == top, 0.0, l - top)
    conf = np.exp(below)
    conf /= conf.sum()
    order = np.argsort(-l, kind="stable")                   # by the logits: their distances from the largest may round to one
    T = 1.0 if temperature is None else float(temperature)
    if not T > 0:
        return int(order[0]), 1.0, conf[order[0]], 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(np.isneginf(below), 0.0, np.exp(np.where(np.isneginf(below), 0.0, below) / T))[order]
    cum = np.cumsum(w)
    n = int((w > 0).sum())
    k = len(w) if top_k is None or top_k <= 0 else min(int(top_k), len(w))
    k = min(k, n)
    n = k
    if top_p is not None and top_p < 1:
        n = min(n, 1 + int(np.searchsorted(cum[:k], max(float(top_p), 0.0) * cum[k - 1])))
    if min_p is not None and min_p > 0:
        n = min(n, int((w >= min(float(min_p), 1.0)).sum()))
    S = cum[n - 1]
    share = min(max(float(u), 0.0), 1.0) if not math.isnan(u) else 0.0
    i = min(int(np.searchsorted(cum[:n], share * S, side="right")), n - 1)
    return int(order[i]), w[i] / S, conf[order[i]], S


def check(ctx, logits, u, per=1, flags=0, **settings):
    """logits: a tensor on the device; settings: lists (None: not asked for)."""
    rows, vocab = logits.shape
    u = np.asarray(u, np.float32)
    on = {k: None if v is None else torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device=DEV) for k, v in settings.items()}
    token = torch.full((rows,), -7, dtype=torch.int32, device=DEV)
    prob, conf = (torch.full((rows,), -7.0, device=DEV) for _ in range(2))
    ctx.sample_tokens(logits, torch.tensor(u, device=DEV), token, prob=prob, confidence=conf, rows_per_setting=per, **on)
    assert ctx.poll_status() == flags
    host = logits.float().cpu().numpy()
    token, prob, conf = token.cpu().numpy(), prob.cpu().numpy().astype(np.float64), conf.cpu().numpy().astype(np.float64)
    for r in range(rows):
        t, p, c, S = reference(host[r], u[r], **{k: None if v is None else v.cpu().numpy()[r // per] for k, v in on.items()})
        assert token[r] == t, (r, token[r], t, host[r][token[r]], host[r][t])
        assert abs(prob[r] - p) <= 2 ** -24 * p + (vocab * 2 ** -45 * p + 2 ** -45) / S, (r, prob[r], p)
        assert abs(conf[r] - c) <= 2 ** -17 * c, (r, conf[r], c)
    return token


def draw(rng, rows, vocab, dtype, spread=2.3):
    x = rng.standard_normal((rows, vocab)) * spread
    m = min(20, vocab)
    for r in range(rows):
        x[r, rng.integers(0, vocab, m)] += rng.random(m) * 12
    return torch.tensor(x, dtype=torch.float32, device=DEV).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 31, 640, 1003, 16384, 16385, 40000, 126464, 131073, 262144])
def test_settings(ctx, vocab, dtype):
    rng = np.random.default_rng(vocab)
    n = 12
    logits, u = draw(rng, n, vocab, dtype), rng.random(n)
    pick = lambda *v: [v[i % len(v)] for i in range(n)]  # noqa: E731
    check(ctx, logits, u)
    check(ctx, logits, u, temperature=pick(0.0, 0.5, 1.7, 8.0))
    check(ctx, logits, u, temperature=pick(0.7), top_k=pick(1, 2, 50, 0, -3, 1000, vocab, vocab + 5))
    check(ctx, logits, u, temperature=pick(0.8, 2.0), top_p=pick(0.9, 0.5, 0.0, 1.0, 1e-6, 0.999999, 2.0, -1.0))
    check(ctx, logits, u, min_p=pick(0.05, 0.0, 1.0, 1e-9, 3.0, -1.0))
    check(ctx, logits, u, temperature=pick(1.3, 0.3, 3.0), top_k=pick(5, 40, 700, 0, 2000), top_p=pick(0.95, 0.7, 1.0, 0.3), min_p=pick(0.0, 0.02, 0.3))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_equal_logits_go_by_their_index(ctx, dtype):
    rng = np.random.default_rng(3)
    for vocab in (5, 1000, 126464):
        logits = torch.full((8, vocab), 1.25, dtype=dtype, device=DEV)
        u = np.array([0.0, 0.25, 0.5, 0.9999999, 0.125, 0.75, 0.3, 0.6], np.float32)
        token = check(ctx, logits, u)
        assert token[0] == 0 and token[2] == vocab // 2 and token[3] == min(vocab - 1, int(float(u[3]) * vocab))
        check(ctx, logits, u, top_k=[3, 1, 700, vocab, 2, 64, 65, 4], temperature=[0.1, 5.0] * 4)
        check(ctx, logits, u, top_p=[0.5, 0.1, 0.25, 0.75, 1e-7, 0.125, 0.5, 0.0])
        check(ctx, logits, u, temperature=[0.0] * 8)
        few = torch.tensor(rng.integers(0, 4, (8, vocab)) / 4 - 0.5, dtype=dtype, device=DEV)      # 0 and -0 among them
        few[3] *= -1
        check(ctx, few, u, temperature=[0.3, 1.0, 2.0, 0.0] * 2, top_k=[0, vocab // 3 + 1] * 4, top_p=[1.0, 1.0, 0.8, 0.4] * 2)


def test_masked_and_infinite_logits(ctx):
    rng = np.random.default_rng(4)
    vocab = 5000
    logits = draw(rng, 12, vocab, torch.float32)
    u = rng.random(12)
    logits[0, 1:] = -INF                                     # one token left
    logits[1] = -INF
    logits[2, ::2] = torch.finfo(torch.float32).min
    logits[3, 7] = INF
    logits[4, [9, 70, 4000]] = INF
    logits[5, 100:] = -INF
    logits[6] = torch.finfo(torch.float32).min
    logits[7] = torch.finfo(torch.float32).max
    logits[8, 3] = torch.finfo(torch.float32).max
    logits[9, :] = INF
    logits[10, 11] = 3e38
    logits[10, 12] = -3e38
    for settings in (dict(), dict(top_k=[3] * 12), dict(top_p=[0.9] * 12, temperature=[1.5] * 12), dict(min_p=[0.1] * 12), dict(temperature=[0.0] * 12),
                     dict(temperature=[INF] * 12), dict(temperature=[1e-30] * 12), dict(temperature=[1e30] * 12, top_k=[100] * 12)):
        check(ctx, logits, u, **settings)


def test_nan_counts_as_minus_infinity_and_is_reported(ctx):
    rng = np.random.default_rng(5)
    for dtype in (torch.bfloat16, torch.float32):
        logits = draw(rng, 3, 3001, dtype)
        logits[0, 17] = math.nan
        logits[1, :] = math.nan
        logits[2, 3000] = -math.nan
        check(ctx, logits, rng.random(3), flags=ab.FLAG_NONFINITE)


def test_settings_and_random_numbers_out_of_range(ctx):
    rng = np.random.default_rng(6)
    logits = draw(rng, 8, 1000, torch.float32)
    u = [0.0, 1.0 - 2 ** -24, 1.0, 2.0, -1.0, math.nan, INF, -INF]
    check(ctx, logits, u)
    check(ctx, logits, u, temperature=[-1.0, math.nan, -INF, 1e-45, 1e-38, INF, -0.0, 3e38])
    check(ctx, logits, u, top_p=[math.nan, INF, -INF, -1.0, 1e-45, 0.99999994, 1.0, 0.0], top_k=[2 ** 31 - 1, -2 ** 31, 0, 1, 7, 999, 1000, 1001])
    check(ctx, logits, u, min_p=[math.nan, INF, -INF, 1.0, 1e-45, 0.5, 1.0000001, 0.0])


def test_many_different_logits_in_one_bin(ctx):
    """An outlier far below stretches the histogram: the rest differ by less than a bin, and by less than a bin of the next."""
    rng = np.random.default_rng(7)
    for vocab in (3000, 126464):
        x = rng.random((6, vocab)) * 1e-4 + 3.0
        x[:3, 5] = -30.0
        x[1, 6] = -25.0
        x[2, :vocab // 2] += 1e-2
        x[3] = 1.0 + rng.integers(0, 3, vocab) * 2.0 ** -23           # neighbours
        x[4] = np.linspace(-1e-30, 1e-30, vocab)
        x[5, :] = rng.random(vocab) * 1e-38
        x[5, 0] = -20.0
        logits = torch.tensor(x, dtype=torch.float32, device=DEV)
        for u in (rng.random(6), np.full(6, 0.5), np.full(6, 0.99999)):
            check(ctx, logits, u)
            check(ctx, logits, u, top_k=[vocab // 2] * 6, top_p=[0.7] * 6)
            check(ctx, logits, u, top_k=[777] * 6)


def test_rows_that_lie_apart_and_begin_anywhere(ctx):
    rng = np.random.default_rng(8)
    for dtype in (torch.bfloat16, torch.float32):
        wide = draw(rng, 9, 20011, dtype)
        for first, vocab in ((0, 20000), (1, 19999), (3, 1003), (7, 17), (5, 20006), (11, 1)):
            wide[:, first + vocab:first + vocab + 1] = 100.0                  # what is behind a row is not its
            view = wide[:, first:first + vocab]
            check(ctx, view, rng.random(9), top_p=[0.95] * 9)
            wide[:, first + vocab:first + vocab + 1] = 0.0
        check(ctx, wide[2:3, 1:300], rng.random(1))
        one = draw(rng, 1, 300, dtype)
        check(ctx, one.expand(4, 300).contiguous().view(2, 600)[:, :300], [0.3, 0.8])


def test_a_setting_for_several_rows(ctx):
    rng = np.random.default_rng(9)
    logits = draw(rng, 11, 2000, torch.float32)
    check(ctx, logits, rng.random(11), per=4, temperature=[0.0, 0.7, 2.0], top_k=[0, 5, 40], top_p=[1.0, 0.9, 0.5])
    check(ctx, logits, rng.random(11), per=100, temperature=[1.2])


def test_many_rows_and_frequencies(ctx):
    """20000 draws from one distribution: each token's share is within five standard deviations of its probability."""
    vocab, rows = 50, 20000
    gen = torch.Generator(device=DEV).manual_seed(1)
    logits = torch.randn((1, vocab), generator=gen, device=DEV).repeat(rows, 1)
    u = torch.rand((rows,), generator=gen, device=DEV)
    token = torch.empty((rows,), dtype=torch.int32, device=DEV)
    ctx.sample_tokens(logits, u, token)
    p = torch.softmax(logits[0].double(), 0).cpu()
    share = torch.bincount(token.long().cpu(), minlength=vocab).double() / rows
    assert ((share - p).abs() <= 5 * (p * (1 - p) / rows).sqrt()).all()


def test_again_on_another_stream_and_in_a_graph(ctx):
    rng = np.random.default_rng(10)
    logits = draw(rng, 5, 126464, torch.bfloat16)
    u = torch.tensor(rng.random(5), dtype=torch.float32, device=DEV)
    T, p = torch.full((5,), 0.9, device=DEV), torch.full((5,), 0.9, device=DEV)
    token, prob = torch.empty(5, dtype=torch.int32, device=DEV), torch.empty(5, device=DEV)
    ctx.sample_tokens(logits, u, token, prob=prob, temperature=T, top_p=p)
    want = token.clone(), prob.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.sample_tokens(logits, u, token, prob=prob, temperature=T, top_p=p)
    for _ in range(3):
        token.zero_()
        graph.replay()
        assert torch.equal(token, want[0]) and torch.equal(prob, want[1])
    other = draw(rng, 5, 126464, torch.bfloat16)
    logits.copy_(other)
    graph.replay()
    host = other.float().cpu().numpy()
    assert token.tolist() == [reference(host[r], float(u[r]), 0.9, None, np.float32(0.9))[0] for r in range(5)]
    ctx.sample_tokens(logits, u, token)                      # without prob and confidence


def test_refusals(ctx):
    logits, u = torch.zeros((2, 100), device=DEV), torch.zeros(2, device=DEV)
    token = torch.zeros(2, dtype=torch.int32, device=DEV)
    launches = ctx.launch_count()
    for call in (lambda: ctx.sample_tokens(logits.half(), u, token), lambda: ctx.sample_tokens(logits.t(), u, token), lambda: ctx.sample_tokens(logits.cpu(), u, token),
                 lambda: ctx.sample_tokens(logits, u[:1], token), lambda: ctx.sample_tokens(logits, u, token.long()), lambda: ctx.sample_tokens(logits, u.double(), token),
                 lambda: ctx.sample_tokens(logits, u, token, prob=u[:1]), lambda: ctx.sample_tokens(logits, u, token, confidence=u.double()),
                 lambda: ctx.sample_tokens(logits, u, token, temperature=u[:1]), lambda: ctx.sample_tokens(logits, u, token, top_k=u),
                 lambda: ctx.sample_tokens(logits, u, token, top_p=u, rows_per_setting=2)):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: ctx.sample_tokens(logits, u, token, rows_per_setting=0), ab.ERR_INVALID_ARG),
                       (lambda: ctx.sample_tokens(torch.zeros((2, 262145), device=DEV), u, token), ab.ERR_UNSUPPORTED_SHAPE),
                       (lambda: ctx.sample_tokens(logits[:, :0], u, token), ab.ERR_INVALID_ARG),
                       (lambda: ctx.sample_tokens(logits[:1].expand(2, 100), u, token), ab.ERR_INVALID_ARG)):
        with pytest.raises(ab.AcacheError) as e:
            call()
        assert e.value.status == code
    ctx.sample_tokens(logits[:0], u[:0], token[:0])
    assert ctx.launch_count() == launches


@pytest.mark.parametrize("shape,V,B,h_rows,n_blk", [(wl.TINY, 1280, 2, 40, 32), (wl.TINY, 128, 1, 5, 3), (wl.TINY, 2688, 3, 50, 43), (wl.TINY, 16640, 9, 40, 32)])
def test_predict_sample(shape, V, B, h_rows, n_blk):
    """The logits are the LM head's; the tokens are drawn from them; without a temperature they and the commits are predict_commit's."""
    D, rows = shape.hidden, B * n_blk
    gen = torch.Generator(device=DEV).manual_seed(V)
    w_lm = (torch.randn((V, D), generator=gen, device=DEV) * 0.2).bfloat16()
    gain = (1 + 0.05 * torch.randn((D,), generator=gen, device=DEV)).bfloat16()
    h = torch.randn((B, h_rows, D), generator=gen, device=DEV).bfloat16()
    block_rows = torch.stack([torch.randperm(h_rows, generator=gen, device=DEV)[:n_blk] for _ in range(B)]).to(torch.int32) if h_rows >= n_blk else \
        torch.randint(h_rows, (B, n_blk), generator=gen, device=DEV).to(torch.int32)
    ctx = ab.Context.for_shape(shape, B, 64, 32, 8, 8, DEV, max_vocab=V, max_block=n_blk)
    new = lambda: (torch.full((B, n_blk), -1, dtype=torch.int32, device=DEV), torch.zeros((B, n_blk), device=DEV), torch.full((B, n_blk), -1, dtype=torch.int32, device=DEV))  # noqa: E731
    token, conf, commit = new()
    ctx.predict_commit(h, h_rows, block_rows, B, n_blk, gain, w_lm, V, 0.3, token, conf, commit)
    logits = torch.full((rows, V), 7.0, device=DEV)
    u = torch.rand((B, n_blk), generator=gen, device=DEV)
    zero = torch.zeros(B, device=DEV)
    got = new()
    ctx.predict_sample(h, h_rows, block_rows, B, n_blk, gain, w_lm, V, logits, u, 0.3, *got, temperature=zero, rows_per_setting=n_blk)
    assert torch.equal(got[0], token) and torch.equal(got[2], commit)
    assert ((got[1] - conf).abs() <= 2e-5 * conf).all()                       # both from fp32 sums of the same logits, the other by a fast exponential
    x = h.gather(1, block_rows.long()[..., None].expand(B, n_blk, D)).double()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + shape.rms_eps) * gain.double()
    ref = (x.reshape(rows, D) @ w_lm.double().T)
    size = x.reshape(rows, D).abs() @ w_lm.double().abs().T
    assert ((logits.double() - ref).abs() <= (2 ** -8 + (D + 8) * 2 ** -24) * size).all()      # the normed row is rounded to bf16; sums in fp32
    T, k, p = torch.full((rows,), 0.8, device=DEV), torch.full((rows,), 30, dtype=torch.int32, device=DEV), torch.full((rows,), 0.9, device=DEV)
    ctx.predict_sample(h, h_rows, block_rows, B, n_blk, gain, w_lm, V, logits, u, 0.3, *got, temperature=T, top_k=k, top_p=p)
    host = logits.cpu().numpy()
    flat_u, flat_t, flat_c = u.view(-1).tolist(), got[0].view(-1).tolist(), got[1].view(-1).tolist()
    for r in range(rows):
        t, _, c, _ = reference(host[r], flat_u[r], np.float32(0.8), 30, np.float32(0.9))
        assert flat_t[r] == t and abs(flat_c[r] - c) <= 2 ** -17 * c
    over = got[1] > 0.3
    best = got[1].argmax(1)
    want = torch.where(over.any(1, keepdim=True), over, torch.arange(n_blk, device=DEV) == best[:, None])
    assert torch.equal(got[2] != 0, want)
    assert ctx.poll_status() == 0
