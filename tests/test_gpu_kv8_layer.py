"""The layer-step on an 8-bit cache apart from scoring, selecting and recomputing in one call (test_gpu_kv8.py): scores without a selection,
before and after the rows are written, accumulated, without a recompute; compact inputs; nothing to do; what its stages take."""
import numpy as np
import pytest
import torch

from oracle import acache_oracle as orc
from paper_2608_26140_b200 import binding as ab
from paper_2608_26140_b200 import workloads as wl

from helpers import DEV, DeviceCase

pytestmark = pytest.mark.gpu

MID = wl.LayerShape(512, 8, 2, 128, 768, 1e-6, True, 1e6, "mid-gqa")


class Step:
    """A case on the device and 8-bit caches made of its bf16 one."""

    def __init__(self, shape, lay, block, fmt):
        self.case, self.shape, self.lay, self.block, self.fmt = wl.make_case(shape, lay, 0.0, 0), shape, lay, block, fmt
        self.dc = DeviceCase(self.case)
        self.ctx = self.dc.ctx

    def cache(self):
        keep, c = self.ctx.new_kv8(self.lay.batch, self.lay.ctx_len, self.block, self.fmt)
        T = self.lay.ctx_len
        self.ctx.kv8_write(c, self.lay.batch, T, self.dc.ck[:, :T], self.dc.cv[:, :T])
        return keep, c

    def keys(self, c):
        lay = self.lay
        k = torch.empty((lay.batch, lay.ctx_len, self.shape.n_kv_heads, self.shape.head_dim), dtype=torch.bfloat16, device=DEV)
        self.ctx.kv8_read(c, lay.batch, lay.ctx_len, k, None)
        return orc.bf16_bits_to_f64(ab.to_host_bits(k))

    def scores(self, keys, norm_full):
        """The oracle's, on these keys."""
        case, lay = self.case, self.lay
        out = []
        for b in range(lay.batch):
            pos = lay.masked_pos[b]
            q = orc.masked_queries(case.weights, self.shape, orc.bf16_bits_to_f64(case.x[b])[pos], pos, case.rope_cos, case.rope_sin)
            out.append(orc.score_anchors(q, keys[b][lay.affix_start:lay.affix_start + lay.affix_len], keys[b], lay.affix_start, norm_full))
        return np.stack(out)

    def run(self, c, flags, scores=None, anchors=None, ratio=0.0, x=None, req=None):
        rows = orc.k_from_ratio(self.lay.affix_len, ratio) + self.lay.n_extra
        y = torch.full((self.lay.batch, rows, self.shape.hidden), 7.0, dtype=torch.bfloat16, device=DEV)
        self.ctx.layer_step_kv8(self.dc.lw, req or self.dc.req, c, self.dc.x if x is None else x, int(x is not None), ratio, flags, scores, anchors, y)
        return y


def assert_scores(got, ref):
    # Eq. 4-5 from bf16 products summed in fp32: the bound the other scoring tests use
    assert np.all(np.abs(got.cpu().numpy() - ref) <= 1e-3 * np.maximum(ref, ref.mean(axis=1, keepdims=True)))


LAYOUTS = [(wl.TINY, (2, 8, 131, 37, 32, 32, "all"), 16, "int8"), (MID, (3, 5, 300, 33, 40, 32, "all"), 64, "e4m3"), (MID, (1, 0, 257, 9, 32, 20, "masked"), 128, "int8")]


@pytest.mark.parametrize("norm_full", [False, True])
@pytest.mark.parametrize("shape,layout,block,fmt", LAYOUTS)
def test_scores_of_a_probe(shape, layout, block, fmt, norm_full):
    """No anchors, no selection: with the softmax over all keys the scores are of the cache with the fresh rows in it, else of the cache as
    given.  Rows, cache and output are what they are without scores, and with the rows of x alone."""
    s = Step(shape, wl.make_layout(*layout), block, fmt)
    keep, c = s.cache()
    before = s.keys(c)
    flags = ab.F_SCORE_NORM_FULL if norm_full else 0
    scores = torch.full((s.lay.batch, s.lay.affix_len), 5.0, dtype=torch.float32, device=DEV)
    y = s.run(c, ab.F_SCORE | flags, scores)
    assert s.ctx.poll_status() == 0
    after = s.keys(c)
    assert not np.array_equal(before, after)
    assert_scores(scores, s.scores(after if norm_full else before, norm_full))
    keep2, c2 = s.cache()
    y2 = s.run(c2, 0)
    compact = torch.gather(s.dc.x, 1, torch.from_numpy(s.lay.extra_rows).long().to(DEV)[:, :, None].expand(-1, -1, shape.hidden)).contiguous()
    keep3, c3 = s.cache()
    scores3 = torch.zeros_like(scores)
    y3 = s.run(c3, ab.F_SCORE | flags, scores3, x=compact)
    assert torch.equal(y, y2) and torch.equal(y, y3) and torch.equal(scores, scores3)
    assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(keep, keep2, keep3))
    assert s.ctx.poll_status() == 0


@pytest.mark.parametrize("norm_full", [False, True])
@pytest.mark.parametrize("shape,layout,block,fmt", LAYOUTS)
def test_scores_alone(shape, layout, block, fmt, norm_full):
    """Without a recompute, added to what is there or not: cache and output are left alone.  What earlier calls left in the workspace does not
    matter: the call before read a cache of NaN back."""
    s = Step(shape, wl.make_layout(*layout), block, fmt)
    keep, c = s.cache()
    odd, codd = s.ctx.new_kv8(s.lay.batch, s.lay.ctx_len, block, "e4m3")
    odd[0].fill_(0x7F)
    odd[2].fill_(127)
    flags = ab.F_SCORE | ab.F_NO_RECOMPUTE | (ab.F_SCORE_NORM_FULL if norm_full else 0)
    before, was = s.keys(c), [t.clone() for t in keep]
    ref = s.scores(before, norm_full)
    for accumulate in (False, True):
        scores = torch.zeros((s.lay.batch, s.lay.affix_len), dtype=torch.float32, device=DEV)
        s.run(codd, ab.F_SCORE | ab.F_NO_RECOMPUTE | ab.F_SCORE_NORM_FULL, scores)
        scores.fill_(2.0)
        y = s.run(c, flags | (ab.F_ACCUMULATE if accumulate else 0), scores)
        assert_scores(scores - 2.0 if accumulate else scores, ref)
        assert (y == 7.0).all() and all(torch.equal(p, q) for p, q in zip(keep, was))
    assert s.ctx.poll_status() == 0


@pytest.mark.parametrize("shape,layout,block,fmt", LAYOUTS)
def test_compact_rows_with_anchors(shape, layout, block, fmt):
    s = Step(shape, wl.make_layout(*layout), block, fmt)
    ratio, L = 0.2, s.lay.affix_len
    K = orc.k_from_ratio(L, ratio)
    g = np.random.default_rng(1)
    a = np.stack([np.sort(g.choice(L, K, replace=False)) for _ in range(s.lay.batch)]).astype(np.int32)
    anchors = torch.from_numpy(a).to(DEV)
    rows = np.concatenate([a + s.lay.affix_start, s.lay.extra_rows], axis=1)
    compact = torch.gather(s.dc.x, 1, torch.from_numpy(rows).long().to(DEV)[:, :, None].expand(-1, -1, shape.hidden)).contiguous()
    results = []
    for x in (None, compact):
        keep, c = s.cache()
        results.append([s.run(c, 0, None, anchors, ratio, x), *keep])
    assert all(torch.equal(p, q) for p, q in zip(*results)) and s.ctx.poll_status() == 0


def test_nothing_to_do():
    s = Step(MID, wl.make_layout(2, 0, 200, 8, 32, 32, "masked"), 32, "int8")
    keep, c = s.cache()
    was = [t.clone() for t in keep]
    scores = torch.full((2, 200), 5.0, dtype=torch.float32, device=DEV)
    K = orc.k_from_ratio(200, 0.25)
    anchors = torch.full((2, K), -1, dtype=torch.int32, device=DEV)
    launched = s.ctx.launch_count()
    none = ab.Context.request(0, s.lay.ctx_len, 0, 200, s.dc.masked, s.dc.extra, s.dc.cos, s.dc.sin)
    s.run(c, ab.F_SCORE | ab.F_SELECT, scores, anchors, 0.25, req=none)
    assert s.ctx.launch_count() == launched
    # no masked rows: zero scores, the lowest positions
    unmasked = ab.Context.request(2, s.lay.ctx_len, 0, 200, None, s.dc.extra, s.dc.cos, s.dc.sin)
    s.run(c, ab.F_SCORE | ab.F_SELECT | ab.F_NO_RECOMPUTE, scores, anchors, 0.25, req=unmasked)
    assert (scores == 0).all() and torch.equal(anchors, torch.arange(K, dtype=torch.int32, device=DEV).expand(2, K))
    assert all(torch.equal(p, q) for p, q in zip(keep, was)) and s.ctx.poll_status() == 0


def test_stage_times_hold_the_keys_that_are_read_back():
    """Scores on many keys: the stages' times add up to the call's."""
    shape = wl.LayerShape(512, 32, 32, 128, 512, 1e-5, False, 5e5, "wide-heads")
    B, T = 4, 8192
    s = Step(shape, wl.make_layout(1, 0, T - 40, 8, 32, 32, "masked"), 64, "int8")
    ctx = ab.Context.for_shape(shape, B, T, T - 40, 32, 32, DEV)
    keep, c = ctx.new_kv8(B, T, 64, "int8")
    keep[2].fill_(120)
    x = s.dc.x.expand(B, T, 512).contiguous()
    pos = s.dc.masked.expand(B, 32).contiguous()
    req = ab.Context.request(B, T, 0, T - 40, pos, pos, s.dc.cos, s.dc.sin)
    scores = torch.zeros((B, T - 40), dtype=torch.float32, device=DEV)
    shares = []
    ctx.stage_timing(True)
    for i in range(12):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        ctx.layer_step_kv8(s.dc.lw, req, c, x, 0, 0.0, ab.F_SCORE | ab.F_SCORE_NORM_FULL | ab.F_NO_RECOMPUTE, scores, None, None)
        b.record()
        shares.append(sum(ctx.read_stage_times().values()) / a.elapsed_time(b))
    assert ctx.poll_status() == 0
    assert np.median(shares[2:]) > 0.8, shares
