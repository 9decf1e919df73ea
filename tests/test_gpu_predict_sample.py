"""Predict-then-commit with drawn tokens (acache_predict_sample): rows that have no token, beside the commit of the same rows to the sequence."""
import pytest
import torch

from paper_2608_26140_b200 import binding as ab
from paper_2608_26140_b200 import workloads as wl

from helpers import DEV

pytestmark = pytest.mark.gpu


class Head:
    """A context, an LM head and the block rows of a few requests."""

    def __init__(self, V, B, n_blk, seed, shape=wl.TINY):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.V, self.B, self.n, D = V, B, n_blk, shape.hidden
        self.w_lm = (torch.randn((V, D), generator=gen, device=DEV) * 0.2).bfloat16()
        self.gain = torch.ones((D,), device=DEV).bfloat16()
        self.h = torch.randn((B, n_blk, D), generator=gen, device=DEV).bfloat16()
        self.rows = torch.arange(n_blk, device=DEV).to(torch.int32).repeat(B, 1).contiguous()
        self.u = torch.rand((B, n_blk), generator=gen, device=DEV)
        self.logits = torch.empty((B * n_blk, V), device=DEV)
        self.ctx = ab.Context.for_shape(shape, B, 64, 32, 8, 8, DEV, max_vocab=V, max_block=n_blk)

    def out(self):
        i32 = dict(dtype=torch.int32, device=DEV)
        return torch.full((self.B, self.n), 7, **i32), torch.full((self.B, self.n), 7.0, device=DEV), torch.full((self.B, self.n), 7, **i32)

    def sample(self, threshold, **settings):
        out = self.out()
        self.ctx.predict_sample(self.h, self.n, self.rows, self.B, self.n, self.gain, self.w_lm, self.V, self.logits, self.u, threshold, *out, **settings)
        return out


@pytest.mark.parametrize("n_blk", [1, 3, 33, 70])
@pytest.mark.parametrize("threshold", [-1.0, 0.0, 2.0])
def test_a_row_without_a_token_is_not_committed(n_blk, threshold):
    """Hidden rows of NaN have logits of NaN, and those no token.  Request 0 has none at all, request 1 one row that has a token, request 2 all but one."""
    head = Head(640, 3, n_blk, 5)
    nan = torch.zeros((3, n_blk), dtype=torch.bool, device=DEV)
    nan[0] = True
    nan[1] = torch.arange(n_blk, device=DEV) != n_blk - 1
    nan[2] = torch.arange(n_blk, device=DEV) == n_blk // 2
    head.h[nan] = float("nan")
    token, conf, commit = head.sample(threshold, temperature=torch.full((3 * n_blk,), 0.7, device=DEV))
    assert head.ctx.poll_status() == ab.FLAG_NONFINITE
    assert torch.equal(token < 0, nan) and (token[nan] == -1).all() and (conf[nan] == 0).all()
    assert (conf[~nan] > 0).all()
    over = ~nan & (conf > threshold)
    best = torch.where(nan, -1.0, conf).argmax(1)
    only = (torch.arange(n_blk, device=DEV) == best[:, None]) & ~nan
    want = torch.where(over.any(1, keepdim=True), over, only)
    assert torch.equal(commit != 0, want) and commit.max() <= 1 and commit.min() >= 0
    # the sequence: what has no token stays masked
    ids = torch.full((3, 2 * n_blk), 999, dtype=torch.int32, device=DEV)
    block = (torch.arange(n_blk, device=DEV) * 2 + 1).to(torch.int32).repeat(3, 1).contiguous()
    left = torch.empty(3, dtype=torch.int32, device=DEV)
    head.ctx.commit_update(ids, 2 * n_blk, block, 3, n_blk, token, conf, 999, threshold, left)
    assert torch.equal(ids[:, 1::2], torch.where(want, token, 999)) and (ids[:, ::2] == 999).all()
    assert torch.equal(left, (n_blk - want.sum(1)).to(torch.int32))
    assert head.ctx.poll_status() == 0


def test_tensors_that_do_not_fit_are_refused_before_any_launch():
    head = Head(640, 2, 3, 5)
    token, conf, commit = head.out()
    good = dict(h=head.h, h_rows=3, block_rows=head.rows, batch=2, n_blk=3, final_norm_g=head.gain, w_lm=head.w_lm, vocab=640, logits=head.logits, u=head.u, threshold=0.5,
                token=token, confidence=conf, commit=commit)
    launches = head.ctx.launch_count()
    for bad in (dict(token=token.long()), dict(token=token.cpu()), dict(token=token[:1]), dict(confidence=conf.double()), dict(confidence=conf.view(-1)[:5]), dict(commit=commit[:1]),
                dict(commit=commit.cpu()), dict(h=head.h.cpu()), dict(h=head.h.float()), dict(h=head.h[:1]), dict(h=head.h.transpose(0, 1)), dict(block_rows=head.rows.long()),
                dict(block_rows=head.rows[:1]), dict(final_norm_g=head.gain.float()), dict(w_lm=head.w_lm[:639]), dict(w_lm=head.w_lm.cpu())):
        with pytest.raises(ValueError):
            head.ctx.predict_sample(**{**good, **bad})
    assert head.ctx.launch_count() == launches
    head.ctx.predict_sample(**good)
    assert head.ctx.launch_count() > launches and head.ctx.poll_status() == 0 and (token >= 0).all()


def committed(conf, threshold):
    over = conf > threshold
    first = torch.arange(conf.shape[1], device=DEV) == conf.argmax(1)[:, None]
    return torch.where(over.any(1, keepdim=True), over, first).to(torch.int32)


@pytest.mark.parametrize("V,B,n_blk", [(16640, 9, 32), (640, 2, 40)])
def test_without_a_temperature(V, B, n_blk):
    """Tokens are the arg max's, and each call's commits follow from its own confidences, also at thresholds that one of those equals.

    How far the confidences may differ, in roundings of 2^-24.  An exponential is off by 4 + 2.4 |x| of them (2 + 1.17 |x| units in the last place), |x| on
    average over a row's weight at most ln(262144) = 12.5: 34.  One call adds 128 terms in a row (128) with 4 corrections of 6 (24) and joins some 14 such sums by
    two exponentials, two products and an addition each (112); the other adds 36 in a row, behind up to 32 corrections of 6 (228).  560 in all, below 2^-14."""
    head = Head(V, B, n_blk, V)
    zero = torch.zeros(B, device=DEV)
    conf = head.sample(0.5, temperature=zero, rows_per_setting=n_blk)[1]
    for t in (0.9, 0.3, 0.0, float(conf[0, 0]), float(conf[-1, -1]), float(conf.max()), float(conf.min())):
        token, conf, commit = head.sample(t, temperature=zero, rows_per_setting=n_blk)
        arg = head.out()
        head.ctx.predict_commit(head.h, n_blk, head.rows, B, n_blk, head.gain, head.w_lm, V, t, *arg)
        assert torch.equal(token, arg[0]) and torch.equal(token.view(-1), head.logits.argmax(1).to(torch.int32))
        assert ((conf - arg[1]).abs() <= 2 ** -14 * arg[1]).all()
        assert torch.equal(commit, committed(conf, t)) and torch.equal(arg[2], committed(arg[1], t))
