"""Sampling of so many rows that other kernels are used (rows in larger parts, read again instead of held), against 64 bits as
in test_gpu_sample.py."""
import math

import numpy as np
import pytest
import torch

from paper_2608_26140_b200 import binding as ab

from helpers import DEV
from test_gpu_sample import check, ctx, draw  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(40, 126464), (39, 126465), (19, 262143), (297, 1280), (300, 17)])
def test_settings(ctx, rows, vocab, dtype):  # noqa: F811
    rng = np.random.default_rng(vocab)
    logits, u = draw(rng, rows, vocab, dtype), rng.random(rows)
    pick = lambda *v: [v[i % len(v)] for i in range(rows)]  # noqa: E731
    check(ctx, logits, u, temperature=pick(0.0, 0.5, 1.7, 8.0, 1.0), top_p=pick(0.9, 1.0, 0.3))
    check(ctx, logits, u, temperature=pick(1.3, 0.3, 3.0), top_k=pick(5, 40, 700, 0, 2000, 1024, 1025), top_p=pick(0.95, 0.7, 1.0, 0.3), min_p=pick(0.0, 0.02, 0.3))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_are_odd(ctx, dtype):  # noqa: F811
    """NaN, infinities, masks, ties, neighbours in one bin, rows that begin anywhere."""
    rng = np.random.default_rng(1)
    rows, vocab = 320, 5003
    wide = draw(rng, rows, vocab + 9, dtype)
    logits = wide[:, 3:3 + vocab]
    wide[:, 2], wide[:, 3 + vocab] = 90.0, 90.0               # not theirs
    logits[0] = -math.inf
    logits[1, 7] = math.inf
    logits[2, [1, 4000, vocab - 1]] = math.inf
    logits[3] = 0.5
    logits[4] = torch.finfo(dtype).min
    logits[5, ::3] = torch.finfo(dtype).min
    logits[6] = torch.tensor(rng.integers(0, 3, vocab) / 2.0)
    logits[7] = torch.tensor(rng.random(vocab) * 1e-4 + 3.0)
    logits[7, 11] = -30.0
    logits[8, 1:] = -math.inf
    logits[9, :vocab - 1] = -math.inf
    u = rng.random(rows)
    for settings in (dict(), dict(top_k=[600] * rows), dict(top_p=[0.8] * rows, temperature=[1.5] * rows), dict(temperature=[0.0] * rows), dict(min_p=[0.05] * rows)):
        check(ctx, logits, u, **settings)
    logits[10, 20] = math.nan
    logits[11] = math.nan
    logits[12, 1:] = math.nan
    logits[13, 0], logits[13, vocab - 1] = math.nan, -math.nan
    for settings in (dict(), dict(top_k=[50] * rows), dict(temperature=[0.0] * rows)):
        check(ctx, logits, u, flags=ab.FLAG_NONFINITE, **settings)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_row_gives_the_same_alone_and_among_others(ctx, dtype):  # noqa: F811
    """Sums are exact, so the token and its probability do not depend on how the row is cut."""
    rng = np.random.default_rng(2)
    rows, vocab = 64, 100000
    logits = draw(rng, rows, vocab, dtype)
    u = torch.tensor(rng.random(rows), dtype=torch.float32, device=DEV)
    T, p = torch.full((rows,), 1.1, device=DEV), torch.full((rows,), 0.95, device=DEV)
    token, prob = torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV)
    ctx.sample_tokens(logits, u, token, prob=prob, temperature=T, top_p=p)
    one, one_prob = torch.empty(1, dtype=torch.int32, device=DEV), torch.empty(1, device=DEV)
    for r in (0, 17, 63):
        ctx.sample_tokens(logits[r:r + 1], u[r:r + 1], one, prob=one_prob, temperature=T[r:r + 1], top_p=p[r:r + 1])
        assert one[0] == token[r] and one_prob[0] == prob[r]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 8191), (5, 4097), (16, 32003), (33, 262144), (64, 50257), (65, 8200), (129, 40961), (257, 9000), (70, 151937), (130, 65537)])
def test_rows_cut_in_every_way(ctx, rows, vocab, dtype):  # noqa: F811
    rng = np.random.default_rng(rows)
    logits, u = draw(rng, rows, vocab, dtype), rng.random(rows)
    pick = lambda *v: [v[i % len(v)] for i in range(rows)]  # noqa: E731
    check(ctx, logits, u, temperature=pick(1.0, 0.6, 2.5, 0.0), top_k=pick(0, 0, 30, 900, 3000), top_p=pick(1.0, 0.9, 0.4), min_p=pick(0.0, 0.0, 0.0, 0.05))


@pytest.mark.parametrize("dtype,rows,vocab", [(torch.float32, 33, 262144), (torch.bfloat16, 300, 80000), (torch.float32, 257, 65536)])
def test_sums_that_fill_their_words(ctx, dtype, rows, vocab):  # noqa: F811
    """All but one token weigh a unit less than the largest, so that each of a weight's parts is as large as it can be; in whole numbers."""
    shift = 46 if vocab <= 65536 else 45 if vocab <= 131072 else 44
    logits = torch.zeros((rows, vocab), device=DEV, dtype=dtype)
    logits[:, 77] = 1.0
    temperature = torch.full((rows,), 2.0 ** shift, device=DEV)
    unit, less = 1 << shift, (1 << shift) - 1                # 2^shift exp(-2^-shift) = 2^shift - 1 + 2^-(shift + 1)
    u = torch.linspace(0.0, 1.0, rows, device=DEV)
    u[-1] = 0.999999
    token, prob = torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV)
    ctx.sample_tokens(logits, u, token, prob=prob, temperature=temperature)
    kept = unit + (vocab - 1) * less
    for r, share in enumerate(u.tolist()):
        drawn = int(share * float(kept))
        i = 0 if drawn < unit else 1 + (drawn - unit) // less          # in the order of falling logits
        assert int(token[r]) == (77 if i == 0 else i - 1 if i - 1 < 77 else i), (r, share)
        assert abs(float(prob[r]) * kept / (unit if i == 0 else less) - 1) <= 2.0 ** -24
    assert ctx.poll_status() == 0
