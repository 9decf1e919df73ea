"""Sampling of so many rows that other kernels are used (bf16 rows in larger parts, fp32 rows that are read again instead of held), against 64 bits as
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
