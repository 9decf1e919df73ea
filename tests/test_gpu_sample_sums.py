"""Searches by weight alone, where no counts were added up, after rows that left counts of their own behind in the same memory."""
import numpy as np
import pytest
import torch

from test_gpu_sample import check, ctx  # noqa: F401  (a fixture)

from helpers import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [640, 5000, 20000, 126464])
def test_a_search_by_weight_after_one_by_rank(ctx, vocab):  # noqa: F811
    rng = np.random.default_rng(vocab)
    rows = 160
    by_rank = torch.tensor(rng.standard_normal((rows, vocab)), dtype=torch.float32, device=DEV)
    x = rng.random((12, vocab)) * 1e-4 + 3.0                     # a bin holds more of them than are sorted at once
    x[:, 7] = -20.0
    close = torch.tensor(x, dtype=torch.float32, device=DEV)
    u = rng.random(12)
    for _ in range(3):
        check(ctx, by_rank, rng.random(rows), top_k=[2000] * rows, top_p=[0.9] * rows)
        check(ctx, close, u, top_p=[0.7] * 12)
        check(ctx, by_rank[:37], rng.random(37), top_k=[1500, 0, 300, 0, 0] * 7 + [0, 5])
        check(ctx, close, u)
        check(ctx, close.bfloat16(), u, min_p=[0.5] * 12)
