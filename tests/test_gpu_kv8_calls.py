"""Calls of the 8-bit cache at the ends of what its arguments may be."""
import numpy as np
import pytest
import torch

from paper_2608_26140_b200 import binding as ab

from helpers import DEV
from test_gpu_kv8 import HEADS, Cache, check_attention, context, filled, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 40])
def test_rows_listed_for_a_context_of_no_tokens(n):
    """No position is inside it: every row is skipped and reported, nothing is written."""
    heads, B, cap = "gqa28", 2, 64
    H, hkv, d = HEADS[heads]
    ctx, cache = context(heads, B, cap), Cache(heads, B, cap, 16, "int8", garbage=True)
    rows = torch.ones((B, n, hkv, d), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros((B, n), dtype=torch.int32, device=DEV)
    ctx.kv8_write(cache.c, B, 0, rows, rows, pos=pos)
    cache.check()
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX
    out = torch.full_like(rows, 7.0)
    ctx.kv8_read(cache.c, B, 0, out, None, pos=pos)
    assert ctx.poll_status() == ab.FLAG_BAD_INDEX and (out == 0).all()
