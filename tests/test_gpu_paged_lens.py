"""A refresh over a cache in pages in which each request has a length of its own: keys behind it do not count, whatever the pages hold there."""
import numpy as np
import pytest
import torch

from oracle import acache_oracle as orc
from paper_2608_26140_b200 import binding as ab
from paper_2608_26140_b200 import workloads as wl

from helpers import DEV, DeviceCase, assert_close_bf16
from test_gpu_paged_layer import MID, back, pages_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("compact", [0, 1])
@pytest.mark.parametrize("shape,page,lens", [(wl.TINY, 16, (20, 330, 377)), (MID, 64, (378, 65, 306)), (MID, 8, (129, 378, 1)), (wl.TINY, 1, (63, 64, 301))])
def test_keys_behind_a_length_do_not_count(shape, page, lens, compact):
    """Two of the rows of R lie behind the length (where it leaves room): they are computed and stored like any other, but attend what
    lies before it.  The places that no row of R takes hold NaN there."""
    rng = np.random.default_rng(page)
    B, start, L, T, e, K = 3, 5, 300, 378, 9, 40
    outside = np.concatenate([np.arange(start), np.arange(start + L, T)])
    extra = np.stack([rng.permutation(outside)[:e] for _ in range(B)]).astype(np.int32)
    masked = np.tile(np.arange(T - 32, T, dtype=np.int32), (B, 1))
    lay = wl.Layout(B, T, start, L, masked, extra)
    case = wl.make_case(shape, lay, 0.0, 0)
    dc = DeviceCase(case, max_rows=K + e)
    anchors = np.stack([np.sort(rng.choice(L, K, replace=False)) for _ in range(B)]).astype(np.int32)
    k_pool, v_pool, table, cache = pages_of(dc.ctx, dc.ck[:, :T], dc.cv[:, :T], page, 3)
    stored = [back(p, table, T).clone() for p in (k_pool, v_pool)]
    # NaN behind each length, where no row of R will be written
    slots = torch.arange(table.shape[1] * page, device=DEV)
    for b in range(B):
        fresh = torch.zeros(len(slots), dtype=torch.bool, device=DEV)
        fresh[torch.from_numpy(np.concatenate([anchors[b] + start, extra[b]])).long().to(DEV)] = True
        at = slots[(slots >= lens[b]) & ~fresh]
        for pool in (k_pool, v_pool):
            pool[table[b].long()[at // page], :, at % page] = float("nan")
    rows = np.concatenate([anchors + start, extra], 1)
    x = dc.x
    if compact:
        x = torch.gather(dc.x, 1, torch.from_numpy(rows.astype(np.int64)).to(DEV)[..., None].expand(-1, -1, shape.hidden)).contiguous()
    y = torch.full((B, K + e, shape.hidden), 7.0, dtype=torch.bfloat16, device=DEV)
    dc.ctx.recompute_paged(dc.lw, dc.req, cache, x, compact, torch.from_numpy(anchors).to(DEV), K, y, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    assert dc.ctx.poll_status() == 0
    for b in range(B):
        want = orc.recompute_rows(case.weights, shape, orc.bf16_bits_to_f64(case.x[b])[rows[b]], rows[b], case.cache_k[b], case.cache_v[b], T, case.rope_cos,
                                  case.rope_sin, True, np.arange(T) < lens[b])
        assert_close_bf16(ab.to_host_bits(y[b]), want["y"], f"y of request {b}, {lens[b]} tokens")
        now = [back(p, table, T)[b] for p in (k_pool, v_pool)]
        for got, old, new in zip(now, stored, (want["k_new"], want["v_new"])):
            assert_close_bf16(ab.to_host_bits(got[rows[b]]), new, f"rows of request {b}")
            keep = np.setdiff1d(np.arange(lens[b]), rows[b])
            assert torch.equal(got[keep], old[b][keep])
