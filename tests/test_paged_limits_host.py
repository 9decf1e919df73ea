"""The largest calls on a cache in pages, without a GPU: what cannot be counted in 32 bits is refused before anything is enqueued."""
import ctypes as C

import pytest
import torch

from paper_2608_26140_b200 import binding as ab
from paper_2608_26140_b200 import build as abuild

B, T, ROWS, HIDDEN, H, HKV, D = 4096, 1 << 20, 2048, 256, 4, 2, 64


@pytest.fixture
def handle():
    if torch.cuda.is_available():
        pytest.skip("the workspace of this test is no memory")
    abuild.build()
    lib, h = ab.load_library(), C.c_void_p()
    assert lib.acache_create(C.byref(ab.ModelDesc(HIDDEN, H, HKV, D, 1024, 1e-5, 0, B, T, 128, ROWS, 32, 0, 0)), C.byref(h)) == ab.OK
    # the address is taken before the call fails for want of a GPU; no refused call touches it
    assert lib.acache_set_workspace(h, 1 << 20, lib.acache_workspace_bytes(h), None) == ab.ERR_CUDA
    yield lib, h
    assert lib.acache_launch_count(h) == 0
    lib.acache_destroy(h)


def refresh(lib, h, batch, ctx_len, rows):
    w = ab.LayerWeights(*[256] * 12)
    kv = ab.PagedKV(4096, 8192, HKV * 64 * D, 8, 64, 256, T // 64)
    req = ab.Request(batch, ctx_len, 0, 0, None, 0, 256, rows, 256, 256, None, 0)
    return lib.acache_recompute_paged(h, C.byref(w), C.byref(req), C.byref(kv), 256, 1, None, 0, None, 256, None)


def attend(lib, h, batch, ctx_len, rows):
    kv = ab.PagedKV(4096, 8192, HKV * 64 * D, 8, 64, 256, 1 << 25)
    return lib.acache_paged_attention(h, C.byref(kv), batch, rows, ctx_len, 256, None, None, 256, None, None)


@pytest.mark.parametrize("call", [refresh, attend])
def test_too_many_units(handle, call):
    """Units: tiles of 32 rows (2048 rows of 2 heads: 128) x KV heads x requests x (keys / 64 and 5 more)."""
    assert call(*handle, B, T, ROWS) == ab.ERR_UNSUPPORTED_SHAPE                 # 2^20 * 16389
    most = (2 ** 31 - 1) // (2 ** 20)                                            # 2047 units an item
    assert call(*handle, B, (most - 5) * 64 + 1, ROWS) == ab.ERR_UNSUPPORTED_SHAPE
    assert call(*handle, B, (most - 5) * 64, ROWS) == ab.ERR_CUDA                # as far as the launch, which wants a GPU
    assert call(*handle, 1, T, 1) == ab.ERR_CUDA


def test_units_that_pass_64_bits(handle):
    """2^25 tiles x 2 x 2^12 x 2^24 units are 2^62, which times a little more would come round to a small number."""
    assert attend(*handle, B, 1 << 30, 1 << 29) == ab.ERR_UNSUPPORTED_SHAPE
    assert attend(*handle, B, 1 << 30, 0) == ab.OK
