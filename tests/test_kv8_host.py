"""Host side of the 8-bit cache, without a GPU: calls that are refused before any launch, the handle's checks, the key mask's bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2608_26140_b200 import binding as ab
from paper_2608_26140_b200 import build as abuild


@pytest.fixture(scope="module")
def lib():
    abuild.build()
    return ab.load_library()


def test_calls_without_workspace_are_rejected(lib):
    h = C.c_void_p()
    assert lib.acache_create(C.byref(ab.ModelDesc(256, 4, 4, 64, 1024, 1e-5, 0, 2, 256, 128, 64, 32, 0, 0)), C.byref(h)) == ab.OK
    kv = ab.KV8(256, 256, 256, 256, 4 * 256 * 64, 256, 64, ab.KV8_FORMATS["int8"])
    assert lib.acache_kv8_write(h, C.byref(kv), 1, 256, 256, 256, 0, 1, None, 0, None) == ab.ERR_WORKSPACE
    assert lib.acache_kv8_read(h, C.byref(kv), 1, 256, 256, 256, 1, None, 0, None) == ab.ERR_WORKSPACE
    assert lib.acache_kv8_attention(h, C.byref(kv), 1, 1, 256, 256, None, None, 256, None, None) == ab.ERR_WORKSPACE
    for call in (lambda: lib.acache_kv8_write(None, C.byref(kv), 1, 256, 256, 256, 0, 1, None, 0, None),
                 lambda: lib.acache_kv8_read(None, C.byref(kv), 1, 256, 256, 256, 1, None, 0, None),
                 lambda: lib.acache_kv8_attention(None, C.byref(kv), 1, 1, 256, 256, None, None, 256, None, None)):
        assert call() == ab.ERR_INVALID_ARG
    assert lib.acache_launch_count(h) == 0
    lib.acache_destroy(h)


def test_the_handle_wants_codes_and_exponents_that_go_together():
    codes, exps = torch.zeros((2, 4, 128, 64), dtype=torch.uint8), torch.zeros((2, 4, 2), dtype=torch.uint8)
    c = ab.Context.kv8(codes, codes.clone(), exps, exps.clone(), 64, ab.KV8_FORMATS["e4m3"])
    assert (c.batch_stride, c.ctx_capacity, c.block, c.format) == (4 * 128 * 64, 128, 64, 0)
    assert ab.Context.kv8(codes, codes, exps, exps, 64, 0, shared=True).batch_stride == 0
    apart = torch.zeros((2, 8, 128, 64), dtype=torch.uint8)[:, :4]          # requests further apart than their codes take
    assert ab.Context.kv8(apart, apart.clone().new_zeros((2, 8, 128, 64))[:, :4], exps, exps, 64, 0).batch_stride == 8 * 128 * 64
    for bad in ((codes, codes, exps, exps, 32), (codes, codes[:1], exps, exps, 64), (codes.float(), codes, exps, exps, 64),
                (codes, codes, exps.int(), exps, 64), (codes.transpose(1, 2), codes.transpose(1, 2), exps, exps, 64), (codes, apart, exps, exps, 64)):
        with pytest.raises(ValueError):
            ab.Context.kv8(*bad, 0)


@pytest.mark.parametrize("T", [1, 31, 32, 33, 100])
def test_key_mask_bits(T):
    drop = np.random.default_rng(T).random((3, T)) < 0.5
    words = ab.Context.pack_key_drop(torch.from_numpy(drop)).numpy().view(np.uint32)
    assert words.shape == (3, -(-T // 32))
    for t in range(words.shape[1] * 32):
        want = drop[:, t] if t < T else np.zeros(3, bool)
        assert np.array_equal((words[:, t // 32] >> np.uint32(t % 32)) & 1, want), t
