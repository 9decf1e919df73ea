"""What the binding refuses before acache_predict_sample is called, without a GPU: the current device is made the CPU's number, so that tensors here are where
they should be, and the library is one that notes its calls."""
import types

import pytest
import torch

from paper_2608_26140_b200 import binding as ab

B, H_ROWS, N, D, V = 2, 5, 3, 256, 640


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 5


@pytest.fixture
def ctx(monkeypatch):
    monkeypatch.setattr(ab, "_current_device", lambda: -1)
    monkeypatch.setattr(ab, "_stream", lambda: 0)
    c = ab.Context.__new__(ab.Context)
    c.h, c.gpu, c.heads, c.desc, c.dtypes = None, -1, (4, 2, 64), ab.ModelDesc(hidden=D), (torch.bfloat16, torch.float32, torch.int32)
    how = ab.Sampling()
    c._sampling_arg = (how, how)
    c.calls = []
    c.lib = types.SimpleNamespace(acache_predict_sample=lambda *a: c.calls.append(a) or ab.OK)
    return c


def arguments():
    i32 = lambda: torch.zeros((B, N), dtype=torch.int32)  # noqa: E731
    return dict(h=torch.zeros((B, H_ROWS, D), dtype=torch.bfloat16), h_rows=H_ROWS, block_rows=i32(), batch=B, n_blk=N, final_norm_g=torch.zeros(D, dtype=torch.bfloat16),
                w_lm=torch.zeros((V, D), dtype=torch.bfloat16), vocab=V, logits=torch.zeros((B * N, V)), u=torch.zeros((B, N)), threshold=0.5, token=i32(),
                confidence=torch.zeros((B, N)), commit=i32())


def test_tensors_that_fit_come_through(ctx):
    a = arguments()
    ctx.predict_sample(**a)
    ctx.predict_sample(**{**a, "h": torch.zeros((B + 1, H_ROWS, D), dtype=torch.bfloat16), "token": torch.zeros(B * N + 5, dtype=torch.int32)})       # more than is wanted
    assert len(ctx.calls) == 2
    got = ctx.calls[0]
    assert (got[1], got[3], got[6], got[7], got[12], got[13], got[14]) == \
        (a["h"].data_ptr(), a["block_rows"].data_ptr(), a["final_norm_g"].data_ptr(), a["w_lm"].data_ptr(), 0.5, a["token"].data_ptr(), a["confidence"].data_ptr())
    ctx.predict_sample(**{**a, "token": None})                   # (the library refuses a NULL)
    assert ctx.calls[-1][13] is None


@pytest.mark.parametrize("name", ["h", "block_rows", "final_norm_g", "w_lm", "logits", "u", "token", "confidence", "commit"])
def test_tensors_that_do_not_fit_are_refused(ctx, name):
    a = arguments()
    t = a[name]
    kinds = {torch.bfloat16: torch.float16, torch.float32: torch.float64, torch.int32: torch.int64}
    apart = torch.zeros((*t.shape, 2), dtype=t.dtype)[..., 0]
    for bad in (t.to(kinds[t.dtype]), t.flatten()[:-1], t[:0], apart, t.clone().as_subclass(Elsewhere)):
        with pytest.raises((ValueError, RuntimeError)) as e:     # (RuntimeError: u cannot be seen as one row)
            ctx.predict_sample(**{**a, name: bad})
        assert not isinstance(e.value, ab.AcacheError)
    assert not ctx.calls
