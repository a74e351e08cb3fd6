"""Calls on pages that have nothing to do: no rows or no new tokens, their empty arrays without an address (no GPU needed)."""
import pytest
import torch

import paper_2403_08058_amd as C
from test_paged_refusals import FAKE, NULL, SHAPE, append, attention, gather, step

NO_ROWS = {"B": 0, "table": None}


@pytest.mark.parametrize("f,empty", [
    (attention, ("q", "h2c", "rep", "lens", "out", "ws")),
    (step, ("q", "k_new", "v_new", "h2c", "rep", "lens", "out", "ws")),
    (append, ("k_new", "v_new", "rep", "start")),
    (gather, ("start", "k_out", "v_out")),
])
def test_no_rows(f, empty):
    nothing = {**NO_ROWS, **{name: None for name in empty}}
    assert f(**nothing) == 0
    assert f(**nothing, cache_dtype=2, k_scales=FAKE, v_scales=FAKE) == 0
    assert f(**nothing, k_pages=None) == NULL and f(**nothing, page=12) == SHAPE       # the pool is there all the same
    for name in empty:
        if name != "ws":
            assert f(**{name: None}) in (NULL, SHAPE), name


def test_no_tokens():
    assert append(Tn=0, k_new=None, v_new=None, k_stride=0, v_stride=0) == 0
    assert gather(Tn=0, k_out=None, v_out=None) == 0
    assert append(Tn=0, k_new=None, v_new=None, start=None) == NULL and gather(Tn=0, k_out=None, v_out=None, start=None) == NULL
    assert append(Tn=-1, k_new=None, v_new=None) in (NULL, SHAPE)


class Empty(torch.Tensor):
    """An empty tensor that says it is the device's (one has no address there either)."""
    is_cuda = True


@pytest.mark.parametrize("B,Tn", [(0, 9), (2, 0)])
def test_the_binding_passes_empty_tensors(B, Tn, monkeypatch):
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt).as_subclass(Empty)  # noqa: E731
    i32 = lambda *s: z(*s, dt=torch.int32)  # noqa: E731
    pages = (z(5, 2, 16, 128), z(5, 6, 16, 128))
    from paper_2403_08058_amd import binding
    monkeypatch.setattr(binding, "_stream", lambda stream: 0)
    assert z(0, 3).data_ptr() == 0
    C.chai_paged_append_kv(z(B, 6, Tn, 128), z(B, 6, Tn, 128), i32(B, 2), i32(B, 4), i32(B), None, *pages)
    C.chai_paged_gather_kv(*pages, i32(B, 4), i32(B), i32(B), z(B, 2, Tn, 128), z(B, 6, Tn, 128))
    if B == 0:
        q, out, ws = z(0, 6, 128), z(0, 6, 128, dt=torch.float32), z(256, dt=torch.uint8)
        maps = (i32(0, 6), i32(0, 2), i32(0, 4), i32(0), 64, 0.1, out, ws)
        C.chai_paged_decode_attention(q, *pages, *maps)
        C.chai_paged_decode_step(q, q, q, *pages, *maps)
