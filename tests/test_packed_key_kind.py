"""Packed tokens: keys of all heads and keys by slot have the same shape where every head has a slot (no GPU needed)."""
import pytest
import torch

import paper_2403_08058_amd as C


def call(k, maps, **kw):
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = lambda *s: z(*s, dt=torch.int32)  # noqa: E731
    H = kw.pop("heads", 6)
    C.chai_paged_append_packed(z(5, H, 128), z(5, kw.pop("keys", 6), 128), z(5, H, 128), i(2, k) if maps else None, i(5), i(5), i(5),
                               z(64, dt=torch.float64), z(5, H, 128), z(9, k, 16, 128), z(9, H, 16, 128), **kw)


def test_the_binding_does_not_guess_what_keys_are():
    """With maps that name the heads in an order of their own, one reading writes other heads' keys than the other."""
    with pytest.raises(ValueError, match="k_by_slot"):
        call(6, True)


@pytest.mark.parametrize("kw", [dict(k=6, maps=True, k_by_slot=True), dict(k=6, maps=True, k_by_slot=False), dict(k=6, maps=False), dict(k=2, maps=True),
                                dict(k=2, maps=True, keys=2), dict(k=1, maps=True, heads=1, keys=1)])
def test_what_is_said_or_plain_is_taken(kw):
    with pytest.raises(ValueError, match="device tensors"):                      # (as far as it gets with tensors of the host)
        call(**kw)
