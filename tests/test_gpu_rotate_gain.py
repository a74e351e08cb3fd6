"""Turned rows with a gain that 24 bits do not hold, as models that scale their angles have it (0.1 ln(factor) + 1).  The bar is that of the
other turns (see test_gpu_rotate.py): of the gain's own rounding to 24 bits, up to 2^-24 of every result, there is no room in it."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2403_08058_amd as C
from test_gpu_rotate import D, TYPES, assert_rounded, dev, layout_of, turned

GAINS = [0.1 * math.log(32.0) + 1.0, 0.1 * math.log(5.0) + 1.0, -0.7]


@pytest.mark.parametrize("gain", GAINS)
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_gain_is_held_in_64_bits(dtype, layout, gain):
    print(f"[rotate] {dtype} {layout}, gain {gain}", flush=True)
    g = np.random.default_rng(21)
    B, H, Tn, pos0, rot = 2, 3, 40, 3, 96
    x = torch.from_numpy(g.standard_normal((B, H, Tn, D)).astype(np.float32)).cuda().to(TYPES[dtype])
    freq = C.chai_rotary_frequencies(rot)
    q, keys = torch.full_like(x, 7.0), torch.full((B, H, pos0 + Tn, D), 9.0, dtype=x.dtype, device="cuda")
    C.chai_rotate_qk(x, x, None, freq.cuda(), q, keys, pos0, layout=layout_of(layout), gain=gain)
    # the same tokens one behind the other, into pages of as many
    N = B * Tn
    packed = x.transpose(1, 2).reshape(N, H, D)
    pos = np.tile(np.arange(pos0, pos0 + Tn), B)
    pages = [torch.zeros((B, H, Tn, D), dtype=x.dtype, device="cuda") for _ in "kv"]
    packed_q = torch.zeros_like(packed)
    C.chai_paged_append_packed(packed, packed, packed, None, dev(np.repeat(np.arange(B), Tn)), dev(pos), dev(np.arange(N)), freq.cuda(), packed_q, *pages,
                               layout=layout_of(layout), gain=gain)
    torch.cuda.synchronize()
    want, mag = turned(x.double().cpu().numpy(), np.broadcast_to(pos[:Tn], (B, H, Tn)), freq.numpy(), layout, gain)
    for what, got in (("q", q), ("k", keys[:, :, pos0:]), ("packed q", packed_q.view(B, Tn, H, D).transpose(1, 2)), ("packed k", pages[0])):
        assert_rounded(got, want, mag, dtype, what)
