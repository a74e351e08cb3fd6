"""Projections with adapters where what comes out is known to the last bit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from adapted_cases import CASES, MORE, PARTS
from test_gpu_adapted import Inputs

SIZES = [(kernel, *c) for kernel, cases in CASES.items() for c in cases] + [("parts", *c) for c in PARTS] + [("more", *c) for c in MORE]


@pytest.mark.parametrize("R", [8, 24, 128])
@pytest.mark.parametrize("kernel,B,H,k,Tn,D", SIZES)
def test_the_first_half_has_all_its_bits(kernel, B, H, k, Tn, D, R):
    """t of two ranks is 1.5 (1 + 2^-10 + 2^-20) and 1.5 (1 + 2^-10), 22 bits, and the result their difference, 1.5 * 2^-20.  Every sum on the
    way is a multiple of 2^-21 below 2^2, which 32 bits hold whatever the order."""
    print(f"[adapted] bits of t, {kernel} {B} x {Tn} tokens, {k} of {H}, width {D}, rank {R}", flush=True)
    x = Inputs(7, B, H, k, Tn, D, R, n=3)
    g = np.random.default_rng(B + Tn + R)
    x.ids[:] = g.integers(0, 3, B)
    x.x.fill_(1.0)
    x.scale.fill_(1.5)
    for p in "qk":
        for z in (x.w[p], x.a[p], x.b[p]):
            z.zero_()
    for a in range(3):
        for p in "qk":
            i, j = g.permutation(R)[:2].tolist()
            at = g.permutation(D)[:3].tolist()
            x.a[p][a, i, at] = torch.tensor([1.0, 2.0 ** -10, 2.0 ** -20], dtype=torch.bfloat16, device="cuda")
            x.a[p][a, j, at[:2]] = torch.tensor([1.0, 2.0 ** -10], dtype=torch.bfloat16, device="cuda")
            x.b[p][a, :, i], x.b[p][a, :, j] = 1.0, -1.0
    q, kc = x.run()
    for b in {0, B // 3, B // 2, B - 1}:
        used = x.rep[b][x.rep[b] >= 0]
        assert bool((q[b, used] == 1.5 * 2.0 ** -20).all()), (b, q[b, used].unique())
        assert bool((kc[b, x.rep[b] >= 0] == 1.5 * 2.0 ** -20).all())
