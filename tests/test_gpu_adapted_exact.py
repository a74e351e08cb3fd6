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


@pytest.mark.parametrize("R", [8, 24])
@pytest.mark.parametrize("kernel,B,H,k,Tn,D", SIZES)
def test_infinities_of_adapters_are_the_formulas(kernel, B, H, k, Tn, D, R):
    """An infinite element of B_a gives infinities of the sign that x A_a^T has there, one of A_a those of x times B_a's, and where they meet NaN
    (opposite signs, 0 times infinity); columns without are as without."""
    print(f"[adapted] infinities, {kernel} {B} x {Tn} tokens, {k} of {H}, width {D}, rank {R}", flush=True)
    x = Inputs(13, B, H, k, Tn, D, R, n=4)
    x.ids[:] = np.arange(B) % 4
    inf = float("inf")
    for p in "qk":
        up = x.b[p].view(4, H, 128, R)
        up[0, :, 5, 2], up[0, :, 77, R - 1], up[0, :, 100, 0], up[0, :, 100, 1] = inf, -inf, inf, inf
        up[1, :, 9, 3], up[1, :, 64, 0] = -inf, float("nan")
        x.a[p][2, 6, D // 2] = inf
        up[2, :, 31, 6] = 0.0
        x.a[p][3, 4] = 0.0
        up[3, :, 12, 4] = inf
    q, kc = x.run()
    for b in sorted({0, 1, 2, 3, B // 2, B - 1} & set(range(B))):
        a, rows = int(x.ids[b]), x.x[b].double()
        for p in "qk":
            t = float(x.scale[a]) * (rows @ x.a[p][a].double().t().contiguous())
            for j, r in enumerate(x.rep[b]):
                if r < 0:
                    continue
                cols = slice(r * 128, (r + 1) * 128)
                want = rows @ x.w[p][cols].double().t().contiguous() + t @ x.b[p][a, cols].double().t().contiguous()
                got = (q[b, r] if p == "q" else kc[b, j]).double()
                assert torch.equal(torch.isnan(got), torch.isnan(want)), (b, j, p, a)
                assert torch.equal(torch.where(torch.isinf(got), got, 0.0), torch.where(torch.isinf(want), want, 0.0)), (b, j, p, a)


@pytest.mark.parametrize("kernel,B,H,k,Tn,D", [(kernel, *c[0]) for kernel, c in CASES.items()])
@pytest.mark.parametrize("power", [-95, -118, -126, -140])
def test_small_first_halves(kernel, B, H, k, Tn, D, power):
    """t of about 2^power, down to where 32 bits are subnormal: the bars of test_gpu_adapted.py, and four parts that may lose what they
    have below 2^-126."""
    x = Inputs(15, B, H, k, Tn, D, 16, n=2)
    x.ids[:] = np.arange(B) % 2
    for p in "qk":
        x.w[p].zero_()
        x.a[p].zero_()
        x.a[p][:, :, :8] = torch.randn((2, 16, 8), device="cuda").mul_(2.0 ** -20).to(torch.bfloat16)
        x.b[p].mul_(2.0 ** 100)
    x.scale.fill_(2.0 ** (power + 20) if power > -140 else 2.0 ** -120)
    q, kc = x.run()
    for b in {0, B // 2, B - 1}:
        a, rows = int(x.ids[b]), x.x[b].double()
        for p in "qk":
            down = x.a[p][a].double().t().contiguous()
            s = float(x.scale[a])
            t, mag_t = s * (rows @ down), s * (rows.abs() @ down.abs())
            for j, r in enumerate(x.rep[b]):
                if r < 0:
                    continue
                up = x.b[p][a, r * 128:(r + 1) * 128].double().t().contiguous()
                want = t @ up
                allowed = 2.0 ** -8 * want.abs() + (3e-6 * mag_t + (2.0 ** -17 + 2.0 ** -24 + 3e-6) * t.abs() + 4 * 2.0 ** -126) @ up.abs()
                got = (q[b, r] if p == "q" else kc[b, j]).double()
                assert bool(((got - want).abs() <= allowed).all()), (b, j, p, float(((got - want).abs() / allowed).max()))
