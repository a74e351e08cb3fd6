"""Attention over pages by every way that it is computed: the bound of the lengths alone decides which, so all must answer alike.

Tolerances are those of tests/test_gpu_paged.py.  Where a sum's terms may be smaller than the smallest normal float, each of them
is off by at most half of 2^-149 besides."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from gpu_util import rows_close
from paged_paths import CACHES, PAGE, PATHS
from test_gpu_paged import BAR, D, Setting


def setting(path, cache, seed, lengths=None):
    H, k, bound, rows, _ = PATHS[path]
    print(f"[paged] {path} {cache} H={H} k={k} bound={bound}", flush=True)
    return Setting(seed, cache, H, k, PAGE, rows if lengths is None else lengths, blocks=bound // PAGE), bound


def members(s, b, j):
    h2c, _ = s.maps(b)
    return [h for h in range(s.H) if h2c[h] == j]


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("path", PATHS)
def test_scores_of_minus_infinity_weigh_nothing(path, cache):
    """Whatever the values beside them hold, infinities and NaN among it; heads without another score get 0."""
    s, bound = setting(path, cache, 12000)
    q = s.normal(s.B, s.H, D).abs() + 0.5

    def lowest(at, streams, slot):
        if s.k_scales is None:
            s.k_pages[at, streams, slot] = -float("inf")
        else:                                              # rows of -1, their scale infinite
            s.k_pages[at, streams, slot] = 0xB8
            s.k_scales[at, streams, slot] = float("inf")

    def strange(at, streams, slot, i):
        if s.v_scales is None:
            s.v_pages[at, streams, slot] = (float("inf"), -float("inf"), float("nan"))[i % 3]
        else:
            s.v_pages[at, streams, slot] = (0x38, 0xB8, 0x7F)[i % 3]
            s.v_scales[at, streams, slot] = float("inf")

    _, at0, slot0 = s.places(0, 0, 401)                    # row 0: all streams' first positions, whole shares of them
    for p, t in zip(at0, slot0):
        lowest(p, slice(None), t)
    _, at1, slot1 = s.places(1, 0, 90)                     # row 1: cluster 1 throughout
    for p, t in zip(at1, slot1):
        lowest(p, 1, t)
    _, at2, slot2 = s.places(2, 3, 570)                    # row 2: every third position of cluster 0
    for p, t in zip(at2[::3], slot2[::3]):
        lowest(p, 0, t)
    none = members(s, 1, 1)
    third = members(s, 2, 0)
    assert none and third
    ref = s.expected(q, bound)
    assert bool(ref[1, none].isnan().all())                # (nothing to divide by)
    ref[1, none] = 0.0
    assert bool(ref.isfinite().all())
    for i, (p, t) in enumerate(zip(at0, slot0)):
        strange(p, slice(None), t, i)
    for i, (p, t) in enumerate(zip(at1, slot1)):
        strange(p, none, t, i)
    for i, (p, t) in enumerate(zip(at2[::3], slot2[::3])):
        strange(p, third, t, i)
    out = s.attend(q, bound)
    assert bool((out[1, none] == 0).all())
    ok, worst = rows_close(out.cpu().numpy(), ref.cpu().numpy(), BAR[cache])
    assert ok, f"worst err/allowed {worst:.3g}"
