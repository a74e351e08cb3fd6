"""Attention over pages by every way that it is computed: the bound of the lengths alone decides which, so all must answer alike;
and rows beyond the 64 whose lengths a wave's lanes hold one each, attended to and moved.

Tolerances are those of tests/test_gpu_paged.py.  Where a sum's terms may be smaller than the smallest normal float, each of them
is off by at most half of 2^-149 besides."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2403_08058_amd as C

from gpu_util import guarded, guards_intact, rows_close
from paged_paths import CACHES, LONGEST, MANY_HEADS, MANY_ROWS, MOVED, PAGE, PATHS, many_lengths
from test_gpu_paged import BAR, D, SCALE, Setting, bits, copies, held, put, same_pools


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


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("path", PATHS)
def test_nan_reaches_its_cluster_and_row_alone(path, cache):
    """From a key that is NaN, beside scores of -inf as well."""
    s, bound = setting(path, cache, 12100)
    q = s.normal(s.B, s.H, D)
    _, at, slot = s.places(2, 0, 577)
    for page, place in ((at[350], slot[350]), (at[33], slot[33])):
        if s.k_scales is None:
            s.k_pages[page, 0, place, 5] = float("nan")
        else:
            s.k_pages[page, 0, place, 5] = 0x7F
    out, ref = s.attend(q, bound), s.expected(q, bound)
    nan = members(s, 2, 0)
    assert nan and bool(out[2, nan].isnan().all()) and bool(ref[2, nan].isnan().all())
    out[2, nan], ref[2, nan] = 0.0, 0.0
    ok, worst = rows_close(out.cpu().numpy(), ref.cpu().numpy(), BAR[cache])
    assert ok, f"worst err/allowed {worst:.3g}"


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("path", PATHS)
def test_places_that_are_not_attended_to_may_hold_anything(path, cache):
    """Free pages and places past a row's end: infinities, NaN and the lowest value.  Some of a row's pages are absent."""
    s, bound = setting(path, cache, 12200)
    s.host_table[0, [0, 3, 4, 34]] = [-1, s.n_pages, -5, 1 << 30]
    s.host_table[1, 0] = -1
    s.table.copy_(torch.from_numpy(s.host_table))
    used = torch.zeros((s.n_pages, PAGE), dtype=torch.bool)
    for b in range(s.B):
        _, at, slot = s.places(b, 0, int(s.host_lengths[b]))
        used[torch.from_numpy(at), torch.from_numpy(slot)] = True
    for pages, scales in ((s.k_pages, s.k_scales), (s.v_pages, s.v_scales)):
        for i, (p, t) in enumerate((~used).nonzero().tolist()):
            if scales is not None:
                pages[p, :, t] = (0x7F, 0xFF, 0x7E)[i % 3]
                scales[p, :, t] = (float("nan"), float("inf"), 3e38)[i % 3]
            else:
                pages[p, :, t] = (float("nan"), float("inf"), torch.finfo(pages.dtype).min)[i % 3]
    s.check(s.normal(s.B, s.H, D), bound)
    s.host_lengths[1] = -3
    s.lengths.copy_(torch.from_numpy(s.host_lengths))
    s.check(s.normal(s.B, s.H, D), bound)


@pytest.mark.parametrize("path", PATHS)
def test_values_near_the_largest_and_the_smallest_float(path):
    s, bound = setting(path, "f32", 12300)
    s.k_pages.mul_(1e-3)
    s.v_pages.copy_(torch.where(s.v_pages > 0, 3.3e38, 3.0e38))
    s.check(s.normal(s.B, s.H, D), bound)
    s.v_pages.normal_(generator=s.g).mul_(1e-37)
    q = s.normal(s.B, s.H, D)
    out, ref = s.attend(q, bound).double(), s.expected(q, bound)
    # terms of some 1e-40: each sum of a position, of a part or of a lane group is off by half of 2^-149 at most
    floor = (max(s.host_lengths) + 100) * 2.0 ** -150
    allowed = BAR["f32"] * (ref.abs() + 0.25 * ref.abs().amax(-1, keepdim=True)) + floor
    assert bool(((out - ref).abs() <= allowed).all())


def step_and_check(s, bound, q=None):
    """The step's rows written as by the append, attended to as stored."""
    q = s.normal(s.B, s.H, D) if q is None else q
    k_new, v_new = s.normal(s.B, s.H, D), s.normal(s.B, s.H, D)
    expect = copies(s)
    put(s, expect, k_new.unsqueeze(2), v_new.unsqueeze(2), s.host_lengths - 1, (s.host_lengths > 0).astype(int))
    whole, out = guarded((s.B, s.H, D), torch.float32, float("nan"))
    ws = C.alloc_paged_workspace(s.B, s.H, s.k, bound)
    ws.fill_(0xFF)
    C.chai_paged_decode_step(q, k_new, v_new, s.k_pages, s.v_pages, s.h2c, s.rep, s.table, s.lengths, bound, SCALE, out, ws, **s.scales)
    torch.cuda.synchronize()
    assert guards_intact(whole, out.shape, float("nan"))
    same_pools(s, expect)
    ok, worst = rows_close(out.cpu().numpy(), s.expected(q, bound).cpu().numpy(), BAR[s.cache])
    assert ok, f"worst err/allowed {worst:.3g}"
    return out


@pytest.mark.parametrize("cache", CACHES + ["e4m3/f32"])
@pytest.mark.parametrize("path", PATHS)
def test_step_by_every_way(path, cache):
    s, bound = setting(path, cache, 12400)
    s.host_table[1, 5] = -1                                # of 90 tokens, the last ones and the new one are in no page
    s.table.copy_(torch.from_numpy(s.host_table))
    step_and_check(s, bound)


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("path", PATHS)
def test_rows_that_are_all_empty(path, cache):
    lengths = [0] * len(PATHS[path][3])
    s, bound = setting(path, cache, 12500, lengths)
    q = s.normal(s.B, s.H, D)
    assert bool((s.attend(q, bound) == 0).all())
    assert bool((step_and_check(s, bound, q) == 0).all())


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("B", MANY_ROWS)
@pytest.mark.parametrize("H,k", MANY_HEADS)
def test_many_rows_of_which_one_is_long(H, k, B, cache):
    print(f"[paged] many rows {cache} B={B} H={H} k={k}", flush=True)
    s = Setting(12600 + B, cache, H, k, PAGE, many_lengths(B), blocks=(LONGEST + 8) // PAGE)
    q = s.normal(B, H, D)
    first = s.check(q, LONGEST + 8)
    assert torch.equal(s.attend(q, LONGEST + 8), first)
    step_and_check(s, LONGEST + 8)


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("B,H,k,Tn", MOVED)
def test_many_rows_written_and_read_back(B, H, k, Tn, cache):
    print(f"[paged] many rows moved {cache} B={B} H={H} k={k} Tn={Tn}", flush=True)
    s = Setting(12700 + B, cache, H, k, PAGE, [100] * B)
    s.host_table[B // 2, 2] = -1
    s.table.copy_(torch.from_numpy(s.host_table))
    k_new, v_new = s.normal(B, H, Tn, D), s.normal(B, H, Tn, D)
    start = [(13 * i) % 60 - 3 for i in range(B)]
    n = [min(many_lengths(B)[i], Tn) for i in range(B)]
    expect = copies(s)
    put(s, expect, k_new, v_new, start, n)
    first, counts = (torch.tensor(a, dtype=torch.int32, device="cuda") for a in (start, n))
    C.chai_paged_append_kv(k_new, v_new, s.rep, s.table, first, counts, s.k_pages, s.v_pages, **s.scales)
    torch.cuda.synchronize()
    same_pools(s, expect)
    (kw, k_out), (vw, v_out) = (guarded((B, streams, Tn, D), s.dtype, 7.0) for streams in (k, H))
    C.chai_paged_gather_kv(s.k_pages, s.v_pages, s.table, first, counts, k_out, v_out, **s.scales)
    torch.cuda.synchronize()
    assert guards_intact(kw, k_out.shape, 7.0) and guards_intact(vw, v_out.shape, 7.0)
    for got, pages, scales in ((k_out, s.k_pages, s.k_scales), (v_out, s.v_pages, s.v_scales)):
        for b in range(B):
            i, at, slot = (torch.from_numpy(a).cuda() for a in s.places(b, start[b], n[b]))
            want = torch.full(got.shape[1:], 7.0, dtype=torch.float64, device="cuda")
            want[:, :n[b]] = 0.0
            want[:, i] = (pages[at, :, slot].double() if scales is None else held(pages[at, :, slot], scales[at, :, slot])).transpose(0, 1)
            if scales is None:
                assert torch.equal(bits(got[b]), bits(want.to(s.dtype))), b
            else:                                          # the exact product rounded to fp32 and to bf16: half a step of each
                step = 2.0 ** -8 + 2.0 ** -24
                assert bool(((got[b].double() - want).abs() <= step * want.abs() + 2.0 ** -133).all()), b
