"""Queries and keys turned by their positions, in blocks and packed into pages, against turns in 80 bits.

Tolerance.  The kernels hold angles, turns and products in 64 bits and round once to fp32 and from there to the stored type, so a result
is off by half a step of fp32 (2^-24 of it), and of bf16 besides (2^-8), beside what 64 bits lose: the angle is reduced to 2^-53 of a
turn, the series are cut below 2^-56, products and sum round to 2^-53 each;
16 * 2^-53 of |a| + |b| covers them.  Subnormal results: half of the smallest subnormal instead."""
from fractions import Fraction

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2403_08058_amd as C

D = 128
LONG = np.longdouble
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8 + 2.0 ** -24}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


TURN = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494")


def angles(pos, freq):
    """pos * freq without whole turns: exactly (the product of 32 and 53 bits has no place in 80), then rounded to 80 bits."""
    f = [Fraction(float(x)) for x in freq]
    rest = [[p * x - TURN * round(p * x / TURN) for x in f] for p in np.asarray(pos).ravel().tolist()]
    both = [[(float(x), float(x - Fraction(float(x)))) for x in row] for row in rest]
    both = np.array(both, np.float64).reshape(*np.shape(pos), len(f), 2)
    return both[..., 0].astype(LONG) + both[..., 1].astype(LONG)


def turned(x, pos, freq, layout, gain):
    """x [..,n,128] float64 at pos [..,n]: values in 80 bits and the magnitudes that went into each."""
    rot = 2 * len(freq)
    angle = angles(pos, freq)
    c, s = np.cos(angle) * LONG(gain), np.sin(angle) * LONG(gain)
    y, mag = x.astype(LONG), np.abs(x).astype(np.float64)
    first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = y[..., first].copy(), y[..., second].copy()
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    both = (np.abs(a) + np.abs(b)).astype(np.float64) * abs(gain)
    mag[..., first], mag[..., second] = both, both
    return y, mag


def assert_rounded(got, want, mag, dtype, what):
    got = got.double().cpu().numpy()
    allowed = HALF_STEP[dtype] * np.abs(want).astype(np.float64) + 16 * 2.0 ** -53 * mag + 2.0 ** -149
    if dtype == "bf16":
        allowed += 2.0 ** -134
    off = np.abs(got - want).astype(np.float64) > allowed
    assert not off.any(), (what, int(off.sum()), got[off][:4], want[off][:4])


def maps(g, B, H, k, holes=False):
    rep = np.stack([g.permutation(H)[:k] for _ in range(B)])
    if holes:
        rep[g.random((B, k)) < 0.3] = -1
    return rep


def layout_of(name):
    return C.CHAI_ROPE_HALVES if name == "halves" else C.CHAI_ROPE_PAIRS


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("B,H,k,Tn,pos0,rot,far,dense", [
    (1, 32, 8, 1, 255, 128, False, False), (3, 5, 2, 7, 0, 128, True, False), (2, 12, 12, 33, 5, 96, False, True), (5, 6, 3, 3, 9, 16, True, False),
    (1, 72, 16, 130, 17, 64, False, False), (9, 3, 1, 5, 0, 112, True, False), (2, 4, 4, 257, 3, 32, True, True), (700, 2, 1, 3, 0, 128, False, False)])
def test_blocks(dtype, layout, B, H, k, Tn, pos0, rot, far, dense):
    print(f"[rotate] {dtype} {layout} {B} x {H} in {k}, {Tn} tokens from {pos0}, rot {rot}, far {far}", flush=True)
    g = np.random.default_rng(B * 3 + H * 5 + Tn + rot)
    dt = TYPES[dtype]
    new = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).cuda().to(dt)  # noqa: E731
    rep = None if dense else maps(g, B, H, k, holes=True)
    q, keys = new(B, H, Tn, D), new(B, k, Tn, D)
    pos = g.integers(-(1 << 31), 1 << 31, (B, Tn)) if far else None
    freq = C.chai_rotary_frequencies(rot, kind=C.CHAI_ROPE_TURNS if far else C.CHAI_ROPE_PLAIN, factor=4.0, original_length=512.0)
    gain = 1.25 if far else 1.0
    q_out, k_out = torch.full_like(q, 7.0), torch.full((B, k, pos0 + Tn + 2, D), 9.0, dtype=dt, device="cuda")
    C.chai_rotate_qk(q, keys, None if dense else dev(rep), freq.cuda(), q_out, k_out, pos0, positions=None if pos is None else dev(pos),
                     layout=layout_of(layout), gain=gain)
    torch.cuda.synchronize()
    at = pos if far else np.tile(np.arange(pos0, pos0 + Tn), (B, 1))
    for b in range(B):
        slots = np.arange(k) if dense else np.flatnonzero(rep[b] >= 0)
        heads = slots if dense else rep[b][slots]
        others = np.setdiff1d(np.arange(H), heads)
        assert bool((q_out[b, others] == 7.0).all()), "rows of other heads"
        unused = np.setdiff1d(np.arange(k), slots)
        assert bool((k_out[b, unused] == 9.0).all()) and bool((k_out[b, :, :pos0] == 9.0).all()) and bool((k_out[b, :, pos0 + Tn:] == 9.0).all())
        if b % 97 in (0, 1, 2):
            for got, x, rows in ((q_out[b, heads], q[b], heads), (k_out[b, slots, pos0:pos0 + Tn], keys[b], slots)):
                want, mag = turned(x[rows].double().cpu().numpy(), at[b], freq.numpy(), layout, gain)
                assert_rounded(got, want, mag, dtype, b)
    if rot < D:                                            # what is not turned is copied
        heads = slice(None) if dense else rep[0][rep[0] >= 0]
        assert torch.equal(q_out[0, heads, :, rot:], q[0, heads, :, rot:])


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_equals_elsewhere(dtype, layout):
    """Queries over themselves and keys over their rows of the cache, with a head that stands in three slots."""
    g = np.random.default_rng(11)
    B, H, k, Tn, pos0, cap = 3, 10, 4, 21, 6, 40
    dt = TYPES[dtype]
    new = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).cuda().to(dt)  # noqa: E731
    rep = maps(g, B, H, k)
    rep[1] = [4, 2, 4, 4]
    rep[2] = [H + 3, -1, H - 1, 0]                         # (beyond the heads: the last one)
    q, cache, freq = new(B, H, Tn, D), new(B, k, cap, D), C.chai_rotary_frequencies(128).cuda()
    q_out, k_out = q.clone(), cache.clone()
    C.chai_rotate_qk(q, cache[:, :, pos0:pos0 + Tn], dev(rep), freq, q_out, k_out, pos0, layout=layout_of(layout))
    torch.cuda.synchronize()
    assert not torch.equal(q_out, q)
    C.chai_rotate_qk(q, cache[:, :, pos0:pos0 + Tn], dev(rep), freq, q, cache, pos0, layout=layout_of(layout))
    torch.cuda.synchronize()
    assert torch.equal(q, q_out) and torch.equal(cache, k_out)


def test_queries_or_keys_alone_and_views():
    g = np.random.default_rng(12)
    B, H, k, Tn = 2, 7, 3, 9
    new = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    rep, freq = dev(maps(g, B, H, k)), C.chai_rotary_frequencies(128).cuda()
    wide_q, wide_k = new(B, H, 30, D), new(B, k, 25, D)
    q, keys = wide_q[:, :, 4:4 + Tn], wide_k[:, :, 16:]
    q_out, k_out = torch.zeros((B, H, Tn, D), device="cuda"), torch.zeros((B, k, Tn, D), device="cuda")
    C.chai_rotate_qk(q, keys, rep, freq, q_out, k_out, 0)
    alone_q, alone_k = torch.zeros_like(q_out), torch.zeros_like(k_out)
    C.chai_rotate_qk(q.contiguous(), None, rep, freq, alone_q, None, 0)
    C.chai_rotate_qk(None, keys.contiguous(), rep, freq, None, alone_k, 0)
    torch.cuda.synchronize()
    assert torch.equal(q_out, alone_q) and torch.equal(k_out, alone_k) and bool((alone_k != 0).all())
    with pytest.raises(ValueError):
        C.chai_rotate_qk(wide_q[:, :, ::2][:, :, :Tn], None, rep, freq, alone_q, None, 0)
    with pytest.raises(C.ChaiError):
        C.chai_rotate_qk(wide_q[:, :, :Tn], None, rep, freq, wide_q.view(-1)[:q_out.numel()].view(B, H, Tn, D), None, 0)


def test_turned_back_and_lengths_kept():
    """A turn by -p after one by p gives the row back; scores of a query and a key hang on the distance of their positions alone."""
    g = np.random.default_rng(13)
    H, n = 4, 50
    x = torch.from_numpy(g.standard_normal((1, H, n, D)).astype(np.float32)).cuda()
    pos = dev(g.integers(0, 1 << 20, (1, n)))
    freq = C.chai_rotary_frequencies(128).cuda()
    there, back = torch.zeros_like(x), torch.zeros_like(x)
    C.chai_rotate_qk(x, None, None, freq, there, None, 0, positions=pos)
    C.chai_rotate_qk(there, None, None, freq, back, None, 0, positions=-pos)
    # two roundings of 2^-24 of at most |a| + |b| each, times sqrt(2) by the second turn
    pair = (x[..., :64].abs() + x[..., 64:].abs()).repeat(1, 1, 1, 2)
    assert bool(((back - x).abs() <= 3 * 2.0 ** -24 * pair).all())
    moved, same = torch.zeros_like(x), torch.zeros_like(x)
    C.chai_rotate_qk(x, None, None, freq, moved, None, 0, positions=pos + 1000)
    C.chai_rotate_qk(x.flip(1).contiguous(), None, None, freq, same, None, 0, positions=pos + 1003)
    base, other = torch.zeros_like(x), torch.zeros_like(x)
    C.chai_rotate_qk(x, None, None, freq, base, None, 0)
    C.chai_rotate_qk(x.flip(1).contiguous(), None, None, freq, other, None, 3)
    s = (moved.double() * same.double()).sum(-1)
    C.chai_rotate_qk(x, None, None, freq, base, None, 0, positions=torch.zeros_like(pos))
    C.chai_rotate_qk(x.flip(1).contiguous(), None, None, freq, other, None, 0, positions=torch.full_like(pos, 3))
    t = (base.double() * other.double()).sum(-1)
    # both sides round 128 elements of either row to 2^-24
    bar = 4 * 2.0 ** -24 * (moved.double().abs() * same.double().abs()).sum(-1) + 4 * 2.0 ** -24 * (base.double().abs() * other.double().abs()).sum(-1)
    assert bool(((s - t).abs() <= bar).all())


def test_extreme_values():
    """The largest and the smallest, infinities and NaN stay in their pairs."""
    x = torch.zeros((1, 1, 1, D), device="cuda")
    x[0, 0, 0, :8] = torch.tensor([3.4e38, 1e-45, 1e-38, float("inf"), float("nan"), -0.0, 1.0, -3.4e38])
    out = torch.zeros_like(x)
    C.chai_rotate_qk(x, None, None, C.chai_rotary_frequencies(128).cuda(), out, None, 0, positions=dev([[0]]))
    torch.cuda.synchronize()
    ok = [0, 1, 2, 3, 5, 6, 7] + list(range(8, 67)) + [69] + list(range(72, 128))
    ok = [i for i in ok if i not in (67, 68)]
    assert torch.equal(out[0, 0, 0, ok], x[0, 0, 0, ok])   # position 0: nothing moves (inf * 0 and NaN reach their partners, 67 and 68)
    assert bool(torch.isnan(out[0, 0, 0, [4, 67, 68]]).all()) and bool(torch.isfinite(out[0, 0, 0, [66, 69, 70]]).all())


def test_offsets_beyond_32_bits():
    """The last rows of a cache of more than 2^32 bytes."""
    cap, k, Tn = 1 << 20, 20, 3                            # 20 * 2^20 rows of 256 bytes
    cache = torch.zeros((1, k, cap, D), dtype=torch.bfloat16, device="cuda")
    g = np.random.default_rng(14)
    keys = torch.from_numpy(g.standard_normal((1, k, Tn, D)).astype(np.float32)).cuda().to(torch.bfloat16)
    freq = C.chai_rotary_frequencies(128)
    C.chai_rotate_qk(None, keys, None, freq.cuda(), None, cache, cap - Tn)
    torch.cuda.synchronize()
    want, mag = turned(keys[0].double().cpu().numpy(), np.arange(cap - Tn, cap), freq.numpy(), "halves", 1.0)
    assert_rounded(cache[0, :, cap - Tn:], want, mag, "bf16", "last rows")
    assert int((cache.view(torch.int64) != 0).sum()) <= k * Tn * D // 4


# ------------------------------------------------------------------------------------------------- packed into pages
def packed_case(seed, B, H, k, N, page, cache, by_slot, dense=False, wide=False):
    g = np.random.default_rng(seed)
    dt = torch.float32 if cache in ("f32", "e4m3_f32") else torch.bfloat16
    coded = cache.startswith("e4m3")
    new = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).cuda().to(dt)  # noqa: E731
    s = {"rep": None if dense else maps(g, B, H, k, holes=True)}
    if wide:                                               # parts of one row per token
        fused = new(N, (2 * H + (k if by_slot else H)) * D + 16)
        s["q"], s["v_new"] = fused[:, :H * D].unflatten(1, (H, D)), fused[:, H * D:2 * H * D].unflatten(1, (H, D))
        s["k_new"] = fused[:, 2 * H * D:-16].unflatten(1, (-1, D))
    else:
        s["q"], s["v_new"], s["k_new"] = new(N, H, D), new(N, H, D), new(N, k if by_slot else H, D)
    n_pages = -(-N // page) + 3
    s["rows"] = np.sort(g.integers(0, B, N))
    s["pos"] = g.integers(0, 100000, N)
    s["slots"] = g.permutation(n_pages * page)[:N]
    if N > 4:
        s["slots"][[1, 3]] = [-1, n_pages * page]          # no place
        s["rows"][4] = -1                                  # no token
    s["pages"] = [torch.full((n_pages, st, page, D), 0x55 if coded else 3.0, dtype=torch.uint8 if coded else dt, device="cuda") for st in (k, H)]
    s["scales"] = [torch.full((n_pages, st, page), 5.0, device="cuda") if coded else None for st in (k, H)]
    s["q_out"] = torch.full((N, H, D), 7.0, dtype=dt, device="cuda")
    return s


@pytest.mark.parametrize("layout,rot", [("halves", 128), ("pairs", 96), ("pairs", 128), ("halves", 0)])
@pytest.mark.parametrize("cache", ["bf16", "f32", "e4m3", "e4m3_f32"])
@pytest.mark.parametrize("B,H,k,N,page,by_slot,dense,wide", [
    (1, 32, 8, 1, 16, False, False, False), (3, 5, 2, 23, 8, True, False, True), (2, 4, 4, 9, 24, False, True, False), (16, 32, 8, 16, 64, True, False, False),
    (4, 3, 3, 70, 16, False, False, True), (1, 2, 1, 1500, 32, False, False, False)])
def test_packed(layout, rot, cache, B, H, k, N, page, by_slot, dense, wide):
    print(f"[packed] {cache} {layout} rot {rot} {B} rows {N} tokens {H} in {k} page {page} by slot {by_slot}", flush=True)
    s = packed_case(N * 3 + H + page, B, H, k, N, page, cache, by_slot, dense, wide)
    freq = C.chai_rotary_frequencies(rot).cuda() if rot else None
    C.chai_paged_append_packed(s["q"], s["k_new"], s["v_new"], None if dense else dev(s["rep"]), dev(s["rows"]), dev(s["pos"]), dev(s["slots"]),
                               freq, s["q_out"], *s["pages"], *s["scales"], layout=layout_of(layout), gain=1.5 if rot else 1.0, k_by_slot=by_slot)
    torch.cuda.synchronize()
    # the same rows by the call on blocks (every head, fp32: their values before they are stored)
    def turn(x):
        x = x.float().transpose(0, 1).contiguous()[None]
        if not rot:
            return x[0].transpose(0, 1)
        y = torch.empty_like(x)
        C.chai_rotate_qk(x, None, None, freq, y, None, 0, positions=dev(s["pos"][None]), layout=layout_of(layout), gain=1.5)
        return y[0].transpose(0, 1)
    tq, tk = turn(s["q"]), turn(s["k_new"])
    n_pages = s["pages"][0].shape[0]
    want_q = torch.full_like(s["q_out"], 7.0)
    want = [p.clone() for p in s["pages"]]
    want_scales = [None if x is None else x.clone() for x in s["scales"]]
    for n in range(N):
        b, slot = int(s["rows"][n]), int(s["slots"][n])
        if b < 0:
            continue
        slots = np.arange(k) if dense else np.flatnonzero(s["rep"][b] >= 0)
        heads = slots if dense else s["rep"][b][slots]
        want_q[n, heads] = tq[n, heads].to(want_q.dtype)
        if not 0 <= slot < n_pages * page:
            continue
        rows = (tk[n, slots if by_slot else heads].contiguous(), s["v_new"][n].float().contiguous())
        for i, (at, x) in enumerate(zip((torch.from_numpy(slots).cuda(), torch.arange(H, device="cuda")), rows)):
            if not len(x):
                continue
            if want_scales[i] is None:
                want[i][slot // page, at, slot % page] = x.to(want[i].dtype)
            else:
                want[i][slot // page, at, slot % page], want_scales[i][slot // page, at, slot % page] = C.chai_quantize_rows(x)
    torch.cuda.synchronize()
    assert torch.equal(s["q_out"], want_q)
    for i in range(2):
        assert torch.equal(s["pages"][i], want[i]), i
        assert want_scales[i] is None or torch.equal(s["scales"][i], want_scales[i])


@pytest.mark.parametrize("cache", ["bf16", "e4m3_f32"])
@pytest.mark.parametrize("by_slot", [False, True])
def test_packed_views_of_a_block(cache, by_slot):
    """A row's blocks [heads,N,128] as the projections leave them, queries turned in place, against the same tokens dense."""
    B, H, k, N = 1, 6, 3, 37
    s, t = (packed_case(41, B, H, k, N, 16, cache, by_slot) for _ in range(2))
    freq = C.chai_rotary_frequencies(96).cuda()
    views = {n: s[n].transpose(0, 1).contiguous().transpose(0, 1) for n in ("q", "k_new", "v_new")}
    args = (dev(s["rep"]), dev(s["rows"]), dev(s["pos"]), dev(s["slots"]), freq)
    s["q_out"].copy_(s["q"])
    C.chai_paged_append_packed(s["q"], s["k_new"], s["v_new"], *args, s["q_out"], *s["pages"], *s["scales"], k_by_slot=by_slot)
    C.chai_paged_append_packed(views["q"], views["k_new"], views["v_new"], *args, views["q"], *t["pages"], *t["scales"], k_by_slot=by_slot)
    torch.cuda.synchronize()
    assert torch.equal(views["q"], s["q_out"])
    for i in range(2):
        assert torch.equal(s["pages"][i], t["pages"][i]) and (s["scales"][i] is None or torch.equal(s["scales"][i], t["scales"][i]))


def test_packed_queries_in_place_and_without_queries():
    s, t, u = (packed_case(21, 3, 6, 3, 40, 16, "bf16", False) for _ in range(3))
    freq = C.chai_rotary_frequencies(128).cuda()
    args = lambda x: (dev(x["rep"]), dev(x["rows"]), dev(x["pos"]), dev(x["slots"]), freq)  # noqa: E731
    s["rep"][1] = t["rep"][1] = u["rep"][1] = [2, 2, 2]    # a head in three slots
    s["q_out"].copy_(s["q"])
    C.chai_paged_append_packed(s["q"], s["k_new"], s["v_new"], *args(s), s["q_out"], *s["pages"])
    C.chai_paged_append_packed(t["q"], t["k_new"], t["v_new"], *args(t), t["q"], *t["pages"])
    C.chai_paged_append_packed(None, u["k_new"], u["v_new"], *args(u), None, *u["pages"])
    torch.cuda.synchronize()
    assert torch.equal(s["q_out"], t["q"]) and not torch.equal(s["q"], t["q"])
    for i in range(2):
        assert torch.equal(s["pages"][i], t["pages"][i]) and torch.equal(s["pages"][i], u["pages"][i])


def test_packed_recorded_and_on_another_stream():
    s = packed_case(31, 4, 6, 2, 30, 16, "e4m3", True)
    freq, rep, rows = C.chai_rotary_frequencies(128).cuda(), dev(s["rep"]), dev(s["rows"])
    pos, slots = dev(s["pos"]), dev(s["slots"])
    call = lambda stream=None: C.chai_paged_append_packed(s["q"], s["k_new"], s["v_new"], rep, rows, pos, slots, freq, s["q_out"], *s["pages"],  # noqa: E731
                                                          *s["scales"], k_by_slot=True, stream=stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    g = np.random.default_rng(32)
    for _ in range(4):
        for t in (s["q"], s["k_new"], s["v_new"]):
            t.copy_(torch.from_numpy(g.standard_normal(tuple(t.shape)).astype(np.float32)))
        pos.copy_(dev(g.integers(0, 5000, 30)))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (s["q_out"], *s["pages"], *s["scales"])]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (s["q_out"], *s["pages"], *s["scales"])))


def test_packed_offsets_beyond_32_bits():
    """The last page of pools of more than 2^32 bytes."""
    H, k, page, n_pages, N = 72, 2, 256, 1000, 9
    g = np.random.default_rng(51)
    new = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).cuda().to(torch.bfloat16)  # noqa: E731
    v_pages = torch.zeros((n_pages, H, page, D), dtype=torch.bfloat16, device="cuda")
    k_pages = torch.zeros((n_pages, k, page, D), dtype=torch.bfloat16, device="cuda")
    q, keys, v, freq = new(N, H, D), new(N, k, D), new(N, H, D), C.chai_rotary_frequencies(128)
    slots = (n_pages - 1) * page + page - 1 - np.arange(N)
    pos = np.arange(5, 5 + N)
    C.chai_paged_append_packed(q, keys, v, dev([[1, 70]]), dev(np.zeros(N)), dev(pos), dev(slots), freq.cuda(), q, k_pages, v_pages, k_by_slot=True)
    torch.cuda.synchronize()
    at = torch.from_numpy(slots % page).cuda()
    assert torch.equal(v_pages[-1][:, at], v.transpose(0, 1))
    want, mag = turned(keys.transpose(0, 1).double().cpu().numpy(), pos, freq.numpy(), "halves", 1.0)
    assert_rounded(k_pages[-1][:, at], want, mag, "bf16", "last page")
    v_pages[-1][:, at] = 0
    assert not bool(v_pages.view(torch.int64).any())


def test_empty_calls():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    i = lambda *s: z(*s, dt=torch.int32)  # noqa: E731
    freq = C.chai_rotary_frequencies(128).cuda()
    for B, Tn in ((0, 3), (2, 0)):
        q, kc = z(B, 4, Tn, D), torch.full((B, 2, 5, D), 3.0, device="cuda", dtype=torch.bfloat16)
        C.chai_rotate_qk(q, z(B, 2, Tn, D), i(B, 2), freq, z(B, 4, Tn, D), kc, 1)
        assert bool((kc == 3.0).all())
    pages = torch.full((3, 2, 8, D), 3.0, device="cuda", dtype=torch.bfloat16), torch.full((3, 4, 8, D), 3.0, device="cuda", dtype=torch.bfloat16)
    C.chai_paged_append_packed(z(0, 4, D), z(0, 4, D), z(0, 4, D), i(2, 2), i(0), i(0), i(0), freq, z(0, 4, D), *pages)
    C.chai_paged_place_tokens(i(0), i(0), i(0, 4), i(9), i(1), 8, i(0), i(1), i(0), i(1), i(6), i(6), i(6), C.alloc_paged_place_workspace(0))
    C.chai_paged_release_pages(i(0), i(0), i(0, 4), i(9), i(1), 8, i(0), i(1))
    x = z(0, 3, 64)
    C.chai_project_qk_adapted(x, z(4 * D, 64), z(4 * D, 64), i(0, 2), i(0), z(1, 8, 64), z(1, 4 * D, 8), None, None, None, z(0, 4, 3, D), z(0, 2, 3, D), 0,
                              C.alloc_adapted_workspace(0, 3, 8))
    torch.cuda.synchronize()
    assert all(bool((p == 3.0).all()) for p in pages)
