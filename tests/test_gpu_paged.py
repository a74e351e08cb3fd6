"""Caches in pages on the GPU: writing, attention of one new token per request, both at once, reading back, against a plain
evaluation in 64 bits (attention) or bit for bit (rows that are copied or quantised).

Tolerances: attention is held to the bars of the contiguous decode kernels (gpu_util.RTOL, normwise per output row and per
element), which a single dropped or doubled token of these lengths exceeds by far.  8-bit caches are compared with the codes
they hold, so their rounding is not part of the comparison.  Codes times scales rounded to bf16 are off by at most half a step
of bf16, 2^-8 of the value, and the fp32 product before it by 2^-24."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2403_08058_amd as C
import workloads as W

from gpu_util import RTOL, guarded, guards_intact, rows_close

D = 128
SCALE = float(np.float32(1.0 / np.sqrt(D)))
NEW = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.bfloat16, "e4m3/f32": torch.float32}
BAR = {"f32": RTOL[W.F32], "bf16": RTOL[W.BF16], "e4m3": RTOL[W.BF16], "e4m3/f32": RTOL[W.F32]}


def held(pages, scales):
    """The values that pages hold, in 64 bits."""
    if scales is None:
        return pages.double()
    return pages.view(torch.float8_e4m3fn).double() * scales.double().unsqueeze(-1)


class Setting:
    """A pool of pages with rows of the given lengths in it, in random order."""

    def __init__(self, seed, cache, H, k, page, lengths, blocks=None, free=3, clustered=None):
        self.g = g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        host = np.random.default_rng(seed)
        self.cache, self.H, self.k, self.page, self.B = cache, H, k, page, len(lengths)
        lengths = np.asarray(lengths, np.int64)
        need = -(-np.maximum(lengths, 0) // page)
        self.blocks = blocks = int(max(need.max(initial=0), 1)) if blocks is None else blocks
        self.n_pages = int(need.sum()) + free
        order = host.permutation(self.n_pages)
        table = host.choice([-1, -7, self.n_pages, 1 << 30, -(1 << 31), 0], (self.B, blocks))     # stale entries
        at = 0
        for b in range(self.B):
            table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        self.host_table = table.astype(np.int32)
        self.table = torch.from_numpy(self.host_table).cuda()
        self.lengths = torch.from_numpy(lengths.astype(np.int32)).cuda()
        self.host_lengths = lengths
        self.dtype = NEW[cache]
        self.k_pages, self.k_scales = self.pool(k)
        self.v_pages, self.v_scales = self.pool(H)
        self.scales = {"k_scales": self.k_scales, "v_scales": self.v_scales}
        self.h2c = self.rep = None
        if (k < H) if clustered is None else clustered:
            h2c, rep = W.random_membership(W.rng(seed, 0, "member"), self.B, H, k)
            self.h2c, self.rep = torch.from_numpy(h2c).cuda(), torch.from_numpy(rep).cuda()

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda").to(self.dtype)

    def pool(self, streams):
        shape = (self.n_pages, streams, self.page, D)
        if not self.cache.startswith("e4m3"):
            return self.normal(*shape), None
        x = torch.randn(shape, generator=self.g, device="cuda").mul_(120.0).clamp_(-448.0, 448.0)
        return x.to(torch.float8_e4m3fn).view(torch.uint8), torch.rand(shape[:3], generator=self.g, device="cuda").add_(0.5).mul_(0.008)

    def places(self, b, first, n):
        """(i, page, place) of the positions first + i that are in a page, i < n."""
        t = np.arange(first, first + n)
        i = np.flatnonzero((t >= 0) & (t < self.blocks * self.page))
        at = self.host_table[b, t[i] // self.page]
        ok = (at >= 0) & (at < self.n_pages)
        return i[ok], at[ok].astype(np.int64), (t[i] % self.page)[ok]

    def maps(self, b):
        if self.h2c is None:
            return list(range(self.H)), list(range(self.H))
        return self.h2c[b].tolist(), self.rep[b].tolist()

    def expected(self, q, T_max):
        keys, values = held(self.k_pages, self.k_scales), held(self.v_pages, self.v_scales)
        out = torch.zeros((self.B, self.H, D), dtype=torch.float64, device="cuda")
        for b in range(self.B):
            _, at, slot = self.places(b, 0, int(min(max(self.host_lengths[b], 0), T_max)))
            if not len(at):
                continue
            at, slot = torch.from_numpy(at).cuda(), torch.from_numpy(slot).cuda()
            h2c, rep = self.maps(b)
            s = SCALE * (keys[at, :, slot] * q[b].double()[rep]).sum(-1)                 # [T, k]
            p = torch.softmax(s, 0)[:, h2c]
            out[b] = (p.unsqueeze(-1) * values[at, :, slot]).sum(0)
        return out

    def attend(self, q, T_max, stream=None):
        whole, out = guarded((self.B, self.H, D), torch.float32, float("nan"))
        ws = C.alloc_paged_workspace(self.B, self.H, self.k, T_max)
        ws.fill_(0xFF)
        C.chai_paged_decode_attention(q, self.k_pages, self.v_pages, self.h2c, self.rep, self.table, self.lengths, T_max, SCALE,
                                      out, ws, **self.scales, stream=stream)
        torch.cuda.synchronize()
        assert guards_intact(whole, out.shape, float("nan"))
        return out

    def check(self, q, T_max=None):
        T_max = self.blocks * self.page if T_max is None else T_max
        out, ref = self.attend(q, T_max), self.expected(q, T_max)
        ok, worst = rows_close(out.cpu().numpy(), ref.cpu().numpy(), BAR[self.cache])
        assert ok, f"worst err/allowed {worst:.3g}"
        nothing = [b for b in range(self.B) if not len(self.places(b, 0, int(min(max(self.host_lengths[b], 0), T_max)))[0])]
        assert bool((out[nothing] == 0).all())
        return out


CACHES = ["f32", "bf16", "e4m3", "e4m3/f32"]


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("H,k,page,lengths", [
    (8, 3, 16, [1]),
    (8, 8, 8, [0, 1, 2, 7, 8, 9]),
    (5, 2, 16, [15, 16, 17, 31, 32, 33, 63, 64, 65]),
    (7, 3, 24, [250, 0, 500, 129, 1, 511]),
    (32, 8, 64, [700, 64, 0, 2048]),
    (9, 1, 128, [1300, 5]),
    (6, 6, 40, [333] * 3),
    (4, 2, 16, [4999, 3, 17]),
])
def test_attention(cache, H, k, page, lengths):
    print(f"[paged] attention {cache} H={H} k={k} page={page} lengths={lengths}", flush=True)
    s = Setting(9000 + H * 31 + page, cache, H, k, page, lengths)
    s.check(s.normal(s.B, H, D))


@pytest.mark.parametrize("B", [63, 64, 65, 130, 200])
def test_attention_many_rows(B):
    """More rows than lanes: their lengths are added up in two levels; runs of empty rows at either end and inside."""
    lengths = np.random.default_rng(B).integers(0, 90, B)
    lengths[:3] = 0
    lengths[B // 2:B // 2 + 5] = 0
    lengths[-2:] = 0
    s = Setting(9100 + B, "bf16", 3, 2, 16, lengths)
    s.check(s.normal(B, 3, D))


def test_attention_of_rows_that_are_all_empty():
    s = Setting(9150, "bf16", 4, 2, 16, [0, 0, 0], blocks=4)
    s.check(s.normal(3, 4, D))


@pytest.mark.parametrize("cache", ["f32", "e4m3"])
def test_absent_pages(cache):
    """Pages missing at the start, inside and at the end of rows, and rows without any: as if their positions were not there."""
    s = Setting(9200, cache, 6, 2, 16, [400, 77, 300, 16, 5000])
    s.host_table[0, [0, 3, 24]] = [-1, s.n_pages, -5]
    s.host_table[1, :] = -1
    s.host_table[2, 1:] = 1 << 30
    s.host_table[3, 0] = -1
    s.host_table[4, ::2] = -1
    s.table.copy_(torch.from_numpy(s.host_table))
    s.check(s.normal(s.B, 6, D))


@pytest.mark.parametrize("cache", ["f32", "bf16", "e4m3"])
def test_masked_places_may_hold_anything(cache):
    """Free pages and the places past a row's end hold infinities, NaN and the lowest value; lengths beyond T_max, negative."""
    s = Setting(9300, cache, 6, 3, 16, [37, 0, 201, 64], blocks=20)
    used = torch.zeros((s.n_pages, s.page), dtype=torch.bool)
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
    s.check(s.normal(s.B, 6, D))
    s.host_lengths = np.array([37, -3, 201, 64])
    s.lengths.copy_(torch.tensor([37, -3, 1 << 30, 64]))
    s.check(s.normal(s.B, 6, D), T_max=201)


def test_length_is_taken_into_the_bound():
    s = Setting(9350, "bf16", 4, 2, 16, [300, 100])
    s.check(s.normal(2, 4, D), T_max=133)


def test_scores_of_minus_infinity_and_nan():
    """-inf scores weigh nothing, a head with no others gets 0; NaN reaches the heads of its cluster and row alone."""
    s = Setting(9400, "f32", 6, 2, 16, [600, 90, 700])
    q = s.normal(3, 6, D).abs() + 0.5
    _, at, slot = s.places(0, 0, 600)
    s.k_pages[at[:400], :, slot[:400]] = -float("inf")
    _, at1, slot1 = s.places(1, 0, 90)
    s.k_pages[at1, 1, slot1] = -float("inf")
    _, at2, slot2 = s.places(2, 0, 700)
    s.k_pages[at2[350], 0, slot2[350], 5] = float("nan")
    out, ref = s.attend(q, 704), s.expected(q, 704)
    h2c = s.h2c.tolist()
    none = [h for h in range(6) if h2c[1][h] == 1]
    nan = [h for h in range(6) if h2c[2][h] == 0]
    assert none and nan and bool((out[1, none] == 0).all()) and bool(out[2, nan].isnan().all())
    ref[1, none] = 0.0
    out[2, nan] = 0.0
    ref[2, nan] = 0.0
    ok, worst = rows_close(out.cpu().numpy(), ref.cpu().numpy(), BAR["f32"])
    assert ok, worst


def test_values_near_the_largest_and_the_smallest_float():
    s = Setting(9450, "f32", 4, 4, 16, [3000, 700])
    s.k_pages.mul_(1e-3)
    s.v_pages.copy_(torch.where(s.v_pages > 0, 3.3e38, 3.0e38))
    s.check(s.normal(2, 4, D))
    s.v_pages.normal_(generator=s.g).mul_(1e-37)
    s.check(s.normal(2, 4, D))


def test_large_scores():
    """Scores of some hundreds: one position has all the weight, wherever the running maximum was before."""
    s = Setting(9500, "bf16", 8, 8, 32, [2000, 1500, 40])
    ref_q = s.normal(3, 8, D) * 40
    keys = s.k_pages
    out, ref = s.attend(ref_q, 2016), s.expected(ref_q, 2016)
    # products of this size are rounded in steps of 2^-24 of some hundreds: a weight is off by exp of that, 128 sums of them
    top = float(SCALE * ref_q.float().abs().amax() * keys.float().abs().amax() * D)
    bar = max(BAR["bf16"], 4 * 2.0 ** -24 * top)
    err = (out.double() - ref).abs().amax(-1) / ref.abs().amax(-1)
    assert float(err.max()) <= bar, (float(err.max()), bar)


def test_shared_pages_and_other_streams():
    """Two rows share their first pages; the call runs on a stream of its own."""
    s = Setting(9550, "bf16", 6, 2, 16, [200, 150])
    s.host_table[1, :6] = s.host_table[0, :6]
    s.table.copy_(torch.from_numpy(s.host_table))
    q = s.normal(2, 6, D)
    here = s.check(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(s.attend(q, s.blocks * s.page, stream=side), here)


def test_results_do_not_change_from_call_to_call():
    s = Setting(9600, "e4m3", 16, 4, 16, [900, 1, 333, 0, 2500])
    q = s.normal(5, 16, D)
    first = s.attend(q, 2512)
    for _ in range(5):
        assert torch.equal(s.attend(q, 2512), first)


def test_pool_beyond_four_gigabytes():
    """Rows that lie past 2^32 bytes (and past 2^31 elements) into their pool."""
    page, H, n_pages = 128, 40, 3600                      # 4.7 GB of values, a page holds 1.3 MB of them
    lengths = [300, 129]
    s = Setting(9650, "bf16", H, 2, page, lengths, free=0)
    k_pages = torch.empty((n_pages, 2, page, D), dtype=torch.bfloat16, device="cuda")
    v_pages = torch.empty((n_pages, H, page, D), dtype=torch.bfloat16, device="cuda")
    assert v_pages.numel() * 2 > 2 ** 32 and v_pages.numel() > 2 ** 31
    k_pages[-s.n_pages:], v_pages[-s.n_pages:] = s.k_pages, s.v_pages
    q = s.normal(2, H, D)
    ref = s.expected(q, 384)
    s.k_pages, s.v_pages = k_pages, v_pages
    s.table.add_(n_pages - s.n_pages)
    ok, worst = rows_close(s.attend(q, 384).cpu().numpy(), ref.cpu().numpy(), BAR["bf16"])
    assert ok, worst
    # written and read back there
    k_new, v_new = s.normal(2, H, 200, D), s.normal(2, H, 200, D)
    start = torch.tensor([100, 0], dtype=torch.int32, device="cuda")
    count = torch.tensor([200, 129], dtype=torch.int32, device="cuda")
    C.chai_paged_append_kv(k_new, v_new, s.rep, s.table, start, count, k_pages, v_pages)
    k_out, v_out = torch.zeros((2, 2, 200, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, H, 200, D), dtype=torch.bfloat16, device="cuda")
    C.chai_paged_gather_kv(k_pages, v_pages, s.table, start, count, k_out, v_out)
    torch.cuda.synchronize()
    for b, n in enumerate(count.tolist()):
        assert torch.equal(v_out[b, :, :n], v_new[b, :, :n])
        assert torch.equal(k_out[b, :, :n], k_new[b, s.rep[b].long(), :n])


# ------------------------------------------------------------------------------------------------- writing and reading back
def codes_of(x):
    """E4M3 codes and scales of rows, as they are defined: all in fp32, nearest, ties to even."""
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    largest = torch.full_like(amax, 448.0)                 # (a quotient with a number would be a product with its inverse)
    inv = largest / amax
    y = torch.where(amax == 0, torch.zeros_like(x), (x * inv).clamp(-448.0, 448.0))
    return y.to(torch.float8_e4m3fn).view(torch.uint8), (amax / largest).squeeze(-1)


def put(s, expect, k_new, v_new, start, count):
    """The same rows into copies of the pools, one row at a time."""
    k_pages, v_pages, k_scales, v_scales = expect
    for b in range(s.B):
        i, at, slot = s.places(b, int(start[b]), int(count[b]))
        if not len(i):
            continue
        i, at, slot = (torch.from_numpy(a).cuda() for a in (i, at, slot))
        _, rep = s.maps(b)
        used = torch.tensor([j for j in range(s.k) if rep[j] >= 0], dtype=torch.long, device="cuda")
        heads = torch.tensor([rep[j] for j in used.tolist()], dtype=torch.long, device="cuda")
        for pages, scales, x, streams in ((k_pages, k_scales, k_new[b, heads][:, i], used),
                                          (v_pages, v_scales, v_new[b][:, i], torch.arange(s.H, device="cuda"))):
            x = x.transpose(0, 1)
            if scales is not None:
                x, sc = codes_of(x)
                scales[at[:, None], streams[None, :], slot[:, None]] = sc
            pages[at[:, None], streams[None, :], slot[:, None]] = x


def bits(t):
    return None if t is None else t.view(torch.uint8) if t.dtype == torch.uint8 else t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def same_pools(s, expect):
    for got, want, name in zip((s.k_pages, s.v_pages, s.k_scales, s.v_scales), expect, ("k_pages", "v_pages", "k_scales", "v_scales")):
        assert (got is None) == (want is None) and (got is None or torch.equal(bits(got), bits(want))), name


def copies(s):
    return [None if t is None else t.clone() for t in (s.k_pages, s.v_pages, s.k_scales, s.v_scales)]


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("H,k,page,Tn,start,count", [
    (8, 3, 16, 1, [0, 15, 16, 399], None),
    (5, 5, 8, 1, [3, 7], [1, 0]),
    (6, 2, 24, 100, [0, 5, 23], [100, 37, 0]),
    (33, 7, 64, 300, [10, 0], [290, 131]),
    (4, 2, 16, 50, [-7, 360, 2147483640], None),           # begins before the first position, ends past the table
    (3, 1, 128, 129, [64], [200]),                         # more than there are
    (60, 12, 16, 390, [0] * 11 + [7], None),               # more than 262144 rows: shares of all rows' units
    (100, 28, 24, 333, [3, 0, 67, 200, -5, 1, 9, 0], [333, 0, 1, 200, 32, 31, 33, 64]),
])
def test_append_and_gather(cache, H, k, page, Tn, start, count):
    print(f"[paged] append {cache} H={H} k={k} page={page} Tn={Tn}", flush=True)
    B = len(start)
    s = Setting(9700 + Tn, cache, H, k, page, [400] * B)
    s.host_table[0, 1] = -1                                # nowhere to write to
    if page < 400:
        s.host_table[-1, -1] = s.n_pages
    s.table.copy_(torch.from_numpy(s.host_table))
    if s.rep is not None:
        s.rep[0, k - 1] = -1                               # a slot without a cluster keeps what it holds
    k_new, v_new = s.normal(B, H, Tn + 3, D), s.normal(B, H, Tn, D)
    k_new[0, :, 0], v_new[-1, 0, Tn - 1] = 0.0, 0.0        # rows of zeros
    n = [Tn] * B if count is None else [min(c, Tn) for c in count]
    expect = copies(s)
    put(s, expect, k_new, v_new, start, n)
    first = torch.tensor(start, dtype=torch.int32, device="cuda")
    counts = None if count is None else torch.tensor(count, dtype=torch.int32, device="cuda")
    C.chai_paged_append_kv(k_new, v_new, s.rep, s.table, first, counts, s.k_pages, s.v_pages, Tn, **s.scales)
    torch.cuda.synchronize()
    same_pools(s, expect)

    for dtype in ([s.dtype] if not cache.startswith("e4m3") else [torch.float32, torch.bfloat16]):
        (kw, k_out), (vw, v_out) = (guarded((B, streams, Tn, D), dtype, 7.0) for streams in (k, H))
        C.chai_paged_gather_kv(s.k_pages, s.v_pages, s.table, first, counts, k_out, v_out, **s.scales)
        torch.cuda.synchronize()
        assert guards_intact(kw, k_out.shape, 7.0) and guards_intact(vw, v_out.shape, 7.0)
        for got, pages, scales in ((k_out, s.k_pages, s.k_scales), (v_out, s.v_pages, s.v_scales)):
            want = torch.full(got.shape, 7.0, dtype=torch.float64, device="cuda")
            for b in range(B):
                i, at, slot = (torch.from_numpy(a).cuda() for a in s.places(b, start[b], n[b]))
                want[b, :, :n[b]] = 0.0
                want[b][:, i] = held(pages, scales)[at, :, slot].transpose(0, 1)
            if scales is None:
                assert torch.equal(bits(got), bits(want.to(dtype)))
            else:
                step = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8 + 2.0 ** -24
                tiny = 2.0 ** -149 if dtype == torch.float32 else 2.0 ** -133
                assert bool(((got.double() - want).abs() <= step * want.abs() + tiny).all())


def test_append_of_infinities_and_nan_copies_them():
    for cache in ("f32", "bf16"):
        s = Setting(9800, cache, 4, 2, 16, [64])
        k_new, v_new = s.normal(1, 4, 20, D), s.normal(1, 4, 20, D)
        v_new[0, 1, 3, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), -0.0])
        bits(v_new)[0, 2, 5, 9] = 0x7F81 if cache == "bf16" else 0x7F800001          # a signalling NaN
        expect = copies(s)
        put(s, expect, k_new, v_new, [3], [20])
        start = torch.tensor([3], dtype=torch.int32, device="cuda")
        C.chai_paged_append_kv(k_new, v_new, s.rep, s.table, start, None, s.k_pages, s.v_pages)
        k_out, v_out = torch.zeros((1, 2, 20, D), dtype=s.dtype, device="cuda"), torch.zeros((1, 4, 20, D), dtype=s.dtype, device="cuda")
        C.chai_paged_gather_kv(s.k_pages, s.v_pages, s.table, start, None, k_out, v_out)
        torch.cuda.synchronize()
        same_pools(s, expect)
        assert torch.equal(bits(v_out), bits(v_new))


def test_quantised_rows_are_those_of_the_row_quantiser():
    """Codes and scales bit for bit as chai_quantize_rows gives them, rows with infinities and NaN among them."""
    s = Setting(9850, "e4m3", 6, 6, 16, [96])
    x = s.normal(1, 6, 96, D) * torch.logspace(-30, 30, 96, device="cuda")[:, None].to(torch.bfloat16)
    x[0, 1, 4, 7], x[0, 2, 9, 0], x[0, 3, 10] = float("inf"), float("nan"), 0.0
    codes, scales = C.chai_quantize_rows(x.contiguous())
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    C.chai_paged_append_kv(x.contiguous(), x.contiguous(), None, s.table, start, None, s.k_pages, s.v_pages, **s.scales)
    torch.cuda.synchronize()
    _, at, slot = s.places(0, 0, 96)
    for pages, sc in ((s.k_pages, s.k_scales), (s.v_pages, s.v_scales)):
        assert torch.equal(pages[at, :, slot].transpose(0, 1), codes[0])
        assert torch.equal(bits(sc[at, :, slot].transpose(0, 1).contiguous()), bits(scales[0]))


# ------------------------------------------------------------------------------------------------- the step
@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("H,k,page,lengths", [
    (8, 3, 16, [1]),
    (6, 6, 8, [0, 1, 8, 9, 25]),
    (32, 8, 64, [700, 65, 0, 1024, 129]),
    (5, 2, 24, [2600, 24, 49]),
])
def test_step(cache, H, k, page, lengths):
    """The new rows are written as by the append, and attended to as they were stored."""
    print(f"[paged] step {cache} H={H} k={k} page={page} lengths={lengths}", flush=True)
    s = Setting(9900 + H, cache, H, k, page, lengths)
    if len(lengths) > 3:
        s.host_table[3, -1] = -1                           # perhaps no place for the new row of this one
        s.table.copy_(torch.from_numpy(s.host_table))
    q, k_new, v_new = s.normal(s.B, H, D), s.normal(s.B, H, D), s.normal(s.B, H, D)
    expect = copies(s)
    put(s, expect, k_new.unsqueeze(2), v_new.unsqueeze(2), s.host_lengths - 1, (s.host_lengths > 0).astype(int))
    T_max = s.blocks * page
    whole, out = guarded((s.B, H, D), torch.float32, float("nan"))
    ws = C.alloc_paged_workspace(s.B, H, k, T_max)
    ws.fill_(0xFF)
    C.chai_paged_decode_step(q, k_new, v_new, s.k_pages, s.v_pages, s.h2c, s.rep, s.table, s.lengths, T_max, SCALE, out, ws, **s.scales)
    torch.cuda.synchronize()
    assert guards_intact(whole, out.shape, float("nan"))
    same_pools(s, expect)
    ok, worst = rows_close(out.cpu().numpy(), s.expected(q, T_max).cpu().numpy(), BAR[cache])
    assert ok, worst


# sizes at which rows are shared between waves: up to 512 rows of heads and more, with and without clusters
SHARED = [
    (6, 6, 40, [2999, 1, 0, 700, 2048]),
    (32, 32, 16, [4150] + [17 * i for i in range(20)]),
    (32, 8, 16, [4150] + [17 * i for i in range(20)]),
]


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("H,k,page,lengths", SHARED)
def test_step_of_shared_rows(cache, H, k, page, lengths):
    """The same of long rows: written as by the append, attended to as stored, without the new rows the same again."""
    print(f"[paged] shared rows {cache} H={H} k={k} page={page}", flush=True)
    s = Setting(9960 + H + k, cache, H, k, page, lengths)
    s.host_table[0, 2] = -1
    s.table.copy_(torch.from_numpy(s.host_table))
    q, k_new, v_new = s.normal(s.B, H, D), s.normal(s.B, H, D), s.normal(s.B, H, D)
    expect = copies(s)
    put(s, expect, k_new.unsqueeze(2), v_new.unsqueeze(2), s.host_lengths - 1, (s.host_lengths > 0).astype(int))
    T_max = s.blocks * page
    whole, out = guarded((s.B, H, D), torch.float32, float("nan"))
    ws = C.alloc_paged_workspace(s.B, H, k, T_max)
    ws.fill_(0xFF)
    C.chai_paged_decode_step(q, k_new, v_new, s.k_pages, s.v_pages, s.h2c, s.rep, s.table, s.lengths, T_max, SCALE, out, ws, **s.scales)
    torch.cuda.synchronize()
    assert guards_intact(whole, out.shape, float("nan"))
    same_pools(s, expect)
    ok, worst = rows_close(out.cpu().numpy(), s.expected(q, T_max).cpu().numpy(), BAR[cache])
    assert ok, worst
    s.check(q)


# more than 256 (head, row) pairs of short rows: taken in the order of their lengths, a row's heads in that of their clusters
ORDERED = [
    (32, 8, [40, 0, 300, 300, 1, 40, 555, 0, 300, 17, 64, 65]),
    (52, 52, [100, 700, 0, 700, 3, 699]),
    (100, 30, [33, 400, 33]),                              # two heads per lane
    (130, 20, [200, 5, 90]),                               # more heads than that
    (300, 7, [70, 128]),                                   # one row is more than a workgroup per CU
    (5, 2, [(37 * i) % 211 for i in range(64)]),           # as many rows as lanes
    (5, 2, [(37 * i) % 211 for i in range(65)]),           # one more
    (16, 8, [0] * 20),
    (20, 3, [128] * 51),
]


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("H,k,lengths", ORDERED)
def test_rows_in_the_order_of_their_lengths(cache, H, k, lengths):
    print(f"[paged] ordered rows {cache} H={H} k={k} lengths={lengths}", flush=True)
    s = Setting(9980 + H, cache, H, k, 16, lengths, blocks=64)
    q = s.normal(s.B, H, D)
    first = s.check(q, T_max=999)
    s.lengths.copy_(torch.tensor([n if n else -5 - i for i, n in enumerate(lengths)]))      # rows without a position
    assert torch.equal(s.attend(q, 999), first)
    if len(lengths) > 2:
        s.lengths[2], s.host_lengths[2] = 1 << 30, 500                                      # one longer than the bound
        s.host_table[2, :32] = np.arange(32) % s.n_pages
        s.table.copy_(torch.from_numpy(s.host_table))
        s.check(q, T_max=500)


@pytest.mark.parametrize("maps", ["one", "skewed", "last"])
def test_clusters_of_any_size(maps):
    """All heads in one cluster, one cluster of nearly all, clusters without a head."""
    H, k = 72, 9
    s = Setting(9990, "bf16", H, k, 16, [100, 333, 20, 64])
    h2c, rep = torch.zeros((4, H), dtype=torch.int32), torch.zeros((4, k), dtype=torch.int32)
    if maps == "skewed":
        h2c[:, 3:11] = torch.arange(1, 9, dtype=torch.int32)
        rep[:, 1:] = torch.arange(3, 11, dtype=torch.int32)
    if maps == "last":
        h2c[:], rep[:, k - 1], rep[:, :k - 1] = k - 1, 5, -1
    s.h2c, s.rep = h2c.cuda(), rep.cuda()
    s.check(s.normal(4, H, D))


def test_slots_without_a_cluster():
    """Fewer clusters than slots: what the others' keys hold reaches nobody, short rows and long ones."""
    for T in (100, 3000):
        s = Setting(9965, "bf16", 8, 3, 16, [T, T // 2])
        s.h2c.clamp_(max=1)
        s.rep[:, 2] = -1
        s.k_pages[:, 2] = float("nan")
        q = s.normal(2, 8, D)
        out = s.attend(q, s.blocks * 16)
        s.k_pages[:, 2] = 0.0
        s.rep[:, 2] = 0
        ok, worst = rows_close(out.cpu().numpy(), s.expected(q, s.blocks * 16).cpu().numpy(), BAR["bf16"])
        assert ok, (T, worst)


def test_step_beyond_the_bound_writes_nothing():
    s = Setting(9950, "bf16", 4, 2, 16, [200, 90])
    q, k_new, v_new = s.normal(2, 4, D), s.normal(2, 4, D), s.normal(2, 4, D)
    expect = copies(s)
    put(s, expect, k_new.unsqueeze(2), v_new.unsqueeze(2), [0, 89], [0, 1])
    out = torch.empty((2, 4, D), dtype=torch.float32, device="cuda")
    C.chai_paged_decode_step(q, k_new, v_new, s.k_pages, s.v_pages, s.h2c, s.rep, s.table, s.lengths, 128, SCALE, out,
                             C.alloc_paged_workspace(2, 4, 2, 128))
    torch.cuda.synchronize()
    same_pools(s, expect)
    ok, worst = rows_close(out.cpu().numpy(), s.expected(q, 128).cpu().numpy(), BAR["bf16"])
    assert ok, worst


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_captured_step_replays_with_growing_rows(cache):
    """A step recorded into a graph, replayed with other queries, new rows and lengths, eager work in between."""
    s = Setting(9970, cache, 8, 3, 16, [30, 100, 0], blocks=12, free=40)
    order = np.random.default_rng(1).permutation(s.n_pages)[:36].reshape(3, 12)
    s.host_table = order.astype(np.int32)
    s.table.copy_(torch.from_numpy(s.host_table))
    q, k_new, v_new = s.normal(3, 8, D), s.normal(3, 8, D), s.normal(3, 8, D)
    out = torch.empty((3, 8, D), dtype=torch.float32, device="cuda")
    ws = C.alloc_paged_workspace(3, 8, 3, 192)
    call = lambda: C.chai_paged_decode_step(q, k_new, v_new, s.k_pages, s.v_pages, s.h2c, s.rep, s.table, s.lengths, 192, SCALE,  # noqa: E731
                                            out, ws, **s.scales)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for step in range(6):
        q.normal_(generator=s.g), k_new.normal_(generator=s.g), v_new.normal_(generator=s.g)
        s.host_lengths = np.array([30 + step, 100 + 17 * step, step])
        s.lengths.copy_(torch.from_numpy(s.host_lengths))
        graph.replay()
        torch.cuda.synchronize()
        ok, worst = rows_close(out.cpu().numpy(), s.expected(q, 192).cpu().numpy(), BAR[cache])
        assert ok, (step, worst)


def test_pages_and_contiguous_caches_agree():
    """The same rows in pages and in contiguous caches: the two decode paths against each other."""
    B, H, k, T, page = 3, 12, 4, 333, 32
    s = Setting(9990, "bf16", H, k, page, [T] * B)
    k_full, v_full = s.normal(B, H, T, D), s.normal(B, H, T, D)
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    C.chai_paged_append_kv(k_full, v_full, s.rep, s.table, start, None, s.k_pages, s.v_pages)
    k_compact = torch.zeros((B, k, T, D), dtype=torch.bfloat16, device="cuda")
    C.chai_compact_kcache(k_full, s.rep, k_compact, T)
    q = s.normal(B, H, D)
    ref = torch.empty((B, H, D), dtype=torch.float32, device="cuda")
    C.chai_decode_attention(q, k_compact, v_full, s.h2c, s.rep, T, SCALE, ref, C.alloc_workspace(B, H, k, T, D, C.CHAI_BF16))
    out = s.attend(q, T)
    # both are within the bar of the same values
    assert float(((out - ref).abs().amax(-1) / ref.abs().amax(-1)).max()) <= 2 * BAR["bf16"]
    k_out, v_out = torch.zeros_like(k_compact), torch.zeros_like(v_full)
    C.chai_paged_gather_kv(s.k_pages, s.v_pages, s.table, start, None, k_out, v_out)
    torch.cuda.synchronize()
    assert torch.equal(k_out, k_compact) and torch.equal(v_out, v_full)
