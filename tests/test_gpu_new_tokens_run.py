"""New tokens from activations to attention, as a server makes the calls: places in pages, projections with every request's adapter,
queries and keys turned, rows written, attention; the step recorded once and replayed while rows grow, end and come back.  Every stage is held
to 64 bits of what the one before left (bars: see the tests of the calls)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2403_08058_amd as C
import workloads as W
from gpu_util import RTOL, rows_close

D, BF16, I32 = 128, torch.bfloat16, torch.int32
SCALE = float(np.float32(D ** -0.5))


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


class Layer:
    """One layer of a server of B requests: weights, adapters, maps, pages; what is known of every request's positions on the host."""

    def __init__(self, seed, B, H, k, width, R, n_adapters, page, n_pages, longest, cache, rot, layout):
        self.g, self.gen = np.random.default_rng(seed), torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.B, self.H, self.k, self.width, self.page, self.n_pages, self.longest, self.cache = B, H, k, width, page, n_pages, longest, cache
        new = lambda std, *s: torch.randn(s, generator=self.gen, device="cuda").mul_(std).to(BF16)  # noqa: E731
        self.w = [new(width ** -0.5, H * D, width) for _ in "qk"]
        self.a = [new(width ** -0.5, n_adapters, R, width) for _ in "qk"]
        self.b = [new(R ** -0.5, n_adapters, H * D, R) for _ in "qk"]
        self.scale, self.ids = torch.full((n_adapters,), 1.5, device="cuda"), dev(self.g.integers(-1, n_adapters, B))
        self.rep = np.stack([np.sort(self.g.permutation(H)[:k]) for _ in range(B)])
        h2c = self.g.integers(0, k, (B, H))
        for b in range(B):
            h2c[b, self.rep[b]] = np.arange(k)
        self.h2c, self.rep_d, self.maps = h2c, dev(self.rep), None
        self.h2c_d = dev(h2c)
        blocks = -(-longest // page)
        self.t = {"seq_lens": dev(np.zeros(B)), "block_table": dev(np.full((B, blocks), -1)), "free_pages": dev(self.g.permutation(n_pages)),
                  "n_free": dev([n_pages])}
        self.lens = np.zeros(B, np.int64)
        coded = cache == "e4m3"
        self.pages = [torch.full((n_pages, s, page, D), 0x7f if coded else float("nan"), dtype=torch.uint8 if coded else BF16, device="cuda") for s in (k, H)]
        self.scales = [torch.full((n_pages, s, page), float("nan"), device="cuda") if coded else None for s in (k, H)]
        self.held = {"k_scales": self.scales[0], "v_scales": self.scales[1]}
        self.freq, self.layout, self.R = C.chai_rotary_frequencies(rot, kind=C.CHAI_ROPE_TURNS, factor=8.0, original_length=64.0).cuda(), layout, R
        self.known = {b: [[], []] for b in range(B)}       # keys and values of every position, as they were given to the pages
        self.place_ws, self.project_ws = C.alloc_paged_place_workspace(B), C.alloc_adapted_workspace(B, longest, R)
        self.attend_ws = C.alloc_paged_workspace(B, H, k, longest)
        self.out = torch.zeros((B, H, D), device="cuda")

    def x_of(self, *shape):
        return torch.randn((*shape, self.width), generator=self.gen, device="cuda").to(BF16)

    def places(self, N):
        return {"granted": dev(np.zeros(self.B)), "offsets": dev(np.zeros(self.B + 1)), "token_rows": dev(np.zeros(N)), "positions": dev(np.zeros(N)),
                "slots": dev(np.zeros(N))}

    def place(self, counts, out):
        C.chai_paged_place_tokens(counts, **self.t, page=self.page, new_lens=self.t["seq_lens"], n_left=self.t["n_free"], **out,
                                  workspace=self.place_ws)

    def project(self, x, rows, q, keys):
        C.chai_project_qk_adapted(x, *self.w, self.rep_d[rows], self.ids[rows], self.a[0], self.b[0], self.a[1], self.b[1], self.scale, q, keys,
                                  0, self.project_ws)

    def turned(self, x, pos):
        """x [n,heads,128] at positions pos, in 64 bits."""
        rot = 2 * len(self.freq)
        angle = (torch.from_numpy(np.asarray(pos)).cuda().double()[:, None] * self.freq)[:, None]
        y = x.double().clone()
        i, j = (slice(0, rot, 2), slice(1, rot, 2)) if self.layout == C.CHAI_ROPE_PAIRS else (slice(0, rot // 2), slice(rot // 2, rot))
        a, b = y[..., i].clone(), y[..., j].clone()
        y[..., i], y[..., j] = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
        return y

    def check_projection(self, x, b, q, keys):
        """q [H,n,128], keys [k,n,128] of row b's activations x [n,width]."""
        a = int(self.ids[b])
        x = x.double()
        for p, got in ((0, q[self.rep[b]]), (1, keys)):
            for j, r in enumerate(self.rep[b]):
                cols = slice(r * D, (r + 1) * D)
                w = self.w[p][cols].double().t().contiguous()
                want, allowed = x @ w, 3e-6 * (x.abs() @ w.abs())
                if a >= 0:
                    down, up = self.a[p][a].double().t().contiguous(), self.b[p][a, cols].double().t().contiguous()
                    t = 1.5 * (x @ down)
                    want = want + t @ up
                    allowed = allowed + 3e-6 * 1.5 * (x.abs() @ down.abs()) @ up.abs() + (2.0 ** -17 + 2.0 ** -24 + 3e-6) * t.abs() @ up.abs()
                assert bool(((got[j].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -8 * allowed + allowed).all()), (b, j, p)

    def written(self, b, keys, values):
        """What the pages hold of rows [n,streams,128] (keys turned, in 64 bits)."""
        for i, x in enumerate((keys, values)):
            self.known[b][i].append(x.double())

    def check_pages(self, b):
        n = int(self.lens[b])
        got = [torch.zeros((1, s, n, D), device="cuda", dtype=torch.float32 if self.cache == "e4m3" else BF16) for s in (self.k, self.H)]
        C.chai_paged_gather_kv(*self.pages, self.t["block_table"][b:b + 1], dev([0]), None, *got, **self.held)
        for i in range(2):
            want = torch.cat(self.known[b][i], 0).transpose(0, 1)
            x = got[i][0].double()
            if self.cache == "e4m3":
                # half a step of a code (2^-4 of it, or of the smallest normal, 2^-6, of rows of at most 448 times their scale), and 2^-20 of the rest
                top = want.abs().amax(-1, keepdim=True)
                bar = (2.0 ** -4 + 2.0 ** -20) * want.abs() + 2.0 ** -10 * top / 448 + 2.0 ** -20 * top / 448
            else:
                bar = (2.0 ** -8 + 2.0 ** -20) * want.abs() + 2.0 ** -50
            assert bool(((x - want).abs() <= bar).all()), (b, i, float(((x - want).abs() - bar).max()))
        return got

    def check_attention(self, q, b):
        """out[b] against 64 bits over what the pages hold; q [H,128] as it was attended with."""
        keys, values = (x[0].double() for x in self.check_pages(b))
        s = SCALE * (keys * q[self.rep[b]].double()[:, None]).sum(-1)
        p = torch.softmax(s, -1)[torch.from_numpy(self.h2c[b]).cuda()]
        want = (p[..., None] * values).sum(1)
        ok, worst = rows_close(self.out[b].cpu().numpy(), want.cpu().numpy(), RTOL[W.BF16])
        assert ok, (b, worst)


@pytest.mark.parametrize("cache,rot,layout", [("bf16", 128, C.CHAI_ROPE_HALVES), ("e4m3", 96, C.CHAI_ROPE_PAIRS)])
def test_a_server_of_new_tokens(cache, rot, layout):
    print(f"[new tokens] a run over {cache} pages", flush=True)
    B, H, k, page, longest = 5, 6, 3, 8, 90
    L = Layer(91, B, H, k, 256, 8, 3, page, 30, longest, cache, rot, layout)

    # ---- the step: one token of every row that holds a request (counts say which), recorded once
    N = 8
    counts, x = dev(np.zeros(B)), L.x_of(B, 1)
    q, keys, v = torch.zeros((B, H, 1, D), dtype=BF16, device="cuda"), torch.zeros((B, k, 1, D), dtype=BF16, device="cuda"), torch.zeros((B, H, D), dtype=BF16, device="cuda")
    turned_q = torch.zeros((B, H, D), dtype=BF16, device="cuda")
    every = {n: dev(np.zeros(B)) for n in ("rows", "positions", "slots")}
    places = L.places(N)
    index = torch.arange(B, device="cuda")

    def step():
        L.place(counts, places)
        L.project(x, slice(None), q, keys)
        # the tokens of all B rows: those without one have no slot (their number in the block is the next row's)
        at = places["offsets"][:B].long().clamp(max=N - 1)
        has = (counts > 0) & (places["granted"] > 0)
        every["rows"].copy_(torch.where(has, index, -torch.ones_like(index)))
        every["positions"].copy_(places["positions"][at])
        every["slots"].copy_(torch.where(has, places["slots"][at].long(), -torch.ones_like(at)))
        C.chai_paged_append_packed(q[:, :, 0], keys[:, :, 0], v, L.rep_d, every["rows"], every["positions"], every["slots"], L.freq, turned_q,
                                   *L.pages, **L.held, layout=L.layout, k_by_slot=True)
        C.chai_paged_decode_attention(turned_q, *L.pages, L.h2c_d, L.rep_d, L.t["block_table"], L.t["seq_lens"], longest, SCALE, L.out, L.attend_ws,
                                      **L.held)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                             # (no row has a token: nothing is written)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()

    def prompt(rows):
        """Prompts of several rows {row: tokens}, placed in one block; projected and turned row by row, written together."""
        new = np.zeros(B, np.int64)
        for b, n in rows.items():
            new[b] = n
        total = int(new.sum())
        out = L.places(total + 3)
        L.place(dev(new), out)
        qs, ks, vs = (torch.zeros((total + 3, s, D), dtype=BF16, device="cuda") for s in (H, k, H))
        at = 0
        for b in sorted(rows):
            n = rows[b]
            xb = L.x_of(1, n)
            qb, kb = torch.zeros((1, H, n, D), dtype=BF16, device="cuda"), torch.zeros((1, k, n, D), dtype=BF16, device="cuda")
            L.project(xb, slice(b, b + 1), qb, kb)
            torch.cuda.synchronize()
            L.check_projection(xb[0], b, qb[0], kb[0])
            qs[at:at + n], ks[at:at + n] = qb[0].transpose(0, 1), kb[0].transpose(0, 1)
            vs[at:at + n] = torch.randn((n, H, D), generator=L.gen, device="cuda").to(BF16)
            L.written(b, L.turned(ks[at:at + n], np.arange(L.lens[b], L.lens[b] + n)), vs[at:at + n])
            L.lens[b] += n
            at += n
        C.chai_paged_append_packed(qs, ks, vs, L.rep_d, out["token_rows"], out["positions"], out["slots"], L.freq, qs, *L.pages, **L.held,
                                   layout=L.layout)
        torch.cuda.synchronize()
        assert out["granted"].tolist() == [1] * B and L.t["seq_lens"].tolist() == L.lens.tolist()
        for b in rows:
            L.check_pages(b)

    def steps(count):
        for _ in range(count):
            has = L.lens > 0
            counts.copy_(dev(has))
            x.copy_(L.x_of(B, 1))
            v.copy_(torch.randn((B, H, D), generator=L.gen, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            assert places["granted"].tolist() == [1] * B
            for b in np.flatnonzero(has):
                L.check_projection(x[b], b, q[b], keys[b])
                want = L.turned(q[b, :, 0][None], [L.lens[b]])[0][L.rep[b]]
                got = turned_q[b][L.rep[b]].double()
                assert bool(((got - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs() + 2.0 ** -50).all())
                L.written(b, L.turned(keys[b, :, 0][None], [L.lens[b]]), v[b][None])
                L.lens[b] += 1
            assert L.t["seq_lens"].tolist() == L.lens.tolist()
            for b in range(B):
                if L.lens[b] > 0:
                    L.check_attention(turned_q[b], b)
                else:
                    assert bool((L.out[b] == 0).all())

    def end(b, keep=0):
        kept = dev([keep if r == b else 1 << 20 for r in range(B)])
        C.chai_paged_release_pages(kept, **L.t, page=page, new_lens=L.t["seq_lens"], n_left=L.t["n_free"])
        L.lens[b] = keep
        for i in range(2):
            L.known[b][i] = [torch.cat(L.known[b][i], 0)[:keep]] if keep else []

    prompt({0: 13, 3: 5, 4: 40})
    steps(3)
    prompt({1: 24, 4: 9})                                  # a new request, and one that goes on
    steps(2)
    end(3)
    end(4, keep=50)                                        # two pages less
    steps(2)
    prompt({3: 30, 2: 1})
    steps(3)
    torch.cuda.synchronize()
    held = L.t["block_table"][L.t["block_table"] >= 0].tolist()
    free = L.t["free_pages"][:int(L.t["n_free"])].tolist()
    assert sorted(held + free) == list(range(30))          # no page lost, none in two places
    # a row that there are no pages for gets nothing, and is as it was
    lens, left = L.t["seq_lens"].tolist(), int(L.t["n_free"])
    out = L.places(100)
    L.place(dev([0, 0, 88, 0, 0]), out)
    torch.cuda.synchronize()
    assert (left * page < 88) == (out["granted"].tolist() == [1, 1, 0, 1, 1]) and (left * page >= 88 or L.t["seq_lens"].tolist() == lens)


def test_prompt_attention_behind_turned_projections():
    """Projections with adapters, queries and keys turned in place, prompt attention over the compact cache, the rows copied into pages:
    one step over the pages equals one over the cache."""
    B, H, k, Tn, width, R, page = 2, 8, 3, 75, 192, 16, 16
    L = Layer(17, B, H, k, width, R, 2, page, 40, 96, "bf16", 128, C.CHAI_ROPE_HALVES)
    x, cap = L.x_of(B, Tn), 96
    q, kc = torch.zeros((B, H, Tn, D), dtype=BF16, device="cuda"), torch.zeros((B, k, cap, D), dtype=BF16, device="cuda")
    v = torch.randn((B, H, cap, D), generator=L.gen, device="cuda").to(BF16)
    C.chai_project_qk_adapted(x, *L.w, L.rep_d, L.ids, L.a[0], L.b[0], L.a[1], L.b[1], L.scale, q, kc, 0, L.project_ws)
    torch.cuda.synchronize()
    for b in range(B):
        L.check_projection(x[b], b, q[b], kc[b, :, :Tn])
    want_k = [L.turned(kc[b, :, :Tn].transpose(0, 1), np.arange(Tn)) for b in range(B)]
    C.chai_rotate_qk(q, kc[:, :, :Tn], L.rep_d, L.freq, q, kc, 0)
    out = torch.zeros((B, H, Tn, D), device="cuda")
    ws = torch.empty((C.chai_prefill_workspace_bytes(B, H, k, Tn),), dtype=torch.uint8, device="cuda")
    C.chai_prefill_attention(q, kc, v, L.h2c_d, L.rep_d, 0, SCALE, out, ws)
    torch.cuda.synchronize()
    for b in range(B):
        got = kc[b, :, :Tn].transpose(0, 1).double()
        assert bool(((got - want_k[b]).abs() <= (2.0 ** -8 + 2.0 ** -20) * want_k[b].abs() + 2.0 ** -50).all())
        keys = kc[b, :, :Tn].double()
        s = SCALE * (q[b][L.rep[b]].double() @ keys.transpose(1, 2).contiguous())
        p = torch.softmax(s.masked_fill(torch.ones((Tn, Tn), device="cuda").triu(1).bool(), -float("inf")), -1)[torch.from_numpy(L.h2c[b]).cuda()]
        ok, worst = rows_close(out[b].cpu().numpy(), (p @ v[b, :, :Tn].double()).cpu().numpy(), 2e-3)
        assert ok, worst
    # the same rows, row by row as packed views (turned already: no frequencies), then the last token's query again
    places = L.places(B * Tn)
    L.place(dev([Tn] * B), places)
    for b in range(B):
        part = slice(b * Tn, (b + 1) * Tn)
        C.chai_paged_append_packed(None, kc[b, :, :Tn].transpose(0, 1), v[b, :, :Tn].transpose(0, 1), L.rep_d, places["token_rows"][part], None,
                                   places["slots"][part], None, None, *L.pages, k_by_slot=True)
    last = q[:, :, Tn - 1].contiguous()
    C.chai_paged_decode_attention(last, *L.pages, L.h2c_d, L.rep_d, L.t["block_table"], L.t["seq_lens"], 96, SCALE, L.out, L.attend_ws)
    over_cache = torch.zeros_like(L.out)
    C.chai_decode_attention(last, kc, v, L.h2c_d, L.rep_d, Tn, SCALE, over_cache, C.alloc_workspace(B, H, k, cap, D, C.CHAI_BF16))
    torch.cuda.synchronize()
    ok, worst = rows_close(L.out.cpu().numpy(), over_cache.cpu().numpy(), 2 * RTOL[W.BF16])
    assert ok, worst
