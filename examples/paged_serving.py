"""Requests of different lengths served out of one pool of pages, the way the calls on pages are meant to be used.

    python examples/paged_serving.py [--layers 4] [--heads 32] [--clusters 8] [--rows 16] [--page 64] [--cache bf16|e4m3]
                                     [--requests 48] [--steps 2048] [--eager] [--seed 1]

Requests arrive and leave.  A new one gets pages for its prompt; layer by layer its membership is decided on the first five
positions, its prompt attended to, and its keys (the representatives') and values written into pages.  Every step then adds a
token to every row: one call per layer writes the token's rows and attends, over lengths that only the device reads, so the
step is recorded into a HIP graph once and replayed while rows grow, come and go.  A row may be continued (a conversation's
next turn): its pages are read back into contiguous caches, which prompt attention takes.  Rows that end give their pages back.

There is no model here: Source draws the queries, keys and values that a layer's projections would give.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2403_08058_amd as C  # noqa: E402

D = 128                                    # head dimension
N_TOK = 5                                  # positions that membership is decided on
SCALE = float(np.float32(1.0 / np.sqrt(D)))


class Source:
    """What a model's projections would hand over: q, k, v [B,H,n,128] of a layer's n new tokens."""

    def __init__(self, heads: int, seed: int):
        self.H = heads
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def prompt(self, layer: int, row: int, n: int):
        return [torch.randn((1, self.H, n, D), generator=self.g, device="cuda").to(torch.bfloat16) for _ in range(3)]

    def token(self, layer: int, q, k, v):
        for t in (q, k, v):
            t.normal_(generator=self.g)


class Server:
    """`rows` places for requests of up to `longest` tokens, `n_pages` pages of `page` positions in every layer's pool."""

    def __init__(self, source, layers: int, heads: int, clusters: int, rows: int, longest: int, page: int, n_pages: int,
                 cache: str = "bf16", seed: int = 0):
        self.source, self.L, self.H, self.k = source, layers, heads, clusters
        self.rows, self.longest, self.page, self.n_pages = rows, longest, page, n_pages
        self.blocks = -(-longest // page)
        self.host = np.random.default_rng(seed)
        self.free = list(range(n_pages))
        # the table and the lengths: kept on the host, copied to where the kernels read them
        self.table_h = torch.full((rows, self.blocks), -1, dtype=torch.int32).pin_memory()
        self.lens_h = torch.zeros((rows,), dtype=torch.int32).pin_memory()
        self.table, self.lens = self.table_h.cuda(), self.lens_h.cuda()
        self.pools = [self._pool(cache) for _ in range(layers)]
        new = lambda *shape, dt=torch.bfloat16: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
        self.h2c = [new(rows, heads, dt=torch.int32) for _ in range(layers)]
        self.rep = [new(rows, clusters, dt=torch.int32) for _ in range(layers)]
        self.q, self.k_new, self.v_new = ([new(rows, heads, D) for _ in range(layers)] for _ in range(3))
        self.out = [new(rows, heads, D, dt=torch.float32) for _ in range(layers)]
        self.workspace = C.alloc_paged_workspace(rows, heads, clusters, longest)
        self.scratch = None                # of prompt attention
        self.graph = None

    def _pool(self, cache):
        shape = lambda streams: (self.n_pages, streams, self.page, D)  # noqa: E731
        dt = torch.uint8 if cache == "e4m3" else torch.bfloat16
        k, v = (torch.empty(shape(s), dtype=dt, device="cuda") for s in (self.k, self.H))
        scales = [torch.empty(shape(s)[:3], dtype=torch.float32, device="cuda") if cache == "e4m3" else None for s in (self.k, self.H)]
        return (k, v), {"k_scales": scales[0], "v_scales": scales[1]}

    # ---- pages
    def _grow(self, lengths: dict):
        """Rows get the lengths {row: tokens} and pages for their positions, all of them or, where there are too few, none."""
        for row, length in lengths.items():
            if length > self.longest:
                raise ValueError(f"row {row}: {length} tokens, {self.longest} at most")
        blocks = {row: range(-(-int(self.lens_h[row]) // self.page), -(-length // self.page)) for row, length in lengths.items()}
        need = sum(map(len, blocks.values()))
        if need > len(self.free):
            raise RuntimeError(f"{need} pages needed, {len(self.free)} of {self.n_pages} are free")
        for row, new in blocks.items():
            for block in new:
                self.table_h[row, block] = self.free.pop()
            self.lens_h[row] = lengths[row]

    def _tell_device(self):
        self.table.copy_(self.table_h, non_blocking=True)
        self.lens.copy_(self.lens_h, non_blocking=True)
        torch.cuda.current_stream().synchronize()      # (the host writes to the same memory again)

    # ---- requests
    def _prompt_attention(self, layer, row, q, keys, values, first):
        """Clustered attention of the new tokens' queries over contiguous caches."""
        n = q.shape[2]
        need = C.chai_prefill_workspace_bytes(1, self.H, self.k, first + n)
        if self.scratch is None or self.scratch.numel() < need:
            self.scratch = torch.empty((need,), dtype=torch.uint8, device="cuda")
        out = torch.empty((1, self.H, n, D), dtype=torch.float32, device="cuda")
        return C.chai_prefill_attention(q, keys, values, self.h2c[layer][row:row + 1], self.rep[layer][row:row + 1], first, SCALE, out,
                                        self.scratch)

    def _write(self, layer, row, k, v, start):
        pools, scales = self.pools[layer]
        C.chai_paged_append_kv(k, v, self.rep[layer][row:row + 1], self.table[row:row + 1], start, None, *pools, **scales)

    def admit(self, row: int, n: int):
        """A request with a prompt of n tokens (at least five) takes an empty row; the layers' outputs."""
        self._grow({row: n})
        self._tell_device()
        start = torch.zeros((1,), dtype=torch.int32, device="cuda")
        outs = []
        for l in range(self.L):
            q, k, v = self.source.prompt(l, row, n)
            features = C.chai_score_features(q, k, N_TOK, SCALE)
            first = self.host.permutation(self.H)[:self.k].astype(np.int32)[None]
            maps = {"head_to_cluster": self.h2c[l][row:row + 1], "rep_heads": self.rep[l][row:row + 1]}
            C.chai_assign_clusters(features, torch.from_numpy(first).cuda(), **maps)
            keys = torch.empty((1, self.k, n, D), dtype=torch.bfloat16, device="cuda")
            C.chai_compact_kcache(k, maps["rep_heads"], keys, n)
            outs.append(self._prompt_attention(l, row, q, keys, v, 0))
            self._write(l, row, k, v, start)
        return outs

    def resume(self, row: int, n: int):
        """n more tokens of a row at once, after what its pages hold; the layers' outputs."""
        before = int(self.lens_h[row])
        self._grow({row: before + n})
        self._tell_device()
        at = torch.tensor([before], dtype=torch.int32, device="cuda")
        outs = []
        for l in range(self.L):
            q, k, v = self.source.prompt(l, row, n)
            self._write(l, row, k, v, at)
            keys, values = (torch.empty((1, s, before + n, D), dtype=torch.bfloat16, device="cuda") for s in (self.k, self.H))
            pools, scales = self.pools[l]
            C.chai_paged_gather_kv(*pools, self.table[row:row + 1], torch.zeros_like(at), None, keys, values, **scales)
            outs.append(self._prompt_attention(l, row, q, keys, values, before))
        return outs

    def retire(self, row: int):
        held = self.table_h[row, :-(-int(self.lens_h[row]) // self.page)]
        self.free += held.tolist()
        held.fill_(-1)
        self.lens_h[row] = 0

    # ---- a step of all rows
    def _layers(self):
        for l in range(self.L):
            pools, scales = self.pools[l]
            C.chai_paged_decode_step(self.q[l], self.k_new[l], self.v_new[l], *pools, self.h2c[l], self.rep[l], self.table, self.lens,
                                     self.longest, SCALE, self.out[l], self.workspace, **scales)

    def record(self):
        """The layers' calls as a graph.  (They are made once before, on rows that do not exist: nothing is written.)"""
        lens = self.lens.clone()
        self.lens.zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self._layers()
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._layers()
        self.lens.copy_(lens)

    def step(self):
        """One token more for every row that holds a request; out[layer] [rows,H,128], zeros in the other rows."""
        self._grow({row: n + 1 for row, n in enumerate(self.lens_h.tolist()) if n > 0})
        self._tell_device()
        for l in range(self.L):
            self.source.token(l, self.q[l], self.k_new[l], self.v_new[l])
        if self.graph is not None:
            self.graph.replay()
        else:
            self._layers()
        return self.out


def main():
    ap = argparse.ArgumentParser(description="Requests of different lengths out of one pool of pages.")
    for name, default in (("layers", 4), ("heads", 32), ("clusters", 8), ("rows", 16), ("page", 64), ("requests", 48), ("steps", 2048),
                          ("longest", 2048), ("seed", 1)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--cache", choices=["bf16", "e4m3"], default="bf16")
    ap.add_argument("--eager", action="store_true", help="the step's calls one by one instead of a recorded graph")
    a = ap.parse_args()

    blocks = -(-a.longest // a.page)
    n_pages = max(a.rows * blocks * 3 // 4, blocks)          # fewer than all rows at full length would take, enough for one
    server = Server(Source(a.heads, a.seed), a.layers, a.heads, a.clusters, a.rows, a.longest, a.page, n_pages, a.cache, a.seed)
    if not a.eager:
        server.record()
    g = np.random.default_rng(a.seed)
    waiting = [(int(g.integers(N_TOK, a.longest * 5 // 8)), int(g.integers(1, a.longest // 4))) for _ in range(a.requests)]
    left, promised = [0] * a.rows, [0] * a.rows             # tokens that a row is still to get; pages that it may come to need
    served = tokens = peak = 0
    spent = 0.0
    for _ in range(a.steps):
        for row in range(a.rows):
            if left[row] == 0 and int(server.lens_h[row]) > 0:
                server.retire(row)
                promised[row] = 0
                served += 1
            if int(server.lens_h[row]) == 0 and waiting:
                prompt, answer = waiting[0]
                need = -(-(prompt + answer) // a.page)
                if sum(promised) + need <= n_pages:
                    waiting.pop(0)
                    server.admit(row, prompt)
                    left[row], promised[row] = answer, need
        alive = [row for row in range(a.rows) if left[row] > 0]
        if not alive:
            break
        torch.cuda.synchronize()
        began = time.perf_counter()
        server.step()
        torch.cuda.synchronize()
        spent += time.perf_counter() - began
        tokens += len(alive)
        peak = max(peak, n_pages - len(server.free))
        for row in alive:
            left[row] -= 1
    print(f"{served} of {a.requests} requests ended, {tokens} tokens of {a.layers} layers x {a.heads} heads in {a.clusters} clusters over {a.cache} "
          f"pages: {1e3 * spent:.1f} ms in steps, {tokens / spent if tokens else 0:.0f} tokens/s; at most {peak} of {n_pages} pages in use")


if __name__ == "__main__":
    main()
