"""The serving example: rows that come, grow, are continued and go, against attention in 64 bits over what each of them was given."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import workloads as W
from gpu_util import RTOL, rows_close
from test_gpu_paged import codes_of

_path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")
_spec = importlib.util.spec_from_file_location("paged_serving", _path)
S = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(S)

# prompt attention rounds weights to 11 bits and its sums: the bar that its own tests hold it to
PROMPT_BAR = 2e-3


class Recorded(S.Source):
    """Keeps the keys and values that every row of every layer was given."""

    def __init__(self, heads, layers, rows, seed):
        super().__init__(heads, seed)
        self.kept = {(l, b): [] for l in range(layers) for b in range(rows)}
        self.last_q = None
        self.alive = []

    def prompt(self, layer, row, n):
        q, k, v = super().prompt(layer, row, n)
        self.kept[layer, row].append((k[0].clone(), v[0].clone()))
        self.last_q = q[0]
        return q, k, v

    def token(self, layer, q, k, v):
        super().token(layer, q, k, v)
        for b in self.alive:
            self.kept[layer, b].append((k[b].unsqueeze(1).clone(), v[b].unsqueeze(1).clone()))

    def rows_of(self, layer, row, cache):
        got = []
        for i in range(2):
            x = torch.cat([kv[i] for kv in self.kept[layer, row]], 1)
            if cache == "e4m3":
                codes, scales = codes_of(x)
                got.append(codes.view(torch.float8_e4m3fn).double() * scales.double().unsqueeze(-1))
            else:
                got.append(x.double())
        return got


def expected(server, layer, row, q, keys, values):
    """[H,n,128]: the last n positions' queries over all positions up to their own."""
    h2c, rep = server.h2c[layer][row].long(), server.rep[layer][row].long()
    q = q.double()
    n, T = q.shape[1], keys.shape[1]
    s = S.SCALE * torch.matmul(q[rep.clamp(min=0)], keys[rep.clamp(min=0)].transpose(1, 2).contiguous())
    later = torch.arange(T, device="cuda")[None] > torch.arange(T - n, T, device="cuda")[:, None]
    p = torch.softmax(s.masked_fill(later, -float("inf")), -1)
    return torch.matmul(p[h2c], values)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("longest,recorded", [(300, False), (300, True), (4500, True)])
def test_requests_come_grow_and_go(cache, longest, recorded):
    print(f"[paged] serving {cache} longest {longest} recorded {recorded}", flush=True)
    L, H, k, rows, page = 2, 12, 3, 4, 24
    source = Recorded(H, L, rows, 77)
    server = S.Server(source, L, H, k, rows, longest, page, 40, cache, seed=5)
    for pools, scales in server.pools:                       # pages hold what they were left with
        for t in pools:
            t.view(torch.uint8).fill_(0xFF)
    if recorded:
        server.record()

    def steps(count):
        for _ in range(count):
            source.alive = [b for b in range(rows) if int(server.lens_h[b]) > 0]
            out = server.step()
            torch.cuda.synchronize()
            for l in range(L):
                for b in range(rows):
                    if b not in source.alive:
                        assert bool((out[l][b] == 0).all())
                        continue
                    want = expected(server, l, b, server.q[l][b].unsqueeze(1), *source.rows_of(l, b, cache))[:, 0]
                    ok, worst = rows_close(out[l][b].cpu().numpy(), want.cpu().numpy(), RTOL[W.BF16])
                    assert ok, (l, b, worst)

    def check_prompt(outs, row, compare_codes):
        torch.cuda.synchronize()
        l = L - 1                                            # (the source keeps the last layer's queries)
        want = expected(server, l, row, source.last_q, *source.rows_of(l, row, cache if compare_codes else "bf16"))
        ok, worst = rows_close(outs[l][0].cpu().numpy(), want.cpu().numpy(), PROMPT_BAR)
        assert ok, worst

    check_prompt(server.admit(2, 100), 2, False)
    steps(3)
    check_prompt(server.admit(0, 5), 0, False)
    server.admit(3, 47)
    steps(3)
    if cache == "bf16":                                      # (a row read back from codes is rounded to bf16 besides)
        check_prompt(server.resume(2, 61), 2, False)
    else:
        server.resume(2, 61)
    steps(2)
    free = len(server.free)
    server.retire(3)
    assert len(server.free) == free + 3                      # 47 + 5 tokens
    for l in range(L):
        source.kept[l, 3].clear()
    steps(1)
    server.admit(3, 130)
    server.admit(1, 24)
    steps(3)
    assert sorted(server.free + [p for p in server.table_h.flatten().tolist() if p >= 0]) == list(range(40))
