"""The serving example's account of pages and requests, on the host: the calls on the GPU are left out (no GPU needed)."""
import importlib.util
import os
import sys

import pytest
import torch

_path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")
_spec = importlib.util.spec_from_file_location("paged_serving_host", _path)
S = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(S)


class HostServer(S.Server):
    """The pages of a server without what the device holds."""

    def __init__(self, source, layers, heads, clusters, rows, longest, page, n_pages, cache="bf16", seed=0):
        self.L, self.rows, self.longest, self.page, self.n_pages = 0, rows, longest, page, n_pages
        self.blocks = -(-longest // page)
        self.free = list(range(n_pages))
        self.table_h = torch.full((rows, self.blocks), -1, dtype=torch.int32)
        self.lens_h = torch.zeros((rows,), dtype=torch.int32)
        self.graph, self.out = None, []

    def _tell_device(self):
        pass

    def admit(self, row, n):
        assert int(self.lens_h[row]) == 0 and bool((self.table_h[row] == -1).all())
        self._grow({row: n})


def whole(server):
    """Every page is free or in one place of the table, and a row holds those that its length needs."""
    held = [p for p in server.table_h.flatten().tolist() if p >= 0]
    assert sorted(server.free + held) == list(range(server.n_pages))
    for row in range(server.rows):
        need = -(-int(server.lens_h[row]) // server.page)
        assert bool((server.table_h[row, :need] >= 0).all()) and bool((server.table_h[row, need:] == -1).all())


def test_a_pool_that_is_too_small_is_left_as_it_was():
    server = HostServer(None, 1, 4, 2, rows=3, longest=200, page=8, n_pages=10)
    server._grow({0: 30, 1: 8})                            # four pages and one
    whole(server)
    before = server.table_h.clone(), server.lens_h.clone(), list(server.free)
    with pytest.raises(RuntimeError):
        server._grow({2: 48})                              # six of the five that are left
    with pytest.raises(RuntimeError):
        server._grow({0: 40, 1: 16, 2: 32})                # together too many
    with pytest.raises(ValueError):
        server._grow({2: 1, 0: 201})
    assert torch.equal(server.table_h, before[0]) and torch.equal(server.lens_h, before[1]) and server.free == before[2]
    server._grow({1: 40, 0: 40})
    whole(server)
    assert server.free == []
    with pytest.raises(RuntimeError):
        server.step()                                      # neither row's next token has a place
    whole(server)
    assert server.lens_h.tolist() == [40, 40, 0]
    server.retire(0)
    server.step()
    whole(server)
    assert server.lens_h.tolist() == [0, 41, 0]

def run_main(monkeypatch, capsys, *args):
    monkeypatch.setattr(S, "Server", HostServer)
    monkeypatch.setattr(S, "Source", lambda heads, seed: None)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    monkeypatch.setattr(sys, "argv", ["paged_serving.py", "--eager", "--layers", "0", *args])
    S.main()
    return capsys.readouterr().out


@pytest.mark.parametrize("rows,page,seed", [(1, 64, 1), (1, 64, 2), (1, 2048, 3), (2, 512, 1), (16, 64, 1)])
def test_every_request_is_served(monkeypatch, capsys, rows, page, seed):
    out = run_main(monkeypatch, capsys, "--rows", str(rows), "--page", str(page), "--seed", str(seed), "--requests", "12", "--steps", "20000")
    assert "12 of 12 requests ended" in out


def test_nothing_to_do(monkeypatch, capsys):
    assert "0 of 0 requests ended, 0 tokens" in run_main(monkeypatch, capsys, "--requests", "0")
    assert "0 of 48 requests ended, 0 tokens" in run_main(monkeypatch, capsys, "--steps", "0")
