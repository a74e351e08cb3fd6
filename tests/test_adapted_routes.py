"""Projections with adapters: which kernels the GPU tests' sizes reach, and what the call refuses (no GPU needed)."""
import re

import pytest
import torch

import launch_log
import paper_2403_08058_amd as C
from adapted_cases import CASES, MORE, PARTS, RANKS

FAKE, BIG = 0x1000, 1 << 40
NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED, ALIGN = 1, 2, 3, 4, 5, 7


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    sizes = [(*c, R) for cases in (*CASES.values(), PARTS, MORE) for c in cases for R in RANKS]
    return launch_log.run(tmp_path_factory.mktemp("stand_in"), f"""
        result = []
        for B, H, k, Tn, D, R in {sizes!r}:
            st = L.chai_project_qk_adapted(P, P, P, P, P, P, P, P, P, P, 3, R, B, H, k, Tn, D, 128, 1, P, P, 0, Tn, P, N, None)
            first = launches()
            L.chai_project_qk(P, P, P, P, B, H, k, Tn, D, 128, 1, P, P, 0, Tn, None)
            result.append([st, [B, H, k, Tn, D, R], first, launches()])
    """)


@pytest.mark.parametrize("kernel", CASES)
def test_kernels_of_the_sizes(launched, kernel):
    for case in CASES[kernel]:
        for R in RANKS:
            st, _, got, plain = next(r for r in launched if r[1] == [*case, R])
            assert st == 0 and len(got) == 2 and "adapter_down_kernel" in got[0][0]
            assert got[0][3] <= got[0][4] and got[1][3] <= got[1][4] or "rows" in got[1][0]
            name = re.search(r"project_([a-z]*)_?kernel", got[1][0]).group(1) or "large"
            assert name == kernel, (case, got[1][0])
            # the call without adapters goes the same way
            assert re.search(r"project_[a-z_]*kernel", plain[0][0]).group(0) == re.search(r"project_[a-z_]*kernel", got[1][0]).group(0)
            assert "NoAdapters" in plain[0][0] and "NoAdapters" not in got[1][0]
    if kernel == "large":                                  # a workgroup per tile, and several tiles each
        grids = {r[2][1][1] for r in launched if r[1][:5] in [list(c) for c in CASES["large"]]}
        assert 256 in grids and any(n < 256 for n in grids)


def test_rows_of_too_many_pairs_go_in_parts(launched):
    for case in PARTS:
        st, _, got, plain = next(r for r in launched if r[1] == [*case, 16])
        assert st == 0 and len(plain) == 1 and "14project_kernel" in plain[0][0]
        assert len(got) >= 3 and "adapter_down_kernel" in got[0][0] and not any("14project_kernel" in g[0] for g in got), got
    for case in MORE:
        st, _, got, plain = next(r for r in launched if r[1] == [*case, 16])
        assert st == 0 and "14project_kernel" in plain[0][0] and len(got) == 2 and "project_tile_kernel" in got[1][0]


def test_shapes_of_the_first_half(launched):
    """Every shape of workgroups of it is reached."""
    shapes = {re.search(r"adapter_down_kernelILi(\d+)ELi(\d+)ELi(\d+)E", r[2][0][0]).groups() for r in launched}
    assert shapes == {("1", "1", "16"), ("2", "1", "16"), ("4", "1", "16"), ("1", "2", "16"), ("4", "4", "4")}


def test_the_first_half_of_more_rows_than_a_launch_has_threads_for(tmp_path):
    """A launch has less than 2^32 threads in a direction."""
    got = launch_log.run(tmp_path, """
        result = []
        for B, Tn, R, part in ((5_000_000, 1, 8, None), (5_000_000, 3, 128, P), (40_000, 64, 128, P), (20_000, 64, 128, P), (70_000, 1000, 128, P)):
            st = L.chai_project_qk_adapted(P, P, P, P, P, P, P, part, part, P, 3, R, B, 1, 1, Tn, 256, 128, 1, P, P, 0, Tn, P, N, None)
            result.append([st, launches()])
    """)
    assert [sum("adapter_down_kernel" in n[0] for n in launches) for _, launches in got] == [2, 10, 2, 1, 2]      # rows of a launch: 4194296, 524280, 32766, 65535
    for st, launches in got:
        assert st == 0 and all(n[1] * n[2] < 1 << 32 for n in launches)


def call(**kw):
    fields = (("x", FAKE), ("w_q", FAKE), ("w_k", FAKE), ("rep", FAKE), ("ids", FAKE), ("a_q", FAKE), ("b_q", FAKE), ("a_k", FAKE), ("b_k", FAKE),
              ("scale", FAKE), ("n", 3), ("R", 16), ("B", 2), ("H", 32), ("k", 8), ("Tn", 4), ("D", 512), ("d", 128), ("dtype", 1), ("q_out", FAKE),
              ("kc", FAKE), ("pos0", 3), ("cap", 7), ("ws", FAKE), ("ws_bytes", BIG), ("stream", None))
    assert not set(kw) - {n for n, _ in fields}
    return C.lib().chai_project_qk_adapted(*[kw.get(n, v) for n, v in fields])


def test_refusals():
    for name in ("x", "w_q", "w_k", "rep", "ids", "a_q", "b_q", "a_k", "b_k", "q_out", "kc"):
        assert call(**{name: None}) == NULL, name
    assert call(a_q=None, b_q=None, a_k=None, b_k=None) == NULL
    assert call(dtype=2) == DTYPE and call(n=0) == SHAPE and call(R=0) == SHAPE and call(k=33) == SHAPE and call(pos0=4) == SHAPE
    assert call(dtype=0) == UNSUPPORTED and call(R=12) == UNSUPPORTED and call(R=136) == UNSUPPORTED and call(D=500) == UNSUPPORTED
    assert call(a_q=FAKE + 8) == ALIGN and call(b_k=FAKE + 2) == ALIGN and call(x=FAKE + 8) == ALIGN
    assert call(ws=None) == WORKSPACE and call(ws=FAKE + 16) == WORKSPACE and call(ws_bytes=2 * 4 * 2 * 64 - 1) == WORKSPACE
    assert call(B=0, ws=None) == 0 and call(B=0, x=None, rep=None, ids=None, q_out=None, kc=None, ws=None) == 0 and call(B=0, w_k=None) == NULL


def test_workspace():
    q = C.chai_project_adapted_workspace_bytes
    assert q(0, 1, 8) == 256 and q(3, 5, 24) % 256 == 0 and q(3, 5, 24) >= 3 * 5 * 2 * 24 * 4
    for bad in ((-1, 1, 8), (1, 0, 8), (1, 1, 0), (1, 1, 12), (1, 1, 136)):
        assert q(*bad) == 0
    for sizes in ([q(b, 7, 16) for b in (1, 2, 50)], [q(3, t, 16) for t in (1, 2, 1000)], [q(3, 7, r) for r in (8, 16, 24, 128)]):
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("change", [{"a_k": None}, {"a_q": None, "b_q": None, "a_k": None, "b_k": None}, {"adapter_ids": torch.zeros(3, dtype=torch.int32)},
                                    {"adapter_ids": torch.zeros(2, dtype=torch.int64)}, {"adapter_scale": torch.zeros(4)}, {"b_q": torch.zeros((3, 6 * 128, 8), dtype=torch.bfloat16)},
                                    {"w_k": torch.zeros((5 * 128, 64), dtype=torch.bfloat16)}, {"a_q": torch.zeros((3, 16, 64))}, {}])
def test_the_binding_refuses_what_does_not_fit(change):
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    x = {"x": z(2, 4, 64), "w_q": z(6 * 128, 64), "w_k": z(6 * 128, 64), "rep_heads": z(2, 3, dt=torch.int32), "adapter_ids": z(2, dt=torch.int32),
         "a_q": z(3, 16, 64), "b_q": z(3, 6 * 128, 16), "a_k": z(3, 16, 64), "b_k": z(3, 6 * 128, 16), "adapter_scale": torch.zeros(3),
         "q_out": z(2, 6, 4, 128), "k_compact": z(2, 3, 4, 128), "pos0": 0, "workspace": torch.zeros(4096, dtype=torch.uint8), **change}
    with pytest.raises(ValueError):
        C.chai_project_qk_adapted(**x)
