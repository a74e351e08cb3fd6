"""Which kernels the sizes of the GPU tests reach: a test whose sizes no longer reach what it is there for fails here (no GPU
needed, the runtime's launches are written down by a stand-in)."""
import re

import pytest

import launch_log
from paged_paths import CACHES, LONGEST, MANY_HEADS, MANY_ROWS, MOVED, PAGE, PATHS

CODE = {"f32": (0, 0), "bf16": (1, 1), "e4m3": (1, 2)}


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    attention = [(len(rows), H, k, bound) for H, k, bound, rows, _ in PATHS.values()]
    attention += [(B, H, k, LONGEST + 8) for B in MANY_ROWS for H, k in MANY_HEADS]
    calls = [(*a, *CODE[c]) for a in attention for c in CACHES]
    moves = [(*m, *CODE[c]) for m in MOVED for c in CACHES]
    return launch_log.run(tmp_path_factory.mktemp("stand_in"), f"""
        result = []
        for B, H, k, T, dt, cache in {calls!r}:
            maps = (P, P) if k < H else (None, None)
            sizes = (B, H, k, T, 4096, {PAGE}, -(-T // {PAGE}), 128, dt, cache)
            for step in (False, True):
                if step:
                    st = L.chai_paged_decode_step(P, P, P, P, P, P, P, *maps, P, P, *sizes, ctypes.c_float(0.1), P, P, N, None)
                else:
                    st = L.chai_paged_decode_attention(P, P, P, P, P, *maps, P, P, *sizes, ctypes.c_float(0.1), P, P, N, None)
                result.append([st, B, H, k, T, cache, step, launches()])
        for B, H, k, Tn, dt, cache in {moves!r}:
            sizes = (B, H, k, Tn, 4096, {PAGE}, 64, 128, dt, cache)
            stride = ctypes.c_int64(Tn * 128)
            st = L.chai_paged_append_kv(P, P, stride, stride, P if k < H else None, P, P, P, P, P, P, P, *sizes, None)
            result.append([st, B, H, k, Tn, cache, "append", launches()])
            st = L.chai_paged_gather_kv(P, P, P, P, P, P, P, P, P, *sizes, None)
            result.append([st, B, H, k, Tn, cache, "gather", launches()])
    """)


def kernels(launched, B, H, k, T, what):
    """For each type of cache: the kernels of the calls, their instances and threads of a workgroup."""
    got = [r for r in launched if r[1:5] == [B, H, k, T] and r[6] == what]
    assert len(got) == 3 and all(r[0] == 0 for r in got)
    return [[(re.search(r"paged_[a-z_]*?(?=_kernel)", n[0]).group(0), n[0], n[2]) for n in r[7]] for r in got]


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("step", [False, True])
def test_ways_of_attention(launched, path, step):
    H, k, bound, rows, want = PATHS[path]
    for got in kernels(launched, len(rows), H, k, bound, step):
        assert [g[0] for g in got] == want
        if want == ["paged_rows"]:
            assert got[0][2] == (512 if "eight" in path else 256)
            assert ("in order" in path) == (256 < len(rows) * H <= 1024)
        else:
            assert ("many heads" in path) == (len(rows) * H > 512)
            # a mangled name ends its template's arguments with the waves that join a head's parts
            assert ("Li1EE" in got[-1][1]) == ("many heads" in path)


@pytest.mark.parametrize("B", MANY_ROWS)
@pytest.mark.parametrize("H,k", MANY_HEADS)
@pytest.mark.parametrize("step", [False, True])
def test_many_rows_are_shared(launched, B, H, k, step):
    want = ["paged_scores", "paged_values", "paged_join"] if k < H else ["paged_attend", "paged_join"]
    for got in kernels(launched, B, H, k, LONGEST + 8, step):
        assert [g[0] for g in got] == want


@pytest.mark.parametrize("what", ["append", "gather"])
@pytest.mark.parametrize("B,H,k,Tn", MOVED)
def test_moves_of_many_rows_are_dealt_out(launched, B, H, k, Tn, what):
    assert B > 64
    for got in kernels(launched, B, H, k, Tn, what):
        assert [g[0] for g in got] == [f"paged_{what}_stream"]
