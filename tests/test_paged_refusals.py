"""Caches in pages: what the calls refuse, on the host and before any launch (no GPU needed)."""
import pytest
import torch

import paper_2403_08058_amd as C

FAKE, BIG = 0x1000, 1 << 40           # a 256-byte aligned address that is never dereferenced


def call(name, fields, **kw):
    unknown = set(kw) - {n for n, _ in fields}
    assert not unknown, unknown
    return getattr(C.lib(), name)(*[kw.get(n, dflt) for n, dflt in fields])


SIZES = (("n_pages", 40), ("page", 16), ("max_blocks", 8), ("d", 128), ("dtype", 1), ("cache_dtype", 1))


def attention(**kw):
    return call("chai_paged_decode_attention", (
        ("q", FAKE), ("k_pages", FAKE), ("v_pages", FAKE), ("k_scales", None), ("v_scales", None), ("h2c", FAKE), ("rep", FAKE),
        ("table", FAKE), ("lens", FAKE), ("B", 2), ("H", 32), ("k", 8), ("T_max", 128), *SIZES, ("scale", 0.1), ("out", FAKE),
        ("ws", FAKE), ("ws_bytes", BIG), ("stream", None)), **kw)


def step(**kw):
    return call("chai_paged_decode_step", (
        ("q", FAKE), ("k_new", FAKE), ("v_new", FAKE), ("k_pages", FAKE), ("v_pages", FAKE), ("k_scales", None), ("v_scales", None),
        ("h2c", FAKE), ("rep", FAKE), ("table", FAKE), ("lens", FAKE), ("B", 2), ("H", 32), ("k", 8), ("T_max", 128), *SIZES,
        ("scale", 0.1), ("out", FAKE), ("ws", FAKE), ("ws_bytes", BIG), ("stream", None)), **kw)


def append(**kw):
    return call("chai_paged_append_kv", (
        ("k_new", FAKE), ("v_new", FAKE), ("k_stride", 4 * 128), ("v_stride", 4 * 128), ("rep", FAKE), ("table", FAKE),
        ("start", FAKE), ("count", None), ("k_pages", FAKE), ("v_pages", FAKE), ("k_scales", None), ("v_scales", None), ("B", 2),
        ("H", 32), ("k", 8), ("Tn", 4), *SIZES, ("stream", None)), **kw)


def gather(**kw):
    return call("chai_paged_gather_kv", (
        ("k_pages", FAKE), ("v_pages", FAKE), ("k_scales", None), ("v_scales", None), ("table", FAKE), ("start", FAKE),
        ("count", None), ("k_out", FAKE), ("v_out", FAKE), ("B", 2), ("H", 32), ("k", 8), ("Tn", 4), *SIZES, ("stream", None)), **kw)


NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED, ALIGN = 1, 2, 3, 4, 5, 7


@pytest.mark.parametrize("f", [attention, step, append, gather])
def test_common_checks(f):
    for name in ("k_pages", "v_pages", "table"):
        assert f(**{name: None}) == NULL
    assert f(cache_dtype=2) == NULL                        # codes without scales
    assert f(cache_dtype=2, k_scales=FAKE) == NULL
    assert f(dtype=2) == DTYPE and f(dtype=0) == DTYPE and f(cache_dtype=3) == DTYPE and f(cache_dtype=0) == DTYPE
    assert f(dtype=2, cache_dtype=2, k_scales=FAKE, v_scales=FAKE) == DTYPE
    assert f(B=-1) == SHAPE and f(H=0) == SHAPE and f(k=0) == SHAPE and f(k=33) == SHAPE
    assert f(n_pages=0) == SHAPE and f(page=0) == SHAPE and f(page=4) == SHAPE and f(page=20) == SHAPE and f(max_blocks=0) == SHAPE
    assert f(d=64) == UNSUPPORTED and f(B=4097) == UNSUPPORTED and f(H=65535) == UNSUPPORTED
    assert f(n_pages=1 << 23) == UNSUPPORTED               # 2^23 * 32 * 16 rows
    assert f(k_pages=FAKE + 8) == ALIGN and f(v_pages=FAKE + 4) == ALIGN
    assert f(B=0) == 0                                     # an empty batch: nothing to do


@pytest.mark.parametrize("f", [attention, step])
def test_decode_checks(f):
    for name in ("q", "lens", "out", "rep", "h2c"):        # (one map alone is no layout)
        assert f(**{name: None}) == NULL
    assert f(rep=None, h2c=None) == SHAPE                  # every head its own cluster, but k < H
    assert f(T_max=0) == SHAPE and f(T_max=129) == SHAPE
    assert f(T_max=(1 << 24) + 1, max_blocks=1 << 21) == UNSUPPORTED
    assert f(B=4096, H=256, k=256, T_max=1 << 16, max_blocks=1 << 12) == UNSUPPORTED
    assert f(ws=None) == WORKSPACE and f(ws=FAKE + 16) == WORKSPACE and f(ws_bytes=255) == WORKSPACE
    assert f(ws_bytes=C.chai_paged_workspace_bytes(2, 32, 8, 128) - 1) == WORKSPACE
    assert f(q=FAKE + 2) == ALIGN and f(out=FAKE + 4) == ALIGN
    assert f(B=0, ws=None) == 0
    if f is step:
        assert f(k_new=None) == NULL and f(v_new=None) == NULL and f(k_new=FAKE + 8) == ALIGN


def test_append_and_gather_checks():
    assert append(k_new=None) == NULL and append(v_new=None) == NULL and append(start=None) == NULL
    assert append(rep=None) == SHAPE                       # k < H needs representatives
    assert append(Tn=-1) == SHAPE and append(Tn=5) == SHAPE and append(k_stride=513) == SHAPE and append(v_stride=516) == SHAPE
    assert append(Tn=(1 << 24) + 1, k_stride=1 << 40, v_stride=1 << 40) == UNSUPPORTED
    assert append(k_new=FAKE + 2) == ALIGN and append(v_new=FAKE + 8) == ALIGN
    assert append(Tn=0) == 0
    assert gather(start=None) == NULL and gather(k_out=None) == NULL and gather(v_out=None) == NULL
    assert gather(Tn=-1) == SHAPE and gather(k_out=FAKE + 8) == ALIGN
    assert gather(Tn=0) == 0


def test_workspace_query():
    q = C.chai_paged_workspace_bytes
    assert q(16, 32, 8, 2048) > 0 and q(16, 32, 8, 2048) % 256 == 0 and q(0, 32, 8, 2048) == 256
    for bad in ((-1, 32, 8, 64), (4097, 32, 8, 64), (1, 0, 1, 64), (1, 32, 33, 64), (1, 32, 0, 64), (1, 32, 8, 0),
                (1, 32, 8, (1 << 24) + 1), (1, 32, 8, 64, 64), (4096, 256, 8, 1 << 16), (1, 65535, 1, 64)):
        assert q(*bad) == 0, bad
    for sizes in ([q(b, 32, 8, 700) for b in (1, 2, 3, 16, 65, 700)], [q(3, h, 3, 700) for h in (3, 4, 31, 72, 256)],
                  [q(3, 32, k, 700) for k in (1, 2, 8, 31, 32)], [q(3, 32, 8, t) for t in (1, 2, 63, 64, 65, 700, 4097, 1 << 20)]):
        assert sizes == sorted(sizes)


def tensors():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    return {"q": z(2, 6, 128), "k_new": z(2, 6, 128), "v_new": z(2, 6, 128), "k_pages": z(5, 2, 16, 128), "v_pages": z(5, 6, 16, 128),
            "head_to_cluster": z(2, 6, dt=torch.int32), "rep_heads": z(2, 2, dt=torch.int32), "block_table": z(2, 4, dt=torch.int32),
            "seq_lens": z(2, dt=torch.int32), "out": z(2, 6, 128, dt=torch.float32)}


@pytest.mark.parametrize("change,error", [
    ({"seq_lens": torch.zeros(2, dtype=torch.int64)}, ValueError),
    ({"seq_lens": torch.zeros(3, dtype=torch.int32)}, ValueError),
    ({"block_table": torch.zeros((2, 4), dtype=torch.int64)}, ValueError),
    ({"block_table": torch.zeros((3, 4), dtype=torch.int32)}, ValueError),
    ({"head_to_cluster": torch.zeros((2, 5), dtype=torch.int32)}, ValueError),
    ({"rep_heads": torch.zeros((2, 3), dtype=torch.int32)}, ValueError),
    ({"q": torch.zeros((2, 5, 128), dtype=torch.bfloat16)}, ValueError),
    ({"q": torch.zeros((2, 6, 128), dtype=torch.float16)}, TypeError),
    ({"k_new": torch.zeros((2, 6, 128), dtype=torch.float32)}, ValueError),
    ({"out": torch.zeros((2, 6, 128), dtype=torch.bfloat16)}, ValueError),
    ({"v_pages": torch.zeros((4, 6, 16, 128), dtype=torch.bfloat16)}, ValueError),
    ({"v_pages": torch.zeros((5, 6, 16, 128), dtype=torch.float32)}, ValueError),
    ({"k_pages": torch.zeros((5, 2, 16, 128), dtype=torch.uint8), "v_pages": torch.zeros((5, 6, 16, 128), dtype=torch.uint8)}, ValueError),
    ({}, ValueError),                                      # tensors of the host
])
def test_the_binding_refuses_tensors_that_do_not_fit(change, error):
    x = {**tensors(), **change}
    with pytest.raises(error):
        C.chai_paged_decode_step(x["q"], x["k_new"], x["v_new"], x["k_pages"], x["v_pages"], x["head_to_cluster"], x["rep_heads"],
                                 x["block_table"], x["seq_lens"], 64, 0.1, x["out"], torch.zeros(1 << 20, dtype=torch.uint8))


def test_the_binding_refuses_new_rows_and_results_that_do_not_fit():
    x = tensors()
    i32 = torch.zeros(2, dtype=torch.int32)
    new = torch.zeros((2, 6, 9, 128), dtype=torch.bfloat16)
    for kw in ({"v_new": new[:, :5]}, {"v_new": new.float()}, {"start": i32.long()}, {"start": i32[:1]}, {"count": i32[:1]}):
        a = {"k_new": new, "v_new": new, "start": i32, "count": i32, **kw}
        with pytest.raises(ValueError):
            C.chai_paged_append_kv(a["k_new"], a["v_new"], x["rep_heads"], x["block_table"], a["start"], a["count"], x["k_pages"], x["v_pages"])
    out = torch.zeros((2, 2, 9, 128), dtype=torch.bfloat16)
    for kw in ({"k_out": out[:, :1]}, {"v_out": new[:, :, :8]}, {"v_out": new.float()}, {"count": i32.long()}):
        a = {"k_out": out, "v_out": new, "start": i32, "count": i32, **kw}
        with pytest.raises(ValueError):
            C.chai_paged_gather_kv(x["k_pages"], x["v_pages"], x["block_table"], a["start"], a["count"], a["k_out"], a["v_out"])
