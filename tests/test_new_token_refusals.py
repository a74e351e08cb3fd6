"""New tokens' places, turned rows and packed writes: what the calls refuse, before any launch, and the frequencies (no GPU needed)."""
import math

import numpy as np
import pytest
import torch

import paper_2403_08058_amd as C

FAKE, BIG = 0x1000, 1 << 40           # a 256-byte aligned address that is never dereferenced
NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED, ALIGN = 1, 2, 3, 4, 5, 7


def call(name, fields, **kw):
    unknown = set(kw) - {n for n, _ in fields}
    assert not unknown, unknown
    return getattr(C.lib(), name)(*[kw.get(n, dflt) for n, dflt in fields])


def place(**kw):
    return call("chai_paged_place_tokens", (
        ("counts", FAKE), ("lens", FAKE), ("table", FAKE), ("free", FAKE), ("n_free", FAKE), ("B", 2), ("N", 16), ("n_pages", 40),
        ("page", 16), ("max_blocks", 8), ("new_lens", FAKE), ("n_left", FAKE), ("granted", FAKE), ("offsets", FAKE), ("rows", FAKE),
        ("positions", FAKE), ("slots", FAKE), ("ws", FAKE), ("ws_bytes", BIG), ("stream", None)), **kw)


def release(**kw):
    return call("chai_paged_release_pages", (
        ("keep", FAKE), ("lens", FAKE), ("table", FAKE), ("free", FAKE), ("n_free", FAKE), ("B", 2), ("n_pages", 40), ("page", 16),
        ("max_blocks", 8), ("new_lens", FAKE), ("n_left", FAKE), ("stream", None)), **kw)


def rotate(**kw):
    return call("chai_rotate_qk", (
        ("q", FAKE), ("k", FAKE), ("q_stride", 4 * 128), ("k_stride", 4 * 128), ("rep", FAKE), ("positions", None), ("freq", FAKE),
        ("B", 2), ("H", 32), ("k_slots", 8), ("Tn", 4), ("pos0", 3), ("Tc_cap", 7), ("d", 128), ("rot", 128), ("layout", 0),
        ("dtype", 1), ("gain", 1.0), ("q_out", 2 * FAKE), ("k_out", 2 * FAKE), ("stream", None)), **kw)


def packed(**kw):
    return call("chai_paged_append_packed", (
        ("q", FAKE), ("k_new", FAKE), ("v_new", FAKE), ("q_stride", 32 * 128), ("q_head", 128), ("k_stride", 32 * 128), ("k_head", 128),
        ("v_stride", 32 * 128), ("v_head", 128), ("k_by_slot", 0), ("rep", FAKE), ("rows", FAKE), ("positions", FAKE), ("slots", FAKE),
        ("freq", FAKE), ("q_out", 2 * FAKE), ("out_stride", 32 * 128), ("out_head", 128),
        ("k_pages", FAKE), ("v_pages", FAKE), ("k_scales", None), ("v_scales", None), ("N", 5), ("B", 2), ("H", 32), ("k", 8),
        ("n_pages", 40), ("page", 16), ("d", 128), ("rot", 128), ("layout", 0), ("dtype", 1), ("cache_dtype", 1), ("gain", 1.0),
        ("stream", None)), **kw)


@pytest.mark.parametrize("f,pointers", [
    (place, ("counts", "lens", "table", "free", "n_free", "new_lens", "n_left", "granted", "offsets", "rows", "positions", "slots")),
    (release, ("keep", "lens", "table", "free", "n_free", "new_lens", "n_left"))])
def test_places(f, pointers):
    for name in pointers:
        assert f(**{name: None}) == NULL, name
    assert f(B=-1) == SHAPE and f(n_pages=0) == SHAPE and f(page=4) == SHAPE and f(page=20) == SHAPE and f(max_blocks=0) == SHAPE
    assert f(B=4097) == UNSUPPORTED and f(n_pages=1 << 27) == UNSUPPORTED
    assert f(**{"B": 0, **{name: None for name in pointers}}) == 0
    if f is place:
        assert f(N=-1) == SHAPE and f(N=(1 << 24) + 1) == UNSUPPORTED
        assert f(ws=None) == WORKSPACE and f(ws=FAKE + 8) == WORKSPACE and f(ws_bytes=31) == WORKSPACE
        assert f(B=0, ws=None) == 0


def test_workspace_of_places():
    q = C.chai_paged_place_workspace_bytes
    assert q(-1) == 0 and q(4097) == 0 and q(0) == 256
    sizes = [q(b) for b in (1, 16, 17, 1024, 4096)]
    assert sizes == sorted(sizes) and all(s > 0 and s % 256 == 0 for s in sizes)


def test_rotated_blocks():
    for name in ("q", "k", "q_out", "k_out", "freq"):
        assert rotate(**{name: None}) == NULL, name
    assert rotate(q=None, q_out=None, k=None, k_out=None) == NULL
    assert rotate(rep=None) == SHAPE                       # every head, but k < H
    assert rotate(dtype=2) == DTYPE
    assert rotate(B=-1) == SHAPE and rotate(k_slots=33) == SHAPE and rotate(H=0) == SHAPE and rotate(Tn=-1) == SHAPE
    assert rotate(pos0=-1) == SHAPE and rotate(pos0=4) == SHAPE and rotate(Tn=5) == SHAPE
    assert rotate(q_stride=511) == SHAPE and rotate(q_stride=516) == SHAPE and rotate(k_stride=508) == SHAPE
    assert rotate(q_out=FAKE, q_stride=8 * 128) == SHAPE   # in place, but rows lie elsewhere
    assert rotate(k_out=FAKE - 3 * 256) == SHAPE           # the same for keys: 3 = pos0 rows of 256 bytes before them
    assert rotate(rot=0) == SHAPE and rotate(rot=-16) == SHAPE and rotate(rot=144) == SHAPE and rotate(layout=2) == SHAPE
    assert rotate(rot=24) == UNSUPPORTED and rotate(d=64, rot=64) == UNSUPPORTED
    assert rotate(B=1 << 20, Tn=1 << 12, q_stride=1 << 20, k_stride=1 << 20, Tc_cap=1 << 13) == UNSUPPORTED
    assert rotate(B=1, H=1, k_slots=1, Tn=(1 << 26) + 1, q_stride=1 << 40, k_stride=1 << 40, Tc_cap=1 << 30) == UNSUPPORTED
    assert rotate(q=FAKE + 8) == ALIGN and rotate(k_out=FAKE + 4) == ALIGN and rotate(freq=FAKE + 4) == ALIGN
    assert rotate(B=0) == 0 and rotate(Tn=0) == 0


def test_packed_tokens():
    for name in ("k_new", "v_new", "rows", "positions", "slots", "q", "q_out", "k_pages", "v_pages", "freq"):
        assert packed(**{name: None}) == NULL, name
    assert packed(rep=None) == SHAPE
    assert packed(dtype=2) == DTYPE and packed(cache_dtype=0) == DTYPE and packed(cache_dtype=2) == NULL
    assert packed(N=-1) == SHAPE and packed(B=0) == SHAPE and packed(k=33) == SHAPE and packed(page=20) == SHAPE
    assert packed(k_stride=8 * 128) == SHAPE and packed(v_stride=32 * 128 - 8) == SHAPE and packed(q_stride=32 * 128 + 4) == SHAPE
    assert packed(q_out=FAKE, q_stride=33 * 128) == SHAPE and packed(q_out=FAKE, q_head=256, q_stride=64 * 128) == SHAPE
    assert packed(v_head=64) == SHAPE and packed(k_head=132) == SHAPE and packed(out_head=0) == SHAPE and packed(v_stride=-128, v_head=640) == SHAPE
    assert packed(v_stride=1 << 41) == SHAPE
    # rows of one head one behind the other: five tokens of 128 elements, no fewer
    assert packed(v_stride=128, v_head=5 * 128 - 8) == SHAPE and packed(k_stride=128, k_head=4 * 128) == SHAPE
    assert packed(rot=136) == SHAPE and packed(layout=-1) == SHAPE and packed(rot=40) == UNSUPPORTED and packed(d=64, rot=64) == UNSUPPORTED
    assert packed(N=(1 << 24) + 1) == UNSUPPORTED and packed(n_pages=1 << 27, H=1, k=1) == UNSUPPORTED and packed(B=4097) == UNSUPPORTED
    assert packed(N=1 << 24, H=1000, k=1000, q_stride=128000, k_stride=128000, v_stride=128000, out_stride=128000) == UNSUPPORTED
    assert packed(k_new=FAKE + 2) == ALIGN and packed(k_pages=FAKE + 8) == ALIGN and packed(q_out=FAKE + 8) == ALIGN
    assert packed(N=0) == 0 and packed(N=0, B=0, k_new=None, v_new=None, rows=None, positions=None, slots=None) == 0


def test_frequencies():
    plain = 10000.0 ** (-np.arange(32) / 32.0)
    assert np.allclose(C.chai_rotary_frequencies(64).numpy(), plain, rtol=1e-14, atol=0)
    linear = C.chai_rotary_frequencies(64, kind=C.CHAI_ROPE_LINEAR, factor=4.0).numpy()
    assert np.allclose(linear, plain / 4, rtol=1e-14, atol=0)
    base = C.chai_rotary_frequencies(64, kind=C.CHAI_ROPE_BASE, factor=8.0).numpy()
    assert base[0] == 1.0 and math.isclose(base[-1], plain[-1] / 8, rel_tol=1e-12)       # the fastest stays, the slowest is divided
    turns = C.chai_rotary_frequencies(64, kind=C.CHAI_ROPE_TURNS, factor=16.0, original_length=2048.0, slow=1.0, fast=32.0).numpy()
    made = 2048.0 * plain / (2 * math.pi)
    assert np.array_equal(turns[made >= 32], C.chai_rotary_frequencies(64).numpy()[made >= 32])
    assert np.allclose(turns[made <= 1], plain[made <= 1] / 16, rtol=1e-14, atol=0)
    between = (made > 1) & (made < 32)
    share = (made[between] - 1) / 31
    assert between.any() and np.allclose(turns[between], share * plain[between] + (1 - share) * plain[between] / 16, rtol=1e-13, atol=0)
    for bad in (dict(rot=0), dict(rot=63), dict(rot=130), dict(rot=64, theta=0.0), dict(rot=64, theta=float("inf")), dict(rot=64, kind=4),
                dict(rot=64, kind=1, factor=0.0), dict(rot=2, kind=2, factor=2.0), dict(rot=64, kind=3, factor=2.0),
                dict(rot=64, kind=3, factor=2.0, original_length=100.0, slow=2.0, fast=2.0)):
        with pytest.raises(C.ChaiError):
            C.chai_rotary_frequencies(**bad)
    assert C.lib().chai_rotary_frequencies(64, 10000.0, 0, 1.0, 0.0, 1.0, 32.0, None) == NULL


def _z(*shape, dt=torch.bfloat16):
    return torch.zeros(shape, dtype=dt)


@pytest.mark.parametrize("change", [{"counts": _z(2, dt=torch.int64)}, {"seq_lens": _z(3, dt=torch.int32)}, {"n_free": _z(2, dt=torch.int32)},
                                    {"offsets": _z(2, dt=torch.int32)}, {"positions": _z(15, dt=torch.int32)}, {}])
def test_the_binding_refuses_places_that_do_not_fit(change):
    i = lambda *s: _z(*s, dt=torch.int32)  # noqa: E731
    x = {"counts": i(2), "seq_lens": i(2), "block_table": i(2, 4), "free_pages": i(9), "n_free": i(1), "page": 16, "new_lens": i(2),
         "n_left": i(1), "granted": i(2), "offsets": i(3), "token_rows": i(16), "positions": i(16), "slots": i(16),
         "workspace": torch.zeros(256, dtype=torch.uint8), **change}
    with pytest.raises(ValueError):                        # (the last: tensors of the host)
        C.chai_paged_place_tokens(**x)


@pytest.mark.parametrize("change", [{"q_out": _z(2, 6, 3, 128, dt=torch.float32)}, {"k": _z(2, 3, 3, 128)}, {"k_out": _z(2, 2, 9, 64)},
                                    {"rep_heads": _z(2, 3, dt=torch.int32)}, {"positions": _z(2, 4, dt=torch.int32)},
                                    {"positions": _z(2, 3, dt=torch.int64)}, {"freq": _z(64, dt=torch.float32)}, {"k_out": None},
                                    {"q": None, "q_out": None, "k": None, "k_out": None}, {}])
def test_the_binding_refuses_rows_to_turn_that_do_not_fit(change):
    x = {"q": _z(2, 6, 3, 128), "k": _z(2, 2, 3, 128), "rep_heads": _z(2, 2, dt=torch.int32), "freq": _z(64, dt=torch.float64),
         "q_out": _z(2, 6, 3, 128), "k_out": _z(2, 2, 9, 128), "pos0": 4, "positions": None, **change}
    with pytest.raises(ValueError):
        C.chai_rotate_qk(**x)


@pytest.mark.parametrize("change", [{"q_out": _z(4, 6, 128)}, {"k_new": _z(5, 3, 128)}, {"k_new": _z(4, 6, 128)}, {"v_new": _z(5, 6, 128, dt=torch.float32)},
                                    {"rep_heads": _z(2, 3, dt=torch.int32)}, {"slots": _z(5, dt=torch.int64)}, {"token_rows": _z(4, dt=torch.int32)},
                                    {"freq": _z(64, dt=torch.float32)}, {"v_pages": _z(9, 5, 16, 128)}, {"q": None}, {}])
def test_the_binding_refuses_tokens_that_do_not_fit(change):
    i = lambda *s: _z(*s, dt=torch.int32)  # noqa: E731
    x = {"q": _z(5, 6, 128), "k_new": _z(5, 6, 128), "v_new": _z(5, 6, 128), "rep_heads": i(2, 2), "token_rows": i(5), "positions": i(5),
         "slots": i(5), "freq": _z(64, dt=torch.float64), "q_out": _z(5, 6, 128), "k_pages": _z(9, 2, 16, 128),
         "v_pages": _z(9, 6, 16, 128), **change}
    with pytest.raises(ValueError):
        C.chai_paged_append_packed(**x)
