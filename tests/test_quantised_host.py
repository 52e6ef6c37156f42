"""The calls on an 8-bit cache and on a model's own rotary positions refuse bad arguments before they touch a device.
No GPU needed."""

import ctypes
import re

import pytest
import torch

import paper_2609_32518_b200 as U
from paper_2609_32518_b200 import binding
from test_overlap_sources import kernels

FAKE = 0x10000  # a non-null, 16-byte aligned address that is never dereferenced
INVALID, UNSUPPORTED = -1, -2


def good_shape(**kw):
    args = dict(batch=2, heads=2, chunk_frames=2, grid_h=8, grid_w=8, ring_frames=6)
    args.update(kw)
    return U.Shape.make(**args)


def starts(values):
    return None if values is None else (ctypes.c_int32 * len(values))(*values)


def table(shape, rope, start=0, cos=FAKE, sin=FAKE):
    return U.lib().unstep_rotary_table(ctypes.byref(shape), rope and ctypes.byref(rope), start, cos, sin, None)


def apply(shape, rope, transposed=0, ptrs=(FAKE,) * 4, stride=0):
    x, cos, sin, y = ptrs
    return U.lib().unstep_rotary_apply(ctypes.byref(shape), rope and ctypes.byref(rope), transposed, x, cos, sin, stride, y, None)


def append(shape, rope, sink=0, first=(0, 2), ptrs=(FAKE,) * 10, gains=(None, None), eps=0.0, stride=0):
    q, k, v, cos, sin, qo, ck, sk, cv, sv = ptrs
    return U.lib().unstep_rotary_kv_append_q8(ctypes.byref(shape), rope and ctypes.byref(rope), sink, starts(first), q, k, v,
                                              *gains, eps, cos, sin, stride, qo, ck, sk, cv, sv, None)


def read(shape, sink=0, first=(0, 2), n=2, ptrs=(FAKE,) * 6):
    return U.lib().unstep_kv_read_q8(ctypes.byref(shape), sink, starts(first), n, *ptrs, None)


def attn(shape, sink=0, first=(0, 2), recent=2, attend=0, ptrs=(FAKE,) * 6):
    q, ck, sk, cv, sv, out = ptrs
    return U.lib().unstep_window_attn_q8(ctypes.byref(shape), sink, starts(first), recent, attend, q, ck, sk, cv, sv, out, None)


@pytest.mark.parametrize("kw", [dict(chunk_frames=0), dict(grid_h=0), dict(bands=(43, 43, 42)), dict(bands=(44, 42, 44)),
                                dict(bands=(8, 4, 2)), dict(bands=(0, 0, 0)), dict(bands=(-16, 16, 16)),
                                dict(bands=(24, 24, 24)), dict(bands=(2 ** 31 - 2, 2, 16)), dict(rope_base=0.0), dict(head_dim=0)])
def test_bad_shapes_are_rejected_everywhere(kw):
    sh, rope = good_shape(**kw), U.Rope.make()
    assert table(sh, rope) == INVALID
    assert apply(sh, rope) == INVALID
    assert append(sh, rope) == INVALID
    assert read(sh) == INVALID
    assert attn(sh) == INVALID


def test_head_dim_other_than_128_is_unsupported():
    sh = good_shape(head_dim=64, bands=(32, 16, 16))
    assert table(sh, U.Rope.make()) == UNSUPPORTED and attn(sh) == UNSUPPORTED and read(sh) == UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(factor=(0.5, 1, 1)), dict(factor=(1, float("nan"), 1)), dict(factor=(1, 1, float("inf"))),
                                dict(trained=(-1, 0, 0)), dict(factor=(2, 1, 1), trained=(21, 0, 0), beta=(4.0, 4.0)),
                                dict(factor=(2, 1, 1), trained=(21, 0, 0), beta=(-1.0, 4.0)),
                                dict(factor=(2, 1, 1), trained=(21, 0, 0), beta=(1.0, float("nan"))),
                                dict(magnitude=0.0), dict(magnitude=float("nan")), dict(magnitude=-1.0)])
def test_bad_rotary_positions_are_rejected(kw):
    sh, rope = good_shape(), U.Rope.make(**kw)
    assert table(sh, rope) == apply(sh, rope) == append(sh, rope) == INVALID


def test_layout_has_to_be_one_of_two_and_the_pointer_there():
    sh = good_shape()
    rope = U.Rope.make()
    rope.half = 2
    for r in (rope, None):
        assert table(sh, r) == apply(sh, r) == append(sh, r) == INVALID


def each_bad_pointer(call, n, scales=()):
    for i in range(n):
        for bad in (None, FAKE + (2 if i in scales else 8)):
            ptrs = [FAKE] * n
            ptrs[i] = bad
            assert call(tuple(ptrs)) == INVALID, (i, bad)


def test_pointers():
    sh, rope = good_shape(), U.Rope.make()
    for kw in (dict(cos=None), dict(sin=FAKE + 4), dict(start=-1), dict(start=2 ** 31 - 1)):
        assert table(sh, rope, **kw) == INVALID
    each_bad_pointer(lambda p: apply(sh, rope, ptrs=p), 4)
    each_bad_pointer(lambda p: append(sh, rope, ptrs=p), 10, (7, 9))
    each_bad_pointer(lambda p: read(sh, ptrs=p), 6, (1, 3))
    each_bad_pointer(lambda p: attn(sh, ptrs=p), 6, (2, 4))


def test_other_arguments():
    sh, rope = good_shape(), U.Rope.make()
    assert apply(sh, rope, transposed=2) == apply(sh, rope, stride=-4) == apply(sh, rope, stride=2) == INVALID
    assert apply(good_shape(batch=0), rope) == apply(good_shape(heads=0), rope) == apply(good_shape(heads=5000), rope) == INVALID
    assert append(sh, rope, first=None) == append(sh, rope, first=(0, -1)) == append(sh, rope, first=(2 ** 31 - 1, 0)) == INVALID
    assert append(sh, rope, sink=-1) == append(sh, rope, sink=5000) == append(sh, rope, stride=6) == INVALID
    assert append(sh, rope, gains=(FAKE, None)) == append(sh, rope, gains=(None, FAKE)) == INVALID
    assert append(sh, rope, gains=(FAKE, FAKE + 8)) == append(sh, rope, gains=(FAKE, FAKE), eps=-1.0) == INVALID
    assert append(sh, rope, gains=(FAKE, FAKE), eps=float("nan")) == INVALID
    assert append(good_shape(ring_frames=1), rope) == INVALID
    assert read(sh, n=0) == read(sh, first=None) == read(sh, first=(-1, 0)) == read(sh, first=(0, 2 ** 31 - 1)) == INVALID
    assert read(sh, n=7) == read(sh, sink=2, first=(0, 1), n=9) == read(sh, sink=2, first=(0, 3), n=7) == INVALID
    assert attn(sh, recent=1) == attn(sh, recent=7) == attn(sh, attend=1) == attn(sh, sink=1, attend=2) == INVALID
    assert attn(sh, first=(-1, 0)) == attn(sh, first=None) == INVALID


def tensors(sh):
    act = (sh.batch, sh.chunk_tokens, sh.heads, 128)
    cache = (sh.batch, sh.ring_frames, sh.tokens_per_frame, sh.heads)
    return {"x": torch.zeros(act, dtype=torch.bfloat16), "tab": torch.zeros((sh.chunk_tokens, 64)),
            "code": torch.zeros(cache + (128,), dtype=torch.uint8).view(torch.float8_e4m3fn),
            "scale": torch.zeros(cache + (4,), dtype=torch.uint8).view(torch.float8_e8m0fnu)}


def test_binding_refuses_cpu_tensors_and_what_is_no_rope():
    sh, rope = good_shape(), U.Rope.make()
    t = tensors(sh)
    cache = (t["code"], t["scale"], t["code"], t["scale"])
    calls = [lambda r: U.rotary_table(sh, r, 0, t["tab"], t["tab"]),
             lambda r: U.rotary_apply(sh, r, t["x"], t["tab"], t["tab"], t["x"]),
             lambda r: U.rotary_kv_append_q8(sh, r, 0, [0, 2], t["x"], t["x"], t["x"], t["tab"], t["tab"], t["x"], *cache),
             lambda r: U.kv_read_q8(sh, 0, [0, 2], 2, *cache, t["x"], t["x"]),
             lambda r: U.window_attn_q8(sh, 0, [0, 2], 2, 0, t["x"], *cache, t["x"])]
    for call in calls:
        with pytest.raises(TypeError, match="expected a CUDA tensor"):
            call(rope)
    for call in calls[:3]:
        with pytest.raises(TypeError, match="rope"):
            call(None)
    for call in (lambda: U.kv_read_q8(sh, 0, [0], 2, *cache, t["x"], t["x"]),
                 lambda: U.window_attn_q8(sh, 0, [0], 2, 0, t["x"], *cache, t["x"])):
        with pytest.raises(ValueError, match="one entry per stream"):
            call()


def test_native_marshalling_answers_none_for_what_is_not_well_formed():
    sh, rope = good_shape(), U.Rope.make()
    native = binding._native()
    t = tensors(sh)
    cache = (t["code"], t["scale"], t["code"], t["scale"])
    assert native.rotary_table(sh, sh, 0, t["tab"], t["tab"], None) is None
    assert native.rotary_table(sh, rope, 1 << 40, t["tab"], t["tab"], None) is None
    assert native.rotary_apply(sh, rope, t["x"], t["tab"], t["tab"], t["x"], 1, 0, None) is None
    assert native.rotary_apply(sh, rope, t["x"], t["tab"], t["tab"], t["x"], False, 1 << 70, None) is None
    assert native.append_q8(sh, rope, 0, [0, 2]) is None
    assert native.read_q8(sh, 0, [0, 2], 0, *cache, t["x"], t["x"], None) is None
    huge = U.Shape.make(2 ** 31 - 1, 2, 2, 8, 8, 6)
    assert native.rotary_apply(huge, rope, t["x"], t["tab"], t["tab"], t["x"], False, 1 << 50, None) is None
    assert native.attn_q8(sh, 0, [0, 2], 2, 0, t["x"], *cache, t["x"], None) is None


def test_inputs_of_overlapped_kernels_are_read_behind_the_wait():
    found = list(kernels("rotary.cu")) + list(kernels("attn_few.cu"))
    assert len(found) == 4
    for name, params, body in found:
        assert "grid_wait()" in body, name
        assert not re.search(r"const\s+(?!__grid_constant__)\w+\s*\*\s*__restrict__", params), name
        assert "__ldg(" not in body, name
        wait = body.index("grid_wait()")
        for load in re.finditer(r"__ldca\(|__ldcs\(|q_in\[|= load_coefficients", body):
            assert load.start() > wait, name
        # addresses take the wait's zero in
        assert re.search(r"\+ behind|\+= behind|\+ __shfl_sync\(0xFFFFFFFFu, grid_wait\(\), 0\)", body), name


def test_runs_of_the_cache_are_those_of_a_walk_over_the_frames():
    # the plan's key tiles of an item against a walk frame by frame, for a ring that wraps behind a sink
    import random
    rng = random.Random(3)
    for _ in range(300):
        tokens, sink, ring = 8 * rng.randint(16, 24), rng.randint(0, 4), rng.randint(1, 9)
        window = rng.randint(1, ring)
        start, attend = rng.randint(0, 40), rng.randint(0, sink)
        sh = U.Shape.make(1, 1, 1, 8, tokens // 8, ring)
        hi = start + 1
        lo = max(0, hi - window)
        runs, prev = [], None
        for p in list(range(min(attend, lo))) + list(range(lo, hi)):
            slot = p if p < sink else sink + (p - sink) % ring
            if slot != prev:
                runs.append(0)
            runs[-1] += tokens
            prev = slot + 1
        segs = U.window_attn_plan(sh, [start], window, 148, sink, attend)
        assert segs[0][7] == sum((r + 127) // 128 for r in runs), (tokens, sink, ring, window, start, attend)


def test_way_of_a_call():
    def way(batch, heads, queries, keys, workers=148, **kw):
        # one frame of `queries` tokens, keys / queries of them in the window
        n = keys // queries
        sh = U.Shape.make(batch, heads, 1, 1, queries, n, **kw)
        return U.window_attn_q8_way(sh, 0, [n + 5] * batch, n, 0, workers)

    assert {way(b, h, q, k) for b in (1, 40) for h in (1, 4096) for q in (1, 8) for k in (8, 800)} == {"few"}
    assert way(1, 2, 100, 300) == "few" and way(1, 40, 100, 300) == "tiles" and way(1, 2, 100, 300, 4) == "tiles"
    assert way(1, 2, 768, 1 << 20) == "tiles" and way(1, 2, 769, 769 << 10) == "unpacked"
    # the largest that the checks let through: 2^30 cache rows less one frame of them, all heads, all streams
    assert way(1 << 20, 2, 1 << 20, 1023 << 20) == "unpacked"
    assert way(1 << 20, 4096, 1 << 15, 16 << 15, 65536) == "unpacked" and way(1, 4096, 1 << 19, 1 << 19, 1) == "unpacked"


def test_way_of_a_call_refuses():
    def way(shape=good_shape(), sink=0, first=(0, 2), recent=2, attend=0, workers=148, out=True):
        got = ctypes.c_int32(7)
        rc = U.lib().unstep_window_attn_q8_way(ctypes.byref(shape), sink, starts(first), recent, attend, workers,
                                               ctypes.byref(got) if out else None)
        assert rc == 0 or got.value == 7
        return rc

    assert way() == 0
    for kw in (dict(sink=-1), dict(first=None), dict(first=(0, -1)), dict(recent=1), dict(recent=7), dict(attend=1),
               dict(workers=0), dict(workers=65537), dict(out=False), dict(shape=good_shape(batch=0))):
        assert way(**kw) == INVALID, kw
    assert way(shape=good_shape(head_dim=64)) == UNSUPPORTED
