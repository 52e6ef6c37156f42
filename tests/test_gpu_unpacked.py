"""Attention over unpacked windows where they can go wrong, and the other two ways beside it: what lies outside the window or
is left in the buffer from another call, blocks that are NaN, values and keys far from one, infinite queries, windows
that are larger than the buffer."""

import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_32518_b200 as U
import workloads as W
from harness import attn_errors, to_bits
from oracle import quantised_oracle as Q
from quant_harness import CODES, SCALES, Layer

pytestmark = pytest.mark.gpu

MAX_ABS, MEAN_ABS, REL_L2 = 2e-2, 2e-3, 1.5e-2     # the bounds of the other attention tests
# heads, grid of a frame: one launch of each way over a window of three frames
WAYS = {"few": (2, (8, 20)), "tiles": (12, (8, 20)), "unpacked": (3, (25, 33))}


def make(way, frames=3, batch=1):
    heads, grid = WAYS[way]
    layer = Layer(W.Shape(batch=batch, heads=heads, chunk_frames=1, grid_h=grid[0], grid_w=grid[1], ring_frames=frames))
    assert_way(layer, way, [frames - 1] * batch, frames)
    return layer


def assert_way(layer, way, starts, recent, attend=0):
    got = U.window_attn_q8_way(layer.abi, layer.sink, starts, recent, attend, U.attn_workers()[0])
    assert got == way, f"{got} instead of {way}"


def check(got, ref, what):
    mx, mean, rel = attn_errors(to_bits(got), ref)
    assert np.isfinite(O.bf16_bits_to_f32(to_bits(got))).all(), what
    assert mx <= MAX_ABS and mean <= MEAN_ABS and rel <= REL_L2, f"{what}: {mx:.3e} {mean:.3e} {rel:.3e}"


def test_slots_outside_the_window_are_left_alone():
    layer = Layer(W.Shape(batch=2, heads=3, chunk_frames=2, grid_h=20, grid_w=21, ring_frames=8), 2)
    layer.fill(30)
    starts, recent, attend = (9, 15), 5, 1
    assert_way(layer, "unpacked", starts, recent, attend)
    for b, s in enumerate(starts):
        held = {O.sink_slot(p, 2, 8) for p in O.sink_window_frames(s, 2, recent, attend)}
        for slot in set(range(10)) - held:
            for c, e in ((layer.ora.cache_k, layer.ora.scale_k), (layer.ora.cache_v, layer.ora.scale_v)):
                c[b, slot], e[b, slot] = 0x7F, 255
    layer.upload()
    q, rows = layer.queries(31), W.sample_rows(layer.sh.chunk_tokens)
    check(layer.attend(starts, recent, attend, q)[:, rows], layer.attend_oracle(starts, recent, attend, q, rows=rows), "poisoned")


def test_what_a_former_call_left_in_the_buffer_is_not_attended():
    # a long window of NaN blocks, then shorter ones that end inside a tile, of streams that differ in length
    for frames, starts, poison in ((9, (8, 8), True), (3, (2, 0), False), (2, (1, 1), False)):
        layer = make("unpacked", frames, batch=2)
        layer.fill(32)
        if poison:
            for field in ("cache_k", "cache_v"):
                getattr(layer.ora, field)[...] = 0x7E
            for field in ("scale_k", "scale_v"):
                getattr(layer.ora, field)[...] = 255
            layer.upload()
        q = layer.queries(33)
        got = layer.attend(starts, frames, 0, q)
        if poison:
            assert torch.isnan(got).all()
            continue
        rows = W.sample_rows(layer.sh.chunk_tokens)
        check(got[:, rows], layer.attend_oracle(starts, frames, 0, q, rows=rows), f"{frames} frames")
    assert U.poll_status() == 0


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("keys", [False, True])
def test_a_nan_block(way, keys):
    # of a key: every query of its head has a NaN score; of a value: its 32 dims of that head
    layer = make(way)
    layer.fill(34)
    (layer.ora.scale_k if keys else layer.ora.scale_v)[0, 1, 77, 1, 2] = 255
    layer.upload()
    q = layer.queries(35)
    got = layer.attend([2], 3, 0, q)
    nan = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    nan[:, :, 1, slice(None) if keys else slice(64, 96)] = True
    assert torch.equal(torch.isnan(got), nan)
    rows, others = W.sample_rows(layer.sh.chunk_tokens), [h for h in range(layer.sh.heads) if h != 1]
    check(got[:, rows][:, :, others], layer.attend_oracle([2], 3, 0, q, rows=rows, heads=others), "the other heads")


@pytest.mark.parametrize("way", WAYS)
def test_keys_and_values_under_large_scales_are_those_near_one_bit_for_bit(way):
    # Scale bytes above 134 are decoded with two factors.  Keys times 2^24 and queries times 2^-24 give the same scores, values times
    # 2^40 the same result times 2^40: all of it powers of two, within range, and exact.
    layer = make(way)
    layer.fill(36, k_scale=2.0)
    q = layer.queries(37)
    want = layer.attend([2], 3, 0, q)
    assert layer.ora.scale_k.max() <= 134 and layer.ora.scale_v.max() <= 134
    layer.ora.scale_k += 24
    layer.ora.scale_v += 40
    assert layer.ora.scale_k.min() > 134 and layer.ora.scale_v.min() > 134
    layer.upload()
    got = layer.attend([2], 3, 0, q * 2.0 ** -24)
    assert torch.equal((got * 2.0 ** -40).view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("power", [-100, 60, 100])
def test_values_far_from_one(power):
    layer = make("unpacked")
    layer.fill(38, v_power=power)
    q, rows = layer.queries(39), W.sample_rows(layer.sh.chunk_tokens)
    got = layer.attend([2], 3, 0, q)[:, rows].double().cpu().numpy()
    ref = layer.attend_oracle([2], 3, 0, q, rows=rows)
    assert np.isfinite(got).all()
    assert np.linalg.norm((got - ref) * 2.0 ** -power) <= REL_L2 * np.linalg.norm(ref * 2.0 ** -power)


def test_peaked_scores():
    layer = make("unpacked")
    layer.fill(40, k_scale=40.0)
    q, rows = layer.queries(41), W.sample_rows(layer.sh.chunk_tokens)
    check(layer.attend([2], 3, 0, q)[:, rows], layer.attend_oracle([2], 3, 0, q, rows=rows), "peaked")


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_query_that_is_not_finite_is_nan_alone(way, value):
    # an infinite query has scores of both signs of infinity: NaN, for itself and nobody else
    layer = make(way)
    layer.fill(42)
    q = layer.queries(43)
    at = layer.sh.chunk_tokens // 2 + 1
    q[0, at, 1, 5] = value
    got = layer.attend([2], 3, 0, q)
    nan = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    nan[0, at, 1] = True
    assert torch.equal(torch.isnan(got), nan)
    near = [r for r in range(at - 40, at + 40) if r != at and 0 <= r < layer.sh.chunk_tokens]
    clean = layer.queries(43)
    check(got[:, near], layer.attend_oracle([2], 3, 0, clean, rows=near), "the others")


@pytest.mark.parametrize("grid", [(10, 32), (17, 19)])       # a window of whole tiles, and one that ends inside a tile
def test_unpacked_is_the_bf16_attention_over_the_cache_read_back_bit_for_bit(grid):
    # decoding is exact, and over one run of frames tiles and split are the same
    layer = Layer(W.Shape(batch=1, heads=4, chunk_frames=3, grid_h=grid[0], grid_w=grid[1], ring_frames=6))
    layer.fill(44)
    assert_way(layer, "unpacked", [3], 6)
    q = layer.queries(45)
    back = [torch.empty((1, 6, grid[0] * grid[1], 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    U.kv_read_q8(layer.abi, 0, [0], 6, *layer.cache, *back)
    out = torch.empty_like(q)
    U.window_attn(layer.abi, [3], 6, q, *back, out)
    assert torch.equal(layer.attend([3], 6, 0, q).view(torch.int16), out.view(torch.int16))


def test_a_head_whose_window_exceeds_the_buffer_is_decoded_as_it_goes():
    # 524 700 keys x 512 bytes are more than 256 MB: nothing is unpacked, and the result is that of float64
    tokens, frames = 1100, 477
    abi = U.Shape.make(1, 1, 1, 11, 100, frames)
    assert U.window_attn_q8_way(abi, 0, [frames], frames, 0, U.attn_workers()[0]) == "unpacked"   # as far as there is room
    gen = torch.Generator(device="cuda").manual_seed(46)
    dims = (1, frames, tokens, 1)

    def codes():
        c = torch.randint(0, 256, dims + (128,), generator=gen, device="cuda", dtype=torch.uint8)
        c[(c & 127) == 127] = 0
        return c.view(CODES)

    def scales():
        return torch.randint(114, 119, dims + (4,), generator=gen, device="cuda", dtype=torch.uint8).view(SCALES)

    cache = (codes(), scales(), codes(), scales())
    q = torch.randn((1, tokens, 1, 128), generator=gen, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    launches = U.launch_count()
    U.window_attn_q8(abi, 0, [frames], frames, 0, q, *cache, out)
    assert U.launch_count() - launches == 1
    rows = W.sample_rows(tokens)[::2]
    # code times the power of two of its block, from torch's own types
    k, v = ((c.float().double().view(-1, 4, 32) * torch.exp2(e.view(torch.uint8).double().view(-1, 4, 1) - 127)).view(-1, 128)
            for c, e in (cache[:2], cache[2:]))
    ref = torch.softmax(q[0, rows, 0].double() @ k.T / 128 ** 0.5, dim=-1) @ v
    check(out[0, rows, 0], ref.cpu().numpy(), "long window")
    assert U.poll_status() == 0
