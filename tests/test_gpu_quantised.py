"""GPU parity of the 8-bit cache and its rotary positions against the oracle (through the C ABI).

Table: at most one unit in the last place of float32 (one rounding of a double that may differ in its last bits).
Rotation, append without the norm and read: bit for bit.  Append with the norm: the sum of squares runs in float32 in
another order than the oracle's, so values move by parts in 2^20; bounds below.  Attention: the bounds of the other
attention tests, against float64 over the decoded cache."""

import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_32518_b200 as U
import workloads as W
from harness import attn_errors, to_bits, to_dev
from oracle import quantised_oracle as Q
from quant_harness import BANDS, Layer, bytes_host, device_rope, random_qkv

pytestmark = pytest.mark.gpu

MAX_ABS, MEAN_ABS, REL_L2 = 2e-2, 2e-3, 1.5e-2


def shape(batch, heads, chunk_frames, grid_h, grid_w, ring):
    return W.Shape(batch=batch, heads=heads, chunk_frames=chunk_frames, grid_h=grid_h, grid_w=grid_w, ring_frames=ring)


# ------------------------------------------------------------------ table

@pytest.mark.parametrize("rotated", [128, 96, 64, 16])
@pytest.mark.parametrize("start,grid,fc", [(0, (1, 1), 1), (123, (9, 17), 3), (2_000_000_000, (8, 8), 2)])
def test_table(rotated, start, grid, fc):
    for rope in (Q.Rope(), Q.Rope(factor=(4.0, 1.0, 2.0), trained=(21, 0, 30), beta=(1.0, 4.0), magnitude=1.25)):
        abi = U.Shape.make(1, 1, fc, *grid, fc, bands=BANDS[rotated])
        cos = torch.full((fc * grid[0] * grid[1], rotated // 2), float("nan"), device="cuda")
        sin = cos.clone()
        U.rotary_table(abi, device_rope(rope), start, cos, sin)
        for got, want in zip((cos, sin), Q.rotary_table(start, fc, *grid, BANDS[rotated], rope)):
            got = got.cpu().numpy()
            # at 2e9 a double's last bit moves the angle by 2^-23, which small cosines and sines show in full
            far = 2.0 ** -52 * (start + fc)
            assert (np.abs(got - want) <= np.spacing(np.abs(want)) + 2 * far).all()
    assert U.poll_status() == 0


def test_plain_rotary_table_is_the_rope_table():
    abi = U.Shape.make(1, 1, 2, 9, 13, 2)
    tabs = [torch.empty((abi.chunk_tokens, 64), device="cuda") for _ in range(4)]
    U.rope_table(abi, 7, *tabs[:2])
    U.rotary_table(abi, U.Rope.make(half=True), 7, *tabs[2:])
    assert torch.equal(tabs[0], tabs[2]) and torch.equal(tabs[1], tabs[3])


# ------------------------------------------------------------------ rotation

@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("rotated", [128, 96, 64, 16])
@pytest.mark.parametrize("batch,heads,grid,fc", [(1, 1, (1, 1), 1), (2, 5, (3, 7), 2), (3, 12, (1, 5), 1), (1, 33, (2, 2), 1)])
def test_rotation_and_its_transpose(half, rotated, batch, heads, grid, fc):
    sh = shape(batch, heads, fc, *grid, fc)
    abi = U.Shape.make(batch, heads, fc, *grid, fc, bands=BANDS[rotated])
    rope = Q.Rope(half=half, magnitude=1.25)
    x = random_qkv(sh, 3)[0]
    x[0, 0, 0, :3] = (0x7F80, 0x8000, 0x7FC0)                     # infinity, -0, NaN
    tables = [Q.rotary_table(5 + b, fc, *grid, BANDS[rotated], rope) for b in range(batch)]
    for transposed in (False, True):
        for shared in (True, False):
            cos, sin = (tables[0][i] if shared else np.stack([t[i] for t in tables]) for i in range(2))
            want = Q.rotary_apply(x, cos, sin, half, transposed)
            for in_place in (False, True):
                dx = to_dev(x)
                y = dx if in_place else torch.empty_like(dx)
                U.rotary_apply(abi, device_rope(rope), dx, torch.from_numpy(np.ascontiguousarray(cos)).cuda(),
                               torch.from_numpy(np.ascontiguousarray(sin)).cuda(), y, transposed=transposed,
                               table_stream_stride=0 if shared else cos.shape[1] * cos.shape[2])
                got = to_bits(y)
                nan = np.isnan(O.bf16_bits_to_f32(want))
                assert np.array_equal(np.isnan(O.bf16_bits_to_f32(got)), nan)
                assert np.array_equal(got[~nan], want[~nan]), (half, rotated, transposed, shared, in_place)


def test_rotation_undone_by_its_transpose_and_gradient_by_differences():
    # y = R x in bf16: g . (R(x + d) - R(x - d)) against (R^T g) . 2 d.  Powers of two in x, g, d: roundings of y to
    # bf16 (2^-8 of up to 4) in 2 x 128 terms, of R^T g (2^-8 of up to 2) in one, sums exact enough.
    abi = U.Shape.make(1, 1, 1, 1, 1, 1, bands=(64, 0, 0))
    rope = U.Rope.make(half=True)
    cos, sin = (torch.empty((1, 32), device="cuda") for _ in range(2))
    U.rotary_table(abi, rope, 3, cos, sin)

    def rotate(x, transposed=False):
        y = torch.empty_like(x)
        U.rotary_apply(abi, rope, x, cos, sin, y, transposed=transposed)
        return y

    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, 1, 1, 128), generator=gen, device="cuda").to(torch.bfloat16)
    g = torch.randn((1, 1, 1, 128), generator=gen, device="cuda").sign().to(torch.bfloat16)
    grad = rotate(g, True).float()
    for i in (0, 5, 31, 32, 63, 64, 127):
        d = torch.zeros_like(x)
        d[..., i] = 1.0
        diff = (g.float() * (rotate(x + d).float() - rotate(x - d).float())).sum() / 2
        # only the two outputs of the pair differ; x + d is itself rounded to bf16
        bound = 2 * 2 * 2.0 ** -8 * 8 + 2.0 ** -8 * 2
        assert abs(diff.item() - grad[..., i].item()) <= bound
    back = rotate(rotate(x), True).float()
    # two roundings to bf16 of values at most sqrt(2) times a pair's largest
    assert (back - x.float()).abs().max() <= 2 * 2.0 ** -8 * 1.5 * x.float().abs().max()


# ------------------------------------------------------------------ append and read

@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("rotated", [128, 96, 16])
@pytest.mark.parametrize("batch,heads,grid,fc,ring,sink", [
    (1, 1, (1, 1), 1, 3, 0), (2, 3, (3, 5), 2, 4, 1), (1, 12, (2, 9), 3, 3, 0), (35, 2, (1, 3), 1, 2, 2), (2, 17, (1, 7), 1, 2, 0),
    (1, 4, (1, 41), 1, 2, 0), (2, 7, (1, 19), 1, 2, 1), (1, 32, (1, 5), 1, 2, 0), (1, 33, (1, 3), 2, 3, 1), (2, 48, (1, 2), 1, 2, 0),
    (1, 49, (1, 3), 1, 2, 1), (1, 65, (1, 3), 1, 2, 0)])
def test_append_is_bit_exact_and_read_gives_it_back(half, rotated, batch, heads, grid, fc, ring, sink):
    sh = shape(batch, heads, fc, *grid, ring)
    layer = Layer(sh, sink, Q.Rope(half=half), rotated)
    for step in range(4):
        starts = [step * fc + (b % 3) * fc for b in range(batch)]
        q, k, v = random_qkv(sh, 10 + step, spread=step % 2 == 1)
        got, want = layer.append(starts, q, k, v, in_place=step == 2)
        assert np.array_equal(to_bits(got), want)
        layer.assert_same()                                      # slots that were not written among them
    n = min(fc + 1, ring)
    first = [s + fc - n for s in starts]
    out = [torch.full((batch, n, sh.tokens_per_frame, heads, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
           for _ in range(2)]
    U.kv_read_q8(layer.abi, sink, first, n, *layer.cache, *out)
    for b in range(batch):
        for got, want in zip(out, Q.kv_frames(layer.ora, b, range(first[b], first[b] + n))):
            got = got[b].double().cpu().numpy()
            assert np.array_equal(got, want, equal_nan=True)
    assert U.poll_status() == 0


def test_blocks_that_are_not_finite_or_at_the_ends_of_the_range():
    sh = shape(1, 2, 1, 1, 8, 2)
    layer = Layer(sh, 0, Q.Rope())
    q, k, v = random_qkv(sh, 5)
    top = [0x7F80, 0xFF80, 0x7FC0, 0x7F78, 0x7F77, 0x0001, 0x0000, 0x0080]   # inf, -inf, NaN, ends of the range, subnormals
    for n, bits in enumerate(top):
        v[0, n, 1, 40] = bits
        if n >= 5:
            v[0, n, 1, 32:64] = bits
    got, want = layer.append([0], q, k, v)
    assert np.array_equal(to_bits(got), want)
    layer.assert_same()
    out = [torch.empty((1, 1, 8, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    U.kv_read_q8(layer.abi, 0, [0], 1, *layer.cache, *out)
    want_k, want_v = Q.kv_frames(layer.ora, 0, [0])
    assert np.array_equal(out[0][0].double().cpu().numpy(), want_k)
    assert np.array_equal(out[1][0].double().cpu().numpy(), want_v, equal_nan=True)
    assert np.isnan(want_v[0, :4, 1, 32:64]).all() and np.isfinite(want_v[0, 4:]).all()


def test_read_decodes_every_code_under_every_scale():
    sh = shape(1, 2, 1, 16, 8, 1)                                 # 256 rows of 128 dims
    layer = Layer(sh)
    codes = np.arange(256, dtype=np.uint8)
    codes[(codes & 127) == 127] = 0                              # the append writes none of these
    layer.ora.cache_k = np.tile(codes.reshape(2, 128)[None, None, None], (1, 1, 128, 1, 1)).copy()
    layer.ora.cache_v = layer.ora.cache_k[..., ::-1].copy()
    scales = np.concatenate([np.arange(3, 248), [255] * 11]).astype(np.uint8).reshape(1, 1, 128, 2)
    layer.ora.scale_k = np.repeat(scales[..., :1], 8, axis=-1).reshape(1, 1, 128, 2, 4).copy()
    layer.ora.scale_v = np.repeat(scales[..., 1:], 8, axis=-1).reshape(1, 1, 128, 2, 4).copy()
    layer.upload()
    out = [torch.empty((1, 1, 128, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    U.kv_read_q8(layer.abi, 0, [0], 1, *layer.cache, *out)
    for got, want in zip(out, Q.kv_frames(layer.ora, 0, [0])):
        with np.errstate(over="ignore"):
            want = want.astype(np.float32)                       # 2^128 and more: an infinity of the same sign
        assert np.array_equal(got[0].float().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("heads", [1, 5, 6, 7, 12, 13, 17, 31, 32, 33, 40, 64, 70])   # both sides of each way to lay out a token
def test_append_behind_the_norm(half, heads):
    sh = shape(2, heads, 1, 3, 5, 2)
    layer = Layer(sh, 0, Q.Rope(half=half), 96)
    rng = np.random.default_rng(6)
    gains = tuple((1.0 + 0.2 * rng.standard_normal(heads * 128)).astype(np.float32) for _ in range(2))
    q, k, v = random_qkv(sh, 7)
    got, want = layer.append([0, 1], q, k, v, gains, 1e-6, in_place=heads % 2 == 0)
    # The mean is a sum of up to 2^14 squares in float32, in threads of at most 2^7 terms, warps and blocks: relative
    # error below 2^-15; half of it in the root: values move by 2^-16 of themselves, and of what is subtracted from them.
    # Rounded to bf16, two values that are 2^-16 of a magnitude m apart differ by at most that and one unit, 2^-7 of themselves.
    got, want = O.bf16_bits_to_f32(to_bits(got)), O.bf16_bits_to_f32(want)
    assert (np.abs(got - want) <= 2.0 ** -7 * np.abs(want) + 2.0 ** -15 * np.abs(want).max()).all()
    assert (got != want).mean() <= 2.0 ** -5
    assert np.array_equal(bytes_host(layer.cache_v), layer.ora.cache_v)
    assert np.array_equal(bytes_host(layer.scale_v), layer.ora.scale_v)
    # One code step is at most 2^-3 of a value, or 2^-9 of its scale
    k_got = Q.decode(bytes_host(layer.cache_k), bytes_host(layer.scale_k))
    k_want = Q.decode(layer.ora.cache_k, layer.ora.scale_k)
    fresh = np.isfinite(k_want)
    assert np.array_equal(fresh, np.isfinite(k_got))
    step = np.maximum(2.0 ** -3 * np.abs(k_want), 2.0 ** -9 * np.repeat(np.exp2(layer.ora.scale_k.astype(float) - 127), 32, -1))
    assert (np.abs(k_got - k_want)[fresh] <= step[fresh]).all()
    assert (k_got != k_want)[fresh].mean() <= 2.0 ** -9           # 2^-16 of a value against steps of 2^-4 and more


# ------------------------------------------------------------------ attention

def check(got: torch.Tensor, ref, what):
    bits = to_bits(got)
    mx, mean, rel = attn_errors(bits, ref)
    assert np.isfinite(O.bf16_bits_to_f32(bits)).all(), what
    assert mx <= MAX_ABS and mean <= MEAN_ABS and rel <= REL_L2, f"{what}: {mx:.3e} {mean:.3e} {rel:.3e}"


def assert_way(layer: Layer, want: str, starts, recent, attend=0):
    """A call on so many streams, heads, queries and keys reaches the kernel that its test is about."""
    way = U.window_attn_q8_way(layer.abi, layer.sink, starts, recent, attend, U.attn_workers()[0])
    assert way == want, f"{way} instead of {want}"


ATTN = [
    # batch, heads, grid, chunk, ring, sink, recent, sink_attend, starts
    ("one_key", (1, 1, (1, 1), 1, 1, 0, 1, 0, (0,))),
    ("17_queries_33_keys", (1, 3, (1, 17), 1, 2, 0, 2, 0, (50,))),
    ("one_query_37_keys", (1, 3, (1, 1), 1, 37, 0, 37, 0, (50,))),
    ("tokens", (3, 5, (1, 1), 1, 700, 2, 650, 2, (1500, 3, 699))),
    ("127_keys", (1, 2, (1, 127), 1, 1, 0, 1, 0, (4,))),
    ("128_keys", (1, 2, (8, 16), 1, 1, 0, 1, 0, (4,))),
    ("129_keys", (1, 2, (3, 43), 1, 1, 0, 1, 0, (4,))),
    ("short_frames_wrapped", (2, 3, (5, 7), 2, 9, 1, 7, 1, (31, 8))),
    ("first_chunk", (1, 2, (8, 25), 3, 7, 3, 7, 3, (0,))),
    ("ragged", (2, 3, (8, 25), 3, 7, 0, 5, 0, (12, 3))),
    ("sink_and_ring_wrapped", (2, 2, (8, 25), 3, 6, 3, 6, 2, (13, 6))),
    ("37_streams", (37, 1, (4, 10), 1, 4, 0, 4, 0, tuple(3 + b % 5 for b in range(37)))),
    ("17_queries_33_keys_many_heads", (1, 200, (1, 17), 1, 2, 0, 2, 0, (50,))),
    ("127_keys_many_heads", (1, 20, (1, 127), 1, 1, 0, 1, 0, (4,))),
    ("128_keys_many_heads", (1, 20, (8, 16), 1, 1, 0, 1, 0, (4,))),
    ("129_keys_many_heads", (1, 20, (3, 43), 1, 1, 0, 1, 0, (4,))),
    ("short_frames_wrapped_many_heads", (2, 20, (5, 7), 2, 9, 1, 7, 1, (31, 8))),
    ("first_chunk_many_heads", (1, 12, (8, 25), 3, 7, 3, 7, 3, (0,))),
    ("37_streams_many_heads", (37, 12, (4, 10), 1, 4, 0, 4, 0, tuple(3 + b % 5 for b in range(37)))),
    ("one_tile_clusters_many_heads", (1, 20, (1, 20), 1, 150, 1, 140, 1, (300,))),
    ("clusters", (1, 8, (10, 32), 1, 17, 0, 17, 0, (20,))),
    ("one_tile_many_items", (2, 90, (4, 30), 1, 9, 0, 9, 0, (20, 5))),
    ("one_tile_shares", (1, 200, (1, 100), 1, 25, 0, 25, 0, (60,))),
    ("one_tile_clusters", (1, 6, (1, 20), 1, 150, 1, 140, 1, (300,))),
    ("768_queries", (1, 3, (3, 256), 1, 3, 0, 3, 0, (7,))),
    ("whole_and_parts", (1, 150, (5, 8), 4, 8, 0, 8, 0, (4,))),
    ("shares", (1, 80, (5, 8), 5, 64, 0, 64, 0, (59,))),
]
TILES = ("ragged", "sink_and_ring_wrapped", "clusters", "one_tile_many_items", "one_tile_shares", "768_queries",
         "whole_and_parts", "shares")


@pytest.mark.parametrize("name", [n for n, _ in ATTN])
def test_attention(name):
    batch, heads, grid, fc, ring, sink, recent, attend, starts = dict(ATTN)[name]
    sh = shape(batch, heads, fc, *grid, ring)
    layer = Layer(sh, sink)
    assert_way(layer, "tiles" if name in TILES or name.endswith("many_heads") else "few", starts, recent, attend)
    layer.fill(20, k_scale=2.0)
    q = layer.queries(21)
    some = sorted({0, heads // 2, heads - 1})
    for rep in range(2):                                          # counters and scratch are as the next call wants them
        got = layer.attend(starts, recent, attend, q)
        check(got[:, :, some], layer.attend_oracle(starts, recent, attend, q, heads=some), f"{name} {rep}")
        assert U.poll_status() == 0
        q = q.flip(1).contiguous()


# Few queries, or few keys: keys go straight from memory into warp-level products, for 8 queries at a time.
FEW = [
    ("8_queries_one_key", (1, 1, (1, 8), 1, 1, 0, 1, 0, (0,))),
    ("9_queries", (2, 3, (3, 3), 1, 40, 2, 33, 1, (100, 7))),
    ("16_queries_wrapped", (1, 5, (2, 4), 2, 30, 0, 29, 0, (77,))),
    ("15_keys", (1, 2, (1, 3), 1, 5, 0, 5, 0, (9,))),
    ("17_keys", (2, 2, (1, 1), 1, 17, 0, 17, 0, (40, 16))),
    ("34_streams", (34, 3, (1, 2), 1, 90, 1, 70, 1, tuple(3 * b for b in range(34)))),
    ("long", (1, 1, (1, 1), 1, 9001, 0, 9001, 0, (20000,))),
    ("many_items", (3, 40, (1, 1), 1, 200, 0, 200, 0, (300, 10, 199))),
    ("17_queries", (1, 2, (1, 17), 1, 9, 0, 9, 0, (20,))),
    ("33_queries_one_frame", (3, 2, (3, 11), 1, 2, 0, 1, 0, (0, 7, 1))),
    ("63_queries_wrapped", (2, 3, (3, 7), 3, 19, 2, 16, 2, (40, 3))),
    ("100_queries_whole_items", (1, 5, (10, 10), 1, 1, 0, 1, 0, (6,))),
    ("303_queries_parts", (1, 1, (3, 101), 1, 11, 0, 11, 0, (30,))),
    ("35_streams_of_10_queries", (35, 1, (2, 5), 1, 30, 1, 27, 1, tuple(2 * b for b in range(35)))),
    ("801_queries", (1, 1, (9, 89), 1, 1, 0, 1, 0, (2,))),
]


@pytest.mark.parametrize("name", [n for n, _ in FEW])
@pytest.mark.parametrize("v_power", [0, 60])
def test_attention_of_few_queries(name, v_power):
    batch, heads, grid, fc, ring, sink, recent, attend, starts = dict(FEW)[name]
    sh = shape(batch, heads, fc, *grid, ring)
    layer = Layer(sh, sink)
    assert_way(layer, "few", starts, recent, attend)
    layer.fill(70, k_scale=2.0, v_power=v_power)
    q = layer.queries(71)
    got, ref = layer.attend(starts, recent, attend, q), layer.attend_oracle(starts, recent, attend, q)
    if v_power == 0:
        check(got, ref, name)
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all() and np.linalg.norm(got - ref) <= REL_L2 * np.linalg.norm(ref)
    assert U.poll_status() == 0


def shifted(t: torch.Tensor, nbytes: int) -> torch.Tensor:
    """A copy of t whose address is `nbytes` behind a multiple of 256."""
    raw = torch.zeros(t.numel() * t.element_size() + 256 + nbytes, dtype=torch.uint8, device="cuda")
    lo = -raw.data_ptr() % 256 + nbytes
    out = raw[lo:lo + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
    out.view(torch.uint8).copy_(t.view(torch.uint8))
    assert out.data_ptr() % 256 == nbytes
    return out


@pytest.mark.parametrize("tokens,heads,way", [(2, 3, "few"), (30, 3, "few"), (30, 90, "tiles"), (200, 20, "tiles"),
                                               (900, 3, "unpacked")])
def test_buffers_at_the_least_alignment(tokens, heads, way):
    # activations and codes on 16 bytes, scales on 4
    sh = shape(1, heads, 1, 1, tokens, max(3, 300 // tokens))
    layer = Layer(sh)
    assert_way(layer, way, [sh.ring_frames + 1], sh.ring_frames)
    layer.fill(74)
    q = layer.queries(75)
    n = sh.ring_frames
    want = layer.attend([n + 1], n, 0, q)
    layer.cache_k, layer.cache_v = shifted(layer.cache_k, 16), shifted(layer.cache_v, 16)
    layer.scale_k, layer.scale_v = shifted(layer.scale_k, 4), shifted(layer.scale_v, 4)
    out = shifted(torch.full_like(q, float("nan")), 16)
    U.window_attn_q8(layer.abi, 0, [n + 1], n, 0, shifted(q, 16), *layer.cache, out)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))
    back, moved = ([torch.empty((1, n, tokens, heads, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2))
    moved = [shifted(x, 16) for x in moved]
    U.kv_read_q8(layer.abi, 0, [1], n, *layer.cache, *moved)
    layer.upload()
    U.kv_read_q8(layer.abi, 0, [1], n, *layer.cache, *back)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(back, moved))
    assert U.poll_status() == 0


@pytest.mark.parametrize("tokens,heads,way", [(3, 40, "few"), (25, 3, "few"), (100, 12, "tiles"), (300, 12, "tiles"),
                                               (900, 6, "unpacked")])
def test_calls_that_overlap_on_three_streams(tokens, heads, way):
    # each stream has a scratch of its own: parts, counters and unpacked windows
    layers = []
    for i in range(3):
        layer = Layer(shape(1, heads, 1, 1, tokens, 2500 // tokens + 1))
        layer.fill_codes(80 + i)
        layers.append((layer, layer.queries(85 + i)))
    n = layers[0][0].sh.ring_frames
    assert_way(layers[0][0], way, [n], n)
    want = [layer.attend([n], n, 0, q) for layer, q in layers]
    streams, outs = [torch.cuda.Stream() for _ in range(3)], [torch.empty_like(q) for _, q in layers]
    torch.cuda.synchronize()
    for _ in range(8):
        for (layer, q), st, o in zip(layers, streams, outs):
            U.window_attn_q8(layer.abi, 0, [n], n, 0, q, *layer.cache, o, stream=st)
    torch.cuda.synchronize()
    for a, b in zip(want, outs):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert U.poll_status() == 0


@pytest.mark.parametrize("tokens,frames", [(2, 700), (28, 50)])
def test_few_queries_of_peaked_keys_in_rising_order(tokens, frames):
    # every step of a warp has a larger maximum than the one before: sums and results are rescaled each time
    sh = shape(1, 2, 1, 1, tokens, frames)
    layer = Layer(sh)
    rng = np.random.default_rng(72)
    k = rng.standard_normal(layer.ora.cache_k.shape).astype(np.float32)
    k[..., 0] = np.linspace(0, 200, frames, dtype=np.float32)[None, :, None, None]
    layer.ora.cache_k, layer.ora.scale_k = Q.quantise(k)
    layer.ora.cache_v, layer.ora.scale_v = Q.quantise(rng.standard_normal(k.shape).astype(np.float32))
    layer.upload()
    q = layer.queries(73)
    q[..., 0] = 3.0
    assert_way(layer, "few", [frames - 1], frames)
    check(layer.attend([frames - 1], frames, 0, q), layer.attend_oracle([frames - 1], frames, 0, q), "rising")


# From four pairs of query tiles on the window is unpacked first.
UNPACKED = [
    ("769_queries", (1, 3, (1, 769), 1, 3, 0, 3, 0, (7,))),
    ("1025_queries", (1, 2, (5, 205), 1, 2, 0, 2, 0, (3,))),
    ("small_frames_wrapped", (2, 3, (7, 9), 20, 23, 1, 21, 1, (80, 20))),
    ("sink_and_ring_wrapped", (2, 2, (20, 21), 3, 6, 3, 6, 2, (13, 6))),
    ("first_chunk", (3, 2, (20, 21), 3, 6, 3, 6, 3, (0, 3, 1))),
    ("34_streams", (34, 1, (11, 100), 1, 2, 0, 2, 0, tuple(b % 4 for b in range(34)))),
]


@pytest.mark.parametrize("name", [n for n, _ in UNPACKED])
def test_attention_over_unpacked_windows(name):
    batch, heads, grid, fc, ring, sink, recent, attend, starts = dict(UNPACKED)[name]
    sh = shape(batch, heads, fc, *grid, ring)
    layer = Layer(sh, sink)
    assert_way(layer, "unpacked", starts, recent, attend)
    layer.fill_codes(50)
    q = layer.queries(51)
    rows = W.sample_rows(sh.chunk_tokens)
    for rep in range(2):
        launches = U.launch_count()
        got = layer.attend(starts, recent, attend, q)
        assert U.launch_count() - launches == 2 * ((batch + 31) // 32)
        check(got[:, rows], layer.attend_oracle(starts, recent, attend, q, rows=rows), f"{name} {rep}")
        layer.fill_codes(52)                                      # the scratch holds the former window
    assert U.poll_status() == 0


def test_heads_in_groups_where_the_unpacked_windows_exceed_the_scratch():
    # 40 heads x 13 200 keys x 512 bytes are 270 MB: two groups of 20 heads; three streams of 17 heads: 9 and 8 heads of each
    for batch, heads, frames in ((1, 40, 12), (3, 17, 12)):
        sh = shape(batch, heads, 1, 11, 100, frames)
        layer = Layer(sh)
        layer.fill_codes(53)
        q = layer.queries(54)
        starts = [frames + 3 + b for b in range(batch)]
        launches = U.launch_count()
        got = layer.attend(starts, frames, 0, q)
        assert U.launch_count() - launches == 4
        rows, some = W.sample_rows(sh.chunk_tokens)[::4], sorted({0, heads // 2 - 1, heads // 2, heads - 1})
        check(got[:, rows][:, :, some], layer.attend_oracle(starts, frames, 0, q, rows=rows, heads=some), f"{heads} heads")
    assert U.poll_status() == 0


def test_unpacked_window_of_a_captured_graph_survives_larger_calls():
    small, large = Layer(shape(1, 2, 1, 11, 100, 2)), Layer(shape(1, 4, 1, 11, 100, 9))
    for layer, seed in ((small, 55), (large, 56)):
        layer.fill_codes(seed)
    q, q_large = small.queries(57), large.queries(58)
    side = torch.cuda.Stream()
    out, want = torch.zeros_like(q), torch.zeros_like(q)
    torch.cuda.synchronize()

    def call(layer, x, o, start, n):
        U.window_attn_q8(layer.abi, 0, [start], n, 0, x, *layer.cache, o, stream=side)

    call(small, q, want, 4, 2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(small, q, out, 4, 2)
    call(large, q_large, torch.empty_like(q_large), 11, 9)        # a larger scratch on the same stream
    side.synchronize()
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
    assert_way(small, "unpacked", [4], 2)
    # a capture on a stream that has no scratch yet decodes inside the attention, within the bounds
    fresh, other = torch.cuda.Stream(), torch.zeros_like(q)
    few = Layer(shape(1, 60, 1, 4, 10, 2))
    assert_way(few, "tiles", [4], 2)
    few.fill_codes(59)
    q_few = few.queries(60)
    torch.cuda.synchronize()
    U.window_attn_q8(few.abi, 0, [4], 2, 0, q_few, *few.cache, torch.empty_like(q_few), stream=fresh)   # counters
    graph2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph2, stream=fresh):
        U.window_attn_q8(small.abi, 0, [4], 2, 0, q, *small.cache, other, stream=fresh)
    graph2.replay()
    torch.cuda.synchronize()
    check(other, small.attend_oracle([4], 2, 0, q), "captured without scratch")
    assert U.poll_status() == 0


@pytest.mark.parametrize("heads,way", [(2, "few"), (12, "tiles")])
def test_attention_leaves_what_it_does_not_attend_alone(heads, way):
    # every slot outside the window holds NaN blocks, and codes that nobody writes
    sh = shape(2, heads, 2, 3, 19, 8)
    layer = Layer(sh, 2)
    layer.fill(30)
    starts, recent, attend = (9, 15), 5, 1
    assert_way(layer, way, starts, recent, attend)
    for b, s in enumerate(starts):
        frames = O.sink_window_frames(s, 2, recent, attend)
        held = {O.sink_slot(p, 2, 8) for p in frames}
        for slot in set(range(10)) - held:
            for c, e in ((layer.ora.cache_k, layer.ora.scale_k), (layer.ora.cache_v, layer.ora.scale_v)):
                c[b, slot], e[b, slot] = 0x7F, 255
    layer.upload()
    q = layer.queries(31)
    check(layer.attend(starts, recent, attend, q), layer.attend_oracle(starts, recent, attend, q), "poisoned")


@pytest.mark.parametrize("heads,way", [(2, "few"), (12, "tiles")])
def test_attention_over_a_nan_block_is_nan_for_its_head_only(heads, way):
    sh = shape(1, heads, 1, 8, 20, 3)
    layer = Layer(sh)
    assert_way(layer, way, [2], 3)
    layer.fill(32)
    layer.ora.scale_v[0, 1, 77, 1, 2] = 255
    layer.upload()
    q = layer.queries(33)
    got, ref = layer.attend([2], 3, 0, q), layer.attend_oracle([2], 3, 0, q)
    nan = np.isnan(ref)
    assert nan[:, :, 1, 64:96].all() and nan.sum() == 160 * 32
    assert np.array_equal(np.isnan(got.float().cpu().numpy()), nan)
    others = [h for h in range(heads) if h != 1]
    check(got[:, :, others], ref[:, :, others], "the other heads")


@pytest.mark.parametrize("heads,way", [(2, "few"), (12, "tiles")])
@pytest.mark.parametrize("power", [-100, -40, 20, 60, 100])
def test_attention_with_values_far_from_one(power, heads, way):
    # scale bytes above 134 take a second factor; the result is the one of values near 1, scaled: 2^-11 of the unscaled
    # relative error is lost nowhere
    sh = shape(1, heads, 1, 7, 23, 3)
    layer = Layer(sh)
    assert_way(layer, way, [2], 3)
    layer.fill(34, v_power=power)
    q = layer.queries(35)
    got = layer.attend([2], 3, 0, q).double().cpu().numpy()
    ref = layer.attend_oracle([2], 3, 0, q)
    assert np.isfinite(got).all()
    assert np.linalg.norm((got - ref) * 2.0 ** -power) <= REL_L2 * np.linalg.norm(ref * 2.0 ** -power)


@pytest.mark.parametrize("heads,way", [(2, "few"), (3, "tiles")])
def test_attention_with_peaked_scores(heads, way):
    sh = shape(1, heads, 2, 8, 25, 6)
    layer = Layer(sh)
    assert_way(layer, way, [9], 6)
    layer.fill(36, k_scale=40.0)
    q = layer.queries(37)
    check(layer.attend([9], 6, 0, q), layer.attend_oracle([9], 6, 0, q), "peaked")


def test_same_as_the_bf16_attention_over_the_cache_read_back():
    # decoding is exact, so where the tiles and the split are the same the results are, bit for bit
    sh = shape(1, 4, 3, 10, 32, 6)
    layer = Layer(sh)
    layer.fill(38)
    q = layer.queries(39)
    back = [torch.empty((1, 6, 320, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    U.kv_read_q8(layer.abi, 0, [0], 6, *layer.cache, *back)
    out = torch.empty_like(q)
    U.window_attn(layer.abi, [3], 6, q, *back, out)
    got = layer.attend([3], 6, 0, q)
    assert (got.float() - out.float()).abs().max() <= 2 * 2.0 ** -8 * out.float().abs().max()


def test_calls_on_two_streams_and_a_replayed_graph():
    sh = shape(1, 12, 1, 9, 31, 6)
    layer = Layer(sh)
    layer.fill(40)
    q = layer.queries(41)
    want = layer.attend([5], 6, 0, q)
    side = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(q) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, o in zip(side, outs):
            U.window_attn_q8(layer.abi, 0, [5], 6, 0, q, *layer.cache, o, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o.view(torch.int16), want.view(torch.int16)) for o in outs)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(graph, stream=side[0]):
        U.window_attn_q8(layer.abi, 0, [5], 6, 0, q, *layer.cache, out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
    assert U.poll_status() == 0
