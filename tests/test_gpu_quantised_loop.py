"""The calls on an 8-bit cache together, as they are used: table, rotation and append, attention and read of a stack of
layers over many chunks, eagerly and as a replayed graph; and the native marshalling of each against the general path."""

import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_32518_b200 as U
import workloads as W
from harness import attn_errors, to_bits, to_dev
from oracle import quantised_oracle as Q
from paper_2609_32518_b200 import binding
from paper_2609_32518_b200.layer_loop import ChunkStepper
from quant_harness import BANDS, device_rope, random_qkv

pytestmark = pytest.mark.gpu


def make(sh, bands=BANDS[128]):
    return U.Shape.make(sh.batch, sh.heads, sh.chunk_frames, sh.grid_h, sh.grid_w, sh.ring_frames, bands=bands)


@pytest.mark.parametrize("half,rotated,factor", [(False, 128, 1.0), (True, 96, 4.0)])
def test_chunks_through_a_stack_of_layers_against_the_oracle(half, rotated, factor):
    # 9 chunks of 2 frames through 1 sink + 5 ring frames, two layers, positions up to 4x those "trained on"
    sh = W.Shape(batch=2, heads=3, chunk_frames=2, grid_h=5, grid_w=9, ring_frames=5)
    rope = Q.Rope(half=half, factor=(factor, 1.0, 1.0), trained=(6, 0, 0), beta=(0.1, 0.5), magnitude=1.0 + 0.1 * np.log(factor))
    stepper = ChunkStepper(make(sh, BANDS[rotated]), 2, 5, 1, 1, quantised=True, rope=device_rope(rope))
    states = [Q.QuantState(2, 1, 5, sh.tokens_per_frame, 3) for _ in range(2)]
    for state, layer in zip(states, range(2)):      # what no chunk has written yet is alike on both sides
        for mine, theirs in ((state.cache_k, stepper.cache_k), (state.scale_k, stepper.scale_k),
                             (state.cache_v, stepper.cache_v), (state.scale_v, stepper.scale_v)):
            theirs[layer].view(torch.uint8).copy_(torch.from_numpy(mine))
    dims = (2, sh.chunk_tokens, 3, 128)
    for chunk in range(9):
        start = 2 * chunk
        bits = [random_qkv(sh, 100 + 2 * chunk + layer) for layer in range(2)]
        qkv = [tuple(to_dev(x) for x in b) for b in bits]
        q_rot = [torch.empty(dims, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        outs = [torch.empty_like(q) for q in q_rot]
        stepper.chunk_step(start, qkv, q_rot, outs)
        cos, sin = stepper.table(start)
        for layer in range(2):
            want = Q.kv_append(states[layer], [start] * 2, *bits[layer], cos.cpu().numpy(), sin.cpu().numpy(), half)
            assert np.array_equal(to_bits(q_rot[layer]), want)
            ref = Q.window_attn_q8(states[layer], [start] * 2, 5, 1, want, 2)
            mx, mean, rel = attn_errors(to_bits(outs[layer]), ref)
            assert mx <= 2e-2 and mean <= 2e-3 and rel <= 1.5e-2, (chunk, layer, mx, mean, rel)
    for layer in range(2):
        assert np.array_equal(stepper.cache_k[layer].view(torch.uint8).cpu().numpy(), states[layer].cache_k)
        k, v = stepper.read_frames(layer, 14, 4)
        for b in range(2):
            want_k, want_v = Q.kv_frames(states[layer], b, range(14, 18))
            assert np.array_equal(k[b].double().cpu().numpy(), want_k)
            assert np.array_equal(v[b].double().cpu().numpy(), want_v)
    assert U.poll_status() == 0


def test_read_frames_of_a_bf16_cache_are_its_slots():
    sh = W.Shape(batch=1, heads=2, chunk_frames=1, grid_h=2, grid_w=3, ring_frames=3)
    stepper = ChunkStepper(make(sh), 1, 3, 1, 1)
    for slot in range(4):
        stepper.cache_k[0][:, slot] = slot
    k, _ = stepper.read_frames(0, 6, 3)              # frames 6, 7, 8 behind one sink frame: slots 3, 1, 2
    assert k[0, :, 0, 0, 0].tolist() == [3.0, 1.0, 2.0]
    with pytest.raises(ValueError, match="bf16 cache"):
        ChunkStepper(make(sh), 1, 3, rope=U.Rope.make(half=True))


@pytest.mark.parametrize("quantised", [False, True])
def test_read_frames_refuses_what_no_cache_holds(quantised):
    sh = W.Shape(batch=1, heads=2, chunk_frames=1, grid_h=2, grid_w=3, ring_frames=3)
    stepper = ChunkStepper(make(sh), 1, 3, 1, 1, quantised=quantised)
    for first, n in ((-1, 2), (0, 0), (0, 5), (2, 4)):
        with pytest.raises(ValueError, match="hold at once"):
            stepper.read_frames(0, first, n)
    assert stepper.read_frames(0, 0, 4)[0].shape == (1, 4, 6, 2, 128)    # the sink frame and three of the ring


@pytest.mark.parametrize("grid", [(8, 8), (20, 20)])   # a window decoded in the attention, and one unpacked for it
def test_graph_of_a_chunk_replays_what_the_calls_do(grid):
    sh = W.Shape(batch=1, heads=4, chunk_frames=2, grid_h=grid[0], grid_w=grid[1], ring_frames=6)
    stepper = ChunkStepper(make(sh), 3, 6, quantised=True)
    dims = (1, sh.chunk_tokens, 4, 128)
    gen = torch.Generator(device="cuda").manual_seed(3)

    def normal():
        return torch.randn(dims, generator=gen, device="cuda").to(torch.bfloat16)

    qkv = [(normal(), normal(), normal()) for _ in range(3)]
    q_rot, outs = [torch.empty(dims, dtype=torch.bfloat16, device="cuda") for _ in range(3)], [normal() for _ in range(3)]
    for start in (0, 2):
        stepper.chunk_step(start, qkv, q_rot, outs)
    graphs = {start: stepper.chunk_graph(start, qkv, q_rot, outs) for start in (4, 6)}
    for start in (4, 6):
        for layer in range(3):
            qkv[layer][0].copy_(normal())
            qkv[layer][1].copy_(normal())
        stepper.chunk_step(start, qkv, q_rot, outs)
        want, caches = [o.clone() for o in outs], [c.view(torch.uint8).clone() for c in stepper.cache_k]
        for o in outs:
            o.zero_()
        graphs[start].replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        for a, b in zip(caches, stepper.cache_k):
            assert torch.equal(a, b.view(torch.uint8))
    assert U.poll_status() == 0


def test_native_and_general_marshalling_do_the_same():
    sh = W.Shape(batch=2, heads=3, chunk_frames=2, grid_h=9, grid_w=16, ring_frames=5)
    shape, rope = make(sh, BANDS[96]), U.Rope.make(half=True, magnitude=1.5)
    gen = torch.Generator(device="cuda").manual_seed(5)
    act, cache = (2, sh.chunk_tokens, 3, 128), (2, 6, sh.tokens_per_frame, 3)

    def fresh():
        gen.manual_seed(5)
        t = {n: torch.randn(act, generator=gen, device="cuda").to(torch.bfloat16) for n in ("q", "k", "v", "y", "out")}
        for n in ("ck", "cv"):
            t[n] = torch.randn(cache + (128,), generator=gen, device="cuda").to(torch.float8_e4m3fn)
            t["s" + n[1]] = torch.randint(120, 126, cache + (4,), generator=gen, device="cuda", dtype=torch.uint8).view(
                torch.float8_e8m0fnu)
        t["cos"], t["sin"] = (torch.empty((sh.chunk_tokens, 48), device="cuda") for _ in range(2))
        t["g"] = torch.rand(384, generator=gen, device="cuda")
        t["rk"], t["rv"] = (torch.empty((2, 3, sh.tokens_per_frame, 3, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return t

    def run(t):
        c = (t["ck"], t["sk"], t["cv"], t["sv"])
        U.rotary_table(shape, rope, 11, t["cos"], t["sin"])
        U.rotary_apply(shape, rope, t["q"], t["cos"], t["sin"], t["y"], transposed=True)
        U.rotary_kv_append_q8(shape, rope, 1, [11, 4], t["q"], t["k"], t["v"], t["cos"], t["sin"], t["q"], *c, gain_q=t["g"],
                              gain_k=t["g"], eps=1e-5)
        U.rotary_kv_append_q8(shape, rope, 1, [13, 6], t["q"], t["k"], t["v"], t["cos"], t["sin"], t["q"], *c)
        U.kv_read_q8(shape, 1, [11, 4], 3, *c, t["rk"], t["rv"])
        U.window_attn_q8(shape, 1, [13, 6], 4, 1, t["q"], *c, t["out"])
        torch.cuda.synchronize()

    native, general = fresh(), fresh()
    before = U.launch_count()
    run(native)
    per_run = U.launch_count() - before
    saved, binding._fast = binding._fast, binding._NoMarshal()
    try:
        run(general)
    finally:
        binding._fast = saved
    assert not isinstance(saved, binding._NoMarshal)
    assert U.launch_count() - before == 2 * per_run
    for name in native:
        assert torch.equal(native[name].contiguous().view(torch.uint8), general[name].contiguous().view(torch.uint8)), name


def test_refusals_on_the_device(monkeypatch):
    sh = W.Shape(batch=1, heads=2, chunk_frames=1, grid_h=4, grid_w=4, ring_frames=3)
    shape = make(sh)
    q = torch.zeros((1, 16, 2, 128), dtype=torch.bfloat16, device="cuda")
    code = torch.zeros((1, 3, 16, 2, 128), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((1, 3, 16, 2, 4), dtype=torch.uint8, device="cuda")
    good = (code.view(torch.float8_e4m3fn), scale.view(torch.float8_e8m0fnu)) * 2
    U.window_attn_q8(shape, 0, [2], 3, 0, q, *good, torch.empty_like(q))
    for bad in ((code,) + good[1:], good[:1] + (scale,) + good[2:], (good[0][:, :2],) + good[1:],
                (good[0].transpose(2, 3),) + good[1:]):
        with pytest.raises(ValueError, match="cache_k|scale_k"):
            U.window_attn_q8(shape, 0, [2], 3, 0, q, *bad, torch.empty_like(q))
    with pytest.raises(U.UnstepError):
        U.window_attn_q8(shape, 0, [2], 4, 0, q, *good, torch.empty_like(q))          # window longer than the ring
    with pytest.raises(U.UnstepError):
        U.kv_read_q8(shape, 0, [0], 4, *good, *(torch.empty((1, 4, 16, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    odd = torch.zeros(q.numel() + 4, dtype=torch.bfloat16, device="cuda")[4:].view(q.shape)   # 8 bytes off
    with pytest.raises(U.UnstepError):
        U.window_attn_q8(shape, 0, [2], 3, 0, odd, *good, torch.empty_like(q))
    # tensors of another device than the current one
    launches = U.launch_count()
    monkeypatch.setattr(binding, "_fast", binding._NoMarshal())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        U.window_attn_q8(shape, 0, [2], 3, 0, q, *good, torch.empty_like(q))
    assert U.launch_count() == launches
