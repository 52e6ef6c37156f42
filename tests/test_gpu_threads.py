"""Calls that several host threads make at once: the library is entered without the interpreter's lock, so the launches
of two calls can be enqueued in turn."""

import threading

import pytest
import torch

import paper_2609_32518_b200 as U
import workloads as W
from quant_harness import Layer

pytestmark = pytest.mark.gpu


def together(*bodies):
    """Runs the bodies in a thread each, from a common start on; what one of them raises is raised here."""
    start, failed = threading.Barrier(len(bodies)), []

    def run(body):
        try:
            start.wait(60)
            body()
        except BaseException as e:   # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=run, args=(body,)) for body in bodies]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if failed:
        raise failed[0]


# one group of heads, and 40 heads x 13 200 keys x 512 bytes of unpacked window, which go in two
@pytest.mark.parametrize("heads,grid,frames,calls", [(6, (9, 100), (3, 2), 300), (40, (11, 100), (12, 11), 40)])
@pytest.mark.parametrize("side", [False, True])
def test_two_threads_on_one_stream_with_unpacked_windows(heads, grid, frames, calls, side):
    # Unpacking and attention are launches of their own that share the stream's window buffer: those of one call have
    # to come one behind the other.  The result of a call alone is the one of every call, bit for bit.
    stream = torch.cuda.Stream() if side else torch.cuda.current_stream()
    work = []
    for seed, n in enumerate(frames):
        layer = Layer(W.Shape(batch=1, heads=heads, chunk_frames=1, grid_h=grid[0], grid_w=grid[1], ring_frames=n))
        assert U.window_attn_q8_way(layer.abi, 0, [n], n, 0, U.attn_workers()[0]) == "unpacked"
        layer.fill_codes(90 + seed)
        q = layer.queries(95 + seed)
        outs = torch.empty((calls,) + q.shape, dtype=q.dtype, device="cuda")
        work.append((layer, q, outs, layer.attend([n], n, 0, q)))
    assert not torch.equal(work[0][3], work[1][3])
    torch.cuda.synchronize()

    def body(layer, q, outs, _):
        n = layer.sh.ring_frames
        for i in range(calls):
            U.window_attn_q8(layer.abi, 0, [n], n, 0, q, *layer.cache, outs[i], stream=stream)

    body(*work[0])                                                # the buffer of this stream is there
    torch.cuda.synchronize()
    together(*(lambda w=w: body(*w) for w in work))
    torch.cuda.synchronize()
    for _, _, outs, want in work:
        wrong = [i for i in range(calls) if not torch.equal(outs[i].view(torch.int16), want.view(torch.int16))]
        assert not wrong, f"{len(wrong)} of {calls} calls, the first is number {wrong[0]}"
    assert U.poll_status() == 0


class PerThread:
    """cudaStreamPerThread: one handle, a stream of its own in every host thread."""
    cuda_stream = 2


@pytest.mark.parametrize("quantised,tokens,heads,way", [(False, 200, 80, None), (True, 3, 40, "few"),
                                                        (True, 300, 12, "tiles"), (True, 900, 6, "unpacked")])
def test_the_per_thread_streams_of_two_threads_have_a_scratch_each(quantised, tokens, heads, way):
    work, calls, n = [], 60, 2500 // tokens + 1
    for seed in range(2):
        layer = Layer(W.Shape(batch=1, heads=heads, chunk_frames=1, grid_h=1, grid_w=tokens, ring_frames=n))
        layer.fill_codes(60 + seed)
        if quantised:
            assert U.window_attn_q8_way(layer.abi, 0, [n], n, 0, U.attn_workers()[0]) == way
            call = lambda q, o, st, x=layer: U.window_attn_q8(x.abi, 0, [n], n, 0, q, *x.cache, o, stream=st)
        else:
            ring = [torch.empty((1, n, tokens, heads, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            U.kv_read_q8(layer.abi, 0, [0], n, *layer.cache, *ring)
            call = lambda q, o, st, x=layer, r=ring: U.window_attn(x.abi, [n - 1], n, q, *r, o, stream=st)
            # parts that are merged through the scratch
            plan = U.window_attn_plan(layer.abi, [n - 1], n, U.attn_workers()[0], clusters=U.attn_clusters())
            assert any(s[9] >= 0 for s in plan)
        q = layer.queries(65 + seed)
        want = torch.empty_like(q)
        call(q, want, None)
        work.append((call, q, torch.empty((calls,) + q.shape, dtype=q.dtype, device="cuda"), want))
    torch.cuda.synchronize()

    def body(call, q, outs, _):
        for i in range(calls):
            call(q, outs[i], PerThread)

    for _ in range(2):
        together(*(lambda w=w: body(*w) for w in work))           # threads that have ended leave the others' scratch alone
    torch.cuda.synchronize()
    for _, _, outs, want in work:
        assert all(torch.equal(o.view(torch.int16), want.view(torch.int16)) for o in outs)
    assert U.poll_status() == 0
