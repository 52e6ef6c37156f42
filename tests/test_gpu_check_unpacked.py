"""The checking build (every global store tested against the extent of its buffer) over attention that unpacks its windows,
with guard bands around the result.  Loaded in a child process, so the normal library of this process is untouched."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _child():
    sys.path.insert(0, ROOT)
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    import torch
    import paper_2609_32518_b200 as U
    import workloads as W
    from harness import attn_errors, to_bits
    from quant_harness import Layer

    assert os.path.basename(U.lib()._name) == "libunstep_check.so"
    band, mark = 8192, 0x5A5A

    def run(name, batch, heads, fc, grid, ring, sink, starts, recent, attend, launches, far=False):
        layer = Layer(W.Shape(batch=batch, heads=heads, chunk_frames=fc, grid_h=grid[0], grid_w=grid[1], ring_frames=ring), sink)
        way = U.window_attn_q8_way(layer.abi, sink, starts, recent, attend, U.attn_workers()[0])
        assert way == "unpacked", (name, way)
        layer.fill_codes(3)
        if far:                                                   # a second factor for every block
            layer.ora.scale_v += 40
            layer.upload()
        q = layer.queries(4)
        raw = torch.full((q.numel() + 2 * band,), mark, dtype=torch.int16, device="cuda")
        out = raw[band:-band].view(torch.bfloat16).view(q.shape)
        before = U.launch_count()
        U.window_attn_q8(layer.abi, sink, starts, recent, attend, q, *layer.cache, out)
        assert U.launch_count() - before == launches, (name, U.launch_count() - before)
        torch.cuda.synchronize()
        assert U.poll_status() == 0, "a store was refused"
        assert bool((raw[:band] == mark).all() and (raw[-band:] == mark).all()), "a store landed outside its buffer"
        rows, some = W.sample_rows(layer.sh.chunk_tokens)[::4], sorted({0, heads // 2, heads - 1})
        ref = layer.attend_oracle(starts, recent, attend, q, rows=rows, heads=some)
        got = out[:, rows][:, :, some]
        if far:
            got, ref = got * 2.0 ** -40, ref * 2.0 ** -40
        mx, mean, rel = attn_errors(to_bits(got), ref)
        assert mx <= 2e-2 and mean <= 2e-3 and rel <= 1.5e-2, (name, mx, mean, rel)
        print("ok", name, flush=True)

    run("wrapped behind a sink", 2, 3, 2, (20, 21), 8, 2, [13, 6], 5, 1, 2)
    run("streams of other lengths, large scales", 3, 2, 3, (17, 19), 7, 1, [0, 3, 40], 7, 1, 2, far=True)
    run("least queries", 1, 5, 1, (1, 769), 2, 0, [1], 2, 0, 2)
    # 17 heads x 3 streams x 13 200 keys x 512 bytes are 345 MB: 9 heads of each stream, then 8
    run("unequal groups of heads", 3, 17, 1, (11, 100), 12, 0, [15, 16, 17], 12, 0, 4)
    # 132 000 keys x 512 bytes a head and stream: three streams at a time, then two
    run("groups of streams", 5, 1, 1, (11, 100), 120, 0, [130, 125, 140, 119, 150], 120, 0, 4)
    run("34 streams", 34, 1, 1, (11, 100), 2, 0, [b % 4 for b in range(34)], 2, 0, 4)
    print("all ok")


@pytest.mark.gpu
def test_no_store_of_an_unpacked_window_or_behind_it_leaves_its_buffer():
    env = dict(os.environ, UNSTEP_LIB_VARIANT="check")
    res = subprocess.run([sys.executable, os.path.abspath(__file__), "--child"], env=env, capture_output=True,
                         text=True, timeout=900)
    assert res.returncode == 0 and "all ok" in res.stdout, res.stdout[-2000:] + res.stderr[-4000:]


if __name__ == "__main__":
    if "--child" in sys.argv:
        _child()
