"""The checking build (every global store tested against the extent of its buffer) over the calls on an 8-bit cache, with
guard bands around every output.  Loaded in a child process, so the normal library of this process is untouched."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _child():
    sys.path.insert(0, ROOT)
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    import numpy as np
    import torch
    import oracle as O
    import paper_2609_32518_b200 as U
    import workloads as W
    from harness import attn_errors, to_bits, to_dev
    from oracle import quantised_oracle as Q
    from quant_harness import BANDS, CODES, SCALES, Layer, device_rope, random_qkv

    assert os.path.basename(U.lib()._name) == "libunstep_check.so"
    band, mark = 8192, 0xA5

    class Guarded:
        """Bytes of a buffer between two bands of marks."""

        def __init__(self, dims, dtype, like=None):
            self.n = int(np.prod(dims)) * torch.empty((), dtype=dtype).element_size()
            self.raw = torch.full((self.n + 2 * band,), mark, dtype=torch.uint8, device="cuda")
            self.t = self.raw[band:band + self.n].view(dtype).view(dims)
            if like is not None:
                self.t.view(torch.uint8).copy_(like.contiguous().view(torch.uint8))

        def intact(self):
            return bool((self.raw[:band] == mark).all() and (self.raw[band + self.n:] == mark).all())

    def settled(*buffers):
        torch.cuda.synchronize()
        assert U.poll_status() == 0, "a store was refused"
        assert all(b.intact() for b in buffers), "a store landed outside its buffer"

    def run(name, sh, sink, starts, recent, attend, rotated, half, norm=False):
        rope = Q.Rope(half=half, factor=(2.0, 1.0, 1.0), trained=(21, 0, 0), beta=(1.0, 4.0))
        layer = Layer(sh, sink, rope, rotated)
        layer.fill(3)
        tab = [Guarded((sh.chunk_tokens, rotated // 2), torch.float32) for _ in range(2)]
        U.rotary_table(layer.abi, layer.abi_rope, starts[0], tab[0].t, tab[1].t)
        settled(*tab)
        guards = {}
        for field, dtype in (("cache_k", CODES), ("scale_k", SCALES), ("cache_v", CODES), ("scale_v", SCALES)):
            guards[field] = Guarded(getattr(layer, field).shape, dtype, getattr(layer, field))
            setattr(layer, field, guards[field].t)
        q, k, v = random_qkv(sh, 4)
        dims = (sh.batch, sh.chunk_tokens, sh.heads, 128)
        cos, sin = layer.tables(starts)
        dev_tab = [torch.from_numpy(x).cuda() for x in (cos, sin)]
        stride = cos.shape[1] * cos.shape[2]
        q_out = Guarded(dims, torch.bfloat16)
        rng = np.random.default_rng(5)
        gains = [(1.0 + 0.1 * rng.standard_normal(sh.heads * 128)).astype(np.float32) if norm else None for _ in range(2)]
        dev_gains = [None if g is None else torch.from_numpy(g).cuda() for g in gains]
        U.rotary_apply(layer.abi, layer.abi_rope, to_dev(q), *dev_tab, q_out.t, table_stream_stride=stride)
        settled(q_out)
        assert np.array_equal(to_bits(q_out.t), Q.rotary_apply(q, cos, sin, half))
        U.rotary_kv_append_q8(layer.abi, layer.abi_rope, sink, starts, to_dev(q), to_dev(k), to_dev(v), *dev_tab, q_out.t,
                              *layer.cache, gain_q=dev_gains[0], gain_k=dev_gains[1], eps=1e-6, table_stream_stride=stride)
        settled(q_out, *guards.values())
        Q.kv_append(layer.ora, starts, q, k, v, cos, sin, half, *gains, 1e-6)
        if norm:
            # the sum of squares runs in another order here, so the oracle goes on with what the device has
            for field in ("cache_k", "scale_k", "cache_v", "scale_v"):
                getattr(layer.ora, field)[...] = getattr(layer, field).view(torch.uint8).cpu().numpy()
        else:
            layer.assert_same()
        n = min(recent, min(starts) + sh.chunk_frames)
        first = [s + sh.chunk_frames - n for s in starts]
        back = [Guarded((sh.batch, n, sh.tokens_per_frame, sh.heads, 128), torch.bfloat16) for _ in range(2)]
        U.kv_read_q8(layer.abi, sink, first, n, *layer.cache, back[0].t, back[1].t)
        settled(*back)
        for b in range(sh.batch):
            for got, want in zip(back, Q.kv_frames(layer.ora, b, range(first[b], first[b] + n))):
                assert np.array_equal(got.t[b].double().cpu().numpy(), want)
        out = Guarded(dims, torch.bfloat16)
        U.window_attn_q8(layer.abi, sink, starts, recent, attend, q_out.t, *layer.cache, out.t)
        settled(out, q_out, *guards.values())
        mx, mean, rel = attn_errors(to_bits(out.t), layer.attend_oracle(starts, recent, attend, q_out.t))
        assert mx <= 2e-2 and mean <= 2e-3 and rel <= 1.5e-2, (name, mx, mean, rel)
        print("ok", name, flush=True)

    def shape(batch, heads, fc, gh, gw, ring):
        return W.Shape(batch=batch, heads=heads, chunk_frames=fc, grid_h=gh, grid_w=gw, ring_frames=ring)

    run("token", shape(1, 1, 1, 1, 1, 5), 0, [7], 5, 0, 128, False)
    run("ragged", shape(2, 3, 3, 8, 25, 7), 0, [12, 3], 7, 0, 128, True)
    run("sink", shape(2, 5, 2, 3, 7, 9), 2, [21, 8], 8, 1, 96, True)
    run("sink, many heads", shape(2, 40, 2, 3, 7, 9), 2, [21, 8], 8, 1, 96, True)
    run("groups", shape(1, 2, 1, 7, 13, 6), 0, [9], 6, 0, 128, True)
    run("37 streams", shape(37, 1, 1, 4, 10, 4), 0, [3 + b % 5 for b in range(37)], 4, 0, 16, False)
    run("norm", shape(2, 12, 1, 3, 11, 4), 1, [5, 9], 4, 1, 128, True, norm=True)
    run("wide norm", shape(1, 70, 1, 1, 9, 3), 0, [4], 3, 0, 64, False, norm=True)
    run("parts", shape(1, 150, 4, 5, 8, 8), 0, [4], 8, 0, 128, False)
    run("shares", shape(1, 80, 5, 5, 8, 64), 0, [59], 64, 0, 128, False)
    print("all ok")


@pytest.mark.gpu
def test_no_store_of_the_quantised_calls_leaves_its_buffer():
    env = dict(os.environ, UNSTEP_LIB_VARIANT="check")
    res = subprocess.run([sys.executable, os.path.abspath(__file__), "--child"], env=env, capture_output=True,
                         text=True, timeout=900)
    assert res.returncode == 0 and "all ok" in res.stdout, res.stdout[-2000:] + res.stderr[-4000:]


if __name__ == "__main__":
    if "--child" in sys.argv:
        _child()
