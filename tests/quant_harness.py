"""Shared plumbing of the GPU tests of the 8-bit cache: the same bytes on the oracle's side and on the device's."""

from __future__ import annotations

import numpy as np
import torch

import oracle as O
import paper_2609_32518_b200 as U
import workloads as W
from harness import to_bits, to_dev
from oracle import quantised_oracle as Q

CODES, SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu
BANDS = {128: (44, 42, 42), 96: (32, 32, 32), 64: (24, 20, 20), 16: (16, 0, 0)}


def bytes_dev(a: np.ndarray, dtype) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().view(dtype)


def bytes_host(t: torch.Tensor) -> np.ndarray:
    return t.view(torch.uint8).cpu().numpy()


def device_rope(rope: Q.Rope) -> U.Rope:
    return U.Rope.make(half=rope.half, factor=rope.factor, trained=rope.trained, beta=rope.beta, magnitude=rope.magnitude)


class Layer:
    """One layer's 8-bit cache on both sides."""

    def __init__(self, sh: W.Shape, sink: int = 0, rope: Q.Rope = Q.Rope(), rotated: int = 128):
        self.sh, self.sink, self.rope, self.bands = sh, sink, rope, BANDS[rotated]
        self.abi = U.Shape.make(sh.batch, sh.heads, sh.chunk_frames, sh.grid_h, sh.grid_w, sh.ring_frames, bands=self.bands)
        self.abi_rope = device_rope(rope)
        self.ora = Q.QuantState(sh.batch, sink, sh.ring_frames, sh.tokens_per_frame, sh.heads)
        self.upload()

    def upload(self):
        o = self.ora
        self.cache_k, self.cache_v = bytes_dev(o.cache_k, CODES), bytes_dev(o.cache_v, CODES)
        self.scale_k, self.scale_v = bytes_dev(o.scale_k, SCALES), bytes_dev(o.scale_v, SCALES)

    @property
    def cache(self):
        return self.cache_k, self.scale_k, self.cache_v, self.scale_v

    def fill(self, seed: int, k_scale: float = 1.0, v_power: int = 0):
        """Random keys and values in every slot, values times 2^v_power."""
        rng = np.random.default_rng(seed)
        rows = self.ora.cache_k.shape
        self.ora.cache_k, self.ora.scale_k = Q.quantise((k_scale * rng.standard_normal(rows)).astype(np.float32))
        v = (rng.standard_normal(rows) * 2.0 ** v_power).astype(np.float32)
        self.ora.cache_v, self.ora.scale_v = Q.quantise(v)
        self.upload()

    def fill_codes(self, seed: int):
        """Random codes and scales in every slot, values below 1: large caches, quickly."""
        rng = np.random.default_rng(seed)
        for c, e in (("cache_k", "scale_k"), ("cache_v", "scale_v")):
            codes = rng.integers(0, 256, getattr(self.ora, c).shape, dtype=np.uint8)
            codes[(codes & 127) == 127] = 0
            setattr(self.ora, c, codes)
            setattr(self.ora, e, rng.integers(114, 119, getattr(self.ora, e).shape, dtype=np.uint8))
        self.upload()

    def tables(self, starts):
        sh = self.sh
        t = [Q.rotary_table(int(s), sh.chunk_frames, sh.grid_h, sh.grid_w, self.bands, self.rope) for s in starts]
        return np.stack([x[0] for x in t]), np.stack([x[1] for x in t])

    def append(self, starts, q, k, v, gains=(None, None), eps=0.0, in_place=False):
        """The append on both sides; q_out bits of the device and of the oracle."""
        starts = [int(s) for s in starts]
        cos, sin = self.tables(starts)
        dq = to_dev(q)
        q_out = dq if in_place else torch.empty_like(dq)
        g = [None if x is None else torch.from_numpy(x).cuda() for x in gains]
        U.rotary_kv_append_q8(self.abi, self.abi_rope, self.sink, starts, dq, to_dev(k), to_dev(v),
                              torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), q_out, *self.cache,
                              gain_q=g[0], gain_k=g[1], eps=eps,
                              table_stream_stride=cos.shape[1] * cos.shape[2])
        return q_out, Q.kv_append(self.ora, starts, q, k, v, cos, sin, self.rope.half, gains[0], gains[1], eps)

    def assert_same(self):
        for name in ("cache_k", "scale_k", "cache_v", "scale_v"):
            got, want = bytes_host(getattr(self, name)), getattr(self.ora, name)
            assert np.array_equal(got, want), f"{name}: {(got != want).sum()} of {want.size} differ"

    def attend(self, starts, recent, sink_attend, q: torch.Tensor) -> torch.Tensor:
        out = torch.full_like(q.view(torch.int16), 0x7FC1).view(torch.bfloat16)
        U.window_attn_q8(self.abi, self.sink, [int(s) for s in starts], recent, sink_attend, q, *self.cache, out)
        return out

    def attend_oracle(self, starts, recent, sink_attend, q: torch.Tensor, rows=None, heads=None):
        return Q.window_attn_q8(self.ora, starts, recent, sink_attend, to_bits(q), self.sh.chunk_frames, rows, heads)

    def queries(self, seed: int) -> torch.Tensor:
        gen = torch.Generator(device="cuda").manual_seed(seed)
        dims = (self.sh.batch, self.sh.chunk_tokens, self.sh.heads, 128)
        return torch.randn(dims, generator=gen, device="cuda").to(torch.bfloat16)


def random_qkv(sh: W.Shape, seed: int, spread: bool = False):
    """bf16 bits of q, k, v; `spread`: magnitudes from 2^-40 to 2^40 by blocks of 32 dims."""
    rng = np.random.default_rng(seed)
    dims = (sh.batch, sh.chunk_tokens, sh.heads, 4, 32)
    out = []
    for _ in range(3):
        x = rng.standard_normal(dims)
        if spread:
            x = x * 2.0 ** rng.integers(-40, 41, dims[:-1] + (1,))
        out.append(O.f32_to_bf16_bits_rne(x.astype(np.float32).reshape(dims[:3] + (128,))))
    return out
