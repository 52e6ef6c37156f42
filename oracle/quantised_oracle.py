"""Plain CPU definition of the 8-bit cache and of the rotary positions that go with it.

TEST INFRASTRUCTURE ONLY -- never on the product path.  numpy; shares nothing with the CUDA library.

  Q1  frequencies of the rotated pairs, scaled for positions beyond those a model was trained on
  Q2  the table: magnitude * cos and sin of position * frequency, float64, rounded once to float32
  Q3  the rotation in both layouts, of a part of the head, and its transpose
  Q4  blocks of 32 dims as e4m3 codes and a power of two
  Q5  the append into a cache of such blocks, and its frames read back
  Q6  attention over the decoded window, float64

Rotation and block scales are pinned operation by operation (float32), so the cache is one bit pattern.
"""

from __future__ import annotations

import math
from dataclasses import dataclass, field

import numpy as np

from .unstep_oracle import (HEAD_DIM, attention_rows, bf16_bits_to_f32, f32_to_bf16_bits_rne, sink_slot,
                            sink_window_frames, token_positions)

BLOCK = 32
NAN_BYTE = 255


@dataclass
class Rope:
    """Q1: layout and scaling; the axes are (frame, row, column)."""
    half: bool = False
    factor: tuple = (1.0, 1.0, 1.0)
    trained: tuple = (0, 0, 0)
    beta: tuple = (1.0, 32.0)
    magnitude: float = 1.0


def rotary_frequencies(bands, rope: Rope, base: float = 10000.0):
    """(frequency, axis) of the sum(bands) / 2 rotated pairs, float64."""
    omega, axis = [], []
    for a, dims in enumerate(bands):
        for i in range(dims // 2):
            w = math.pow(base, -(2.0 * i) / dims)
            if rope.factor[a] != 1.0:
                keep = 0.0
                if rope.trained[a] > 0:
                    turns = rope.trained[a] * w / (2.0 * math.pi)
                    keep = min(1.0, max(0.0, (turns - rope.beta[0]) / (rope.beta[1] - rope.beta[0])))
                w *= keep + (1.0 - keep) / rope.factor[a]
            omega.append(w)
            axis.append(a)
    return np.array(omega), np.array(axis, dtype=np.int64)


def rotary_table(start_frame, chunk_frames, grid_h, grid_w, bands, rope: Rope, base: float = 10000.0):
    """Q2: (cos, sin), float32 [L, sum(bands) / 2]."""
    omega, axis = rotary_frequencies(bands, rope, base)
    pos = np.stack(token_positions(start_frame, chunk_frames, grid_h, grid_w), axis=1).astype(np.float64)
    theta = pos[:, axis] * omega[None, :]
    return tuple(np.ascontiguousarray(rope.magnitude * f(theta), dtype=np.float32) for f in (np.cos, np.sin))


def rotate_f32(x: np.ndarray, cos: np.ndarray, sin: np.ndarray, half: bool, transposed: bool = False) -> np.ndarray:
    """Q3: float32 x[..., L, Hn, 128] by tables [.., L, R/2]; every operation rounded to float32 by itself."""
    x = np.asarray(x, dtype=np.float32)
    c = np.asarray(cos, dtype=np.float32)[..., :, None, :]
    s = np.asarray(sin, dtype=np.float32)[..., :, None, :]
    if transposed:
        s = -s
    r = 2 * c.shape[-1]
    a, b = (slice(0, r // 2), slice(r // 2, r)) if half else (slice(0, r, 2), slice(1, r, 2))
    y = x.copy()
    with np.errstate(all="ignore"):
        y[..., a] = (x[..., a] * c).astype(np.float32) - (x[..., b] * s).astype(np.float32)
        y[..., b] = (x[..., a] * s).astype(np.float32) + (x[..., b] * c).astype(np.float32)
    return y


def rotary_apply(x_bits, cos, sin, half, transposed=False):
    """Q3 on bf16 bits: rotated dims rounded to bf16, the others bit copies."""
    y = f32_to_bf16_bits_rne(rotate_f32(bf16_bits_to_f32(x_bits), cos, sin, half, transposed))
    r = 2 * cos.shape[-1]
    y[..., r:] = x_bits[..., r:]
    return y


def e4m3_value(code: np.ndarray) -> np.ndarray:
    """float64 values of e4m3 codes (sign, 4 exponent bits of bias 7, 3 mantissa bits; no infinities, 0x7F is NaN)."""
    c = np.asarray(code, dtype=np.int64)
    exponent, mantissa = (c >> 3) & 15, c & 7
    v = np.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * 2.0 ** (exponent - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


_GRID = e4m3_value(np.arange(127))          # 0, 2^-9, .. 448: increasing


def e4m3_code(x: np.ndarray) -> np.ndarray:
    """Codes of float values of magnitude at most 448 + half a step: nearest value, ties to the even code."""
    a = np.abs(np.asarray(x, dtype=np.float64))
    hi = np.minimum(np.searchsorted(_GRID, a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _GRID[hi] - a, a - _GRID[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def quantise(x: np.ndarray):
    """Q4: float32 x[..., 128] -> codes uint8 [..., 128] and scale bytes uint8 [..., 4]."""
    b = np.asarray(x, dtype=np.float32).reshape(x.shape[:-1] + (HEAD_DIM // BLOCK, BLOCK))
    with np.errstate(invalid="ignore"):
        top = np.abs(b).max(axis=-1).astype(np.float64)
        bad = ~(top < 1.9375 * 2.0 ** 127)                    # a NaN is not
    safe = np.where(bad, 1.0, top)
    e = np.full(safe.shape, -124.0)
    for k in range(-123, 121):                                # least e with top <= 448 * 2^e
        e = np.where(safe > 448.0 * 2.0 ** (k - 1), float(k), e)
    scaled = np.where(bad[..., None], 0.0, b.astype(np.float64)) * np.exp2(-e)[..., None]
    codes = np.where(bad[..., None], 0, e4m3_code(scaled))
    bytes_ = np.where(bad, NAN_BYTE, e + 127)
    return codes.astype(np.uint8).reshape(x.shape), bytes_.astype(np.uint8)


def decode(codes: np.ndarray, bytes_: np.ndarray) -> np.ndarray:
    """Values of codes [..., 128] with scale bytes [..., 4], float64."""
    scale = np.where(bytes_ == NAN_BYTE, np.nan, np.exp2(bytes_.astype(np.float64) - 127.0))
    return e4m3_value(codes) * np.repeat(scale, BLOCK, axis=-1)


@dataclass
class QuantState:
    """Q5: cache of one layer, codes [B, sink + C, T, Hn, 128] and scale bytes [.., 4]."""
    batch: int
    sink_frames: int
    ring_frames: int
    tokens_per_frame: int
    heads: int
    cache_k: np.ndarray = field(init=False)
    scale_k: np.ndarray = field(init=False)
    cache_v: np.ndarray = field(init=False)
    scale_v: np.ndarray = field(init=False)

    def __post_init__(self):
        rows = (self.batch, self.sink_frames + self.ring_frames, self.tokens_per_frame, self.heads)
        # what no append has written reads as NaN
        self.cache_k, self.cache_v = (np.full(rows + (HEAD_DIM,), 0x39, dtype=np.uint8) for _ in range(2))
        self.scale_k, self.scale_v = (np.full(rows + (4,), NAN_BYTE, dtype=np.uint8) for _ in range(2))


def norm_f32(x: np.ndarray, gain: np.ndarray, eps: float) -> np.ndarray:
    """RMS norm over all channels of a token [.., Hn, 128]: mean of squares in float64, the rest in float32."""
    wide = x.reshape(x.shape[:-2] + (-1,))
    ms = (wide.astype(np.float64) ** 2).mean(axis=-1).astype(np.float32)
    r = np.float32(1.0) / np.sqrt(ms + np.float32(eps))
    return ((wide * r[..., None]).astype(np.float32) * gain).astype(np.float32).reshape(x.shape)


def kv_append(state: QuantState, start_frames, q_bits, k_bits, v_bits, cos, sin, half, gain_q=None, gain_k=None,
              eps: float = 0.0):
    """Q5 for one chunk of every stream; returns q_out bits."""
    q, k, v = (bf16_bits_to_f32(x) for x in (q_bits, k_bits, v_bits))
    if gain_q is not None:
        q, k = norm_f32(q, gain_q, eps), norm_f32(k, gain_k, eps)
    q, k = rotate_f32(q, cos, sin, half), rotate_f32(k, cos, sin, half)
    T = state.tokens_per_frame
    for x, cache, scale in ((k, state.cache_k, state.scale_k), (v, state.cache_v, state.scale_v)):
        codes, bytes_ = quantise(x)
        for b, s in enumerate(start_frames):
            for f in range(x.shape[1] // T):
                slot = sink_slot(int(s) + f, state.sink_frames, state.ring_frames)
                cache[b, slot], scale[b, slot] = codes[b, f * T:(f + 1) * T], bytes_[b, f * T:(f + 1) * T]
    return f32_to_bf16_bits_rne(q)


def kv_frames(state: QuantState, b: int, frames, heads=slice(None)):
    """Frames of stream b read back, float64: (k, v) [F, T, heads, 128]."""
    slots = [sink_slot(int(p), state.sink_frames, state.ring_frames) for p in frames]
    return tuple(np.stack([decode(c[b, s][:, heads], e[b, s][:, heads]) for s in slots])
                 for c, e in ((state.cache_k, state.scale_k), (state.cache_v, state.scale_v)))


def window_attn_q8(state: QuantState, start_frames, recent_frames, sink_attend, q_bits, chunk_frames, rows=None,
                   heads=None):
    """Q6: float64 [B, rows, heads, 128]."""
    B, L, Hn, _ = q_bits.shape
    rows = np.arange(L) if rows is None else np.asarray(rows)
    heads = list(range(Hn)) if heads is None else list(heads)
    out = np.empty((B, len(rows), len(heads), HEAD_DIM))
    for b in range(B):
        frames = sink_window_frames(int(start_frames[b]), chunk_frames, recent_frames, sink_attend)
        k, v = kv_frames(state, b, frames, heads)
        for i, h in enumerate(heads):
            out[b, :, i] = attention_rows(bf16_bits_to_f32(q_bits[b, rows, h]).astype(np.float64),
                                          k[:, :, i].reshape(-1, HEAD_DIM), v[:, :, i].reshape(-1, HEAD_DIM))
    return out
