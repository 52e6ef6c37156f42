// Rotation of one tensor by a table (HBM bound), and the append that quantises into an 8-bit cache, with the
// read of its frames.
#include <cuda_bf16.h>

#include "common.h"
#include "quant.cuh"

namespace unstep {

// What a thread rotates: 8 neighbouring dims (a 16-byte vector) at place u = 0 .. 15 of a head.
struct RotaryPlace {
  int32_t rows;        // float4 of a table row: R / 8
  int32_t shift;       // halves: vectors from one half of the rotated part to the other, R / 16
  int64_t stride4;     // table stride of a stream in float4
  uint32_t flip;       // sign bit: the transpose
};

// Coefficients of a thread's vector.  Interleaved: of its four pairs, in the first halves of c and s.  Halves: of the 8
// pairs that its dims belong to, s with the sign with which the partner's value comes in; y = x * c + partner * s
// then rounds as x * c - partner * |s| does.
template <bool kHalf>
struct Coefficients {
  float c[kHalf ? 8 : 4], s[kHalf ? 8 : 4];
};
// `load(i)`: cosines and sines of quad i of the table's row.
template <bool kHalf, typename Load>
__device__ __forceinline__ Coefficients<kHalf> coefficients(const RotaryPlace& p, int u, const Load& load) {
  Coefficients<kHalf> k;
  constexpr int kQuads = kHalf ? 2 : 1;
  const bool second = kHalf && u >= p.shift;
  const int at = kHalf ? 2 * (second ? u - p.shift : u) : u;
#pragma unroll
  for (int i = 0; i < kQuads; ++i) {
    float4 c, s;
    load(at + i, c, s);
    k.c[4 * i] = c.x, k.c[4 * i + 1] = c.y, k.c[4 * i + 2] = c.z, k.c[4 * i + 3] = c.w;
    k.s[4 * i] = s.x, k.s[4 * i + 1] = s.y, k.s[4 * i + 2] = s.z, k.s[4 * i + 3] = s.w;
  }
  const uint32_t flip = p.flip ^ (kHalf && !second ? 0x80000000u : 0u);
#pragma unroll
  for (int i = 0; i < 4 * kQuads; ++i) k.s[i] = __uint_as_float(__float_as_uint(k.s[i]) ^ flip);
  return k;
}
template <bool kHalf>
__device__ __forceinline__ Coefficients<kHalf> load_coefficients(const RotaryPlace& p, const float4* cos_t, const float4* sin_t,
                                                                 int64_t row, int u) {
  return coefficients<kHalf>(p, u, [&](int i, float4& c, float4& s) {
    c = __ldca(cos_t + row + i);
    s = __ldca(sin_t + row + i);
  });
}

__device__ __forceinline__ void unpack8(uint4 x, float* f) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 y = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

// y = rotation of x, products and sums rounded to float32 one by one.  Halves: all lanes of the warp come here, and
// `from` is the lane with the other half of the pairs; its values are passed as the bf16 pairs that they still are.
__device__ __forceinline__ void rotate_pairs(const float* x, const Coefficients<false>& k, float* y) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __fsub_rn(__fmul_rn(x[2 * i], k.c[i]), __fmul_rn(x[2 * i + 1], k.s[i]));
    y[2 * i + 1] = __fadd_rn(__fmul_rn(x[2 * i], k.s[i]), __fmul_rn(x[2 * i + 1], k.c[i]));
  }
}
// (Products two at a time.  Sums are not: a packed product and a packed sum are contracted to one rounding, .rn or not.)
__device__ __forceinline__ void rotate_halves(const float* x, const float* other, const Coefficients<true>& k, float* y) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint64_t a = ptx::mul_f32x2(ptx::pack_f32x2(x[i], x[i + 1]), ptx::pack_f32x2(k.c[i], k.c[i + 1]));
    const uint64_t b = ptx::mul_f32x2(ptx::pack_f32x2(other[i], other[i + 1]), ptx::pack_f32x2(k.s[i], k.s[i + 1]));
    float a0, a1, b0, b1;
    ptx::unpack_f32x2(a, a0, a1);
    ptx::unpack_f32x2(b, b0, b1);
    y[i] = __fadd_rn(a0, b0);
    y[i + 1] = __fadd_rn(a1, b1);
  }
}
__device__ __forceinline__ uint4 shuffle16(uint4 x, int from) {
  return make_uint4(__shfl_sync(0xFFFFFFFFu, x.x, from), __shfl_sync(0xFFFFFFFFu, x.y, from),
                    __shfl_sync(0xFFFFFFFFu, x.z, from), __shfl_sync(0xFFFFFFFFu, x.w, from));
}
__device__ __forceinline__ int partner_lane(const RotaryPlace& p, int lane, int u, bool rotated) {
  return rotated ? (u >= p.shift ? lane - p.shift : lane + p.shift) : lane;
}

// --------------------------------------------------------------------------
// Rotation of one tensor, HBM bound.  A thread has the same place of up to kApplyHeads heads of a token: it fetches
// its coefficients once, and its loads are in flight together.  Halves: the two halves of a pair are 8 vectors or less
// apart, in the same 16 lanes, and meet by a shuffle, so that every element is read once and in place works.  40
// heads x 10800 tokens, halves of the first 96 dims (225 MB): 37.2 us, 6.06 TB/s, 0.92 of the measured copy rate.
// --------------------------------------------------------------------------
constexpr int kApplyHeads = 4;

struct ApplyParams {
  RotaryPlace place;
  int64_t vec_per_stream;      // L * Hn * 16
  int64_t threads_per_stream;  // L * width
  int32_t width;               // threads of a token: 16 * ceil(Hn / kApplyHeads)
  int32_t vec_per_token;       // Hn * 16
  int* status;
  int64_t extent;
};

template <bool kHalf>
__global__ void __launch_bounds__(256)
rotary_apply_kernel(const ApplyParams p, const uint4* x_in, const float4* cos_t, const float4* sin_t, uint4* y_out) {
  grid_launch_next();
  const int64_t id = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int b = blockIdx.y;
  const bool live = id < p.threads_per_stream;
  const int64_t n = id / p.width;
  const int i0 = static_cast<int>(id - n * p.width), u = i0 & 15;
  const bool rotated = u < p.place.rows;
  const int behind = grid_wait();
  const int64_t base = static_cast<int64_t>(b) * p.vec_per_stream + n * p.vec_per_token + behind;
  uint4 x[kApplyHeads];
#pragma unroll
  for (int j = 0; j < kApplyHeads; ++j) {
    const int i = i0 + j * p.width;
    x[j] = make_uint4(0, 0, 0, 0);
    if (live && i < p.vec_per_token) x[j] = __ldcs(x_in + base + i);
  }
  Coefficients<kHalf> k = {};
  if (live && rotated) k = load_coefficients<kHalf>(p.place, cos_t, sin_t, b * p.place.stride4 + n * p.place.rows + behind, u);
  const int from = partner_lane(p.place, threadIdx.x & 31, u, rotated);
#pragma unroll
  for (int j = 0; j < kApplyHeads; ++j) {
    const int i = i0 + j * p.width;
    float f[8], y[8];
    unpack8(x[j], f);
    if constexpr (kHalf) {
      float other[8];
      unpack8(shuffle16(x[j], from), other);
      rotate_halves(f, other, k, y);
    } else {
      rotate_pairs(f, k, y);
    }
    if (live && i < p.vec_per_token) UNSTEP_STORE(y_out, base + i, p.extent, rotated ? pack8(y) : x[j], p.status);
  }
}

// --------------------------------------------------------------------------
// Append into the 8-bit cache.  `width` threads have a token: a thread the same place of kU heads in q, k and v, `width`
// vectors apart (kWide: more than that, kU at a time); a block has one token with the norm, whose sum meets in shared memory, else
// `tokens` of them.  Four neighbouring threads hold a block of 32 dims and find its largest magnitude with two shuffles.
//
// HBM bound without the norm: four streams of 4680 tokens x 12 heads (299 MB) 50.2 us, 6.0 TB/s, 0.91 of the measured copy rate.
// With the norm a block's chain bounds it (loads, sum over
// the block, gains, rotation, conversion; 4.7 long-scoreboard stalls an issue): one stream (75 MB) 20.1 us, 3.7 TB/s.  Halves
// behind the norm pass 8 floats for each vector of q and of k from lane to lane, and are the one form that spills: two heads a
// thread have 64 registers (four blocks of 256 threads) and store 28 and load 48 bytes a thread.  There (halves)
// 10 blocks of 96 threads an SM 20.3, 8 21.3, 11 and 12 (which spill more) 22.6, 192 threads 22.9, 64 21.9; without the gains 16.0; the
// table's row in registers from the start, as without the norm, 22.3; v behind the sum 22.9.  Gains brought to shared memory
// meanwhile: 19.3, but interleaved 18.4 instead of 17.8 and 10800 tokens 42.5 instead of 41.4; blocks that go through the
// tokens with the next one's vectors on their way 34.  With four heads a thread at least two blocks an SM (128
// registers) for interleaved pairs, 40 heads 61.1 -> 54.5, 48 82.8 -> 65.7, and not for halves, which then spill (64.6 -> 67.5).
// --------------------------------------------------------------------------
struct Append8Params {
  RotaryPlace place;
  int32_t L, T, C, S, vec_per_token, width, tokens;
  int32_t frame0;                  // with the norm: first frame of this launch inside the chunk
  int64_t vec_per_stream;          // L * Hn * 16
  int64_t cache_vec_per_stream;    // (S + C) * T * Hn * 16 vectors of 8 codes
  float eps, channels;             // channels: Hn * 128
  int32_t start[kMaxStreamsPerLaunch];
  int32_t prefetch;                // 1: the first blocks prefetch their inputs to L2
  int* status;                     // extents of q_out (16-byte vectors), codes (8-byte vectors) and scale bytes
  int64_t extent_act, extent_code, extent_scale;
};

__device__ __forceinline__ float warp_sum32(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}
// Sum of the squares of a vector, added to the two halves of `acc`.
__device__ __forceinline__ uint64_t squares32(uint4 x, uint64_t acc) {
  float f[8];
  unpack8(x, f);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint64_t v = ptx::pack_f32x2(f[i], f[i + 1]);
    acc = ptx::fma_f32x2(v, v, acc);
  }
  return acc;
}
// f * r * gain, each product rounded to float32
__device__ __forceinline__ void gain8(float* f, float r, const float4* gain, int vi) {
  const float4 g0 = __ldca(gain + 2 * vi), g1 = __ldca(gain + 2 * vi + 1);
  const float g[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
  const uint64_t r2 = ptx::pack_f32x2(r, r);
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    ptx::unpack_f32x2(ptx::mul_f32x2(ptx::mul_f32x2(ptx::pack_f32x2(f[i], f[i + 1]), r2), ptx::pack_f32x2(g[i], g[i + 1])), f[i], f[i + 1]);
}

template <int kU, bool kHalf, bool kNorm, bool kWide>
__global__ void __launch_bounds__(256, kNorm && kU <= 2 ? 4 : kNorm && !kHalf && !kWide ? 2 : 1)
rotary_kv_append_q8_kernel(const Append8Params p, const uint4* q_in, const uint4* k_in, const uint4* v_in,
                           const float4* gain_q, const float4* gain_k, const float4* cos_t, const float4* sin_t,
                           uint4* q_out, uint2* cache_k, uint8_t* scale_k, uint2* cache_v, uint8_t* scale_v) {
  __shared__ float part[2][8];
  __shared__ float4 table[2][16];   // with the norm: the token's row, which is used behind the sum
  grid_launch_next();
  const int b = blockIdx.z;
  int n, f, t, i0 = threadIdx.x;
  bool live = true;
  if (kNorm) {
    t = blockIdx.x;
    f = p.frame0 + blockIdx.y;
    n = f * p.T + t;
  } else {
    const int token = i0 / p.width;   // one more than there are where the block is filled up to whole warps
    n = blockIdx.x * p.tokens + token;
    i0 -= token * p.width;
    live = token < p.tokens && n < p.L;
    f = n / p.T;
    t = n - f * p.T;
  }
  const int frame = p.start[b] + f;
  const int slot = frame < p.S ? frame : p.S + (frame - p.S) % p.C;
  const int u = i0 & 15;
  const bool rotated = u < p.place.rows;
  if (kNorm && p.prefetch && threadIdx.x == 0 && (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x < kEarlyBlocks) {
    const int64_t first = static_cast<int64_t>(b) * p.vec_per_stream + static_cast<int64_t>(n) * p.vec_per_token;
    prefetch_l2(q_in + first, p.vec_per_token);
    prefetch_l2(k_in + first, p.vec_per_token);
    prefetch_l2(v_in + first, p.vec_per_token);
  }
  const int behind = grid_wait();
  i0 += behind;   // every load below goes by i0
  const int64_t in_base = static_cast<int64_t>(b) * p.vec_per_stream + static_cast<int64_t>(n) * p.vec_per_token;
  const int64_t cache_base = static_cast<int64_t>(b) * p.cache_vec_per_stream +
                             (static_cast<int64_t>(slot) * p.T + t) * p.vec_per_token;
  const int from = partner_lane(p.place, threadIdx.x & 31, u, rotated);
  const int step = p.width * kU;
  const uint4 zero = make_uint4(0, 0, 0, 0);

  uint4 xq[kU], xk[kU], xv[kU];
  auto load = [&](int at) {
#pragma unroll
    for (int j = 0; j < kU; ++j) {
      const int i = at + j * p.width;
      const bool mine = live && i < p.vec_per_token;
      xq[j] = mine ? q_in[in_base + i] : zero;   // plain load: q_out may be the same buffer
      xk[j] = mine ? __ldca(k_in + in_base + i) : zero;
      xv[j] = mine ? __ldcs(v_in + in_base + i) : zero;
    }
  };
  auto put = [&](const float* y, int i, uint2* cache, uint8_t* scale) {
    uint32_t byte;
    const uint2 codes = q8::quantise8(y, &byte);
    if (live && i < p.vec_per_token) {
      const int64_t dst = cache_base + i;
      UNSTEP_STORE(cache, dst, p.extent_code, codes, p.status);
      // a word of the head's four bytes from one lane costs two more shuffles: 62 instead of 58 us for four streams
      if ((u & 3) == 0) UNSTEP_STORE(scale, dst >> 2, p.extent_scale, static_cast<uint8_t>(byte), p.status);
    }
  };
  float rq = 1.f, rk = 1.f;
  load(i0);
  Coefficients<kHalf> k = {};
  const int64_t table_row = b * p.place.stride4 + static_cast<int64_t>(n) * p.place.rows + behind;
  if (kNorm) {
    if (threadIdx.x < 32 && u < p.place.rows) table[threadIdx.x >> 4][u] = __ldca((threadIdx.x < 16 ? cos_t : sin_t) + table_row + u);
    // v does without the sum, and its registers are free behind this
    if (!kWide) {
#pragma unroll
      for (int j = 0; j < kU; ++j) {
        float y[8];
        unpack8(xv[j], y);
        put(y, i0 + j * p.width, cache_v, scale_v);
      }
    }
    uint64_t sq2 = 0, sk2 = 0;
    for (int at = i0;;) {
#pragma unroll
      for (int j = 0; j < kU; ++j) {
        sq2 = squares32(xq[j], sq2);
        sk2 = squares32(xk[j], sk2);
      }
      at += step;
      if (!kWide || at - i0 >= p.vec_per_token) break;
      load(at);
    }
    float a, d;
    ptx::unpack_f32x2(sq2, a, d);
    const float sq = warp_sum32(a + d);
    ptx::unpack_f32x2(sk2, a, d);
    const float sk = warp_sum32(a + d);
    if ((threadIdx.x & 31) == 0) {
      part[0][threadIdx.x >> 5] = sq;
      part[1][threadIdx.x >> 5] = sk;
    }
    __syncthreads();
    // even lanes finish q, odd lanes k: one division and one root per warp
    float sum = 0.f;
    for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) sum += part[threadIdx.x & 1][w];
    const float r = __frcp_rn(__fsqrt_rn(__fadd_rn(__fdiv_rn(sum, p.channels), p.eps)));
    rq = __shfl_sync(0xFFFFFFFFu, r, 0);
    rk = __shfl_sync(0xFFFFFFFFu, r, 1);
    if (kWide) load(i0);
    if (rotated)
      k = coefficients<kHalf>(p.place, u, [&](int i, float4& c, float4& s) {
        c = table[0][i];
        s = table[1][i];
      });
  } else if (live && rotated) {
    k = load_coefficients<kHalf>(p.place, cos_t, sin_t, table_row, u);
  }
  // float32 values behind the norm and the rotation
  auto turn = [&](uint4 x, float r, const float4* gain, int vi, float* y) {
    float v[8];
    unpack8(x, v);
    if (kNorm && vi < p.vec_per_token) gain8(v, r, gain, vi);
    if constexpr (kHalf) {
      float other[8];
      if (kNorm) {
#pragma unroll
        for (int e = 0; e < 8; ++e) other[e] = __shfl_sync(0xFFFFFFFFu, v[e], from);
      } else {
        unpack8(shuffle16(x, from), other);
      }
      rotate_halves(v, other, k, y);
    } else {
      rotate_pairs(v, k, y);
    }
    if (!rotated) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = v[e];
    }
  };
  for (int at = i0;;) {
#pragma unroll
    for (int j = 0; j < kU; ++j) {
      const int i = at + j * p.width;
      float y[8];
      turn(xq[j], rq, gain_q, i, y);
      if (live && i < p.vec_per_token) UNSTEP_STORE(q_out, in_base + i, p.extent_act, pack8(y), p.status);
      turn(xk[j], rk, gain_k, i, y);
      put(y, i, cache_k, scale_k);
      if (!kNorm || kWide) {
        unpack8(xv[j], y);
        put(y, i, cache_v, scale_v);
      }
    }
    at += step;
    if (!kWide || at - i0 >= p.vec_per_token) break;
    load(at);
  }
}

// --------------------------------------------------------------------------
// Frames of the 8-bit cache as bf16, HBM bound.  A thread decodes 16 codes of k and of v; a block stays in one frame, so
// that nothing is divided.  12 frames of 3600 tokens x 40 heads (1.34 GB): 230 us, 5.8 TB/s, 0.89 of the measured copy rate.
// --------------------------------------------------------------------------
struct Read8Params {
  int32_t C, S, n_frames, frame0;      // frame0: first frame of this launch inside the read
  int64_t vec_per_frame;               // T * Hn * 8 vectors of 16 codes
  int64_t cache_vec_per_stream;
  int32_t first[kMaxStreamsPerLaunch];
  int* status;
  int64_t extent;                      // 16-byte vectors of an output
};

__device__ __forceinline__ void store_decoded(uint4* out, int64_t dst, int64_t extent, uint4 x, uint32_t byte, int* status) {
  const uint32_t f1 = q8::factor1(byte);
  uint4 lo = q8::decode8(x.x, x.y, f1), hi = q8::decode8(x.z, x.w, f1);
  if (!q8::one_factor(byte)) {
    const uint32_t f2 = q8::factor2(byte);
    lo = q8::mul8(lo, f2);
    hi = q8::mul8(hi, f2);
  }
  UNSTEP_STORE(out, dst, extent, lo, status);
  UNSTEP_STORE(out, dst + 1, extent, hi, status);
}

__global__ void __launch_bounds__(256)
kv_read_q8_kernel(const Read8Params p, const uint4* cache_k, const uint8_t* scale_k, const uint4* cache_v,
                  const uint8_t* scale_v, uint4* out_k, uint4* out_v) {
  grid_launch_next();
  const int64_t v = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int behind = grid_wait();
  if (v >= p.vec_per_frame) return;
  const int b = blockIdx.z, f = p.frame0 + blockIdx.y;
  const int frame = p.first[b] + f;
  const int slot = frame < p.S ? frame : p.S + (frame - p.S) % p.C;
  const int64_t src = b * p.cache_vec_per_stream + slot * p.vec_per_frame + v + behind;
  const uint4 xk = __ldcs(cache_k + src), xv = __ldcs(cache_v + src);
  const uint32_t ek = __ldca(scale_k + (src >> 1)), ev = __ldca(scale_v + (src >> 1));
  const int64_t dst = 2 * ((static_cast<int64_t>(b) * p.n_frames + f) * p.vec_per_frame + v);
  store_decoded(out_k, dst, p.extent, xk, ek, p.status);
  store_decoded(out_v, dst, p.extent, xv, ev, p.status);
}

static RotaryPlace rotary_place(const unstep_shape_t* s, int64_t table_stream_stride, bool transposed) {
  const int32_t rotated = s->band_t + s->band_h + s->band_w;
  RotaryPlace p;
  p.rows = rotated / 8;
  p.shift = rotated / 16;
  p.stride4 = table_stream_stride / 4;
  p.flip = transposed ? 0x80000000u : 0u;
  return p;
}

static bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace unstep

using namespace unstep;

extern "C" int unstep_rotary_apply(const unstep_shape_t* shape, const unstep_rope_t* rope, int32_t transposed,
                                   const void* x, const float* cos, const float* sin, int64_t table_stream_stride,
                                   void* y, void* cuda_stream) {
  int rc = check_shape(shape, false, true);
  if (rc == UNSTEP_OK) rc = check_rope(rope);
  if (rc != UNSTEP_OK) return rc;
  if (shape->batch <= 0 || shape->batch > (1 << 20) || shape->heads <= 0 || shape->heads > 4096) return UNSTEP_ERR_INVALID_ARG;
  if (transposed < 0 || transposed > 1) return UNSTEP_ERR_INVALID_ARG;
  const void* ptrs[] = {x, cos, sin, y};
  for (const void* ptr : ptrs)
    if (ptr == nullptr || !aligned16(ptr)) return UNSTEP_ERR_INVALID_ARG;
  if (table_stream_stride < 0 || (table_stream_stride & 3)) return UNSTEP_ERR_INVALID_ARG;
  rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  const int64_t L = static_cast<int64_t>(shape->grid_h) * shape->grid_w * shape->chunk_frames;
  ApplyParams p;
  p.place = rotary_place(shape, table_stream_stride, transposed != 0);
  p.vec_per_token = shape->heads * 16;
  p.width = 16 * ((shape->heads + kApplyHeads - 1) / kApplyHeads);
  p.vec_per_stream = L * p.vec_per_token;
  p.threads_per_stream = L * p.width;
  const int64_t blocks = (p.threads_per_stream + 255) / 256;
  if (blocks > INT32_MAX) return UNSTEP_ERR_INVALID_ARG;
  p.status = status_word();
  constexpr int kMaxStreams = 65535;
  for (int b0 = 0; b0 < shape->batch; b0 += kMaxStreams) {
    const int nb = shape->batch - b0 < kMaxStreams ? shape->batch - b0 : kMaxStreams;
    p.extent = nb * p.vec_per_stream;
    const int64_t off = b0 * p.vec_per_stream, tab = b0 * table_stream_stride;
    const cudaError_t err = launch_overlapped(
        true, rope->half ? rotary_apply_kernel<true> : rotary_apply_kernel<false>, dim3(static_cast<unsigned>(blocks), nb), 256,
        0, static_cast<cudaStream_t>(cuda_stream), p, static_cast<const uint4*>(x) + off,
        reinterpret_cast<const float4*>(cos + tab), reinterpret_cast<const float4*>(sin + tab), static_cast<uint4*>(y) + off);
    g_launches.fetch_add(1);
    if (err != cudaSuccess) return UNSTEP_ERR_CUDA;
  }
  return UNSTEP_OK;
}

namespace unstep {
typedef void (*Append8Kernel)(const Append8Params, const uint4*, const uint4*, const uint4*, const float4*, const float4*,
                              const float4*, const float4*, uint4*, uint2*, uint8_t*, uint2*, uint8_t*);
template <bool kHalf>
static Append8Kernel append8_kernel(bool norm, int per_thread, bool wide) {
  if (!norm) {
    if (wide) return rotary_kv_append_q8_kernel<4, kHalf, false, true>;
    switch (per_thread) {
      case 2: return rotary_kv_append_q8_kernel<2, kHalf, false, false>;
      case 3: return rotary_kv_append_q8_kernel<3, kHalf, false, false>;
      default: return rotary_kv_append_q8_kernel<4, kHalf, false, false>;
    }
  }
  if (wide) return rotary_kv_append_q8_kernel<4, kHalf, true, true>;
  switch (per_thread) {
    case 1: return rotary_kv_append_q8_kernel<1, kHalf, true, false>;
    case 2: return rotary_kv_append_q8_kernel<2, kHalf, true, false>;
    default: return rotary_kv_append_q8_kernel<4, kHalf, true, false>;
  }
}
}  // namespace unstep

extern "C" int unstep_rotary_kv_append_q8(const unstep_shape_t* shape, const unstep_rope_t* rope, int32_t sink_frames,
                                          const int32_t* start_frame, const void* q_in, const void* k_in,
                                          const void* v_in, const float* gain_q, const float* gain_k, float eps,
                                          const float* cos, const float* sin, int64_t table_stream_stride, void* q_out,
                                          void* cache_k, void* scale_k, void* cache_v, void* scale_v, void* cuda_stream) {
  int rc = check_shape(shape, true, true);
  if (rc == UNSTEP_OK) rc = check_rope(rope);
  if (rc != UNSTEP_OK) return rc;
  const bool norm = gain_q != nullptr;
  if (sink_frames < 0 || sink_frames > 4096 || norm != (gain_k != nullptr) || (norm && !(eps >= 0.f)))
    return UNSTEP_ERR_INVALID_ARG;
  const void* ptrs[] = {q_in, k_in, v_in, cos, sin, q_out, cache_k, cache_v};
  for (const void* ptr : ptrs)
    if (ptr == nullptr || !aligned16(ptr)) return UNSTEP_ERR_INVALID_ARG;
  if (start_frame == nullptr || scale_k == nullptr || scale_v == nullptr || !aligned4(scale_k) || !aligned4(scale_v) ||
      !aligned16(gain_q) || !aligned16(gain_k))
    return UNSTEP_ERR_INVALID_ARG;
  if (table_stream_stride < 0 || (table_stream_stride & 3)) return UNSTEP_ERR_INVALID_ARG;
  for (int b = 0; b < shape->batch; ++b)
    if (start_frame[b] < 0 || start_frame[b] > INT32_MAX - shape->chunk_frames) return UNSTEP_ERR_INVALID_ARG;
  rc = check_device();
  if (rc != UNSTEP_OK) return rc;

  const int64_t T = static_cast<int64_t>(shape->grid_h) * shape->grid_w;
  const int64_t L = T * shape->chunk_frames;
  Append8Params p;
  p.place = rotary_place(shape, table_stream_stride, false);
  p.L = static_cast<int32_t>(L);
  p.T = static_cast<int32_t>(T);
  p.C = shape->ring_frames;
  p.S = sink_frames;
  p.vec_per_token = shape->heads * 16;
  p.vec_per_stream = L * p.vec_per_token;
  p.cache_vec_per_stream = (static_cast<int64_t>(shape->ring_frames) + sink_frames) * T * p.vec_per_token;
  p.eps = eps;
  p.channels = static_cast<float>(shape->heads * kHeadDim);
  p.status = status_word();
  int threads = 256, per_thread = 1;
  bool wide = false;
  int64_t blocks;
  if (norm) {
    // Two heads a thread while a block has the threads: all loads of a token are in flight with 64 registers.  Halves /
    // interleaved, 4680 tokens, us, two : three or four of them: 14 heads 24.5 / 20.9 : 27.9 / 26.2, 20 33.2 / 29.2 : 38.3 / 36.4,
    // 32 49.2 / 42.7 : 51.4 / 47.6; with 36 in blocks of 288 threads 84.5 / 70.5 : 62.3 / 59.3.
    per_thread = p.vec_per_token <= 96 ? 1 : p.vec_per_token <= 512 ? 2 : 4;
    threads = (((p.vec_per_token + per_thread - 1) / per_thread) + 31) & ~31;
    wide = threads > 256;
    if (wide) threads = 256;
    p.width = threads;
    p.tokens = 1;
    blocks = T;
  } else {
    // Three heads a thread, or two (of few heads, four) where that leaves fewer threads without work; four where a block
    // would not have the threads.  Halves / interleaved, 4680 tokens, us, one : two : three : four of them: 4 heads 5.8 / 5.0 :
    // 5.7 / 4.3 : 6.6 / 5.8 : 4.6 / 4.3, 7 9.4 / 8.6 : 9.2 / 7.8 : 10.2 / 9.4 : 8.5 / 8.3, 12 16.4 / 15.4 : 15.7 / 14.6 : 15.1 / 14.6 :
    // 17.8 / 17.7, 14 two 17.7 / 17.0, three 19.0 / 18.2, four 20.7 / 20.3, 20 24.8 / 22.6, 25.4 / 22.2 and 27.5 / 27.0.
    // 40 heads three : four 46.4 / 40.2 : 43.4 / 42.7: the layouts differ there, and the rule goes by their sum.
    wide = shape->heads > 64;
    per_thread = shape->heads > 48 ? 4 : 3;
    auto places = [&](int u) { return (shape->heads + u - 1) / u * u; };
    if (shape->heads <= 8 && places(4) < places(per_thread)) per_thread = 4;
    if (shape->heads <= 32 && places(2) < places(per_thread)) per_thread = 2;
    p.width = wide ? 256 : 16 * ((shape->heads + per_thread - 1) / per_thread);
    p.tokens = 256 / p.width;
    threads = (p.width * p.tokens + 31) & ~31;
    blocks = (L + p.tokens - 1) / p.tokens;
  }
  if (blocks > INT32_MAX) return UNSTEP_ERR_INVALID_ARG;
  const Append8Kernel kernel = rope->half ? append8_kernel<true>(norm, per_thread, wide) : append8_kernel<false>(norm, per_thread, wide);
  for (int b0 = 0; b0 < shape->batch; b0 += kMaxStreamsPerLaunch) {
    const int nb = shape->batch - b0 < kMaxStreamsPerLaunch ? shape->batch - b0 : kMaxStreamsPerLaunch;
    for (int i = 0; i < nb; ++i) p.start[i] = start_frame[b0 + i];
    p.extent_act = nb * p.vec_per_stream;
    p.prefetch = 3 * p.extent_act <= kPrefetchVectors;
    p.extent_code = nb * p.cache_vec_per_stream;
    p.extent_scale = p.extent_code / 4;
    const int64_t in = b0 * p.vec_per_stream, cache = b0 * p.cache_vec_per_stream, tab = b0 * table_stream_stride;
    constexpr int kMaxFrames = 65535;
    for (p.frame0 = 0; p.frame0 < shape->chunk_frames; p.frame0 += kMaxFrames) {
      const int left = shape->chunk_frames - p.frame0;
      const int frames = norm ? (left < kMaxFrames ? left : kMaxFrames) : 1;
      const cudaError_t err = launch_overlapped(
          true, kernel, dim3(static_cast<unsigned>(blocks), frames, nb), threads, 0, static_cast<cudaStream_t>(cuda_stream), p,
          static_cast<const uint4*>(q_in) + in, static_cast<const uint4*>(k_in) + in, static_cast<const uint4*>(v_in) + in,
          reinterpret_cast<const float4*>(gain_q), reinterpret_cast<const float4*>(gain_k),
          reinterpret_cast<const float4*>(cos + tab), reinterpret_cast<const float4*>(sin + tab), static_cast<uint4*>(q_out) + in,
          static_cast<uint2*>(cache_k) + cache, static_cast<uint8_t*>(scale_k) + cache / 4, static_cast<uint2*>(cache_v) + cache,
          static_cast<uint8_t*>(scale_v) + cache / 4);
      g_launches.fetch_add(1);
      if (err != cudaSuccess) return UNSTEP_ERR_CUDA;
      if (!norm || left <= kMaxFrames) break;
    }
  }
  return UNSTEP_OK;
}

extern "C" int unstep_kv_read_q8(const unstep_shape_t* shape, int32_t sink_frames, const int32_t* first_frame,
                                 int32_t n_frames, const void* cache_k, const void* scale_k, const void* cache_v,
                                 const void* scale_v, void* out_k, void* out_v, void* cuda_stream) {
  int rc = check_shape(shape, true, true);
  if (rc != UNSTEP_OK) return rc;
  if (sink_frames < 0 || sink_frames > 4096 || n_frames < 1 || first_frame == nullptr) return UNSTEP_ERR_INVALID_ARG;
  const void* ptrs[] = {cache_k, cache_v, out_k, out_v};
  for (const void* ptr : ptrs)
    if (ptr == nullptr || !aligned16(ptr)) return UNSTEP_ERR_INVALID_ARG;
  if (scale_k == nullptr || scale_v == nullptr || !aligned4(scale_k) || !aligned4(scale_v)) return UNSTEP_ERR_INVALID_ARG;
  for (int b = 0; b < shape->batch; ++b) {
    if (first_frame[b] < 0 || first_frame[b] > INT32_MAX - n_frames) return UNSTEP_ERR_INVALID_ARG;
    const int32_t ring0 = first_frame[b] > sink_frames ? first_frame[b] : sink_frames;   // first one behind the sink
    if (first_frame[b] + n_frames - ring0 > shape->ring_frames) return UNSTEP_ERR_INVALID_ARG;
  }
  rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  const int64_t T = static_cast<int64_t>(shape->grid_h) * shape->grid_w;
  Read8Params p;
  p.C = shape->ring_frames;
  p.S = sink_frames;
  p.n_frames = n_frames;
  p.vec_per_frame = T * shape->heads * 8;
  p.cache_vec_per_stream = (static_cast<int64_t>(shape->ring_frames) + sink_frames) * p.vec_per_frame;
  p.status = status_word();
  const int64_t blocks = (p.vec_per_frame + 255) / 256;
  if (blocks > INT32_MAX) return UNSTEP_ERR_INVALID_ARG;
  constexpr int kMaxFrames = 65535;
  for (int b0 = 0; b0 < shape->batch; b0 += kMaxStreamsPerLaunch) {
    const int nb = shape->batch - b0 < kMaxStreamsPerLaunch ? shape->batch - b0 : kMaxStreamsPerLaunch;
    for (int i = 0; i < nb; ++i) p.first[i] = first_frame[b0 + i];
    const int64_t cache = b0 * p.cache_vec_per_stream;
    const int64_t out = 2 * static_cast<int64_t>(b0) * n_frames * p.vec_per_frame;
    p.extent = 2 * static_cast<int64_t>(nb) * n_frames * p.vec_per_frame;
    for (p.frame0 = 0; p.frame0 < n_frames; p.frame0 += kMaxFrames) {
      const int nf = n_frames - p.frame0 < kMaxFrames ? n_frames - p.frame0 : kMaxFrames;
      const cudaError_t err = launch_overlapped(
          true, kv_read_q8_kernel, dim3(static_cast<unsigned>(blocks), nf, nb), 256, 0, static_cast<cudaStream_t>(cuda_stream),
          p, static_cast<const uint4*>(cache_k) + cache, static_cast<const uint8_t*>(scale_k) + cache / 2,
          static_cast<const uint4*>(cache_v) + cache, static_cast<const uint8_t*>(scale_v) + cache / 2,
          static_cast<uint4*>(out_k) + out, static_cast<uint4*>(out_v) + out);
      g_launches.fetch_add(1);
      if (err != cudaSuccess) return UNSTEP_ERR_CUDA;
      if (n_frames - p.frame0 <= kMaxFrames) break;
    }
  }
  return UNSTEP_OK;
}
