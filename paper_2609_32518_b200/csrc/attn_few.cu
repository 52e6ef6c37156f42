// Attention of few queries, or over few keys, of an 8-bit cache (sm_100a): single tokens, and launches that would be over
// before the kernel with tiles has its first one done.
//
// DRAM bound: every cached key and value is read once, and a query tile of the tensor-memory kernel would be next to empty,
// while it waits for tiles to be decoded into shared memory.  Here a warp takes 16 keys at a time straight from global memory
// into the operands of warp-level matrix products (mma.sync, m16n8k16, bf16 with float32 sums):
//     S^T = K Q^T   16 keys x 8 queries    O^T = V^T P^T   16 dims x 8 queries
// The dims of K, summed over, and those of V, independent of each other, may come in any order, so every thread
// reads 16 or 32 neighbouring codes of a row and needs no exchange; P^T turns from result to operand by a
// transpose of its 8 x 8 blocks.  Each warp has its own running maximum and sum; the warps of a block merge through
// shared memory, the blocks of an item (stream, head, 8 queries) through the scratch: the one that is done last reads the
// others' parts, in part order, so the result does not depend on which one that is.  Streams of different length get
// different numbers of blocks, which clusters could not have.
//
// Measured: one token each of three streams, 12 heads, 4096, 1235 and 4096 keys (30 MB) 13.0 us, of which 3.4 are what a call with next
// to no keys takes; 148 heads x 16384 keys (640 MB) 140 us, 4.6 TB/s; one head x 16384 keys 8.2 us.  The kernel with tiles took
// 29.7 for the first.  Bound by the instructions of a step (16 keys, a warp; 16 warps an SM by 128 registers) and the
// waits between them: 2.1 us, with the ALU pipe, which issues every other cycle, half busy.  The second of these cases with
// steps three ahead in shared memory by cp.async 212 instead of 155 us (more instructions than wait), with the maximum of
// every step by shuffles 155 instead of 151, with the branch for the second factor inside the loops 157 instead of 140, with two
// sums for S 142.  16 queries a warp, which would read keys half as often: 241 registers, one block an SM, slower than tiles
// from 9 queries on; groups of 8 find the keys in L2.  K as fp16, for which two codes are one instruction and a block's scale
// comes behind the products, but whose loads are 8 instead of 32 bytes: 14.1 instead of 12.7 for one token each, the second 137.
#include <cuda_bf16.h>

#include "attn_sched.h"
#include "common.h"
#include "ptx.cuh"
#include "quant.cuh"

namespace unstep {

using namespace ptx;

constexpr int kFewThreads = 32 * kFewWarps;
constexpr int kFewParts = 64;                   // most blocks of an item: two for each lane of a warp that merges them
constexpr float kFewJump = 57.f;                // as far (log2) a score may be above the reference, as in attn.cu

struct FewParams {
  int32_t Hn, L, groups, n_streams;             // groups of kFewQueries queries
  int64_t cache_rows;                           // rows of a stream's cache
  float scale_log2e;
  float* part;                                  // scratch: part_floats for every block
  int* counters;                                // scratch: arrivals per item, zero between launches
  int* status;
  int64_t extent_out, extent_part, extent_counters;   // 4-byte words of `out`, floats of `part`, ints of `counters`
  int32_t parts[kMaxStreamsPerLaunch], block0[kMaxStreamsPerLaunch];   // blocks of an item of a stream, its first block
  int32_t run_row0[kMaxStreamsPerLaunch][3], run_end[kMaxStreamsPerLaunch][3];   // rows of the runs, added up
};

struct Yes {
  __device__ constexpr operator bool() const { return true; }
};
struct No {
  __device__ constexpr operator bool() const { return false; }
};

// D (16 x 8) += A (16 x 16) B (16 x 8)
__device__ __forceinline__ void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Four codes as bf16 pairs, (0, 2) in x and (1, 3) in y, of 2^-120 times their values: without the bytes of q8::spread4
// brought back in order, which is the caller's to choose here.
__device__ __forceinline__ uint2 spread_pairs(uint32_t w) {
  return make_uint2(((w << 8) & 0x80008000u) | ((w << 4) & 0x07F007F0u), (w & 0x80008000u) | ((w >> 4) & 0x07F007F0u));
}
// The multiplier of q8::factor1, for scale bytes up to 134.
__device__ __forceinline__ uint32_t factor_small(uint32_t byte) { return byte * 0x00800080u + 120u * 0x00800080u; }

// What a warp leaves in shared memory: O as [query][dim], then (m, l).
constexpr int kFewWarpBytes = kFewQueries * (kHeadDim + 2) * static_cast<int>(sizeof(float));
// A block's part in the scratch: O as [query][dim], then (m, l) as [query].
constexpr int kFewPartFloats = kFewQueries * kHeadDim + kFewQueries * 2;

// kWide: cache_k is 32-byte aligned.
template <bool kWide>
__global__ void __launch_bounds__(kFewThreads, kFewBlocks)
window_attn_few_kernel(const __grid_constant__ FewParams p, const uint4* q_rot, const uint4* cache_k, const uint8_t* scale_k,
                       const uint4* cache_v, const uint8_t* scale_v, uint32_t* out) {
  __shared__ __align__(16) uint8_t few_smem[kFewWarps * kFewWarpBytes];
  auto slab = [&](int w, int query) { return reinterpret_cast<float*>(few_smem + w * kFewWarpBytes) + query * kHeadDim; };
  auto slab_ml = [&](int w) { return reinterpret_cast<float2*>(slab(w, kFewQueries)); };
  __shared__ int last;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int block = static_cast<int>(blockIdx.x);
  int b = 0;
  while (b + 1 < p.n_streams && p.block0[b + 1] <= block) ++b;
  const int parts = p.parts[b], item = (block - p.block0[b]) / parts, part = block - p.block0[b] - item * parts;
  const int h = item / p.groups, query0 = kFewQueries * (item - h * p.groups), queries = min(kFewQueries, p.L - query0);
  const int end0 = p.run_end[b][0], end1 = p.run_end[b][1], keys = p.run_end[b][2];
  const int row0 = p.run_row0[b][0], row1 = p.run_row0[b][1] - end0, row2 = p.run_row0[b][2] - end1;
  const int steps = (keys + kFewKeys - 1) / kFewKeys;
  const int lo = static_cast<int>(static_cast<int64_t>(steps) * part / parts);
  const int hi = static_cast<int>(static_cast<int64_t>(steps) * (part + 1) / parts);
  // the row of key j in this stream's cache; keys behind the last are the last again, and masked
  auto row_of = [&](int j) {
    j = min(j, keys - 1);
    return static_cast<uint32_t>(j + (j < end0 ? row0 : (j < end1 ? row1 : row2)));
  };
  // from here on everything is read, at addresses that take the wait's 0 in (through a shuffle, so that they are
  // known to be the same in all lanes)
  const int64_t head = b * p.cache_rows * p.Hn + h + __shfl_sync(0xFFFFFFFFu, grid_wait(), 0);
  const uint4* const head_k = cache_k + head * 8;
  const uint4* const head_v = cache_v + head * 8;
  const uint8_t* const head_ek = scale_k + head * 4;
  const uint8_t* const head_ev = scale_v + head * 4;
  const uint4* const head_q = q_rot + ((b * (static_cast<int64_t>(p.L) - p.cache_rows) + query0) * p.Hn + head) * 16;
  const uint32_t row_codes = 8u * p.Hn, row_scales = 4u * p.Hn;

  // B of S^T: thread (g, c) has query g, dims 32 c .. in pairs (0, 2) and (1, 3) of four, as spread_pairs makes them
  uint32_t q[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint4 x = make_uint4(0, 0, 0, 0);
    if (g < queries) x = __ldca(head_q + static_cast<int64_t>(g) * p.Hn * 16 + 4 * c + i);
    q[4 * i] = __byte_perm(x.x, x.y, 0x5410), q[4 * i + 1] = __byte_perm(x.x, x.y, 0x7632);
    q[4 * i + 2] = __byte_perm(x.z, x.w, 0x5410), q[4 * i + 3] = __byte_perm(x.z, x.w, 0x7632);
  }
  float o[8][4];   // O^T: dims 16 g + 2 t and + 2 t + 1, queries 2 c and + 1
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int t = 0; t < 8; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;

  // codes of keys g, g + 8 (dims 32 c ..) and of keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9 (dims 16 g ..), a step ahead
  uint32_t xk[2][8];
  uint4 xv[4];
  uint32_t ek[2], ev[4];
  // A step whose keys lie in one run has its rows at fixed distances from the first one's; the others are looked up.
  const uint32_t off_k = (g * row_codes + 2 * c) * 16, off_v = (2 * c * row_codes + g) * 16;
  const uint32_t off_ek = g * row_scales + c, off_ev = 2 * c * row_scales + (g >> 1);
  auto plain = [&](int step) {
    const int j = step * kFewKeys, e = j + kFewKeys;
    return j >= end1 ? e <= keys : (j >= end0 ? e <= end1 : e <= end0);
  };
  auto load_row = [&](const void* from, uint32_t* x) {   // 32 codes
    if (kWide) {
      ld_global_32(from, x);
    } else {
      const uint4 a = __ldcs(static_cast<const uint4*>(from)), d = __ldcs(static_cast<const uint4*>(from) + 1);
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = d.x, x[5] = d.y, x[6] = d.z, x[7] = d.w;
    }
  };
  auto load_k = [&](int step) {
    if (__builtin_expect(plain(step), 1)) {
      const uint64_t r = row_of(step * kFewKeys);
      const char* const k0 = reinterpret_cast<const char*>(head_k + r * row_codes);
      const uint8_t* const e0 = head_ek + r * row_scales;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        load_row(k0 + (off_k + 8 * i * row_codes * 16), xk[i]);
        ek[i] = __ldca(e0 + (off_ek + 8 * i * row_scales));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint64_t r = row_of(step * kFewKeys + g + 8 * i);
        load_row(head_k + r * row_codes + 2 * c, xk[i]);
        ek[i] = __ldca(head_ek + r * row_scales + c);
      }
    }
  };
  auto load_v = [&](int step) {
    if (__builtin_expect(plain(step), 1)) {
      const uint64_t r = row_of(step * kFewKeys);
      const char* const v0 = reinterpret_cast<const char*>(head_v + r * row_codes);
      const uint8_t* const e0 = head_ev + r * row_scales;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        xv[i] = __ldcs(reinterpret_cast<const uint4*>(v0 + (off_v + ((i & 1) + 8 * (i >> 1)) * row_codes * 16)));
        ev[i] = __ldca(e0 + (off_ev + ((i & 1) + 8 * (i >> 1)) * row_scales));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint64_t r = row_of(step * kFewKeys + 2 * c + (i & 1) + 8 * (i >> 1));
        xv[i] = __ldcs(head_v + r * row_codes + g);
        ev[i] = __ldca(head_ev + r * row_scales + (g >> 1));
      }
    }
  };
  int step = lo + warp;
  bool first = true;
  if (step < hi) {
    load_k(step);
    load_v(step);
  }
#pragma unroll 1
  for (; step < hi; step += kFewWarps) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    // One factor up to a scale byte of 134, else 2^120 and another: two loops, as a branch in the one would keep the compiler
    // from interleaving its turns.
    auto scores = [&](auto two) {
      uint32_t f[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) f[i] = two ? q8::factor1(ek[i]) : factor_small(ek[i]);
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        uint2 y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          y[i] = spread_pairs(xk[i][w]);
          y[i].x = q8::mul_bf16x2(y[i].x, f[i]);
          y[i].y = q8::mul_bf16x2(y[i].y, f[i]);
          if (two) {
            y[i].x = q8::mul_bf16x2(y[i].x, q8::factor2(ek[i]));
            y[i].y = q8::mul_bf16x2(y[i].y, q8::factor2(ek[i]));
          }
        }
        mma16816(s, y[0].x, y[1].x, y[0].y, y[1].y, q[2 * w], q[2 * w + 1]);
      }
    };
    if (__builtin_expect(__any_sync(0xFFFFFFFFu, max(ek[0], ek[1]) > 134u), 0)) scores(Yes{});
    else scores(No{});
    const int next = step + kFewWarps;
    if (next < hi) load_k(next);
    const int left = keys - step * kFewKeys;   // keys of this step
    if (g >= left) s[0] = s[1] = -INFINITY;
    if (g + 8 >= left) s[2] = s[3] = -INFINITY;
    bool jump = first;
#pragma unroll
    for (int e = 0; e < 2; ++e) jump = jump || (fmaxf(s[e], s[2 + e]) - m[e]) * p.scale_log2e > kFewJump;
    // The reference is the first step's maximum, and moves only where a score is far above it: up to there weights and
    // sums have the precision that they have near 1.
    if (__builtin_expect(__any_sync(0xFFFFFFFFu, jump), 0)) {
      first = false;
      float alpha[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float top = fmaxf(s[e], s[2 + e]);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        const float now = fmaxf(m[e], top);
        alpha[e] = ex2((m[e] - now) * p.scale_log2e);
        m[e] = now;
        l[e] *= alpha[e];
      }
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        o[t][0] *= alpha[0];
        o[t][1] *= alpha[1];
        o[t][2] *= alpha[0];
        o[t][3] *= alpha[1];
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float ref = m[e] * p.scale_log2e;
      s[e] = ex2(fmaf(s[e], p.scale_log2e, -ref));
      s[2 + e] = ex2(fmaf(s[2 + e], p.scale_log2e, -ref));
      l[e] += s[e] + s[2 + e];
    }
    // P is rounded to bf16, as the operand that the matrix product takes
    const uint32_t pt0 = transpose8x8(pack_bf16x2(s[0], s[1])), pt1 = transpose8x8(pack_bf16x2(s[2], s[3]));
    auto values = [&](auto two) {
      // factors of the two keys of a pair side by side
      uint32_t f[2], f2[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t e0 = ev[2 * i], e1 = ev[2 * i + 1];
        f[i] = two ? __byte_perm(q8::factor1(e0), q8::factor1(e1), 0x5410) : __byte_perm(factor_small(e0), factor_small(e1), 0x5410);
        f2[i] = two ? __byte_perm(q8::factor2(e0), q8::factor2(e1), 0x5410) : 0u;
      }
#pragma unroll
      for (int w = 0; w < 8; ++w) {   // two of the thread's 16 dims
        uint2 y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 a = xv[2 * i], d = xv[2 * i + 1];
          const uint32_t wa = w < 2 ? a.x : w < 4 ? a.y : w < 6 ? a.z : a.w, wd = w < 2 ? d.x : w < 4 ? d.y : w < 6 ? d.z : d.w;
          // two codes of each key: their pairs are those of a dim
          y[i] = spread_pairs(__byte_perm(wa, wd, (w & 1) ? 0x7632 : 0x5410));
          y[i].x = q8::mul_bf16x2(y[i].x, f[i]);
          y[i].y = q8::mul_bf16x2(y[i].y, f[i]);
          if (two) {
            y[i].x = q8::mul_bf16x2(y[i].x, f2[i]);
            y[i].y = q8::mul_bf16x2(y[i].y, f2[i]);
          }
        }
        mma16816(o[w], y[0].x, y[0].y, y[1].x, y[1].y, pt0, pt1);
      }
    };
    if (__builtin_expect(__any_sync(0xFFFFFFFFu, max(max(ev[0], ev[1]), max(ev[2], ev[3])) > 134u), 0)) values(Yes{});
    else values(No{});
    if (next < hi) load_v(next);
  }

  // ---- warps of the block ----
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], d);
    const int query = 2 * c + e;
    if (g == 0) slab_ml(warp)[query] = make_float2(m[e], l[e]);
    if (query < queries) {
      float* const to = slab(warp, query) + 16 * g;
#pragma unroll
      for (int t = 0; t < 8; ++t) *reinterpret_cast<float2*>(to + 2 * t) = make_float2(o[t][e], o[t][2 + e]);
    }
  }
  __syncthreads();
  // weights of parts that saw no key are 0: their reference is -inf, the one of all is not where it counts
  auto weight = [&](float ref, float all) { return ref == -INFINITY ? 0.f : ex2((ref - all) * p.scale_log2e); };
  auto add = [](float4& acc, float4 x, float f) {
    acc.x = fmaf(x.x, f, acc.x);
    acc.y = fmaf(x.y, f, acc.y);
    acc.z = fmaf(x.z, f, acc.z);
    acc.w = fmaf(x.w, f, acc.w);
  };
  auto store = [&](int query, int col, float4 acc, float inv) {
    const int64_t dst = (((static_cast<int64_t>(b) * p.L + query0 + query) * p.Hn + h) * kHeadDim + 4 * col) / 2;
    UNSTEP_STORE(out, dst, p.extent_out, pack_bf16x2(acc.x * inv, acc.y * inv), p.status);
    UNSTEP_STORE(out, dst + 1, p.extent_out, pack_bf16x2(acc.z * inv, acc.w * inv), p.status);
  };
  constexpr int kCols = kHeadDim / 4;
  float4* const part4 = reinterpret_cast<float4*>(p.part);
  float2* const part2 = reinterpret_cast<float2*>(p.part);
  constexpr int kPart4 = kFewPartFloats / 4, kMl2 = kFewQueries * kHeadDim / 2, kPart2 = kFewPartFloats / 2;
  // the first `slabs` results in shared memory as one, to the scratch or to the result
  auto merge_slabs = [&](int slabs, bool to_scratch) {
    for (int i = threadIdx.x; i < queries * kCols; i += kFewThreads) {
      const int query = i / kCols, col = i - query * kCols;
      float all = -INFINITY, sum = 0.f;
      float2 ml[kFewWarps];
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w) {
        ml[w] = w < slabs ? slab_ml(w)[query] : make_float2(-INFINITY, 0.f);
        all = fmaxf(all, ml[w].x);
      }
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w)
        if (w < slabs) {
          const float f = weight(ml[w].x, all);
          sum = fmaf(ml[w].y, f, sum);
          add(acc, reinterpret_cast<const float4*>(slab(w, query))[col], f);
        }
      if (to_scratch) {
        UNSTEP_STORE(part4, static_cast<int64_t>(block) * kPart4 + i, p.extent_part / 4, acc, p.status);
        if (col == 0)
          UNSTEP_STORE(part2, static_cast<int64_t>(block) * kPart2 + kMl2 + query, p.extent_part / 2, make_float2(all, sum), p.status);
      } else {
        store(query, col, acc, 1.f / sum);
      }
    }
  };
  merge_slabs(kFewWarps, parts > 1);
  if (parts == 1) return;
  // ---- blocks of the item ----
  const int64_t counter = static_cast<int64_t>(b) * p.Hn * p.groups + item;
  __syncthreads();   // all of this part is stored, and shared memory is free
  if (threadIdx.x == 0) {
    int before = -1;
#ifdef UNSTEP_CHECK
    if (counter >= p.extent_counters) atomicExch(p.status, static_cast<int>(UNSTEP_ERR_BOUNDS));
    else
#endif
    // release: the block's stores (ordered before this thread by the barrier) become visible before the count;
    // acquire: the last block sees the others' stores
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(p.counters + counter) : "memory");
    last = before == parts - 1;
    if (last) UNSTEP_STORE(p.counters, counter, p.extent_counters, 0, p.status);   // ready for the next launch
  }
  __syncthreads();
  if (!last) return;
  __threadfence();   // acquire side for every thread that reads the other parts below
  // A warp has a query (the warps that are left over share the parts of one), a lane four dims of it, and what the
  // warps of a query have is merged as above.
  const int64_t part0 = block - part;
  const int shares = queries <= 1 ? 8 : queries <= 2 ? 4 : queries <= 4 ? 2 : 1, query = warp / shares, share = warp - query * shares;
  if (query < queries) {
    // Lane j looks up the references of the j-th and the (j + 32)-th part of this warp; then all lanes add part by part.
    const int mine = (parts - share + shares - 1) / shares;
    float2 ml[2];
    float all = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = share + shares * (lane + 32 * i);
      ml[i] = k < parts ? __ldcg(part2 + (part0 + k) * kPart2 + kMl2 + query) : make_float2(-INFINITY, 0.f);
      all = fmaxf(all, ml[i].x);
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) all = fmaxf(all, __shfl_xor_sync(0xFFFFFFFFu, all, d));
    const float f0 = weight(ml[0].x, all), f1 = weight(ml[1].x, all);
    float sum = fmaf(ml[0].y, f0, ml[1].y * f1);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int j = 0; j < mine; ++j) {
      const float f = __shfl_sync(0xFFFFFFFFu, j < 32 ? f0 : f1, j & 31);
      add(acc, __ldcg(part4 + (part0 + share + shares * j) * kPart4 + query * kCols + lane), f);
    }
    reinterpret_cast<float4*>(slab(share, query))[lane] = acc;
    if (lane == 0) slab_ml(share)[query] = make_float2(all, sum);
  }
  __syncthreads();
  merge_slabs(shares, false);
}

int launch_few(const AttnParams& a, int nb, int sm_count, const void* q_rot, const void* cache_k, const void* scale_k,
               const void* cache_v, const void* scale_v, void* out, cudaStream_t st) {
  FewParams p;
  p.Hn = a.Hn;
  p.L = a.L;
  p.groups = few_groups(a.L);
  p.n_streams = nb;
  p.cache_rows = a.cache_rows;
  p.scale_log2e = a.scale_log2e;
  p.part = a.part;
  p.counters = a.counters;
  p.status = a.status;
  p.extent_out = static_cast<int64_t>(nb) * a.L * a.Hn * (kHeadDim / 2);
  p.extent_part = a.extent_part;
  p.extent_counters = a.extent_counters;
  int64_t steps[kMaxStreamsPerLaunch], all = 0;
  for (int i = 0; i < nb; ++i) {
    int32_t end = 0;
    for (int r = 0; r < 3; ++r) {
      p.run_row0[i][r] = a.run_row0[i][r];
      p.run_end[i][r] = end += a.run_rows[i][r];
    }
    steps[i] = (end + kFewKeys - 1) / kFewKeys;
    all += steps[i] * a.Hn * p.groups;
  }
  // The shortest share of steps for a block with which all blocks run at once (a second wave would take as long as
  // the first), but at least one for each of its warps; with more items than blocks an item is not split.
  const int64_t room = static_cast<int64_t>(sm_count) * kFewBlocks;
  const int64_t part_room = p.extent_part / kFewPartFloats;
  int64_t share = (all + room - 1) / room, blocks = 0;
  if (share < kFewWarps) share = kFewWarps;
  for (int i = 0; i < nb; ++i)   // and no more than kFewParts blocks, which one of them merges
    if (share < (steps[i] + kFewParts - 1) / kFewParts) share = (steps[i] + kFewParts - 1) / kFewParts;
  for (;; share += share / 16 + 1) {
    blocks = 0;
    bool split = false;
    for (int i = 0; i < nb; ++i) {
      const int64_t parts = (steps[i] + share - 1) / share;
      p.parts[i] = static_cast<int32_t>(parts);
      p.block0[i] = static_cast<int32_t>(blocks);
      blocks += parts * a.Hn * p.groups;
      split = split || parts > 1;
    }
    if (!split || (blocks <= room && blocks <= part_room)) break;
  }
  const bool wide = (reinterpret_cast<uintptr_t>(cache_k) & 31u) == 0;   // heads are 128 bytes
  const cudaError_t err = launch_overlapped(
      true, wide ? window_attn_few_kernel<true> : window_attn_few_kernel<false>, dim3(static_cast<unsigned>(blocks)), kFewThreads, 0, st, p, static_cast<const uint4*>(q_rot),
      static_cast<const uint4*>(cache_k), static_cast<const uint8_t*>(scale_k), static_cast<const uint4*>(cache_v),
      static_cast<const uint8_t*>(scale_v), static_cast<uint32_t*>(out));
  g_launches.fetch_add(1);
  return err == cudaSuccess ? UNSTEP_OK : UNSTEP_ERR_CUDA;
}

}  // namespace unstep
