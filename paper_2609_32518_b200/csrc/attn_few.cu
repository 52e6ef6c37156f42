// Attention of at most 16 queries a stream over an 8-bit cache (sm_100a): single tokens, and what little more goes with them.
//
// DRAM bound: every cached key and value is read once, and a query tile of the tensor-memory kernel would be next to empty,
// while it waits for tiles to be decoded into shared memory.  Here a warp takes 16 keys at a time straight from global memory
// into the operands of warp-level matrix products (mma.sync, m16n8k16, bf16 with float32 sums):
//     S^T = K Q^T   16 keys x 8 queries    O^T = V^T P^T   16 dims x 8 queries
// The dims of K, summed over, and those of V, independent of each other, may come in any order, so every thread
// reads 16 or 32 neighbouring codes of a row and needs no exchange; P^T turns from result to operand by a
// transpose of its 8 x 8 blocks.  Each warp has its own running maximum and sum; the warps of a block merge through
// shared memory, the blocks of an item (stream, head) are a cluster and merge through each other's.
#include <cuda_bf16.h>

#include "attn_sched.h"
#include "common.h"
#include "ptx.cuh"
#include "quant.cuh"

namespace unstep {

using namespace ptx;

constexpr int kFewWarps = 8, kFewThreads = 32 * kFewWarps;
constexpr int kFewKeys = 16;                    // keys of a warp's step

struct FewParams {
  int32_t Hn, L, parts;
  int64_t cache_rows;                           // rows of a stream's cache
  float scale_log2e;
  int* status;
  int64_t extent_out;                           // 4-byte words of `out`
  int32_t run_row0[kMaxStreamsPerLaunch][3], run_end[kMaxStreamsPerLaunch][3];   // rows of the runs, added up
};

// D (16 x 8) += A (16 x 16) B (16 x 8)
__device__ __forceinline__ void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Four codes times their scale, as two bf16 pairs.
__device__ __forceinline__ uint2 decode4(uint32_t w, uint32_t f1, uint32_t f2, bool two) {
  uint2 y = q8::spread4(w);
  y.x = q8::mul_bf16x2(y.x, f1);
  y.y = q8::mul_bf16x2(y.y, f1);
  if (two) {
    y.x = q8::mul_bf16x2(y.x, f2);
    y.y = q8::mul_bf16x2(y.y, f2);
  }
  return y;
}

template <int kN>   // groups of 8 queries
constexpr int few_smem_bytes() {
  return (kFewWarps * 8 * kN * kHeadDim + kFewWarps * 8 * kN * 2 + 8 * kN * kHeadDim + 8 * kN * 2) * static_cast<int>(sizeof(float));
}

template <int kN>
__global__ void __launch_bounds__(kFewThreads, kN == 1 ? 2 : 1)
window_attn_few_kernel(const __grid_constant__ FewParams p, const uint4* q_rot, const uint4* cache_k, const uint8_t* scale_k,
                       const uint4* cache_v, const uint8_t* scale_v, uint32_t* out) {
  extern __shared__ __align__(16) float few_smem[];
  float* const slabs = few_smem;                                        // [warp][query][dim]: O of a warp
  float2* const warp_ml = reinterpret_cast<float2*>(slabs + kFewWarps * 8 * kN * kHeadDim);   // [warp][query]
  float* const mine = reinterpret_cast<float*>(warp_ml + kFewWarps * 8 * kN);                 // [query][dim]: O of the block
  float2* const my_ml = reinterpret_cast<float2*>(mine + 8 * kN * kHeadDim);                  // [query]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int item = blockIdx.x / p.parts, part = blockIdx.x - item * p.parts;
  const int b = item / p.Hn, h = item - b * p.Hn;
  const int end0 = p.run_end[b][0], end1 = p.run_end[b][1], keys = p.run_end[b][2];
  const int row0 = p.run_row0[b][0], row1 = p.run_row0[b][1] - end0, row2 = p.run_row0[b][2] - end1;
  const int steps = (keys + kFewKeys - 1) / kFewKeys;
  const int lo = static_cast<int>(static_cast<int64_t>(steps) * part / p.parts);
  const int hi = static_cast<int>(static_cast<int64_t>(steps) * (part + 1) / p.parts);
  const int64_t base = b * p.cache_rows;
  // where key j lies, in rows of a head; keys behind the last are the last again, and masked
  auto row_of = [&](int j) {
    j = min(j, keys - 1);
    return (base + (j < end0 ? row0 + j : (j < end1 ? row1 + j : row2 + j))) * p.Hn + h;
  };
  const int behind = grid_wait();

  // B of S^T: thread (g, c) has query g, dims 32 c ..
  uint32_t q[kN][16];
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    const int query = 8 * n + g;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (query < p.L) x = __ldca(q_rot + ((static_cast<int64_t>(b) * p.L + query) * p.Hn + h) * 16 + 4 * c + i + behind);
      q[n][4 * i] = x.x, q[n][4 * i + 1] = x.y, q[n][4 * i + 2] = x.z, q[n][4 * i + 3] = x.w;
    }
  }
  float o[kN][8][4];   // O^T: dims 16 g + 2 t and + 2 t + 1, queries 8 n + 2 c and + 1
  float m[kN][2], l[kN][2];
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    m[n][0] = m[n][1] = -INFINITY;
    l[n][0] = l[n][1] = 0.f;
#pragma unroll
    for (int t = 0; t < 8; ++t) o[n][t][0] = o[n][t][1] = o[n][t][2] = o[n][t][3] = 0.f;
  }

  uint4 xk[2][2], xv[4];     // codes of keys g, g + 8 (dims 32 c ..) and of keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9 (dims 16 g ..)
  uint32_t ek[2], ev[4];
  auto load_k = [&](int step) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = row_of(step * kFewKeys + g + 8 * i) + behind;
      xk[i][0] = __ldcs(cache_k + r * 8 + 2 * c);
      xk[i][1] = __ldcs(cache_k + r * 8 + 2 * c + 1);
      ek[i] = __ldca(scale_k + r * 4 + c);
    }
  };
  auto load_v = [&](int step) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t r = row_of(step * kFewKeys + 2 * c + (i & 1) + 8 * (i >> 1)) + behind;
      xv[i] = __ldcs(cache_v + r * 8 + g);
      ev[i] = __ldca(scale_v + r * 4 + (g >> 1));
    }
  };
  int step = lo + warp;
  if (step < hi) {
    load_k(step);
    load_v(step);
  }
#pragma unroll 1
  for (; step < hi; step += kFewWarps) {
    float s[kN][4];
#pragma unroll
    for (int n = 0; n < kN; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
    {
      const bool two = __any_sync(0xFFFFFFFFu, !q8::one_factor(ek[0]) || !q8::one_factor(ek[1]));
      const uint32_t fa = q8::factor1(ek[0]), fb = q8::factor1(ek[1]), fa2 = q8::factor2(ek[0]), fb2 = q8::factor2(ek[1]);
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const uint4 ca = xk[0][w >> 2], cb = xk[1][w >> 2];
        const uint2 a = decode4((w & 3) == 0 ? ca.x : (w & 3) == 1 ? ca.y : (w & 3) == 2 ? ca.z : ca.w, fa, fa2, two);
        const uint2 d = decode4((w & 3) == 0 ? cb.x : (w & 3) == 1 ? cb.y : (w & 3) == 2 ? cb.z : cb.w, fb, fb2, two);
#pragma unroll
        for (int n = 0; n < kN; ++n) mma16816(s[n], a.x, d.x, a.y, d.y, q[n][2 * w], q[n][2 * w + 1]);
      }
    }
    const int next = step + kFewWarps;
    if (next < hi) load_k(next);
    const int left = keys - step * kFewKeys;   // keys of this step
    uint32_t pt[kN][2];
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      if (g >= left) s[n][0] = s[n][1] = -INFINITY;
      if (g + 8 >= left) s[n][2] = s[n][3] = -INFINITY;
      float alpha[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float top = fmaxf(s[n][e], s[n][2 + e]);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        // key `step * kFewKeys` is there, so the maximum is one of a score: a first reference, or a larger one
        const float now = fmaxf(m[n][e], top);
        alpha[e] = ex2((m[n][e] - now) * p.scale_log2e);
        m[n][e] = now;
        const float ref = now * p.scale_log2e;
        s[n][e] = ex2(fmaf(s[n][e], p.scale_log2e, -ref));
        s[n][2 + e] = ex2(fmaf(s[n][2 + e], p.scale_log2e, -ref));
        l[n][e] = fmaf(l[n][e], alpha[e], s[n][e] + s[n][2 + e]);
      }
      if (__any_sync(0xFFFFFFFFu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          o[n][t][0] *= alpha[0];
          o[n][t][1] *= alpha[1];
          o[n][t][2] *= alpha[0];
          o[n][t][3] *= alpha[1];
        }
      }
      // P is rounded to bf16, as the operand that the matrix product takes
      pt[n][0] = transpose8x8(pack_bf16x2(s[n][0], s[n][1]));
      pt[n][1] = transpose8x8(pack_bf16x2(s[n][2], s[n][3]));
    }
    {
      const bool two = __any_sync(0xFFFFFFFFu, !q8::one_factor(ev[0]) || !q8::one_factor(ev[1]) || !q8::one_factor(ev[2]) ||
                                                   !q8::one_factor(ev[3]));
      uint32_t f1[4], f2[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f1[i] = q8::factor1(ev[i]);
        f2[i] = q8::factor2(ev[i]);
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint2 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = decode4(w == 0 ? xv[i].x : w == 1 ? xv[i].y : w == 2 ? xv[i].z : xv[i].w, f1[i], f2[i], two);
        // dims 4 w .. 4 w + 3 of the two keys of a pair
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          mma16816(o[n][2 * w], __byte_perm(y[0].x, y[1].x, 0x5410), __byte_perm(y[0].x, y[1].x, 0x7632),
                   __byte_perm(y[2].x, y[3].x, 0x5410), __byte_perm(y[2].x, y[3].x, 0x7632), pt[n][0], pt[n][1]);
          mma16816(o[n][2 * w + 1], __byte_perm(y[0].y, y[1].y, 0x5410), __byte_perm(y[0].y, y[1].y, 0x7632),
                   __byte_perm(y[2].y, y[3].y, 0x5410), __byte_perm(y[2].y, y[3].y, 0x7632), pt[n][0], pt[n][1]);
        }
      }
    }
    if (next < hi) load_v(next);
  }

  // ---- warps of the block ----
#pragma unroll
  for (int n = 0; n < kN; ++n) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, l[n][e], d);
      const int query = 8 * n + 2 * c + e;
      if (g == 0) warp_ml[warp * 8 * kN + query] = make_float2(m[n][e], l[n][e]);
      if (query < p.L) {
        float* const to = slabs + (warp * 8 * kN + query) * kHeadDim + 16 * g;
#pragma unroll
        for (int t = 0; t < 8; ++t) *reinterpret_cast<float2*>(to + 2 * t) = make_float2(o[n][t][e], o[n][t][2 + e]);
      }
    }
  }
  __syncthreads();
  // weights of parts that saw no key are 0: their reference is -inf, the one of all is not where it counts
  auto weight = [&](float ref, float all) { return ref == -INFINITY ? 0.f : ex2((ref - all) * p.scale_log2e); };
  for (int i = threadIdx.x; i < p.L * (kHeadDim / 4); i += kFewThreads) {
    const int query = i / (kHeadDim / 4), col = i - query * (kHeadDim / 4);
    float all = -INFINITY, sum = 0.f;
    float2 ml[kFewWarps];
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      ml[w] = warp_ml[w * 8 * kN + query];
      all = fmaxf(all, ml[w].x);
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float f = weight(ml[w].x, all);
      const float4 x = reinterpret_cast<const float4*>(slabs + (w * 8 * kN + query) * kHeadDim)[col];
      sum = fmaf(ml[w].y, f, sum);
      acc.x = fmaf(x.x, f, acc.x);
      acc.y = fmaf(x.y, f, acc.y);
      acc.z = fmaf(x.z, f, acc.z);
      acc.w = fmaf(x.w, f, acc.w);
    }
    reinterpret_cast<float4*>(mine)[i] = acc;
    if (col == 0) my_ml[query] = make_float2(all, sum);
  }
  // ---- blocks of the cluster ----
  __syncthreads();
  cluster_sync();
  const uint32_t mine_at = smem_u32(mine), ml_at = smem_u32(my_ml);
  for (int i = part * kFewThreads + threadIdx.x; i < p.L * (kHeadDim / 4); i += p.parts * kFewThreads) {
    const int query = i / (kHeadDim / 4), col = i - query * (kHeadDim / 4);
    float all = -INFINITY, sum = 0.f;
    float2 ml[kMaxClusterParts];
#pragma unroll
    for (int k = 0; k < kMaxClusterParts; ++k) {
      ml[k] = k < p.parts ? ld_cluster_8(cluster_addr(ml_at + query * 8, k)) : make_float2(-INFINITY, 0.f);
      all = fmaxf(all, ml[k].x);
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kMaxClusterParts; ++k)
      if (k < p.parts) {
        const float f = weight(ml[k].x, all);
        const float4 x = ld_cluster_16(cluster_addr(mine_at + i * 16, k));
        sum = fmaf(ml[k].y, f, sum);
        acc.x = fmaf(x.x, f, acc.x);
        acc.y = fmaf(x.y, f, acc.y);
        acc.z = fmaf(x.z, f, acc.z);
        acc.w = fmaf(x.w, f, acc.w);
      }
    const float inv = 1.f / sum;
    const int64_t dst = (((static_cast<int64_t>(b) * p.L + query) * p.Hn + h) * kHeadDim + 4 * col) / 2;
    UNSTEP_STORE(out, dst, p.extent_out, pack_bf16x2(acc.x * inv, acc.y * inv), p.status);
    UNSTEP_STORE(out, dst + 1, p.extent_out, pack_bf16x2(acc.z * inv, acc.w * inv), p.status);
  }
  __syncwarp();
  cluster_sync();   // no block leaves while another reads its part
}

bool few_setup() {
  return cudaFuncSetAttribute(window_attn_few_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, few_smem_bytes<1>()) == cudaSuccess &&
         cudaFuncSetAttribute(window_attn_few_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, few_smem_bytes<2>()) == cudaSuccess;
}

int launch_few(const AttnParams& a, int nb, int sm_count, const void* q_rot, const void* cache_k, const void* scale_k,
               const void* cache_v, const void* scale_v, void* out, cudaStream_t st) {
  FewParams p;
  p.Hn = a.Hn;
  p.L = a.L;
  p.cache_rows = a.cache_rows;
  p.scale_log2e = a.scale_log2e;
  p.status = status_word();
  p.extent_out = static_cast<int64_t>(nb) * a.L * a.Hn * (kHeadDim / 2);
  int32_t most = 0;
  for (int i = 0; i < nb; ++i) {
    int32_t end = 0;
    for (int r = 0; r < 3; ++r) {
      p.run_row0[i][r] = a.run_row0[i][r];
      p.run_end[i][r] = end += a.run_rows[i][r];
    }
    most = end > most ? end : most;
  }
  // blocks for two on each SM, but none with less than a step for every warp
  const int64_t items = static_cast<int64_t>(nb) * a.Hn;
  int64_t parts = (2 * sm_count + items - 1) / items;
  const int64_t fill = (most + kFewKeys * kFewWarps - 1) / (kFewKeys * kFewWarps);
  if (parts > fill) parts = fill;
  if (parts > kMaxClusterParts) parts = kMaxClusterParts;
  p.parts = static_cast<int32_t>(parts);
  const bool one = a.L <= 8;
  const cudaError_t err = launch_clusters(
      true, p.parts, one ? window_attn_few_kernel<1> : window_attn_few_kernel<2>, dim3(static_cast<unsigned>(items * parts)),
      kFewThreads, one ? few_smem_bytes<1>() : few_smem_bytes<2>(), st, p, static_cast<const uint4*>(q_rot),
      static_cast<const uint4*>(cache_k), static_cast<const uint8_t*>(scale_k), static_cast<const uint4*>(cache_v),
      static_cast<const uint8_t*>(scale_v), static_cast<uint32_t*>(out));
  g_launches.fetch_add(1);
  return err == cudaSuccess ? UNSTEP_OK : UNSTEP_ERR_CUDA;
}

}  // namespace unstep
