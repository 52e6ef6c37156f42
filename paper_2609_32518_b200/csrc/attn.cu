// Windowed attention of one chunk over the KV ring (sm_100a).
//
// Persistent, warp-specialised kernel, one CTA per SM:
//   warps 0-3   softmax of query tile 0, one thread per query row
//   warps 4-7   softmax of query tile 1
//   warp  8     issues S = Q K^T of both query tiles; owns TMEM
//   warp  9     issues O += P V of both query tiles
//   warp  10    TMA producer (one lane)
//   warps 12-15 (8-bit cache) decode the tiles that TMA brings as codes
// A work item is (stream, head, pair of 128-query tiles): both tiles share every K/V
// tile.  S, P (bf16) and O live in TMEM: one S for both query tiles in turn, a P and an O for each.
// A softmax group takes its scores into registers at once and gives S back, so that the tensor core
// computes the other tile's scores, and then this tile's next ones, while the exponentials run; P V
// follows when P is there.  So the next scores are there when a group is done with its tile, and the
// two groups share the MUFU pipe without waiting for the tensor core.  (With an S for each tile and P over
// S, a tile's next Q K^T had to wait for its P V: exponentials, hand-over, P V and Q K^T were one
// chain of ~3500 clk per key tile.  12 heads, 4680 queries, 32760 keys: 1423-1431 -> 1184-1219 thousand
// cycles and 881-884 -> 808-815 us run on end at the power cap, 755-757 -> 694-697 us in runs of 20.)
//
// What a group does per key tile is as long as the period, so it counts how fast it is fetched: its
// loop over the full tiles is kept short and free of taken branches (rare cases are out of line, one
// masked variant takes first and ragged tiles).  The same pipeline with the variants side by side in one loop
// waited 640 clk per key tile for instructions and took 1425 thousand cycles.
//
// The attended frames are at most three runs of consecutive cache slots (sink prefix, ring
// up to its end, ring from its start).  Key tiles are cut from the runs through a flat
// tensor map over cache rows; only the last tile of a run is ragged, and it is fetched
// through a (token, slot) map whose zero fill ends it exactly at the end of its frame, so
// the cache is never copied and slots outside the window may hold anything.  A ragged tile
// runs with a narrower MMA (N and K rounded up to 16).
#include <cuda.h>
#include <cuda_bf16.h>

#include <atomic>
#include <map>
#include <mutex>
#include <tuple>

#include "common.h"
#include "ptx.cuh"
#include "quant.cuh"
#include "attn_sched.h"
#include "handover.h"

namespace unstep {

using namespace ptx;

__device__ int g_status = 0;

// Optional timeline of CTA 0 (debug builds only): clock64 stamps per role, tile and event.
#ifdef UNSTEP_TRACE
__device__ long long g_trace[12][64][8];
__device__ unsigned long long g_cta_trace[160][16];
__device__ __forceinline__ unsigned long long gtime() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
#define CTRACE(ev)                                                                       \
  do {                                                                                   \
    if (threadIdx.x == 0 && (ev) < 16) g_cta_trace[blockIdx.x][ev] = gtime();            \
  } while (0)
#define TRACE(role, tile, ev)                                                          \
  do {                                                                                 \
    if (blockIdx.x == 0 && (tile) < 64 && (threadIdx.x & 31) == 0) {                   \
      const int w_ = threadIdx.x >> 5;                                                 \
      const int slot_ = (role) < 2 ? (w_ & 3) * 2 + (role) : 8 + (role) - 2;            \
      g_trace[slot_][tile][ev] = clock64();                                            \
    }                                                                                  \
  } while (0)
#else
#define TRACE(role, tile, ev) \
  do {                        \
  } while (0)
#define CTRACE(ev) \
  do {             \
  } while (0)
#endif

constexpr int kHalfBytes = 128 * 64 * 2;    // one TMA box: 128 rows x 64 bf16 (128-byte rows)
constexpr int kTileBytes = 2 * kHalfBytes;  // 128 x 128 bf16
// What the kernel over a bf16 cache and the one over an 8-bit cache have of their own.  The latter has four more
// warps, which decode the tiles that TMA brings as codes (kRawStages buffers) into the bf16 buffers that the other has TMA fill.
// Decoding is exact (quant.cuh), so softmax and products are the same.  It takes ~420 instructions a row and tile, next to a softmax
// that is as long as the period: 4680 queries x 32760 keys x 12 heads 951 us, without the arithmetic of decoding 785, without
// decoding 742, the bf16 kernel 694 (runs of 20).  So launches of many queries unpack their windows in front (kUnpackPairs), and
// this is for the others, in which a head's tiles are decoded only a few times.
//
// Where every item has one query tile (kQ8Lone), the second softmax group has nothing to do and the second Q buffer is free: the
// group then decodes the V tiles and the four warps the K tiles, and K and V have a ring each, of two tiles as codes and
// two as bf16: 100 queries x 16000 keys x 8 heads 39.9 -> 32.9 us, x 24 heads 57.4 -> 49.0.  (Rings that both kinds go through in turn do not do for that: a warp has to see every phase of a barrier
// that it waits at, as it cannot tell one from the phase before the last.)
constexpr int kRawStages = 2, kRawBytes = 128 * 128;
enum Kind { kBf16, kQ8Pairs, kQ8Lone };
constexpr int kKinds = 3;
template <bool kQ8>
struct Form {
  static constexpr int kStages = kQ8 ? 4 : 5;       // 32 KB buffers shared by the K and V tiles
  static constexpr int kThreads = kQ8 ? 512 : 384;
};
constexpr int kTmemCols = 512;
constexpr int kTmemS = 0, kTmemP = 128, kTmemO = 256;   // S (128 columns) | P0 | P1 (64 each) | O0 | O1 (128 each)
constexpr long long kWaitCycles = 2000000000LL;  // about a second: then give up, never hang

constexpr int kSmemQ = 0;
constexpr int kSmemKV = 2 * kTileBytes;
constexpr int kSmemRaw = kSmemKV + Form<true>::kStages * kTileBytes;
constexpr int kSmemBar = kSmemKV + Form<false>::kStages * kTileBytes;
static_assert(kSmemRaw + kRawStages * kRawBytes == kSmemBar, "both forms have their barriers behind their buffers");
constexpr int kAttnSmemBytes = kSmemBar + 256;

// Partial result of one query tile of a split item: O as [col / 4][row][col % 4] (unnormalised,
// relative to the part's own reference maximum; a warp's 16-byte accesses are 512 consecutive
// bytes), then (m, l)[row].  Two tiles per slot, two slots per CTA.
constexpr int kPartTileFloats = 128 * 128 + 2 * 128;
constexpr int kPartFloats = 2 * kPartTileFloats;
struct Waiter {
  volatile int* abort_flag;
  long long limit;   // clock cycles after which a wait gives up
  // Bounded wait: the hardware parks the thread between polls; the clock and the CTA's abort
  // flag are only looked at every 32 polls so that a waiting warp leaves the issue slots alone.
  __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) const {
    if (__builtin_expect(mbar_try_wait(bar, parity) != 0, 1)) return true;
    return wait_long(bar, parity);
  }
  __device__ __forceinline__ bool wait_long(uint32_t bar, uint32_t parity) const {
    const long long t0 = clock64();
#pragma unroll 1
    for (uint32_t spin = 1;; ++spin) {
      if (mbar_try_wait_hint(bar, parity, 2000u)) return true;
      if ((spin & 31u) == 0u) {
        if (*abort_flag) return false;
        if (clock64() - t0 > limit) {
          *abort_flag = 1;
          atomicExch(&g_status, UNSTEP_ERR_TIMEOUT);
          return false;
        }
      }
    }
  }
  // The same by all lanes of a warp, with the warp's answer.
  __device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity) const {
    return __all_sync(0xFFFFFFFFu, wait(bar, parity));
  }
};

// The CTA owns 384 x 168 registers; 128 x 72 for the service warps + 256 x 216 for the softmax
// warps uses exactly that (an increase that the pool cannot satisfy would wait forever).  Nothing spills.
// Over an 8-bit cache 512 x 128: 128 x 56 + 128 x 40 for the decoders + 256 x 208.
constexpr int kRegsService = 72, kRegsSoftmax = 216;
static_assert(128 * kRegsService + 256 * kRegsSoftmax <= 384 * 168, "register redistribution exceeds the CTA's allocation");
static_assert(kRegsService == 72 && kRegsSoftmax == 216, "keep the setmaxnreg literals below in step");
constexpr int kRegsService8 = 56, kRegsDecode8 = 40, kRegsSoftmax8 = 208;
static_assert(128 * kRegsService8 + 128 * kRegsDecode8 + 256 * kRegsSoftmax8 <= 512 * 128, "register redistribution exceeds the CTA's allocation");
static_assert(kRegsService8 == 56 && kRegsDecode8 == 40 && kRegsSoftmax8 == 208, "keep the setmaxnreg literals below in step");
template <bool kQ8>
__device__ __forceinline__ void reg_dealloc_service() {
  if constexpr (kQ8) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  else asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
}
__device__ __forceinline__ void reg_dealloc_decode() { asm volatile("setmaxnreg.dec.sync.aligned.u32 40;"); }
template <bool kQ8>
__device__ __forceinline__ void reg_alloc_softmax() {
  if constexpr (kQ8) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
}

// --------------------------------------------------------------------------------------
// Softmax of one 128 x 128 score tile with one thread per query row (a warpgroup per query
// tile); no data crosses threads.
// --------------------------------------------------------------------------------------
__device__ __forceinline__ void group_barrier(int a) {
  asm volatile("bar.sync %0, 128;" ::"r"(kGroupBarrier + a) : "memory");
}
// The group barrier that also counts the threads with a true predicate: the same answer in every
// thread, with nothing in memory that a warp ahead of the others could overwrite.
__device__ __forceinline__ uint32_t group_count(int a, bool pred) {
  uint32_t n;
  asm volatile("{\n.reg .pred q;\nsetp.ne.u32 q, %2, 0;\nbar.red.popc.u32 %0, %1, 128, q;\n}"
               : "=r"(n) : "r"(kGroupBarrier + a), "r"(static_cast<uint32_t>(pred)) : "memory");
  return n;
}

// Hand-over of P to the P V issuer, and of the read S back to the Q K^T issuer, through named barriers.  An mbarrier lives in shared
// memory, whose bandwidth the MMA operands of Q K^T use up: an arrive or a try_wait there took
// 120-270 clk, several times on every key tile's critical path; a named barrier takes 25-60 clk.
// A named barrier has no bounded wait, so every warp keeps meeting them, once per key tile of its
// segments, after it has given up on an mbarrier as well; handover.h says why all of them end.
__device__ __forceinline__ void p_ready_sync(int a, uint32_t tile) {   // P V issuer: P of group a's tile-th key tile is in TMEM
  asm volatile("bar.sync %0, 160;" ::"r"(p_ready_barrier(a, tile)) : "memory");
}
__device__ __forceinline__ void p_ready_pass(int a, uint32_t tile, bool gave_up) {   // a warp of softmax group a
  if (p_ready_waits(gave_up)) p_ready_sync(a, tile);
  else asm volatile("bar.arrive %0, 160;" ::"r"(p_ready_barrier(a, tile)) : "memory");
}
__device__ __forceinline__ void s_free_sync(int a, uint32_t tile) {   // Q K^T issuer: group a has read S of its tile-th key tile
  asm volatile("bar.sync %0, 160;" ::"r"(s_free_barrier(a, tile)) : "memory");
}
__device__ __forceinline__ void s_free_pass(int a, uint32_t tile, bool gave_up) {   // a warp of softmax group a
  if (p_ready_waits(gave_up)) s_free_sync(a, tile);
  else asm volatile("bar.arrive %0, 160;" ::"r"(s_free_barrier(a, tile)) : "memory");
}

// Exponentials of 32 score columns (registers s) into 16 bf16 pairs (p) and the packed sums.
__device__ __forceinline__ void exp_block32(const uint32_t* s, uint32_t* p, uint64_t c2, uint64_t nm2,
                                            uint64_t* acc) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint64_t x2 = fma_f32x2(pack_f32x2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c2, nm2);
    float x0, x1;
    unpack_f32x2(x2, x0, x1);
    const float p0 = ex2(x0), p1 = ex2(x1);
    acc[i & 3] = add_f32x2(acc[i & 3], pack_f32x2(p0, p1));
    p[i] = pack_bf16x2(p0, p1);
  }
}
__device__ __forceinline__ float max_block32(const uint32_t* s) {
  float m = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
#pragma unroll
  for (int i = 2; i < 32; i += 2) m = max3(m, __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
  return m;
}
template <bool kMasked>
__device__ __forceinline__ void mask_block32(uint32_t* s, int col0, int nvalid) {
  if (kMasked) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (col0 + i >= nvalid) s[i] = 0xFF800000u;  // -inf
  }
}

// One key tile of a row: scores from TMEM (columns t_S ..) into registers, S given back, exponentials against
// the row's reference maximum, P (bf16 pairs, keys 0.. from column t_P on) handed over.  False if a wait gave up;
// S has been given back then, P has not been passed.
//
// The reference is the maximum of the segment's first key tile, so that the largest weight there is exactly 1 (with
// the maximum of 32 scores the error of peaked rows against float64 grew from 2.17e-3 to 2.32e-3).  It moves
// only where a later tile has a score more than kJump = 57 (log2 units) above it: up to there P (bf16) and the
// float32 sums are as accurate as near 1 (same relative precision), and what was accumulated before such a jump
// is negligible exactly as in the true softmax.  A tile's sum of P is at most 128 * 2^57 = 2^64, the sum of n keys
// at most n * 2^57, and O that times |v|: finite for any window that the entry points take (2^30 keys) up to
// |v| = 2^40, for 32760 keys up to 2^55.  (With kJump = 64, tiles of 128 keys 62 above the reference overflowed with |v| =
// 2^60.)  The scores have left TMEM by the time a sum of P could tell, so the maximum is looked for in front: 64
// three-input maxima in the shadow of the other group's exponentials.
//
// P may be stored, and O rescaled, once the P V of the tile before has run.  That barrier, and the one of the next
// tile's scores, are looked at once, ahead of time: the look takes 100-200 clk under the MMAs' traffic, and
// almost always finds what it looks for.
// Tiles of at most 64 keys (frames of up to 64 tokens, the end of a run) leave the other half of the columns
// alone.
constexpr float kJump = 57.f;

template <bool kMasked, int kCols, bool kTight>   // kCols: score columns that hold keys, 64 or 128; kTight: not a segment's first tile
__device__ __forceinline__ bool softmax_row_tile(uint32_t t_S, uint32_t t_P, uint32_t t_O, float c, int nvalid,
                                                 bool first, float& m_run, float& l_run, int a, uint32_t tile,
                                                 const Waiter& w, uint32_t bar_pv, uint32_t bar_s, uint32_t& s_seen) {
  uint32_t s[kCols], p[kCols / 2];
#pragma unroll
  for (int q = 0; q < kCols / 32; ++q) tmem_ld32(t_S + 32 * q, s + 32 * q);
  tc_wait_ld32(s);
#pragma unroll
  for (int q = 1; q < kCols / 32; ++q) reg_fence32(s + 32 * q);
  tc_fence_before();
  s_free_pass(a, tile, false);
  TRACE(a, tile, 2);
#pragma unroll
  for (int q = 0; q < kCols / 32; ++q) mask_block32<kMasked>(s + 32 * q, 32 * q, nvalid);
  float mx = max_block32(s);
#pragma unroll
  for (int q = 1; q < kCols / 32; ++q) mx = fmaxf(mx, max_block32(s + 32 * q));
  if (!kTight && first) {
    m_run = mx;
  } else if (__builtin_expect(__any_sync(0xFFFFFFFFu, (mx - m_run) * c > kJump), 0)) {
    if (!w.wait_warp(bar_pv, (tile - 1) & 1)) return false;
    tc_fence_after();
    float alpha = 1.f;
    if (mx > m_run) {
      alpha = ex2((m_run - mx) * c);
      m_run = mx;
      l_run *= alpha;
    }
#pragma unroll 1
    for (int q = 0; q < 16; ++q) {
      uint32_t o[8];
      tmem_ld8(t_O + q * 8, o);
      tc_wait_ld8(o);
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
      tmem_st8(t_O + q * 8, o);
    }
  }
  const uint64_t c2 = pack_f32x2(c, c), nm2 = pack_f32x2(-m_run * c, -m_run * c);
  uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
  TRACE(a, tile, 3);
#pragma unroll
  for (int q = 0; q < kCols / 32 - 1; ++q) exp_block32(s + 32 * q, p + 16 * q, c2, nm2, acc);
  uint32_t pv_seen = mbar_test(bar_pv, (tile - 1) & 1);
  exp_block32(s + kCols - 32, p + kCols / 2 - 16, c2, nm2, acc);
  if ((kTight || !first) && __builtin_expect(!__all_sync(0xFFFFFFFFu, pv_seen), 0)) {
    if (!w.wait_warp(bar_pv, (tile - 1) & 1)) return false;
  }
  tc_fence_after();
  TRACE(a, tile, 4);
  if (kCols > 64) tmem_st32(t_P, p);
  s_seen = mbar_test(bar_s, (tile + 1) & 1);
  tmem_st32(t_P + kCols / 2 - 32, p + kCols / 2 - 32);
  tc_wait_st();
  tc_fence_before();
  p_ready_pass(a, tile, false);
  TRACE(a, tile, 5);
  const uint64_t t2 = add_f32x2(add_f32x2(acc[0], acc[1]), add_f32x2(acc[2], acc[3]));
  float t0, t1;
  unpack_f32x2(t2, t0, t1);
  l_run += t0 + t1;
  return true;
}

// Real keys of key tile j of a stream, without the divisions of tile_info: only the last tile of a
// run of slots is ragged (frames shorter than a tile: every tile is one frame).
struct ValidKeys {
  int j_last[3], v_last[3], dflt;
  __device__ __forceinline__ ValidKeys(const AttnParams& p, int b) {
    dflt = p.flat ? kTileN : p.T;
#pragma unroll
    for (int r = 0; r < 3; ++r) {
      const int begin = r == 0 ? 0 : p.run_tile_end[b][r - 1];
      const int end = p.run_tile_end[b][r];
      const bool any = p.flat && end > begin;
      j_last[r] = any ? end - 1 : -1;
      v_last[r] = p.run_rows[b][r] - kTileN * (end - begin - 1);
    }
  }
  // first tile from j on that is ragged, at most `end`
  __device__ __forceinline__ int full_until(int j, int end) const {
    if (dflt < kTileN) return j;
    int k = end;
#pragma unroll
    for (int r = 0; r < 3; ++r)
      if (j_last[r] >= j && j_last[r] < k && v_last[r] < kTileN) k = j_last[r];
    return k;
  }
  __device__ __forceinline__ int operator()(int j) const {
    return j == j_last[0] ? v_last[0] : (j == j_last[1] ? v_last[1] : (j == j_last[2] ? v_last[2] : dflt));
  }
};

// Partial results exchanged inside a cluster: where the K and V tiles were, O of both query tiles as
// [tile][col / 4][row][col % 4], then (m, l) as [tile][row].
constexpr int kSwapTileBytes = 128 * 128 * 4;
constexpr int kSwapMl = 2 * kSwapTileBytes;
static_assert(kSwapMl + 2 * 128 * 8 <= kSmemBar - kSmemKV, "the exchange does not fit the K and V stages");

// One row (key) of a K or V tile, codes to bf16: 128 codes at `src`, TMA's 128-byte swizzle by the row, to the two
// 64-column halves of the tile at `dst` with the same swizzle.  Eight neighbouring lanes touch different banks both
// ways.  `word`: the row's four scale bytes.
template <bool kTwoFactors>
__device__ __forceinline__ void decode_row(uint32_t src, uint32_t dst, uint32_t word, uint32_t swizzle) {
#pragma unroll 1
  for (int block = 0; block < 4; ++block) {
    const uint32_t byte = word & 255u, f1 = q8::factor1(byte);
    word >>= 8;
    const uint4 x0 = ld_shared_16(src + (((2 * block) ^ swizzle) << 4)), x1 = ld_shared_16(src + (((2 * block + 1) ^ swizzle) << 4));
    uint4 y[4] = {q8::decode8(x0.x, x0.y, f1), q8::decode8(x0.z, x0.w, f1), q8::decode8(x1.x, x1.y, f1), q8::decode8(x1.z, x1.w, f1)};
    const uint32_t to = dst + (block >> 1) * kHalfBytes;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (kTwoFactors) y[i] = q8::mul8(y[i], q8::factor2(byte));
      st_shared_16(to + (((4 * (block & 1) + i) ^ swizzle) << 4), reinterpret_cast<const uint32_t*>(&y[i]));
    }
  }
}

// kCluster: a launch of one part per block, in which the parts of an item are a cluster and merge through each
// other's shared memory.  The other form merges through global memory, where a part's stores, the fence
// with its count and the last part's loads took 5-10 us one after the other.
// kKind: kBf16, or over an 8-bit cache (kQ8).  Then tm_kf and tm_vf are maps over codes, and tm_k and tm_v are not used: the decoders write
// all rows of a tile, so that a ragged one needs no zero fill, and frames of any length lie in runs of keys.
template <bool kCluster, Kind kKind>
__global__ void __launch_bounds__(Form<kKind != kBf16>::kThreads, 1)
window_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_kf,
                   const __grid_constant__ CUtensorMap tm_vf, const AttnParams p,
                   __nv_bfloat16* __restrict__ out) {
  constexpr bool kQ8 = kKind != kBf16, lone = kKind == kQ8Lone;
  constexpr int kStages = Form<kQ8>::kStages;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t smem_base = smem_u32(smem_raw);
  if (smem_base & 1023u) {  // the 128-byte swizzle needs 1024-byte aligned tiles
    if (threadIdx.x == 0) atomicExch(&g_status, UNSTEP_ERR_CUDA);
    return;
  }
  uint8_t* gen = smem_raw;
  const uint32_t sQ = smem_base + kSmemQ;
  const uint32_t sKV = smem_base + kSmemKV;
  const uint32_t sBar = smem_base + kSmemBar;
  // mbarriers (8 bytes each)
  const uint32_t bar_q_full = sBar;                          // [2]  TMA -> Q K^T issuer
  const uint32_t bar_q_empty = sBar + 16;                    // [2]  Q K^T issuer -> TMA
  const uint32_t bar_kv_full = sBar + 32;                    // [kStages] TMA (kQ8: decoders) -> the issuer that reads the stage
  const uint32_t bar_kv_empty = sBar + 32 + 8 * kStages;     // [kStages] that issuer -> TMA
  const uint32_t bar_s_full = sBar + 32 + 16 * kStages;      // [2]  Q K^T issuer -> softmax a
  const uint32_t bar_pv_done = bar_s_full + 16;              // [2]  P V issuer -> softmax a
  const uint32_t bar_raw_full = bar_pv_done + 16;            // kQ8: [2 kRawStages] TMA -> decoders
  const uint32_t bar_raw_empty = bar_raw_full + 16 * kRawStages;  // kQ8: [2 kRawStages] decoders -> TMA
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + kSmemBar + 224);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + kSmemBar + 228);

  const int tid = threadIdx.x;
  const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);   // the same in all lanes, and known to be
  const int lane = tid & 31;
  CTRACE(0);

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_q_full + 8 * i, 1);
      mbar_init(bar_q_empty + 8 * i, 1);
      mbar_init(bar_s_full + 8 * i, 1);
      mbar_init(bar_pv_done + 8 * i, 1);
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(bar_kv_full + 8 * i, kQ8 ? 4 : 1);
      mbar_init(bar_kv_empty + 8 * i, 1);
    }
    for (int i = 0; kQ8 && i < 2 * kRawStages; ++i) {
      mbar_init(bar_raw_full + 8 * i, 1);
      mbar_init(bar_raw_empty + 8 * i, 4);
    }
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 8) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xFFFFFFFFu, *tmem_slot, 0);
  // What comes before a role's grid_wait may run under the kernel before this one.  Every role waits
  // there, so that no bounded wait counts that kernel's time.
  const Waiter w{abort_flag, kWaitCycles};

  // Buffer and phase of a tile that is the `it`-th of all and the `c`-th of its kind.
  auto kv_stage = [&](bool is_v, uint32_t it, uint32_t c) { return lone ? 2 * is_v + (c & 1) : it % kStages; };
  auto kv_phase = [&](uint32_t it, uint32_t c) { return lone ? c >> 1 : it / kStages; };
  auto raw_stage = [&](bool is_v, uint32_t it, uint32_t c) { return lone ? kRawStages * is_v + (c & 1) : it % kRawStages; };
  auto raw_phase = [&](uint32_t it, uint32_t c) { return lone ? c >> 1 : it / kRawStages; };
  auto raw_buffer = [&](uint32_t stage) {
    return smem_base + (stage < kRawStages ? kSmemRaw + stage * kRawBytes : kSmemQ + kTileBytes + (stage - kRawStages) * kRawBytes);
  };
  // kQ8, a decoding warp: thread `row` has that row (key) of every tile, lone: of every K tile or every V tile.  Its scale word
  // comes straight from global memory, a tile ahead.
  auto decode_tiles = [&](const int row, const bool values) {
    Sched sched(p, static_cast<int>(blockIdx.x));
    Seg s;
    const uint32_t swizzle = row & 7;
    uint32_t c0 = 0;   // tiles of a kind before this segment
    bool ok = true;
    while (ok && sched.next(s)) {
      const int tiles = s.t1 - s.t0, n = lone ? tiles : 2 * tiles;
      // The i-th tile: lone, of its kind; else they come as K of the first, then K and V in turn, V of the last.
      auto is_value = [&](int i) { return lone ? values : i > 0 && ((i & 1) == 0 || i == n - 1); };
      auto index = [&](int i) { return lone ? i : i == n - 1 ? tiles - 1 : is_value(i) ? i / 2 - 1 : (i + 1) / 2; };
      auto word_of = [&](int i) {
        const TileInfo ti = tile_info(p, s.b, s.t0 + index(i));
        if (row >= ti.valid) return 0u;   // nobody attends it: any finite value will do
        return ld_global_4((is_value(i) ? p.scale_v : p.scale_k) + (s.b * p.cache_rows + ti.row + row) * p.Hn + s.h);
      };
      uint32_t ahead = word_of(0);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const uint32_t word = ahead;
        if (i + 1 < n) ahead = word_of(i + 1);
        const uint32_t it = 2 * c0 + i, c = c0 + i;   // lone or not, only one of them is looked at
        const bool is_v = lone && values;
        const uint32_t raw = raw_stage(is_v, it, c), st = kv_stage(is_v, it, c);
        ok = w.wait_warp(bar_raw_full + 8 * raw, raw_phase(it, c) & 1);
        if (ok) ok = w.wait_warp(bar_kv_empty + 8 * st, (kv_phase(it, c) & 1) ^ 1);
        if (!ok) break;
        const uint32_t src = raw_buffer(raw) + row * 128, dst = sKV + st * kTileBytes + row * 128;
        if (__all_sync(0xFFFFFFFFu, __vcmpgtu4(word, 0x86868686u) == 0u)) decode_row<false>(src, dst, word, swizzle);
        else decode_row<true>(src, dst, word, swizzle);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar_kv_full + 8 * st);
          mbar_arrive(bar_raw_empty + 8 * raw);
        }
      }
      c0 += tiles;
    }
  };

  const bool softmax_role = lone ? warp < 4 : warp < 8;
  if (kQ8 && (warp >= 12 || (lone && !softmax_role && warp < 8))) {
    // ---------------------------------------------------------------- decoders
    // (one copy of the code for both groups of a lone launch)
    reg_dealloc_decode();
    grid_wait();
    decode_tiles(tid & 127, warp < 8);
  } else if (warp >= 8) {
    reg_dealloc_service<kQ8>();
    if (warp == 10 && lane == 0) {
      // ------------------------------------------------------------ TMA producer
      prefetch_tensormap(&tm_q);
      prefetch_tensormap(&tm_k);
      prefetch_tensormap(&tm_v);
      prefetch_tensormap(&tm_kf);
      prefetch_tensormap(&tm_vf);
      grid_wait();
      Sched sched(p, static_cast<int>(blockIdx.x));
      Seg s;
      uint32_t kv_it = 0, q_it[2] = {0, 0}, kv_c[2] = {0, 0};   // kv_c: kQ8, K and V tiles
      bool ok = true;
      while (ok && sched.next(s)) {
        auto load_q = [&](int a) {
          if (!ok || a >= s.nq) return;
          ok = w.wait(bar_q_empty + 8 * a, (q_it[a] & 1) ^ 1);
          if (!ok) return;
          const uint32_t dst = sQ + a * kTileBytes, bar = bar_q_full + 8 * a;
          const int n0 = (2 * s.qp + a) * kTileM;
          mbar_expect_tx(bar, kTileBytes);
          tma_load_4d(dst, &tm_q, bar, 0, s.h, n0, s.b);
          tma_load_4d(dst + kHalfBytes, &tm_q, bar, 64, s.h, n0, s.b);
          ++q_it[a];
        };
        auto load_kv = [&](const TileInfo& ti, int kv) {
          if constexpr (kQ8) {
            const uint32_t raw = raw_stage(kv == 1, kv_it, kv_c[kv]), bar = bar_raw_full + 8 * raw;
            if (ok) ok = w.wait(bar_raw_empty + 8 * raw, (raw_phase(kv_it, kv_c[kv]) & 1) ^ 1);
            if (!ok) return;
            mbar_expect_tx(bar, kRawBytes);
            tma_load_4d(raw_buffer(raw), kv == 0 ? &tm_kf : &tm_vf, bar, 0, s.h, ti.row, s.b);
            ++kv_it;
            ++kv_c[kv];
            return;
          }
          const uint32_t st = kv_it % kStages;
          if (ok) ok = w.wait(bar_kv_empty + 8 * st, ((kv_it / kStages) & 1) ^ 1);
          if (!ok) return;
          const uint32_t dst = sKV + st * kTileBytes, bar = bar_kv_full + 8 * st;
          mbar_expect_tx(bar, kTileBytes);
          if (ti.framed) {
            const CUtensorMap* tm = kv == 0 ? &tm_k : &tm_v;
            tma_load_5d(dst, tm, bar, 0, s.h, ti.tok0, ti.slot, s.b);
            tma_load_5d(dst + kHalfBytes, tm, bar, 64, s.h, ti.tok0, ti.slot, s.b);
          } else {
            const CUtensorMap* tm = kv == 0 ? &tm_kf : &tm_vf;
            tma_load_4d(dst, tm, bar, 0, s.h, ti.row, s.b);
            tma_load_4d(dst + kHalfBytes, tm, bar, 64, s.h, ti.row, s.b);
          }
          ++kv_it;
        };
        load_q(0);   // what the first S needs comes first: Q of tile 0, then K
        TileInfo ti = tile_info(p, s.b, s.t0);
        load_kv(ti, 0);
        load_q(1);
        for (int j = s.t0; j < s.t1 && ok; ++j) {
          TileInfo tn = ti;
          if (j + 1 < s.t1) {
            tn = tile_info(p, s.b, j + 1);
            load_kv(tn, 0);
          }
          load_kv(ti, 1);
          ti = tn;
        }
      }
    } else if (warp == 8) {
      // ------------------------------------------------------------ Q K^T issuer
      // The K and V tiles come in the order in which they are used: K of tile 0, then K of tile j + 1 and V
      // of tile j.  The whole warp runs the code (the loops stay rolled: instruction fetch is scarce).
      grid_wait();
      Sched sched(p, static_cast<int>(blockIdx.x));
      Seg s;
      uint32_t kv_base = 0, n0 = 0, n1 = 0, q0 = 0, q1 = 0;   // tiles and items per group
      int before = -1;   // group whose scores are in S
      bool ok = true;
      const uint32_t idesc_full = idesc_bf16_f32(kTileM, kTileN, 0);
      const uint64_t dq = smem_desc_sw128(sQ, 16, 1024);    // Q tile 0, K-major
      const uint64_t dk0 = smem_desc_sw128(sKV, 16, 1024);  // stage 0 as a K tile
      while (sched.next(s)) {
        const int n = s.t1 - s.t0;
        const ValidKeys valid_of(p, s.b);
        for (int j = 0; j < n; ++j) {
          const uint32_t it = kv_base + (j > 0 ? 2 * j - 1 : 0), st = kv_stage(false, it, kv_base / 2 + j);   // K's place in the order
          const int valid = valid_of(s.t0 + j);
          const uint32_t idesc = valid == kTileN ? idesc_full : idesc_bf16_f32(kTileM, (valid + 15) & ~15, 0);
          const uint64_t dk = dk0 + static_cast<uint64_t>((st * kTileBytes) >> 4);
#pragma unroll 1
          for (int a = 0; a < s.nq; ++a) {
            if (ok && j == 0) ok = w.wait_warp(bar_q_full + 8 * a, (a == 0 ? q0 : q1) & 1);
            if (ok && a == 0) ok = w.wait_warp(bar_kv_full + 8 * st, kv_phase(it, kv_base / 2 + j) & 1);
            TRACE(2, n0 + n1, 0);
            if (before >= 0) s_free_sync(before, (before == 0 ? n0 : n1) - 1);
            TRACE(2, n0 + n1, 1);
            if (ok) {
              tc_fence_after();
              mma_ss_k128(tmem_base + kTmemS, dq + static_cast<uint64_t>((a * kTileBytes) >> 4), dk, idesc, 0u);
            }
            if (ok) {
              tc_commit(bar_s_full + 8 * a);
              if (a == s.nq - 1) tc_commit(bar_kv_empty + 8 * st);
              if (j == n - 1) tc_commit(bar_q_empty + 8 * a);
            }
            TRACE(2, n0 + n1, 2);
            if (j == 0) ++(a == 0 ? q0 : q1);
            ++(a == 0 ? n0 : n1);
            before = a;
          }
        }
        kv_base += 2 * n;
      }
      if (before >= 0) s_free_sync(before, (before == 0 ? n0 : n1) - 1);
    } else if (warp == 9) {
      // ------------------------------------------------------------ P V issuer
      // The commits that free a stage come behind those that a softmax group waits for, but for the segment's last one:
      // behind that the kernel may end.
      grid_wait();
      Sched sched(p, static_cast<int>(blockIdx.x));
      Seg s;
      uint32_t kv_base = 0, n0 = 0, n1 = 0;
      bool ok = true;
      const uint32_t idesc_pv = idesc_bf16_f32(kTileM, kHeadDim, 1);
      const uint64_t dv0 = smem_desc_sw128(sKV, kHalfBytes, 1024);          // stage 0 as a V tile (MN-major)
      while (sched.next(s)) {
        const int n = s.t1 - s.t0;
        const ValidKeys valid_of(p, s.b);
        for (int j = 0; j < n; ++j) {
          const uint32_t it = kv_base + (j + 1 < n ? 2 * j + 2 : 2 * n - 1), st = kv_stage(true, it, kv_base / 2 + j);
          const int k_steps = (valid_of(s.t0 + j) + 15) >> 4;
          const uint64_t dv = dv0 + static_cast<uint64_t>((st * kTileBytes) >> 4);
          if (ok) ok = w.wait_warp(bar_kv_full + 8 * st, kv_phase(it, kv_base / 2 + j) & 1);
#pragma unroll 1
          for (int a = 0; a < s.nq; ++a) {
            const uint32_t o_tmem = tmem_base + kTmemO + a * 128, p_tmem = tmem_base + kTmemP + a * 64;
            TRACE(3, n0 + n1, 0);
            p_ready_sync(a, a == 0 ? n0 : n1);   // P of this tile is in TMEM, O rescaled if need be
            TRACE(3, n0 + n1, 1);
            if (ok) {
              tc_fence_after();
              if (k_steps == 8) {
                mma_ts_k64(o_tmem, p_tmem, dv, idesc_pv, j > 0 ? 1u : 0u);
                mma_ts_k64(o_tmem, p_tmem + 32, dv + 512u, idesc_pv, 1u);
              } else {
#pragma unroll 1
                for (int k = 0; k < k_steps; ++k)
                  mma_ts(o_tmem, p_tmem + k * 8, dv + static_cast<uint64_t>(k * 128), idesc_pv, (j > 0 || k > 0) ? 1u : 0u);
              }
            }
            if (ok) {
              const bool last_of_stage = a == s.nq - 1;
              if (last_of_stage && j == n - 1) tc_commit(bar_kv_empty + 8 * st);
              tc_commit(bar_pv_done + 8 * a);
              if (last_of_stage && j < n - 1) tc_commit(bar_kv_empty + 8 * st);
            }
            TRACE(3, n0 + n1, 2);
            ++(a == 0 ? n0 : n1);
          }
        }
        kv_base += 2 * n;
      }
    }
  } else {
    // ---------------------------------------------------------------- softmax warpgroups
    // Warps 0-3 own query tile 0, warps 4-7 query tile 1; a thread owns a row from the scores
    // to the output.
    reg_alloc_softmax<kQ8>();
    grid_wait();
    const int a = warp >> 2;               // query tile of this warpgroup
    const int row = tid & 127;             // row inside the tile = TMEM lane
    const uint32_t t_lane = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t t_S = t_lane + kTmemS, t_P = t_lane + kTmemP + a * 64, t_O = t_lane + kTmemO + a * 128;
    Sched sched(p, static_cast<int>(blockIdx.x));
    Seg s;
    Seg seg = {};        // of a cluster's block: its only one
    uint32_t it = 0, s_seen = 0;
    bool ok = true;
    int seg_no = 0;
    CTRACE(1);
    // After a wait gave up (ok == false) a warp keeps walking its segments without working, so that
    // it still meets its group and its issuer at every named barrier.  ok is the same in all threads
    // of a warp: barriers and TMEM accesses are instructions of the whole warp.
    while (sched.next(s)) {
      if (kCluster) seg = s;
      if (a >= s.nq) continue;             // a lone last query tile: nothing for group 1
      float m_run = -INFINITY, l_run = 0.f;
      const ValidKeys valid_of(p, s.b);
      const uint32_t pv = bar_pv_done + 8 * a, sb = bar_s_full + 8 * a;
      // scores of tile `it`: true unless the wait gave up, in which case the issuers still count on this warp
      auto scores = [&](uint32_t tile) {
        if (ok && __builtin_expect(!__all_sync(0xFFFFFFFFu, s_seen), 0)) ok = w.wait_warp(sb, tile & 1);
        s_seen = 0;
        if (__builtin_expect(!ok, 0)) {
          s_free_pass(a, tile, true);
          p_ready_pass(a, tile, true);
          return false;
        }
        tc_fence_after();
        return true;
      };
      int j = s.t0;
#pragma unroll 1
      while (j < s.t1) {
        {   // the segment's first tile, or a ragged one
          const int valid = valid_of(j);
          TRACE(a, it, 0);
          if (scores(it)) {
            TRACE(a, it, 1);
            const bool first = j == s.t0;
            if (valid <= 64)   // frames of at most half a tile, and the end of a run
              ok = softmax_row_tile<true, 64, false>(t_S, t_P, t_O, p.scale_log2e, valid, first, m_run, l_run, a, it, w, pv, sb, s_seen);
            else
              ok = softmax_row_tile<true, kTileN, false>(t_S, t_P, t_O, p.scale_log2e, valid, first, m_run, l_run, a, it, w, pv, sb, s_seen);
            if (!ok) p_ready_pass(a, it, true);
          }
          ++j;
          ++it;
        }
        const int jf = valid_of.full_until(j, s.t1);
#pragma unroll 1
        for (; j < jf; ++j, ++it) {
          TRACE(a, it, 0);
          if (scores(it)) {
            TRACE(a, it, 1);
            ok = softmax_row_tile<false, kTileN, true>(t_S, t_P, t_O, p.scale_log2e, kTileN, false, m_run, l_run, a, it, w, pv, sb, s_seen);
            if (__builtin_expect(!ok, 0)) p_ready_pass(a, it, true);
          }
        }
      }
      CTRACE(8 + seg_no);
      // ---- epilogue of this group's query tile ----
      const bool whole = (s.t0 == 0 && s.t1 == s.tiles);
      // Part of a split item: the arrival counter, looked at under the wait for the last P V
      auto counter = [&] { return p.counters + 2 * s.item + a; };
      int seen = 0;
      if (!kCluster && !whole && row == 0) {
#ifdef UNSTEP_CHECK
        if (2 * s.item + a >= p.extent_counters) atomicExch(p.status, static_cast<int>(UNSTEP_ERR_BOUNDS));
#endif
        asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(counter()) : "memory");
      }
      if (ok) {
        ok = w.wait_warp(bar_pv_done + 8 * a, (it - 1) & 1);
        tc_fence_after();
      }
      const int n = (2 * s.qp + a) * kTileM + row;
      uint4* const out_v = reinterpret_cast<uint4*>(out);
      const int64_t dst = ((static_cast<int64_t>(s.b) * p.L + n) * p.Hn + s.h) * (kHeadDim / 8);   // 16-byte vectors
      auto store_row = [&](int64_t d, const float* v, float inv_l) {   // 32 columns from vector d on
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = pack_bf16x2(v[2 * i] * inv_l, v[2 * i + 1] * inv_l);
        if (p.out_wide) {   // whole 32-byte sectors
          UNSTEP_STORE_32(out_v, d, p.extent_out, w, p.status);
          UNSTEP_STORE_32(out_v, d + 2, p.extent_out, w + 8, p.status);
          return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          UNSTEP_STORE(out_v, d + i, p.extent_out, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]),
                       p.status);
      };
      if (kCluster) {
        // Every block of a cluster holds one part of the same item.  Each puts its part into its own shared memory and
        // then merges a share of the columns of all rows, in part order, reading the others' parts there.
        if (s.nq == 2) asm volatile("bar.sync %0, 256;" ::"r"(kSwapBarrier) : "memory");   // the stages are free behind both P V
        const uint32_t mine = sKV + a * kSwapTileBytes + row * 16;
        if (ok) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t o[32];
            tmem_ld32(t_O + q * 32, o);
            tc_wait_ld32(o);
#pragma unroll
            for (int i = 0; i < 8; ++i) st_shared_16(mine + (q * 8 + i) * 2048, o + 4 * i);
          }
          st_shared_8(sKV + kSwapMl + a * 1024 + row * 8, __float_as_uint(m_run), __float_as_uint(l_run));
        }
      } else if (whole) {
        // O / l -> bf16 -> out[b][n][h][:]: a thread writes its whole 256-byte row
        if (ok) {
          const float inv_l = 1.f / l_run;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float o[32];
            tmem_ld32(t_O + q * 32, reinterpret_cast<uint32_t*>(o));
            tc_wait_ld32(reinterpret_cast<uint32_t*>(o));
            if (n < p.L) store_row(dst + 4 * q, o, inv_l);
          }
        }
      } else {
        // Part of a split item.  The parts of an item's query tile are merged by whichever of
        // them is done last, in part order (a fixed order, so the result does not depend on
        // which one that is); the merging part takes its own accumulator straight from TMEM.
        // A part that finds all others already published merges at once without publishing
        // itself; otherwise it publishes (O, m, l), counts itself in, and merges if that made
        // the count complete.
        const int c_lo = first_part_worker(p, s);
        const int c_hi = last_part_worker(p, s);
        const int others = c_hi - c_lo;
        // one thread says whether all others are in, the others whether their warp gave up (31 or
        // more do then); a group that gave up publishes nothing
        const uint32_t votes = group_count(a, row == 0 ? seen == others : !ok);
        if (votes > 1) ok = false;
        bool last = votes == 1;
        if (ok && !last) {
          const int64_t mine = (static_cast<int64_t>(2 * blockIdx.x + (s.first_in_worker ? 0 : 1)) * kPartFloats +
                                a * kPartTileFloats);   // first float of this part in the scratch
          float4* const part4 = reinterpret_cast<float4*>(p.part);
          const int64_t mine4 = mine / 4 + row;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t o[32];
            tmem_ld32(t_O + q * 32, o);
            tc_wait_ld32(o);
#pragma unroll
            for (int i = 0; i < 8; ++i)
              UNSTEP_STORE(part4, mine4 + (q * 8 + i) * 128, p.extent_part / 4,
                           make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                       __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3])),
                           p.status);
          }
          UNSTEP_STORE(reinterpret_cast<float2*>(p.part), mine / 2 + 128 * 64 + row, p.extent_part / 2,
                       make_float2(m_run, l_run), p.status);
          group_barrier(a);   // all of this part is stored
          int before = -1;
          if (row == 0) {
            // release: the group's stores (ordered before this thread by the barrier) become visible
            // before the count; acquire: a merging part sees the other parts' stores
            asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter()) : "memory");
          }
          last = group_count(a, before == others) != 0;
        }
        if (ok && last) {
          __threadfence();   // acquire side for every thread that reads the other parts below
          if (row == 0) UNSTEP_STORE(p.counters, 2 * s.item + a, p.extent_counters, 0, p.status);   // ready for the next launch
          const int me = static_cast<int>(blockIdx.x);
          const int lo_slot = part_slot(p, c_lo, s.item_step0);   // every later part starts its worker's range
          auto part_of = [&](int c) -> const float* {
            return p.part + (static_cast<int64_t>(2 * c + (c == c_lo ? lo_slot : 0)) * kPartFloats + a * kPartTileFloats);
          };
          auto ml_of = [&](int c) -> float2 {
            return c == me ? make_float2(m_run, l_run)
                           : __ldcg(reinterpret_cast<const float2*>(part_of(c) + 128 * 128) + row);
          };
          float m_all = m_run, l_sum = 0.f;
          if (others <= 3) {   // one round trip for all parts
            float2 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = i <= others ? ml_of(c_lo + i) : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) m_all = fmaxf(m_all, x[i].x);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (i <= others) l_sum += x[i].y * ex2((x[i].x - m_all) * p.scale_log2e);
          } else {
#pragma unroll 4
            for (int c = c_lo; c <= c_hi; ++c) m_all = fmaxf(m_all, ml_of(c).x);
#pragma unroll 4
            for (int c = c_lo; c <= c_hi; ++c) {
              const float2 x = ml_of(c);
              l_sum += x.y * ex2((x.x - m_all) * p.scale_log2e);
            }
          }
          const float inv_l = 1.f / l_sum;
#pragma unroll 1
          for (int q = 0; q < 2; ++q) {   // 64 output columns at a time
            float acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = 0.f;
            for (int c = c_lo; c <= c_hi; ++c) {
              if (c == me) {
                const float sc = ex2((m_run - m_all) * p.scale_log2e);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  uint32_t o[32];
                  tmem_ld32(t_O + 64 * q + 32 * h, o);
                  tc_wait_ld32(o);
#pragma unroll
                  for (int i = 0; i < 32; ++i) acc[32 * h + i] = fmaf(__uint_as_float(o[i]), sc, acc[32 * h + i]);
                }
              } else {
                const float4* pc = reinterpret_cast<const float4*>(part_of(c)) + q * 16 * 128 + row;
                float4 v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __ldcg(pc + i * 128);
                const float sc = ex2((ml_of(c).x - m_all) * p.scale_log2e);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  acc[4 * i] = fmaf(v[i].x, sc, acc[4 * i]);
                  acc[4 * i + 1] = fmaf(v[i].y, sc, acc[4 * i + 1]);
                  acc[4 * i + 2] = fmaf(v[i].z, sc, acc[4 * i + 2]);
                  acc[4 * i + 3] = fmaf(v[i].w, sc, acc[4 * i + 3]);
                }
              }
            }
            if (n < p.L) {
              store_row(dst + 8 * q, acc, inv_l);
              store_row(dst + 8 * q + 4, acc + 32, inv_l);
            }
          }
        }
      }
      tc_fence_before();
      CTRACE(3 + seg_no);
      ++seg_no;
    }
    if (kCluster) {
      __syncwarp();
      cluster_sync();   // all parts are in place
      const int parts = p.parts, part = static_cast<int>(cluster_rank());
      // a lone query tile is shared out to both groups
      const bool whole_share = lone || seg.nq == 2;
      const int tile = seg.nq == 2 ? a : 0, share = whole_share ? part : 2 * part + a, shares = whole_share ? parts : 2 * parts;
      const int n = (2 * seg.qp + tile) * kTileM + row;
      bool good = seg.nq > 0;
      for (int c = 0; c < parts; ++c)   // a block that gave up has left no part
        good = good && ld_cluster_4(cluster_addr(smem_u32(const_cast<int*>(abort_flag)), c)) == 0;
      if (good && n < p.L) {
        float2 x[kMaxClusterParts];
        float m_all = -INFINITY, l_sum = 0.f;
#pragma unroll
        for (int c = 0; c < kMaxClusterParts; ++c)
          x[c] = c < parts ? ld_cluster_8(cluster_addr(sKV + kSwapMl + tile * 1024 + row * 8, c)) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int c = 0; c < kMaxClusterParts; ++c) m_all = fmaxf(m_all, x[c].x);
#pragma unroll
        for (int c = 0; c < kMaxClusterParts; ++c)
          if (c < parts) {
            x[c].x = ex2((x[c].x - m_all) * p.scale_log2e);
            l_sum += x[c].y * x[c].x;
          }
        const float inv_l = 1.f / l_sum;
        uint4* const out_v = reinterpret_cast<uint4*>(out);
        const int64_t dst = ((static_cast<int64_t>(seg.b) * p.L + n) * p.Hn + seg.h) * (kHeadDim / 8);   // 16-byte vectors
        const uint32_t from = sKV + tile * kSwapTileBytes + row * 16;
#pragma unroll 2
        for (int v = 16 * share / shares; v < 16 * (share + 1) / shares; ++v) {
          float acc[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] = 0.f;
#pragma unroll
          for (int c = 0; c < kMaxClusterParts; ++c)
            if (c < parts) {
              const uint32_t at = cluster_addr(from + v * 4096, c);
              const float4 u0 = ld_cluster_16(at), u1 = ld_cluster_16(at + 2048);
              acc[0] = fmaf(u0.x, x[c].x, acc[0]);
              acc[1] = fmaf(u0.y, x[c].x, acc[1]);
              acc[2] = fmaf(u0.z, x[c].x, acc[2]);
              acc[3] = fmaf(u0.w, x[c].x, acc[3]);
              acc[4] = fmaf(u1.x, x[c].x, acc[4]);
              acc[5] = fmaf(u1.y, x[c].x, acc[5]);
              acc[6] = fmaf(u1.z, x[c].x, acc[6]);
              acc[7] = fmaf(u1.w, x[c].x, acc[7]);
            }
          UNSTEP_STORE(out_v, dst + v, p.extent_out,
                       make_uint4(pack_bf16x2(acc[0] * inv_l, acc[1] * inv_l), pack_bf16x2(acc[2] * inv_l, acc[3] * inv_l),
                                  pack_bf16x2(acc[4] * inv_l, acc[5] * inv_l), pack_bf16x2(acc[6] * inv_l, acc[7] * inv_l)),
                       p.status);
        }
      }
    }
  }
  // The other roles meet the softmax groups at the cluster's barrier, and no block leaves while another reads its part.
  if (kCluster) {
    if (!softmax_role) {
      __syncwarp();
      cluster_sync();
    }
    __syncwarp();
    cluster_sync();
  }

  // ---- teardown: every role ends here, also after a timed-out wait --------------------
  tc_fence_before();
  __syncthreads();
  if (warp == 10 && lane == 0 && *abort_flag) {
    // gave up: let copies that are still in flight land (bounded) before smem is released
    const long long t0 = clock64();
    while (clock64() - t0 < 4000000LL) {
    }
  }
  __syncthreads();
  if (warp == 8) tmem_dealloc(tmem_base, kTmemCols);
  CTRACE(7);
}

// A wait on a barrier that nothing ever arrives at, with a short limit: exercises the give-up
// path of Waiter (status word, flag, orderly return) without any other work.
__global__ void wait_limit_probe_kernel(long long limit_cycles) {
  __shared__ __align__(8) uint64_t bar;
  __shared__ int abort_flag;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&bar), 1);
    abort_flag = 0;
    mbar_fence_init();
  }
  __syncthreads();
  const Waiter w{&abort_flag, limit_cycles};
  w.wait(smem_u32(&bar), 0);
  __syncthreads();
}

// --------------------------------------------------------------------------
// Keys and values of an 8-bit cache's windows as bf16, for launches that read them often: per stream and head the
// keys of the window in order, padded with zeros to whole tiles.  A thread decodes 16 dims of k and v of kUnpackRows
// rows, 32 apart; eight threads have a row of a head, 128 bytes in and 256 out.  DRAM bound: 32760 keys x 12 heads
// (305 MB) 46 us, 6.6 TB/s.
// --------------------------------------------------------------------------
constexpr int kUnpackRows = 2;
struct Unpack8Params {
  int32_t Hn, head0, rows;             // heads of the cache, first head of this launch, rows that the output has for a stream
  int64_t cache_rows;
  int32_t run_row0[kMaxStreamsPerLaunch][3], run_end[kMaxStreamsPerLaunch][3];   // rows of the runs, added up
  int* status;
  int64_t extent;                      // 16-byte vectors of an output
};

__device__ __forceinline__ void store_unpacked(uint4* out, int64_t dst, int64_t extent, uint4 x, uint32_t byte, int* status) {
  const uint32_t f1 = q8::factor1(byte);
  uint4 y[2] = {q8::decode8(x.x, x.y, f1), q8::decode8(x.z, x.w, f1)};
  if (!q8::one_factor(byte)) {
    const uint32_t f2 = q8::factor2(byte);
    y[0] = q8::mul8(y[0], f2);
    y[1] = q8::mul8(y[1], f2);
  }
  UNSTEP_STORE_32(out, dst, extent, reinterpret_cast<const uint32_t*>(y), status);
}

__global__ void __launch_bounds__(256)
window_unpack_q8_kernel(const __grid_constant__ Unpack8Params p, const uint4* cache_k, const uint8_t* scale_k, const uint4* cache_v,
                        const uint8_t* scale_v, uint4* out_k, uint4* out_v) {
  grid_launch_next();
  const int b = blockIdx.z, h = blockIdx.y, vec = threadIdx.x & 7;
  const int row0 = static_cast<int>(blockIdx.x) * 32 * kUnpackRows + (threadIdx.x >> 3);
  const int behind = grid_wait();
  uint4 xk[kUnpackRows], xv[kUnpackRows];
  uint32_t ek[kUnpackRows], ev[kUnpackRows];
#pragma unroll
  for (int i = 0; i < kUnpackRows; ++i) {
    const int r = row0 + 32 * i;
    xk[i] = xv[i] = make_uint4(0, 0, 0, 0);
    ek[i] = ev[i] = q8::kLeastByte;
    if (r < p.run_end[b][2]) {
      const int run = r < p.run_end[b][0] ? 0 : (r < p.run_end[b][1] ? 1 : 2);
      const int row = p.run_row0[b][run] + r - (run == 0 ? 0 : p.run_end[b][run - 1]);
      const int64_t src = ((b * p.cache_rows + row) * p.Hn + p.head0 + h) * 8 + vec + behind;
      xk[i] = __ldcs(cache_k + src);
      xv[i] = __ldcs(cache_v + src);
      ek[i] = __ldca(scale_k + (src >> 1));
      ev[i] = __ldca(scale_v + (src >> 1));
    }
  }
#pragma unroll
  for (int i = 0; i < kUnpackRows; ++i) {
    const int r = row0 + 32 * i;
    if (r < (p.run_end[b][2] + kTileN - 1) / kTileN * kTileN) {
      const int64_t dst = 2 * (((static_cast<int64_t>(b) * gridDim.y + h) * p.rows + r) * 8 + vec);
      store_unpacked(out_k, dst, p.extent, xk[i], ek[i], p.status);
      store_unpacked(out_v, dst, p.extent, xv[i], ev[i], p.status);
    }
  }
}

// --------------------------------------------------------------------------
// Host side
// --------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

static EncodeTiledFn get_encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* sym = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(sym);
  });
  return fn;
}

// bf16 (or code) tensor map with 128-byte swizzle, box = 64 (128) elements x 128 rows of dimension `row_dim`.
static bool make_map(CUtensorMap* m, const void* base, int rank, const uint64_t* dims,
                     const uint64_t* strides_bytes, int row_dim, bool codes = false) {
  EncodeTiledFn fn = get_encode_fn();
  if (fn == nullptr) return false;
  cuuint64_t gdim[5], gstride[4];
  cuuint32_t box[5], estr[5];
  for (int i = 0; i < rank; ++i) {
    gdim[i] = dims[i];
    box[i] = 1;
    estr[i] = 1;
    if (i > 0) gstride[i - 1] = strides_bytes[i - 1];
  }
  box[0] = codes ? 128 : 64;
  box[row_dim] = 128;
  return fn(m, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), gdim, gstride, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct DeviceInfo {
  bool ok = false;
  int sm_count = 0;
  int32_t clusters[kKinds][kMaxClusterParts + 1] = {};   // clusters of that many blocks which the device runs at the same time
};

template <Kind kKind>
static bool query_kernels(int32_t* clusters) {
  if (cudaFuncSetAttribute(window_attn_kernel<false, kKind>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmemBytes) != cudaSuccess ||
      cudaFuncSetAttribute(window_attn_kernel<true, kKind>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmemBytes) != cudaSuccess)
    return false;
  for (int parts = 2; parts <= kMaxClusterParts; ++parts) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = parts;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(parts);
    cfg.blockDim = dim3(Form<kKind != kBf16>::kThreads);
    cfg.dynamicSmemBytes = kAttnSmemBytes;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, window_attn_kernel<true, kKind>, &cfg) == cudaSuccess) clusters[parts] = n;
    else cudaGetLastError();   // no clusters of that size, then
  }
  return true;
}

// Set up and queried once per device and process; each thread keeps a copy for the device it uses.
static DeviceInfo query_device(int dev) {
  static std::mutex mutex;
  static std::map<int, DeviceInfo> known;
  std::lock_guard<std::mutex> lock(mutex);
  auto it = known.find(dev);
  if (it != known.end()) return it->second;
  DeviceInfo info;
  info.ok = cudaDeviceGetAttribute(&info.sm_count, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess &&
            query_kernels<kBf16>(info.clusters[kBf16]) &&
            query_kernels<kQ8Pairs>(info.clusters[kQ8Pairs]) && query_kernels<kQ8Lone>(info.clusters[kQ8Lone]);
  if (!info.ok) return info;
  return known[dev] = info;
}

static const DeviceInfo& device_info() {
  static thread_local int cached_dev = -1;
  static thread_local DeviceInfo info;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    info.ok = false;
    return info;
  }
  if (dev != cached_dev || !info.ok) {
    info = query_device(dev);
    cached_dev = dev;
  }
  return info;
}

// Scratch for split items, one per (device, stream): calls on one stream run in order and may
// share it; calls on different streams may overlap on the GPU and must not.  Captured graphs hold
// its addresses, so nothing is given back before unstep_shutdown().  The partial results have two
// slots per SM whatever the launch: the workers of a launch go up and down with the start frame (one
// to all SMs), and a buffer sized by them would move under graphs captured before.  The counters
// go by the work items of the shape and at least double when they grow, so the arrays they have
// left behind are together no larger than the one in use.
struct Workspace {
  float* part = nullptr;
  int* counters = nullptr;
  size_t slots = 0, n_counters = 0;
};
constexpr size_t kLeastCounters = 4096;
constexpr int kMaxGrowths = 32;
constexpr size_t kLeastWindow = size_t{16} << 20;
constexpr int kWindowSizes = 5;                                           // up to 256 MB
constexpr size_t kMostWindow = kLeastWindow << (kWindowSizes - 1);
struct StreamScratch {
  Workspace ws;
  Workspace left[kMaxGrowths];   // counters of former calls; captured graphs may still count in them
  int n_left = 0;
  // unpacked windows of an 8-bit cache: the last one is in use, the smaller ones may be in captured graphs
  void* window[kWindowSizes] = {};
  int n_windows = 0;             // window[i] has kLeastWindow << i bytes, or is null
  std::mutex window_turn;        // held by the call whose launches hand data on through a window (window_turn below)
};
static std::mutex g_ws_mutex;
// (device, stream, host thread): the handle cudaStreamPerThread means another stream in every host thread, so there the
// thread counts too (by a number of its own: the system gives the id of a thread that has ended to another one, whose
// stream could overlap what the ended one left under way); it is 0 with every other handle.
typedef std::tuple<int, cudaStream_t, uint64_t> ScratchKey;
static std::map<ScratchKey, StreamScratch> g_workspaces;
static ScratchKey scratch_key(int dev, cudaStream_t st) {
  static std::atomic<uint64_t> threads{0};
  static thread_local uint64_t number = 0;
  if (st != cudaStreamPerThread) return ScratchKey(dev, st, 0);
  if (number == 0) number = ++threads;
  return ScratchKey(dev, st, number);
}

static int get_workspace(cudaStream_t st, size_t slots, size_t n_counters, Workspace* out) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return UNSTEP_ERR_CUDA;
  std::lock_guard<std::mutex> lock(g_ws_mutex);
  StreamScratch& s = g_workspaces[scratch_key(dev, st)];
  Workspace& ws = s.ws;
  if (ws.part == nullptr) {
    if (cudaMalloc(&ws.part, slots * kPartFloats * sizeof(float)) != cudaSuccess) {
      ws.part = nullptr;
      return UNSTEP_ERR_CUDA;
    }
    ws.slots = slots;
  }
  if (ws.n_counters < n_counters) {
    size_t n = ws.n_counters > 0 ? 2 * ws.n_counters : kLeastCounters;
    while (n < n_counters) n *= 2;
    int* counters = nullptr;
    if (s.n_left == kMaxGrowths || cudaMalloc(&counters, n * sizeof(int)) != cudaSuccess) return UNSTEP_ERR_CUDA;
    // cleared on the caller's stream, so that the clear is ordered before the kernel that follows
    // (a non-blocking stream is not ordered against the legacy default stream)
    if (cudaMemsetAsync(counters, 0, n * sizeof(int), st) != cudaSuccess) {
      cudaFree(counters);
      return UNSTEP_ERR_CUDA;
    }
    if (ws.counters != nullptr) s.left[s.n_left++] = ws;
    ws.counters = counters;
    ws.n_counters = n;
  }
  *out = ws;
  return UNSTEP_OK;
}

// The turn of a call whose launches hand data on through the window buffer of this stream.  Stream order keeps one call's
// launches from the next one's only if they are enqueued one behind the other, and another host thread may be in a call on the
// same stream: so the turn is taken before the buffer is looked up and kept until the last launch that reads it is
// enqueued.  (The calls that launch one kernel need none: it finds its scratch idle and leaves it so.)  g_ws_mutex is taken
// for moments inside a turn, and never the other way round.
static std::unique_lock<std::mutex> window_turn(cudaStream_t st) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return std::unique_lock<std::mutex>();   // get_window finds none then
  std::unique_lock<std::mutex> lock(g_ws_mutex);
  std::mutex& turn = g_workspaces[scratch_key(dev, st)].window_turn;   // stays where it is until unstep_shutdown()
  lock.unlock();
  return std::unique_lock<std::mutex>(turn);
}

// `bytes` (at most kMostWindow) for unpacked windows on this stream, in the caller's turn; null if there is no room, or if the stream
// is being captured and the buffer would have to be made.
static void* get_window(cudaStream_t st, size_t bytes) {
  int dev = 0;
  if (bytes > kMostWindow || cudaGetDevice(&dev) != cudaSuccess) return nullptr;
  int size = 0;
  while (kLeastWindow << size < bytes) ++size;
  std::lock_guard<std::mutex> lock(g_ws_mutex);
  StreamScratch& s = g_workspaces[scratch_key(dev, st)];
  if (s.n_windows > size) return s.window[s.n_windows - 1];
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(st, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone) {
    cudaGetLastError();
    return nullptr;
  }
  void* made = nullptr;
  if (cudaMalloc(&made, kLeastWindow << size) != cudaSuccess) {
    cudaGetLastError();
    return nullptr;
  }
  s.window[size] = made;
  s.n_windows = size + 1;
  return made;
}

// After a kernel gave up, arrival counters may be left non-zero: clear them all.
static void reset_workspace_counters() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return;
  std::lock_guard<std::mutex> lock(g_ws_mutex);
  for (auto& kv : g_workspaces) {
    if (std::get<0>(kv.first) != dev) continue;
    const StreamScratch& s = kv.second;
    if (s.ws.counters != nullptr) cudaMemset(s.ws.counters, 0, s.ws.n_counters * sizeof(int));
    for (int i = 0; i < s.n_left; ++i) cudaMemset(s.left[i].counters, 0, s.left[i].n_counters * sizeof(int));
  }
}

// Device address of g_status on the current device, looked up once per device.
int* status_word() {
  static std::mutex mutex;
  static int* addr[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  std::lock_guard<std::mutex> lock(mutex);
  if (addr[dev] == nullptr) {
    void* ptr = nullptr;
    if (cudaGetSymbolAddress(&ptr, g_status) != cudaSuccess) return nullptr;
    addr[dev] = static_cast<int*>(ptr);
  }
  return addr[dev];
}

}  // namespace unstep

using namespace unstep;

// Hands out the scratch of one launch: `slots` partial-result slots (two per SM) and at least
// `n_counters` zeroed arrival counters.
typedef int (*ScratchFn)(cudaStream_t st, size_t slots, size_t n_counters, Workspace* out);   // an unstep_status

constexpr int kOverlapSteps = 64;   // key-tile steps per worker below which a launch overlaps the kernel before it

// Launches a planned kernel.
//
// Set up under the append before it where the launch is short.  Append and attention (with the pipeline of one
// S per query tile, 10 % slower per step), us not
// overlapped -> overlapped, by steps per worker: in runs of 20 (full clock) 24: 78.9 -> 76.5, 35:
// 94.6 -> 92.6, 57: 143.1 -> 142.3, 114: 242.0 -> 240.6, 226: 446.1 -> 445.5, 394: 754.9 -> 763.7; run
// on end at the power cap 24: 80.2 -> 79.8 (1912 -> 1867 MHz), 57: 155.2 -> 155.8 (1792 -> 1776), 114:
// 276.7 -> 276.6 (1702 -> 1688), 169: 395.4 -> 398.6 (1680 -> 1652), 394: 880.4 -> 895.9 (1635 -> 1605).
// The overlap saves 1.5-6 thousand cycles of a launch at any length; at the cap the clock falls for
// the idling it takes away.  The line lies about where the gain of short runs (0.6 % at 57 steps) has
// come down to the loss of runs at the cap (0.4 %).
static int launch_attn(const AttnParams& p, Kind kind, const CUtensorMap& tm_q, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                       const CUtensorMap& tm_kf, const CUtensorMap& tm_vf, __nv_bfloat16* out, cudaStream_t st) {
  const bool brief = p.all_steps < static_cast<int64_t>(kOverlapSteps) * p.n_workers;
  const cudaError_t err =
      launch_clusters(brief, p.cluster ? p.parts : 1,
                      kind == kBf16      ? (p.cluster ? window_attn_kernel<true, kBf16> : window_attn_kernel<false, kBf16>)
                      : kind == kQ8Pairs ? (p.cluster ? window_attn_kernel<true, kQ8Pairs> : window_attn_kernel<false, kQ8Pairs>)
                                         : (p.cluster ? window_attn_kernel<true, kQ8Lone> : window_attn_kernel<false, kQ8Lone>),
                      p.n_workers, kind == kBf16 ? Form<false>::kThreads : Form<true>::kThreads, kAttnSmemBytes, st, tm_q, tm_k,
                      tm_v, tm_kf, tm_vf, p, out);
  g_launches.fetch_add(1);
  return err == cudaSuccess ? UNSTEP_OK : UNSTEP_ERR_CUDA;
}

// The scratch and the checking build's extents of a planned launch whose results start at `out`, `skip` 16-byte vectors
// into the first stream's.
static int bind_scratch(AttnParams& p, cudaStream_t st, ScratchFn scratch, int sm_count, const void* out, int64_t skip) {
  Workspace ws;
  const int rc = scratch(st, 2 * static_cast<size_t>(sm_count), 2 * static_cast<size_t>(p.n_streams) * p.items_per_stream, &ws);
  if (rc != UNSTEP_OK) return rc;
  p.part = ws.part;
  p.counters = ws.counters;
  p.status = status_word();
  p.out_wide = (reinterpret_cast<uintptr_t>(out) & 31u) == 0;   // rows are multiples of 256 bytes
  p.extent_out = static_cast<int64_t>(p.n_streams) * p.L * p.Hn * (kHeadDim / 8) - skip;
  p.extent_part = static_cast<int64_t>(ws.slots) * kPartFloats;
  p.extent_counters = static_cast<int64_t>(ws.n_counters);
  return UNSTEP_OK;
}

// Validation, work split, tensor maps and launch shared by the attention entry points.
// The cache has `sink_frames` slots in front of the ring (0 for the plain rolling window);
// stream b attends frames [0, min(sink_attend, lo)) and [lo, hi), lo = max(0, hi - window_frames).
// With `scale_k` and `scale_v` the cache is one of 8 bits.
static int window_attn_run(const unstep_shape_t* shape, const int32_t* start_frame,
                           int32_t window_frames, const void* q_rot, const void* ring_k,
                           const void* ring_v, void* out, void* cuda_stream, ScratchFn scratch,
                           int32_t sink_frames = 0, int32_t sink_attend = 0, const void* scale_k = nullptr,
                           const void* scale_v = nullptr) {
  const bool q8 = scale_k != nullptr;
  int rc = check_attn_args(shape, start_frame, window_frames, sink_frames, sink_attend, q8);
  if (rc != UNSTEP_OK) return rc;
  const void* ptrs[] = {q_rot, ring_k, ring_v, out};
  for (const void* ptr : ptrs)
    if (ptr == nullptr || !aligned16(ptr)) return UNSTEP_ERR_INVALID_ARG;
  rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  const DeviceInfo& info = device_info();
  if (!info.ok) return UNSTEP_ERR_CUDA;

  const uint64_t Hn = shape->heads;
  const uint64_t C = static_cast<uint64_t>(shape->ring_frames) + sink_frames;  // cache slots per stream
  const uint64_t T = static_cast<uint64_t>(shape->grid_h) * shape->grid_w;
  const uint64_t L = T * shape->chunk_frames;
  const uint64_t row_bytes = Hn * kHeadDim * 2, cache_row_bytes = q8 ? Hn * kHeadDim : row_bytes;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);

  AttnParams p;
  plan_shape(p, shape, sink_frames);
  const Kind kind = !q8 ? kBf16 : p.q_tiles == 1 ? kQ8Lone : kQ8Pairs;
  if (q8) p.flat = 1;
  p.cache_rows = static_cast<int64_t>(C * T);
  for (int b0 = 0; b0 < shape->batch; b0 += kMaxStreamsPerLaunch) {
    const int nb = shape->batch - b0 < kMaxStreamsPerLaunch ? shape->batch - b0 : kMaxStreamsPerLaunch;
    rc = plan_launch(p, shape, start_frame + b0, nb, window_frames, sink_frames, sink_attend, info.sm_count,
                     info.clusters[kind]);
    if (rc != UNSTEP_OK) return rc;
    rc = bind_scratch(p, st, scratch, info.sm_count, out, 0);
    if (rc != UNSTEP_OK) return rc;
    const char* qb = static_cast<const char*>(q_rot) + static_cast<uint64_t>(b0) * L * row_bytes;
    const char* kb = static_cast<const char*>(ring_k) + static_cast<uint64_t>(b0) * C * T * cache_row_bytes;
    const char* vb = static_cast<const char*>(ring_v) + static_cast<uint64_t>(b0) * C * T * cache_row_bytes;
    p.scale_k = static_cast<const uint32_t*>(scale_k) + (q8 ? b0 * p.cache_rows * p.Hn : 0);
    p.scale_v = static_cast<const uint32_t*>(scale_v) + (q8 ? b0 * p.cache_rows * p.Hn : 0);
    __nv_bfloat16* ob = reinterpret_cast<__nv_bfloat16*>(static_cast<char*>(out) +
                                                         static_cast<uint64_t>(b0) * L * row_bytes);
    CUtensorMap tm_q, tm_k, tm_v, tm_kf, tm_vf;
    const uint64_t qdims[4] = {kHeadDim, Hn, L, static_cast<uint64_t>(nb)};
    const uint64_t qstr[3] = {kHeadDim * 2, row_bytes, L * row_bytes};
    const uint64_t rdims[5] = {kHeadDim, Hn, T, C, static_cast<uint64_t>(nb)};
    const uint64_t rstr[4] = {kHeadDim * 2, row_bytes, T * row_bytes, C * T * row_bytes};
    const uint64_t fdims[4] = {kHeadDim, Hn, C * T, static_cast<uint64_t>(nb)};   // ring rows, flat
    const uint64_t fstr[3] = {cache_row_bytes / Hn, cache_row_bytes, C * T * cache_row_bytes};
    if (!make_map(&tm_q, qb, 4, qdims, qstr, 2) || !make_map(&tm_kf, kb, 4, fdims, fstr, 2, q8) ||
        !make_map(&tm_vf, vb, 4, fdims, fstr, 2, q8))
      return UNSTEP_ERR_CUDA;
    if (q8) {
      tm_k = tm_kf;
      tm_v = tm_vf;
    } else if (!make_map(&tm_k, kb, 5, rdims, rstr, 2) || !make_map(&tm_v, vb, 5, rdims, rstr, 2)) {
      return UNSTEP_ERR_CUDA;
    }
    rc = launch_attn(p, kind, tm_q, tm_k, tm_v, tm_kf, tm_vf, ob, st);
    if (rc != UNSTEP_OK) return rc;
  }
  return UNSTEP_OK;
}


#ifdef UNSTEP_TRACE
extern "C" int unstep_debug_read_cta_trace(unsigned long long* host_out) {
  if (cudaDeviceSynchronize() != cudaSuccess) return UNSTEP_ERR_CUDA;
  return cudaMemcpyFromSymbol(host_out, g_cta_trace, sizeof(unsigned long long) * 160 * 16) == cudaSuccess
             ? UNSTEP_OK : UNSTEP_ERR_CUDA;
}
extern "C" int unstep_debug_read_trace(long long* host_out) {
  if (cudaDeviceSynchronize() != cudaSuccess) return UNSTEP_ERR_CUDA;
  return cudaMemcpyFromSymbol(host_out, g_trace, sizeof(long long) * 12 * 64 * 8) == cudaSuccess
             ? UNSTEP_OK : UNSTEP_ERR_CUDA;
}
#endif

extern "C" int unstep_window_attn(const unstep_shape_t* shape, const int32_t* start_frame,
                                  int32_t window_frames, const void* q_rot, const void* ring_k,
                                  const void* ring_v, void* out, void* cuda_stream) {
  return window_attn_run(shape, start_frame, window_frames, q_rot, ring_k, ring_v, out, cuda_stream,
                         get_workspace);
}

extern "C" int unstep_window_attn_sink(const unstep_shape_t* shape, int32_t sink_frames,
                                       const int32_t* start_frame, int32_t recent_frames,
                                       int32_t sink_attend, const void* q_rot, const void* cache_k,
                                       const void* cache_v, void* out, void* cuda_stream) {
  return window_attn_run(shape, start_frame, recent_frames, q_rot, cache_k, cache_v, out, cuda_stream,
                         get_workspace, sink_frames, sink_attend);
}

// Attention over an 8-bit cache with few queries, or with many, by way of unpacked windows, as many heads at a time as the
// scratch holds.  Leaves `done` false where the kernel that decodes tiles for itself is to do it.  With many queries every
// tile of a head is decoded once here, and by each query pair of the head there, next to a softmax that needs the issue slots.
static int window_attn_q8_run(const unstep_shape_t* shape, int32_t sink_frames, const int32_t* start_frame,
                                int32_t window_frames, int32_t sink_attend, const void* q_rot, const void* cache_k,
                                const void* scale_k, const void* cache_v, const void* scale_v, void* out, cudaStream_t st,
                                bool* done) {
  int rc = check_attn_args(shape, start_frame, window_frames, sink_frames, sink_attend, true);
  if (rc != UNSTEP_OK) return rc;
  AttnParams p;
  plan_shape(p, shape, sink_frames);
  const void* ptrs[] = {q_rot, cache_k, cache_v, out};
  for (const void* ptr : ptrs)
    if (ptr == nullptr || !aligned16(ptr)) return UNSTEP_ERR_INVALID_ARG;
  rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  const DeviceInfo& info = device_info();
  if (!info.ok) return UNSTEP_ERR_CUDA;

  const int64_t Hn = p.Hn, L = p.L, cache_rows = (static_cast<int64_t>(p.C) + sink_frames) * p.T;
  const int64_t row_bytes = Hn * kHeadDim * 2;
  p.flat = p.padded = 1;
  p.cache_rows = cache_rows;
  const Way way = q8_way(p, shape, start_frame, window_frames, sink_attend, info.sm_count);
  if (way == kFew) {
    for (int64_t b0 = 0; b0 < shape->batch; b0 += kMaxStreamsPerLaunch) {
      const int nb = static_cast<int>(shape->batch - b0 < kMaxStreamsPerLaunch ? shape->batch - b0 : kMaxStreamsPerLaunch);
      plan_windows(p, shape, start_frame + b0, nb, window_frames, sink_frames, sink_attend);
      p.items_per_stream = p.Hn * few_groups(p.L);
      rc = bind_scratch(p, st, get_workspace, info.sm_count, out, 0);
      if (rc != UNSTEP_OK) return rc;
      const int64_t act = b0 * L * row_bytes, rows = b0 * cache_rows * Hn;
      rc = launch_few(p, nb, info.sm_count, static_cast<const char*>(q_rot) + act, static_cast<const char*>(cache_k) + rows * kHeadDim,
                      static_cast<const char*>(scale_k) + rows * 4, static_cast<const char*>(cache_v) + rows * kHeadDim,
                      static_cast<const char*>(scale_v) + rows * 4, static_cast<char*>(out) + act, st);
      if (rc != UNSTEP_OK) return rc;
    }
    *done = true;
    return UNSTEP_OK;
  }
  if (way == kTiles) return UNSTEP_OK;
  // the widest window decides how many streams and heads go together
  int64_t rows = 0;
  for (int b = 0; b < shape->batch; ++b) {
    const int64_t hi = static_cast<int64_t>(start_frame[b]) + shape->chunk_frames, lo = hi > window_frames ? hi - window_frames : 0;
    const int64_t keys = ((sink_attend < lo ? sink_attend : lo) + hi - lo) * p.T;
    rows = keys > rows ? keys : rows;
  }
  rows = (rows + kTileN - 1) / kTileN * kTileN;
  const int64_t per_head = 2 * rows * kHeadDim * 2, room = static_cast<int64_t>(kMostWindow) / per_head;
  if (room < 1) return UNSTEP_OK;
  int64_t streams = shape->batch < kMaxStreamsPerLaunch ? shape->batch : kMaxStreamsPerLaunch;
  if (streams > room) streams = room;
  int64_t heads = room / streams < Hn ? room / streams : Hn;
  heads = (Hn + (Hn + heads - 1) / heads - 1) / ((Hn + heads - 1) / heads);   // groups of equal size
  const std::unique_lock<std::mutex> turn = window_turn(st);   // to the end of the call
  uint8_t* const window = static_cast<uint8_t*>(get_window(st, streams * heads * per_head));
  if (window == nullptr) return UNSTEP_OK;

  for (int64_t b0 = 0; b0 < shape->batch; b0 += streams) {
    const int nb = static_cast<int>(shape->batch - b0 < streams ? shape->batch - b0 : streams);
    plan_windows(p, shape, start_frame + b0, nb, window_frames, sink_frames, sink_attend);
    Unpack8Params u;
    u.Hn = p.Hn;
    u.rows = static_cast<int32_t>(rows);
    u.cache_rows = cache_rows;
    u.status = status_word();
    for (int i = 0; i < nb; ++i) {
      int32_t end = 0;
      for (int r = 0; r < 3; ++r) {
        u.run_row0[i][r] = p.run_row0[i][r];
        u.run_end[i][r] = end += p.run_rows[i][r];
      }
      p.tiles[i] = (end + kTileN - 1) / kTileN;
      for (int r = 0; r < 3; ++r) {   // one run, from the first row on
        p.run_row0[i][r] = 0;
        p.run_rows[i][r] = r == 0 ? end : 0;
        p.run_tile_end[i][r] = p.tiles[i];
      }
    }
    for (int64_t h0 = 0; h0 < Hn; h0 += heads) {
      const int64_t g = Hn - h0 < heads ? Hn - h0 : heads;
      p.items_per_stream = static_cast<int32_t>(g) * p.q_pairs;
      plan_split(p, info.sm_count, info.clusters[kBf16]);
      uint8_t* const window_v = window + nb * g * rows * kHeadDim * 2;
      u.head0 = static_cast<int32_t>(h0);
      u.extent = nb * g * rows * (kHeadDim / 8);
      const dim3 grid(static_cast<unsigned>((rows + 32 * kUnpackRows - 1) / (32 * kUnpackRows)), static_cast<unsigned>(g), nb);
      const int64_t row0 = b0 * cache_rows * Hn;
      const cudaError_t err = launch_overlapped(
          true, window_unpack_q8_kernel, grid, 256, 0, st, u, static_cast<const uint4*>(cache_k) + row0 * 8,
          static_cast<const uint8_t*>(scale_k) + row0 * 4, static_cast<const uint4*>(cache_v) + row0 * 8,
          static_cast<const uint8_t*>(scale_v) + row0 * 4, reinterpret_cast<uint4*>(window), reinterpret_cast<uint4*>(window_v));
      g_launches.fetch_add(1);
      if (err != cudaSuccess) return UNSTEP_ERR_CUDA;
      const char* qb = static_cast<const char*>(q_rot) + b0 * L * row_bytes + h0 * kHeadDim * 2;
      char* ob = static_cast<char*>(out) + b0 * L * row_bytes + h0 * kHeadDim * 2;
      rc = bind_scratch(p, st, get_workspace, info.sm_count, ob, h0 * (kHeadDim / 8));
      if (rc != UNSTEP_OK) return rc;
      CUtensorMap tm_q, tm_k, tm_v;
      const uint64_t qdims[4] = {kHeadDim, static_cast<uint64_t>(g), static_cast<uint64_t>(L), static_cast<uint64_t>(nb)};
      const uint64_t qstr[3] = {kHeadDim * 2, static_cast<uint64_t>(row_bytes), static_cast<uint64_t>(L * row_bytes)};
      const uint64_t wdims[4] = {kHeadDim, static_cast<uint64_t>(g), static_cast<uint64_t>(rows), static_cast<uint64_t>(nb)};
      const uint64_t wstr[3] = {static_cast<uint64_t>(rows) * kHeadDim * 2, kHeadDim * 2, static_cast<uint64_t>(g * rows) * kHeadDim * 2};
      if (!make_map(&tm_q, qb, 4, qdims, qstr, 2) || !make_map(&tm_k, window, 4, wdims, wstr, 2) ||
          !make_map(&tm_v, window_v, 4, wdims, wstr, 2))
        return UNSTEP_ERR_CUDA;
      rc = launch_attn(p, kBf16, tm_q, tm_k, tm_v, tm_k, tm_v, reinterpret_cast<__nv_bfloat16*>(ob), st);
      if (rc != UNSTEP_OK) return rc;
    }
  }
  *done = true;
  return UNSTEP_OK;
}

extern "C" int unstep_window_attn_q8(const unstep_shape_t* shape, int32_t sink_frames, const int32_t* start_frame,
                                     int32_t recent_frames, int32_t sink_attend, const void* q_rot, const void* cache_k,
                                     const void* scale_k, const void* cache_v, const void* scale_v, void* out,
                                     void* cuda_stream) {
  if (scale_k == nullptr || scale_v == nullptr || (reinterpret_cast<uintptr_t>(scale_k) & 3u) != 0 ||
      (reinterpret_cast<uintptr_t>(scale_v) & 3u) != 0)
    return UNSTEP_ERR_INVALID_ARG;
  bool done = false;
  const int rc = window_attn_q8_run(shape, sink_frames, start_frame, recent_frames, sink_attend, q_rot, cache_k, scale_k,
                                      cache_v, scale_v, out, static_cast<cudaStream_t>(cuda_stream), &done);
  if (rc != UNSTEP_OK || done) return rc;
  return window_attn_run(shape, start_frame, recent_frames, q_rot, cache_k, cache_v, out, cuda_stream,
                         get_workspace, sink_frames, sink_attend, scale_k, scale_v);
}

// --------------------------------------------------------------------------
// Attention without any allocation: the scratch is a fixed array in the library image.
// --------------------------------------------------------------------------
namespace unstep {

constexpr int kStaticMaxCtas = 148;                      // two partial-result slots per CTA
constexpr int kStaticMaxCounters = 2 * 32768;            // a pair of counters per work item
constexpr size_t kStaticCounterBytes = sizeof(int) * kStaticMaxCounters;
constexpr size_t kStaticScratchBytes =
    kStaticCounterBytes + sizeof(float) * 2 * kStaticMaxCtas * static_cast<size_t>(kPartFloats);

// Counters first, partial results after them.  In host code this name is only a handle for
// cudaGetSymbolAddress: it is not a device address and must never be passed to a kernel.
static __device__ __align__(256) unsigned char g_static_scratch[kStaticScratchBytes];

constexpr int kMaxDevices = 64;
static std::mutex g_static_mutex;
static unsigned char* g_static_addr[kMaxDevices] = {};

// Device address of the array on the current device (looked up once per device).
static unsigned char* static_scratch_base() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
  std::lock_guard<std::mutex> lock(g_static_mutex);
  if (g_static_addr[dev] == nullptr) {
    void* ptr = nullptr;
    if (cudaGetSymbolAddress(&ptr, g_static_scratch) != cudaSuccess || ptr == nullptr) return nullptr;
    g_static_addr[dev] = static_cast<unsigned char*>(ptr);
  }
  return g_static_addr[dev];
}

// Scratch source of the no-allocation entry point: carve the fixed array, clear the counters
// this launch will use (the array keeps the previous call's contents).
static int static_scratch(cudaStream_t st, size_t slots, size_t n_counters, Workspace* out) {
  if (slots > 2 * static_cast<size_t>(kStaticMaxCtas) || n_counters > static_cast<size_t>(kStaticMaxCounters))
    return UNSTEP_ERR_TOO_LARGE;
  unsigned char* base = static_scratch_base();
  if (base == nullptr) return UNSTEP_ERR_CUDA;
  if (cudaMemsetAsync(base, 0, n_counters * sizeof(int), st) != cudaSuccess) return UNSTEP_ERR_CUDA;
  out->counters = reinterpret_cast<int*>(base);
  out->part = reinterpret_cast<float*>(base + kStaticCounterBytes);
  out->slots = slots;
  out->n_counters = n_counters;
  return UNSTEP_OK;
}

}  // namespace unstep

extern "C" int unstep_window_attn_noalloc(const unstep_shape_t* shape, const int32_t* start_frame,
                                          int32_t window_frames, const void* q_rot, const void* ring_k,
                                          const void* ring_v, void* out, void* cuda_stream) {
  // size limits of the fixed array first, so that an oversized problem gets its own clear answer
  int rc = check_shape(shape, true);
  if (rc != UNSTEP_OK) return rc;
  const int64_t L = static_cast<int64_t>(shape->grid_h) * shape->grid_w * shape->chunk_frames;
  const int64_t q_pairs = ((L + kTileM - 1) / kTileM + 1) / 2;
  const int64_t streams = shape->batch < kMaxStreamsPerLaunch ? shape->batch : kMaxStreamsPerLaunch;
  if (2 * streams * shape->heads * q_pairs > kStaticMaxCounters) return UNSTEP_ERR_TOO_LARGE;
  rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  const DeviceInfo& info = device_info();
  if (!info.ok) return UNSTEP_ERR_CUDA;
  if (info.sm_count > kStaticMaxCtas) return UNSTEP_ERR_TOO_LARGE;
  return window_attn_run(shape, start_frame, window_frames, q_rot, ring_k, ring_v, out, cuda_stream,
                         static_scratch);
}

extern "C" int unstep_attn_workers(int32_t* workers, int32_t* ctas_per_worker) {
  if (workers == nullptr || ctas_per_worker == nullptr) return UNSTEP_ERR_INVALID_ARG;
  const int rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  const DeviceInfo& info = device_info();
  if (!info.ok) return UNSTEP_ERR_CUDA;
  *workers = info.sm_count;
  *ctas_per_worker = 1;
  return UNSTEP_OK;
}

extern "C" int unstep_attn_clusters(int32_t* clusters) {
  if (clusters == nullptr) return UNSTEP_ERR_INVALID_ARG;
  const int rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  const DeviceInfo& info = device_info();
  if (!info.ok) return UNSTEP_ERR_CUDA;
  for (int n = 0; n <= kMaxClusterParts; ++n) clusters[n] = info.clusters[kBf16][n];
  return UNSTEP_OK;
}

#ifdef UNSTEP_CHECK
namespace unstep {
// One store just past the end of a 4-element buffer: a checking build must skip it and record it.
__global__ void check_probe_kernel(int* buf, int* status) {
  UNSTEP_STORE(buf, threadIdx.x, 4, 7, status);
}
// Two 32-byte stores into three 16-byte vectors: the second one is half outside and must be skipped whole.
__global__ void check_probe_wide_kernel(int* buf, int* status) {
  const uint32_t w[8] = {7, 7, 7, 7, 7, 7, 7, 7};
  UNSTEP_STORE_32(reinterpret_cast<uint4*>(buf), 2 * threadIdx.x, 3, w, status);
}
}  // namespace unstep

extern "C" int unstep_selftest_bounds_check(int32_t* device_buf5, void* cuda_stream) {
  if (device_buf5 == nullptr) return UNSTEP_ERR_INVALID_ARG;
  const int rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  int* st = status_word();
  if (st == nullptr) return UNSTEP_ERR_CUDA;
  check_probe_kernel<<<1, 5, 0, static_cast<cudaStream_t>(cuda_stream)>>>(device_buf5, st);
  g_launches.fetch_add(1);
  return cudaGetLastError() == cudaSuccess ? UNSTEP_OK : UNSTEP_ERR_CUDA;
}

extern "C" int unstep_selftest_bounds_check_wide(int32_t* device_buf16, void* cuda_stream) {
  if (device_buf16 == nullptr || (reinterpret_cast<uintptr_t>(device_buf16) & 31u) != 0) return UNSTEP_ERR_INVALID_ARG;
  const int rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  int* st = status_word();
  if (st == nullptr) return UNSTEP_ERR_CUDA;
  check_probe_wide_kernel<<<1, 2, 0, static_cast<cudaStream_t>(cuda_stream)>>>(device_buf16, st);
  g_launches.fetch_add(1);
  return cudaGetLastError() == cudaSuccess ? UNSTEP_OK : UNSTEP_ERR_CUDA;
}
#endif

extern "C" int unstep_selftest_wait_limit(int64_t limit_cycles, void* cuda_stream) {
  if (limit_cycles < 1 || limit_cycles > 4000000000LL) return UNSTEP_ERR_INVALID_ARG;
  const int rc = check_device();
  if (rc != UNSTEP_OK) return rc;
  wait_limit_probe_kernel<<<1, 64, 0, static_cast<cudaStream_t>(cuda_stream)>>>(limit_cycles);
  g_launches.fetch_add(1);
  return cudaGetLastError() == cudaSuccess ? UNSTEP_OK : UNSTEP_ERR_CUDA;
}

extern "C" void unstep_shutdown(void) {
  // frees the per-stream scratch buffers of every device; the next attention call makes new ones
  cudaDeviceSynchronize();
  int cur = 0;
  if (cudaGetDevice(&cur) != cudaSuccess) return;
  std::lock_guard<std::mutex> lock(g_ws_mutex);
  for (auto& kv : g_workspaces) {
    if (cudaSetDevice(std::get<0>(kv.first)) != cudaSuccess) continue;
    cudaDeviceSynchronize();
    const StreamScratch& s = kv.second;
    if (s.ws.part != nullptr) cudaFree(s.ws.part);
    if (s.ws.counters != nullptr) cudaFree(s.ws.counters);
    for (int i = 0; i < s.n_left; ++i) cudaFree(s.left[i].counters);
    for (void* window : s.window)
      if (window != nullptr) cudaFree(window);
  }
  g_workspaces.clear();
  cudaSetDevice(cur);
}

extern "C" int unstep_poll_status(void) {
  if (cudaDeviceSynchronize() != cudaSuccess) return UNSTEP_ERR_CUDA;
  int st = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&st, g_status, sizeof(int)) != cudaSuccess) return UNSTEP_ERR_CUDA;
  if (st != 0) {
    if (cudaMemcpyToSymbol(g_status, &zero, sizeof(int)) != cudaSuccess) return UNSTEP_ERR_CUDA;
    if (st == UNSTEP_ERR_TIMEOUT) reset_workspace_counters();
  }
  return st;
}
