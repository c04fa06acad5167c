// Products in 8-bit integers (hsd_gemm_w8), and the rows' codes (hsd_quantize_rows).
//   scale_r = max_k |A_rk| / 127,  a_rk = the whole number nearest to A_rk / scale_r,  out_rn = (sum_k a_rk w_nk) scale_r scale_n
// The sum is exact: tcgen05.mma kind::i8 with 32-bit accumulators, which K below 2^17 cannot leave.  So it does not depend on how K is
// divided, and the result is off by three fp32 roundings (the sum's, two products) and the output's own.
//
// Weight rows lie on the MMA's M side in both kernels: a thread of the finish has one weight row, so that a warp stores 32 neighbours of
// an output row at a time, whatever N is.
// Few rows (w8_stream_kernel): bound by the weight stream (16 rows, 28672 x 4096: 22 us, 0.83 of the copy bandwidth).  A tile is up to 128 weight rows, its tokens (padded to whole 16s) are on
// the N side; with few tiles K is divided over a cluster of CTAs, whose sums are added over distributed shared memory.
// Many rows (w8_pair_kernel): bound by the tensor pipe (4095 rows, 14336 x 4096: 161 us, 2.98 POP/s, alone; 2.35 POP/s among others, under the
// power cap, with the codes' 11 us).  Tiles of 256 weight rows x up to 256 tokens on CTA pairs (cta_group::2), as the
// prompt GEMM's.
// Both: 192 threads (TMA producer, MMA issuer, four finishing warps), k-blocks of 128 codes = one 128-byte swizzle row, every wait bounded
// (a wait that gives up sets the workspace's status word); no waiter can be passed by, as in the bf16 kernels: full has its next loads
// behind empty, which the issuer's commit completes, empty its next products behind the loads, acc_full its next behind acc_empty.
#include <algorithm>
#include <math.h>
#include "gemm_tc.cuh"
#include "paged.cuh"
#include "tc_pair.cuh"

namespace hsd {
namespace {

using namespace ptx;
using namespace pair;

constexpr int kThreads = 192;
constexpr int kTile = 128, kBlock = 128;                      // weight rows of a CTA's tile; codes of a k-block
constexpr int kWBytes = kTile * kBlock;
constexpr int kSmem = 232448;
constexpr int kMaxK = (1 << 17) - 16;                         // (-128)^2 K < 2^31

__device__ __forceinline__ uint32_t idesc_s8(int m, int n) {  // signed x signed -> 32-bit integers
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void umma_s8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void umma_s8_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}

struct W8Args {
  CUtensorMap w, a;                             // codes: boxes of 128 x (tile_rows, or 128 in a pair) and 128 x the tokens a CTA loads
  const float *row_scales, *col_scales;
  void *out;
  int R, N, KB;                                 // k-blocks
  int tile_rows, npad;                          // streaming: weight rows of a tile, tokens padded to whole 16s
  int tokens, m_tiles, tiles;                   // pairs: tokens of a tile (a multiple of 32), token tiles, all tiles
  bool early;                                   // the call's own kernel in front writes the activations' codes: weights do not wait for it
  int *status;
};

__device__ __forceinline__ void store(float *out, float v) { *out = v; }
__device__ __forceinline__ void store(__nv_bfloat16 *out, float v) { *out = __float2bfloat16_rn(v); }
__device__ __forceinline__ float scaled(int sum, float row, float col) { return (float)sum * row * col; }

// ---------------------------------------------------------------------------- few rows
template <int NPAD> struct Stream {
  static constexpr int STAGE = kWBytes + NPAD * kBlock, CTRL = 2048;
  static constexpr int FIT = (kSmem - 1024 - CTRL) / STAGE, STAGES = FIT < 12 ? FIT : 12;
  static constexpr int SMEM = STAGES * STAGE + CTRL + 1024, TMEM = 2 * NPAD;
  static_assert(NPAD * kTile * 4 <= STAGES * STAGE, "a cluster's sums must fit the ring");
};
__device__ __forceinline__ int4 ld_cluster(uint32_t addr, uint32_t rank) {
  int4 v;
  asm volatile("ld.shared::cluster.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(map_to_rank(addr, rank)) : "memory");
  return v;
}
// Weight row m of the tiles from `tile` on, which a wait that gave up left out.
template <typename TO> __device__ __noinline__ void no_result(const W8Args &a, int tile, int end, int step, int m) {
  for (; tile < end; tile += step) {
    const int n = tile * a.tile_rows + m;
    if (m >= a.tile_rows || n >= a.N) continue;
    for (int r = 0; r < a.R; ++r) store(static_cast<TO *>(a.out) + (size_t)r * a.N + n, NAN);
  }
}

template <int NPAD, typename TO>
__global__ void __launch_bounds__(kThreads, 1) w8_stream_kernel(const __grid_constant__ W8Args a, int n_tiles, int S) {
  using C = Stream<NPAD>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float *row_scales = reinterpret_cast<float *>(smem + STAGES * C::STAGE);                 // [256]
  uint64_t *bars = reinterpret_cast<uint64_t *>(row_scales + 256);                         // full, empty [STAGES], acc_full, acc_empty [2]
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * STAGES + 4);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  const uint32_t bar0 = smem_u32(bars), s0 = smem_u32(smem);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
  auto accf_bar = [&](int b) { return bar0 + 8u * (2 * STAGES + b); };
  auto acce_bar = [&](int b) { return bar0 + 8u * (2 * STAGES + 2 + b); };
  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (!a.early) chain_wait();                   // (the kernel behind may only start once what this call reads has been written)
  chain_next();
  // S > 1: the cluster's CTAs share tile blockIdx.x / S; S = 1: tiles blockIdx.x, + gridDim.x, ...
  const int rank = S > 1 ? (int)cluster_rank() : 0;
  const int tile0 = S > 1 ? (int)blockIdx.x / S : (int)blockIdx.x, step = S > 1 ? n_tiles : (int)gridDim.x;
  const int kb0 = a.KB * rank / S, kb1 = a.KB * (rank + 1) / S;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(accf_bar(b), 1); mbar_init(acce_bar(b), 4); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), C::TMEM);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    const bool issuer = elect_one();
    const uint64_t policy = l2_policy_evict_first();
    const uint32_t bytes = (uint32_t)(a.tile_rows + a.npad) * kBlock;
    int s = 0;
    uint32_t ph = 0;
    bool ok = true;
    auto load_w = [&](int tile, int kb, int slot) {
      mbar_expect_tx(full_bar(slot), bytes);
      tma_load_2d_hint(s0 + slot * C::STAGE, &a.w, kb * kBlock, tile * a.tile_rows, full_bar(slot), policy);
    };
    auto load_a = [&](int kb, int slot) { tma_load_2d(s0 + slot * C::STAGE + kWBytes, &a.a, kb * kBlock, 0, full_bar(slot)); };
    for (int tile = tile0; tile < n_tiles && ok; tile += step) {
      int kb = kb0;
      if (tile == tile0) {                      // the ring's first weights before the wait for the activations' codes
        const int ahead = min(STAGES, kb1 - kb0);
        if (issuer)
          for (int i = 0; i < ahead; ++i) load_w(tile, kb0 + i, i);
        chain_wait();
        if (blockIdx.x == 0 && issuer) *a.status = 0;          // (a wait gives up after seconds, long after every CTA has started)
        if (issuer)
          for (int i = 0; i < ahead; ++i) load_a(kb0 + i, i);
        kb += ahead; s = ahead;
        if (s == STAGES) { s = 0; ph ^= 1u; }
      }
      for (; kb < kb1; ++kb) {
        if (!mbar_wait_warp(empty_bar(s), ph ^ 1u, abort_flag)) { ok = false; break; }
        if (issuer) { load_w(tile, kb, s); load_a(kb, s); }
        if (++s == STAGES) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok) {                                  // copies in flight land before the shared memory goes away
      const unsigned long long t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 200000ull) {}
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products
    const bool issuer = elect_one();
    chain_wait();                               // (the limit of the waits below is for this kernel's own work)
    const uint32_t idesc = idesc_s8(kTile, a.npad);
    const uint64_t da0 = umma_desc(s0);
    int s = 0, ti = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int tile = tile0; tile < n_tiles && ok; tile += step, ++ti) {
      const int ab = ti & 1;
      if (!mbar_wait_warp(acce_bar(ab), (uint32_t)((ti >> 1) & 1) ^ 1u, abort_flag)) break;
      tc_fence_after();
      const uint32_t d = tmem + (uint32_t)(ab * NPAD);
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait_warp(full_bar(s), ph, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint64_t da = da0 + (uint64_t)(s * (C::STAGE >> 4)), db = da + (uint64_t)(kWBytes >> 4);
        if (issuer) {
#pragma unroll
          for (int k = 0; k < kBlock / 32; ++k) umma_s8(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, k > 0 || kb > kb0 ? 1u : 0u);
          umma_commit(empty_bar(s));
        }
        if (++s == STAGES) { s = 0; ph ^= 1u; }
      }
      if (ok && issuer) umma_commit(accf_bar(ab));
    }
  } else {
    // ------------------------------------------------------------------ finish (warps 2..5): thread = weight row
    const int q = warp & 3, m = q * 32 + lane;
    chain_wait();
    for (int r = threadIdx.x - 64; r < a.R; r += 128) row_scales[r] = a.row_scales[r];
    asm volatile("bar.sync 1, 128;" ::: "memory");
    int ti = 0, missing = n_tiles;
    bool ok = true;
    for (int tile = tile0; tile < n_tiles; tile += step, ++ti) {
      const int ab = ti & 1, n = tile * a.tile_rows + m;
      const bool mine = m < a.tile_rows && n < a.N;
      const float col = mine && S == 1 ? a.col_scales[n] : 0.f;
      if (lane == 0) ok = mbar_wait(accf_bar(ab), (uint32_t)((ti >> 1) & 1), abort_flag);
      ok = __shfl_sync(0xFFFFFFFFu, ok ? 1 : 0, 0) != 0;
      if (!ok) { missing = tile; break; }
      tc_fence_after();
      const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(ab * NPAD);
      int *part = reinterpret_cast<int *>(smem);                // S > 1: every load of the CTA has been consumed
#pragma unroll 1
      for (int c = 0; c < NPAD && c < a.R; c += 16) {
        float v[16];
        tmem_ld16(from + (uint32_t)c, v);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if (S > 1) part[(c + e) * kTile + m] = __float_as_int(v[e]);
          else if (mine && c + e < a.R) store(static_cast<TO *>(a.out) + (size_t)(c + e) * a.N + n, scaled(__float_as_int(v[e]), row_scales[c + e], col));
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(acce_bar(ab));
    }
    if (S == 1 && missing < n_tiles) no_result<TO>(a, missing, n_tiles, step, m);
  }
  __syncwarp();
  if (S > 1) {
    // ------------------------------------------------------------------ sums across the cluster; each rank finishes its share
    __syncthreads();
    cluster_sync();
    // groups of four weight rows of a token; tiles have whole eights of rows
    const int fours = a.tile_rows / 4, total = a.R * fours, i1 = (int)((long long)total * (rank + 1) / S);
    for (int i = (int)((long long)total * rank / S) + threadIdx.x; i < i1; i += kThreads) {
      const int r = i / fours, m = (i - r * fours) * 4, n = tile0 * a.tile_rows + m;
      int4 x[8];
#pragma unroll
      for (int p = 0; p < 8; ++p)
        if (p < S) x[p] = ld_cluster(s0 + (uint32_t)(r * kTile + m) * 4u, (uint32_t)p);
      int sum[4] = {0, 0, 0, 0};
#pragma unroll
      for (int p = 0; p < 8; ++p)
        if (p < S) { sum[0] += x[p].x; sum[1] += x[p].y; sum[2] += x[p].z; sum[3] += x[p].w; }
      TO *out = static_cast<TO *>(a.out) + (size_t)r * a.N + n;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.N) store(out + e, scaled(sum[e], row_scales[r], a.col_scales[n + e]));
    }
    __syncwarp();
    cluster_sync();                             // nobody leaves while its sums are being read
    if (*abort_flag && threadIdx.x < kTile) no_result<TO>(a, tile0, tile0 + 1, 1, threadIdx.x);        // over what the others made of them
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, C::TMEM);
  if (threadIdx.x == 0 && *abort_flag) atomicExch(a.status, 1);
}

// ---------------------------------------------------------------------------- many rows
constexpr int kPairStages = 6, kHalf = 128;                   // token rows that a CTA of a pair loads at most
constexpr int kPairStage = kWBytes + kHalf * kBlock, kPairSmem = kPairStages * kPairStage + 4096 + 1024;

template <typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) w8_pair_kernel(const __grid_constant__ W8Args a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float *row_scales = reinterpret_cast<float *>(smem + kPairStages * kPairStage);          // [2][256], alternating per tile
  uint64_t *bars = reinterpret_cast<uint64_t *>(row_scales + 512);
  // full[STAGES] (used in the leader) | empty[STAGES] | acc_full[2] | acc_empty[2] (used in the leader)
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * kPairStages + 4);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  volatile int *wait_ok = reinterpret_cast<volatile int *>(tmem_slot + 2);                 // [2], alternating per tile
  const uint32_t bar0 = smem_u32(bars), s0 = smem_u32(smem);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kPairStages + s); };
  auto accf_bar = [&](int b) { return bar0 + 8u * (2 * kPairStages + b); };
  auto acce_bar = [&](int b) { return bar0 + 8u * (2 * kPairStages + 2 + b); };
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  if (!a.early) chain_wait();
  chain_next();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kPairStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(accf_bar(b), 1); mbar_init(acce_bar(b), 8); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();                               // both CTAs' barriers exist, both hold their tensor memory
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int half = a.tokens / 2;                // token rows that each CTA loads

  if (warp == 0) {
    // ------------------------------------------------------------------ producer (one lane of each CTA issues)
    const bool issuer = elect_one();
    const uint32_t bytes = 2u * (uint32_t)(kWBytes + half * kBlock);
    int s = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int t = pair; t < a.tiles && ok; t += pairs) {
      const int n0 = t / a.m_tiles * 2 * kTile + (int)rank * kTile, r0 = t % a.m_tiles * a.tokens + (int)rank * half;
      auto load_w = [&](int kb, int slot) {
        if (rank == 0) mbar_expect_tx(full_bar(slot), bytes);
        tma_load_2d_pair(s0 + slot * kPairStage, &a.w, kb * kBlock, n0, map_to_rank(full_bar(slot), 0));
      };
      auto load_a = [&](int kb, int slot) {
        tma_load_2d_pair(s0 + slot * kPairStage + kWBytes, &a.a, kb * kBlock, r0, map_to_rank(full_bar(slot), 0));
      };
      int kb = 0;
      if (t == pair) {
        kb = min(kPairStages, a.KB);
        if (issuer)
          for (int i = 0; i < kb; ++i) load_w(i, i);
        chain_wait();
        if (blockIdx.x == 0 && issuer) *a.status = 0;
        if (issuer)
          for (int i = 0; i < kb; ++i) load_a(i, i);
        s = kb;
        if (s == kPairStages) { s = 0; ph ^= 1u; }
      }
      for (; kb < a.KB; ++kb) {
        if (!mbar_wait_warp(empty_bar(s), ph ^ 1u, abort_flag)) { ok = false; break; }
        if (issuer) { load_w(kb, s); load_a(kb, s); }
        if (++s == kPairStages) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok) {
      const unsigned long long t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 200000ull) {}
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products (one lane of the leader issues)
    if (rank == 0) {
      const bool issuer = elect_one();
      chain_wait();
      const uint32_t idesc = idesc_s8(2 * kTile, a.tokens);
      const uint64_t da0 = umma_desc(s0);
      int s = 0, ti = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int t = pair; t < a.tiles && ok; t += pairs, ++ti) {
        const int ab = ti & 1;
        ok = mbar_wait_warp(acce_bar(ab), (uint32_t)((ti >> 1) & 1) ^ 1u, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(ab * 256);
        for (int kb = 0; kb < a.KB; ++kb) {
          if (!mbar_wait_warp(full_bar(s), ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint64_t da = da0 + (uint64_t)(s * (kPairStage >> 4)), db = da + (uint64_t)(kWBytes >> 4);
          if (issuer) {
#pragma unroll
            for (int k = 0; k < kBlock / 32; ++k) umma_s8_pair(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, k > 0 || kb > 0 ? 1u : 0u);
            umma_commit_pair(empty_bar(s));
          }
          if (++s == kPairStages) { s = 0; ph ^= 1u; }
        }
        if (ok && issuer) umma_commit_pair(accf_bar(ab));
      }
    }
  } else {
    // ------------------------------------------------------------------ finish (warps 2..5): thread = weight row
    const int q = warp & 3, et = threadIdx.x - 64;
    chain_wait();
    int ti = 0;
    for (int t = pair; t < a.tiles; t += pairs, ++ti) {
      const int ab = ti & 1, n = t / a.m_tiles * 2 * kTile + (int)rank * kTile + q * 32 + lane, r0 = t % a.m_tiles * a.tokens;
      float *rows = row_scales + ab * 256;      // (its last reader is two tiles behind: all four warps have met since)
      for (int r = et; r < a.tokens; r += 128) rows[r] = r0 + r < a.R ? a.row_scales[r0 + r] : 0.f;
      const float col = n < a.N ? a.col_scales[n] : 0.f;
      if (et == 0) wait_ok[ab] = mbar_wait(accf_bar(ab), (uint32_t)((ti >> 1) & 1), abort_flag) ? 1 : 0;
      asm volatile("bar.sync 1, 128;" ::: "memory");
      if (!wait_ok[ab]) {                       // what was not computed is NaN
        for (int x = t; x < a.tiles; x += pairs) {
          const int n = x / a.m_tiles * 2 * kTile + (int)rank * kTile + q * 32 + lane, r0 = x % a.m_tiles * a.tokens, left = min(a.tokens, a.R - r0);
          for (int r = 0; r < left && n < a.N; ++r) store(static_cast<TO *>(a.out) + (size_t)(r0 + r) * a.N + n, NAN);
        }
        break;
      }
      tc_fence_after();
      const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(ab * 256);
      const int left = min(a.tokens, a.R - r0);
      TO *out = static_cast<TO *>(a.out) + (size_t)r0 * a.N + n;
#pragma unroll 1
      for (int c = 0; c < left; c += 32) {
        float v[32];
        tmem_ld32(from + (uint32_t)c, v);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if (n < a.N && c + e < left) store(out + (size_t)(c + e) * a.N, scaled(__float_as_int(v[e]), rows[c + e], col));
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) remote_arrive(map_to_rank(acce_bar(ab), 0));
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync();                               // no signal may arrive in a CTA that has left
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
  if (threadIdx.x == 0 && *abort_flag) atomicExch(a.status, 1);
}

// ---------------------------------------------------------------------------- codes of rows
struct QuantArgs {
  const unsigned char *x;
  long long row_bytes;
  int8_t *codes;
  float *scales;
  int K, rows;
};
// Eight values, as they lie in memory and in fp32.
template <typename T> struct Eight;
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const unsigned char *p) {
    a = __ldg(reinterpret_cast<const float4 *>(p));
    b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float *f) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};
template <> struct Eight<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const unsigned char *p) { v = __ldg(reinterpret_cast<const uint4 *>(p)); }
  __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void get(float *f) const {
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
    f[4] = __uint_as_float(v.z << 16); f[5] = __uint_as_float(v.z & 0xFFFF0000u);
    f[6] = __uint_as_float(v.w << 16); f[7] = __uint_as_float(v.w & 0xFFFF0000u);
  }
};
template <typename T> __device__ __forceinline__ u32 largest(const Eight<T> &x) {       // as bits: NaN lies above infinity, and that above all numbers
  float f[8];
  x.get(f);
  u32 top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
  return top;
}

// A row's scale, and its values' codes: the whole number nearest to x / s, ties to even.
struct Coder {
  float s, inv, half;
  __device__ __forceinline__ explicit Coder(u32 top) {
    s = top < 0x7F800000u ? __fdiv_rn(__uint_as_float(top), 127.f) : __uint_as_float(0x7FC00000u);
    inv = s > 1e-30f ? __fdiv_rn(1.f, s) : 0.f;
    half = 0.5f * s;                            // (exact, but for the smallest scales, which take the quotient)
  }
  // x inv is off by 2^-22 of itself: rounded to a whole number c (by adding 1.5 * 2^23, whose low bits are the number), it is one off at most,
  // where x / s lies next to the middle of two codes.  What is left, x - c s, is exact there, as both are multiples of the smaller one's last
  // place and it is below 1.5 s: above half a scale it says that c is one off, at half a scale that c has to be even.
  __device__ __forceinline__ u32 near(float x, float &rest) const {
    const float big = 12582912.f, biased = __fadd_rn(x * inv, big);
    rest = fmaf(-__fadd_rn(biased, -big), s, x);
    return __float_as_uint(biased);
  }
  __device__ __forceinline__ u32 exact(u32 code, float rest) const {
    const float r = fabsf(rest);
    return r > half || (r == half && (code & 1)) ? code + (rest > 0.f ? 1 : -1) : code;
  }
  // Rows of the smallest scales, and of none (0, or NaN: all codes are 0).
  __device__ __forceinline__ u32 rare(float x) const {
    if (!(s > 0.f)) return 0u;
    float c = rintf(__fdiv_rn(x, s));
    const float rest = fmaf(-c, s, x), twice = 2.f * fabsf(rest);
    if (twice > s || (twice == s && ((int)c & 1))) c += rest > 0.f ? 1.f : -1.f;
    return (u32)max(-127, min(127, (int)c));
  }
  __device__ __forceinline__ u32 operator()(float x) const {
    if (inv == 0.f) return rare(x) & 0xFFu;
    float rest;
    const u32 c = near(x, rest);
    return exact(c, rest) & 0xFFu;
  }
  template <typename T> __device__ __forceinline__ uint2 eight(const Eight<T> &x) const {
    float f[8], rest[8];
    u32 c[8];
    x.get(f);
    if (inv == 0.f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = rare(f[e]);
    } else {
      bool off = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        c[e] = near(f[e], rest[e]);
        off |= fabsf(rest[e]) >= half;
      }
      if (off)
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = exact(c[e], rest[e]);
    }
    const u32 lo = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
    const u32 hi = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
    return make_uint2(lo, hi);
  }
};

// A row a CTA, whose values are in registers between the maximum and the codes: H groups of eight a thread, those past
// H threads' worth are read twice.  H == 0: values at any address, one at a time, read twice.
template <typename T, int H>
__global__ void __launch_bounds__(256) w8_quantize_kernel(QuantArgs a) {
  __shared__ u32 sh[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, thread = threadIdx.x, threads = blockDim.x, step = threads * 8, row = blockIdx.x;
  chain_wait();
  chain_next();
  const unsigned char *x = a.x + (size_t)row * a.row_bytes;
  int8_t *to = a.codes + (size_t)row * a.K;
  u32 top = 0;
  Eight<T> held[H > 0 ? H : 1];
  if constexpr (H > 0) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const int k = i * step + thread * 8;
      held[i].zero();
      if (k < a.K) held[i].load(x + (size_t)k * sizeof(T));
    }
#pragma unroll
    for (int i = 0; i < H; ++i) top = max(top, largest(held[i]));
    for (int k = H * step + thread * 8; k < a.K; k += step) {
      Eight<T> v;
      v.load(x + (size_t)k * sizeof(T));
      top = max(top, largest(v));
    }
  } else {
    for (int k = thread; k < a.K; k += threads) top = max(top, __float_as_uint(to_f32(reinterpret_cast<const T *>(x)[k])) & 0x7FFFFFFFu);
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (lane == 0) sh[warp] = top;
  __syncthreads();
  for (int w = 0; w < threads / 32; ++w) top = max(top, sh[w]);
  const Coder code(top);
  if (thread == 0) a.scales[row] = code.s;
  if constexpr (H > 0) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const int k = i * step + thread * 8;
      if (k < a.K) *reinterpret_cast<uint2 *>(to + k) = code.eight(held[i]);
    }
    for (int k = H * step + thread * 8; k < a.K; k += step) {
      Eight<T> v;
      v.load(x + (size_t)k * sizeof(T));
      *reinterpret_cast<uint2 *>(to + k) = code.eight(v);
    }
  } else {
    for (int k = thread; k < a.K; k += threads) to[k] = (int8_t)code(to_f32(reinterpret_cast<const T *>(x)[k]));
  }
}


constexpr int kManyHeld = 4;                                  // 4095 rows of 4096 bf16: 11.4 us, with 1, 2 or 8 13.8, 13.9 and 11.9
template <typename T> int quantize_t(const QuantArgs &a, cudaStream_t s) {
  const bool vec = a.K % 8 == 0 && ((reinterpret_cast<uintptr_t>(a.x) | (uintptr_t)a.row_bytes) & 15) == 0 && (reinterpret_cast<uintptr_t>(a.codes) & 7) == 0;
  // Threads: of a few rows, a group of eight values each, up to 256 threads with up to eight groups; of many rows, whose CTAs hide one another's
  // trips, kManyHeld groups each
  const int groups = ceil_div(a.K, 8), few = a.rows <= 2 * kMeasuredSMs ? 1 : kManyHeld;
  const int threads = std::min(256, ceil_div(ceil_div(groups, few), 32) * 32), held = ceil_div(groups, threads);
  auto kernel = !vec ? w8_quantize_kernel<T, 0> : held <= 1 ? w8_quantize_kernel<T, 1> : held <= 2 ? w8_quantize_kernel<T, 2> : held <= 4 ? w8_quantize_kernel<T, 4> : w8_quantize_kernel<T, 8>;
  HSD_CUDA_OK(hsd_launch(kernel, dim3(a.rows), threads, 0, s, 0, true, a));
  hsd_count_launches(1);
  return hsd_launch_status();
}
int quantize(const void *x, int dtype, int rows, int K, long long row_stride, void *codes, float *scales, cudaStream_t s) {
  const QuantArgs a = {static_cast<const unsigned char *>(x), row_stride * (dtype == HSD_F32 ? 4 : 2), static_cast<int8_t *>(codes), scales, K, rows};
  return dtype == HSD_F32 ? quantize_t<float>(a, s) : quantize_t<__nv_bfloat16>(a, s);
}

// ---------------------------------------------------------------------------- the call
int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 2) return kMeasuredSMs;
  return sms;
}
// CTAs a tile's k-blocks are divided over, as the bf16 kernel's: while tiles of 128 rows leave half of the SMs idle.
int split_of(int N, int KB, int sms) {
  const int tiles = ceil_div(N, kTile);
  int S = 1;
  while (S < (tiles <= 14 ? 8 : 4) && tiles * S * 2 <= sms && S * 2 <= KB) S *= 2;
  return S;
}
long long ceil_div64(long long a, long long b) { return (a + b - 1) / b; }       // (sizes end close to 2^31)
// Rows of a tile: as many as spread N evenly over the rounds of the SMs, or of the clusters that run at once.
int tile_rows_of(int N, int S, int sms) {
  const long long at_once = S == 2 ? 74 : S == 4 ? 32 : S == 8 ? 14 : sms, rounds = ceil_div64(N, kTile * at_once);
  return (int)std::min<long long>(kTile, ceil_div64(ceil_div64(N, rounds * at_once), 8) * 8);
}
template <int NPAD, typename TO> int run_stream(const W8Args &a, int n_tiles, int S, int grid, cudaStream_t s) {
  static std::atomic<u64> limits{0};
  const int limit = hsd_smem_limit((const void *)w8_stream_kernel<NPAD, TO>, Stream<NPAD>::SMEM, limits);
  if (limit) return limit;
  HSD_CUDA_OK(hsd_launch(w8_stream_kernel<NPAD, TO>, dim3(grid), kThreads, Stream<NPAD>::SMEM, s, S, true, a, n_tiles, S));
  hsd_count_launches(1);
  return hsd_launch_status();
}
template <typename TO> int run(W8Args &a, const void *codes_a, const void *codes_w, int K, cudaStream_t s) {
  const int sms = sm_count();
  // Up to 256 rows by the weight stream, us against the pairs': 2048 x 5632, 16 / 128 / 256 rows 7.4 / 9.5 / 12.8 against 12.6 / 14.8 / 22.5; 4096 x 4096
  // 7.3 / 10.7 / 14.6 against 10.4 / 12.9 / 19.4; 32000 x 2048 13.9 / 18.9 / 27.6 against 16.3 / 20.4 / 28.1 (14336 x 4096: 24.0 against 22.7 with 256)
  if (a.R <= 256) {
    const int S = split_of(a.N, a.KB, sms), npad = tc_npad(a.R);
    a.tile_rows = tile_rows_of(a.N, S, sms);
    a.npad = ceil_div(a.R, 16) * 16;
    int status = tc_make_map_bytes(&a.w, codes_w, a.N, K, a.tile_rows);
    if (!status) status = tc_make_map_bytes(&a.a, codes_a, a.R, K, a.npad);
    if (status) return status;
    const int n_tiles = ceil_div(a.N, a.tile_rows), grid = S > 1 ? n_tiles * S : std::min(n_tiles, sms);
    switch (npad) {
      case 16: return run_stream<16, TO>(a, n_tiles, S, grid, s);
      case 32: return run_stream<32, TO>(a, n_tiles, S, grid, s);
      case 64: return run_stream<64, TO>(a, n_tiles, S, grid, s);
      case 128: return run_stream<128, TO>(a, n_tiles, S, grid, s);
      default: return run_stream<256, TO>(a, n_tiles, S, grid, s);
    }
  }
  // tokens of a tile: as many as spread R evenly over the rounds of the CTA pairs that tiles of 256 need (us against tiles of 256: 3375 rows of
  // 362 x 12528 41 / 48, 512 of 4096 x 4096 14.1 / 20.8, 1000 of 6144 x 4096 26.5 / 32.3, 2000 of 1000 x 2000 12.6 / 17.3)
  const int n_tiles = ceil_div(a.N, 2 * kTile), pairs = sms / 2, most = ceil_div(a.R, 256);
  const long long rounds = ceil_div64((long long)most * n_tiles, pairs), in_them = std::max<long long>(most, std::min<long long>(rounds * pairs / n_tiles, a.R));
  a.tokens = (int)ceil_div64(ceil_div64(a.R, in_them), 32) * 32;
  a.m_tiles = ceil_div(a.R, a.tokens);
  a.tiles = a.m_tiles * ceil_div(a.N, 2 * kTile);
  int status = tc_make_map_bytes(&a.w, codes_w, a.N, K, kTile);
  if (!status) status = tc_make_map_bytes(&a.a, codes_a, a.R, K, a.tokens / 2);
  if (status) return status;
  static std::atomic<u64> limits{0};
  status = hsd_smem_limit((const void *)w8_pair_kernel<TO>, kPairSmem, limits);
  if (status) return status;
  HSD_CUDA_OK(hsd_launch(w8_pair_kernel<TO>, dim3(2 * std::min(sms / 2, a.tiles)), kThreads, kPairSmem, s, 0, true, a));
  hsd_count_launches(1);
  return hsd_launch_status();
}
bool w8_sizes(int R, int N, int K) { return R > 0 && N > 0 && K > 0 && K % 16 == 0; }
bool w8_fits(int R, int N, int K) { return K <= kMaxK && N <= 0x7FFFFF00 && R <= 0x7FFFFF00 && (long long)ceil_div(R, 32) * ceil_div(N, 2 * kTile) < (1ll << 30); }

}  // namespace
}  // namespace hsd

extern "C" int hsd_quantize_rows(const void *x, int dtype, int rows, int K, long long row_stride, void *codes, float *scales, void *stream) {
  using namespace hsd;
  if (!x || !codes || !scales || rows <= 0 || K <= 0 || row_stride < K || (dtype != HSD_F32 && dtype != HSD_BF16)) return HSD_E_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(x) & (dtype == HSD_F32 ? 3 : 1)) || !words(scales, nullptr)) return HSD_E_INVALID_ARG;
  if (K > 0x7FFF0000) return HSD_E_TOO_LARGE;                 // (places past the row's end have to be numbers too)
  return quantize(x, dtype, rows, K, row_stride, codes, scales, (cudaStream_t)stream);
}

extern "C" size_t hsd_gemm_w8_workspace_bytes(int a_dtype, int R, int N, int K) {
  using namespace hsd;
  if (!w8_sizes(R, N, K) || !w8_fits(R, N, K) || (a_dtype != HSD_F32 && a_dtype != HSD_BF16 && a_dtype != HSD_I8)) return 0;
  return 256 + (a_dtype == HSD_I8 ? 0 : ((size_t)R * 4 + 255) / 256 * 256 + (size_t)R * K);      // the status word, the activations' scales and codes
}

extern "C" int hsd_gemm_w8(const void *A, int a_dtype, const float *a_scales, int R, int K, const void *codes, const float *scales, int N,
                           void *out, int out_dtype, void *workspace, size_t workspace_bytes, void *stream) {
  using namespace hsd;
  if (!A || !codes || !scales || !out || !workspace || !w8_sizes(R, N, K)) return HSD_E_INVALID_ARG;
  if ((a_dtype != HSD_F32 && a_dtype != HSD_BF16 && a_dtype != HSD_I8) || (out_dtype != HSD_F32 && out_dtype != HSD_BF16)) return HSD_E_INVALID_ARG;
  if (a_dtype == HSD_I8 ? !a_scales : a_scales != nullptr) return HSD_E_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(A) & (a_dtype == HSD_I8 ? 15 : a_dtype == HSD_F32 ? 3 : 1)) || (reinterpret_cast<uintptr_t>(codes) & 15) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255) || !words(a_scales, scales) ||
      (reinterpret_cast<uintptr_t>(out) & (out_dtype == HSD_F32 ? 3 : 1))) return HSD_E_INVALID_ARG;
  if (!w8_fits(R, N, K)) return HSD_E_TOO_LARGE;
  if (workspace_bytes < hsd_gemm_w8_workspace_bytes(a_dtype, R, N, K)) return HSD_E_WORKSPACE_TOO_SMALL;
  int status = tc_init();
  if (status) return status;
  cudaStream_t s = (cudaStream_t)stream;
  W8Args a = {};
  a.status = static_cast<int *>(workspace);
  float *own_scales = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + 256);
  const void *codes_a = A;
  a.row_scales = a_scales;
  if (a_dtype != HSD_I8) {
    unsigned char *own = static_cast<unsigned char *>(workspace) + 256 + ((size_t)R * 4 + 255) / 256 * 256;
    status = quantize(A, a_dtype, R, K, K, own, own_scales, s);
    if (status) return status;
    codes_a = own;
    a.row_scales = own_scales;
    a.early = true;
  }
  a.col_scales = scales; a.out = out; a.R = R; a.N = N; a.KB = ceil_div(K, kBlock);
  return out_dtype == HSD_F32 ? run<float>(a, codes_a, codes, K, s) : run<__nv_bfloat16>(a, codes_a, codes, K, s);
}
