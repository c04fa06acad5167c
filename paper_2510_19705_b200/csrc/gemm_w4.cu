// Few-row products with 4-bit weights and group scales (hsd_gemm_w4): out[r, n] = sum_k A[r, k] (c[n, k] - 8) s[n, k / group].
// Bound by memory: half a byte a weight.  What stands between that and the products is making bf16 of the codes, eleven operations
// for the eight codes of a word: c less 8 is made from the bits (0x4300 | c is 128 + c in bf16, less 136: exact), a pair at a time, and
// the pairs are (0,4), (1,5), (2,6), (3,7) of a word; the order of k inside a product is free, so the activations are put in the same.
// A group's products are summed in the tensor cores' fp32, then scaled and added in fp32: no rounding to fewer bits anywhere.
// w4_kernel: 128 weight rows a tile, a thread one row.  Codes come by TMA, the pairs go from registers into tensor memory, from where
// tcgen05.mma takes them as its operand A (the activations, at most 64 rows, are B, once put in the pairs' order by w4_stage_kernel);
// a thread reads its row's sums of a group back and scales them.  The tiles' steps (128 of k) stand in one line that is divided evenly over warpgroups, three on an SM (two
// for more than 16 rows), each with a warp of its own that asks for codes and issues products; where a stretch ends inside a tile its sums go to the workspace
// and w4_join_kernel adds them in order.
// w4_small_kernel: see there.
#include <cooperative_groups.h>

#include "gemm_tc.cuh"
#include "tc_ptx.cuh"

namespace hsd {
namespace {

using namespace ptx;

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kChunk = 128;            // k of a warp's step in w4_small_kernel: 16 bytes of codes a lane

struct W4Args {
  const __nv_bfloat16 *a;
  const uint8_t *codes;
  const __nv_bfloat16 *scales;
  float *out;
  int R, K, N, groups;                 // groups of a row
  u32 bits;                            // kCodeBits
};

__device__ __forceinline__ void mma(float *c, const u32 *a, u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Codes i and i + 4 of a word, less 8, as two bf16.  `bits` is 0x43004300 out of the arguments: as a constant it and the mask do not fit
// one instruction.
constexpr u32 kCodeBits = 0x43004300u;
template <int I> __device__ __forceinline__ u32 pair(u32 word, u32 bits) {
  u32 x;
  asm("lop3.b32 %0, %1, 0x000F000F, %2, 0xEA;" : "=r"(x) : "r"(I ? word >> (4 * I) : word), "r"(bits));
  const u32 bias = 0x43084308u;
  const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&bias));
  return *reinterpret_cast<const u32 *>(&y);
}

// ---------------------------------------------------------------------------- small products
// The codes never leave registers: a lane loads 32 of a weight row, and their pairs are its operands of mma.sync with 16 weight rows
// as the tile's rows and up to eight activations as its columns.  A CTA has 16 weight rows; its warps divide k (chunk by chunk in turn, so that
// together they read long pieces of a row), and where the matrix has few rows a cluster divides it once more.
// GW: words of a lane in a group (group = 32 GW); RT: tiles of 8 activation rows; MT: tiles of 16 weight rows.
template <int GW, int RT, int MT>
__global__ void __launch_bounds__(kThreads)
w4_small_kernel(W4Args p) {
  constexpr int GROUPS = 4 / GW;       // of a chunk
  __shared__ __align__(16) float sums[kWarps][MT * 16][RT * 8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 3, lr = lane >> 2;
  const int parts = gridDim.y, part = blockIdx.y, n0 = blockIdx.x * MT * 16;
  float acc[MT][RT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[m][t][x] = 0.f;

  const int chunks = (p.K + kChunk - 1) / kChunk;
  for (int c = part * kWarps + warp; c < chunks; c += parts * kWarps) {
    u32 word[MT][2][4];
    float scale[MT][2][GROUPS];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = min(n0 + m * 16 + h * 8 + lr, p.N - 1);          // rows past the last are read as the last and not stored
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          const int k = c * kChunk + g * GW * 32 + j * GW * 8;
          const bool in = k < p.K;
          const uint8_t *at = p.codes + ((size_t)n * p.K + k) / 2;
          u32 *w = &word[m][h][g * GW];
          if constexpr (GW == 4) {
            const uint4 v = in ? __ldg(reinterpret_cast<const uint4 *>(at)) : make_uint4(0, 0, 0, 0);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
          } else if constexpr (GW == 2) {
            const uint2 v = in ? __ldg(reinterpret_cast<const uint2 *>(at)) : make_uint2(0, 0);
            w[0] = v.x; w[1] = v.y;
          } else {
            w[0] = in ? __ldg(reinterpret_cast<const u32 *>(at)) : 0u;
          }
          const int group = c * GROUPS + g;
          scale[m][h][g] = group < p.groups ? __bfloat162float(p.scales[(size_t)n * p.groups + group]) : 0.f;
        }
      }
    u32 b[RT][4][4];                   // activations of the lane's row and words, as pairs in the codes' order
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int k = c * kChunk + (w / GW) * GW * 32 + j * GW * 8 + (w % GW) * 8, r = t * 8 + lr;
        const uint4 v = r < p.R && k < p.K ? __ldg(reinterpret_cast<const uint4 *>(p.a + (size_t)r * p.K + k)) : make_uint4(0, 0, 0, 0);
        b[t][w][0] = __byte_perm(v.x, v.z, 0x5410);
        b[t][w][1] = __byte_perm(v.x, v.z, 0x7632);
        b[t][w][2] = __byte_perm(v.y, v.w, 0x5410);
        b[t][w][3] = __byte_perm(v.y, v.w, 0x7632);
      }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        float sum[RT][4];
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) sum[t][x] = 0.f;
#pragma unroll
        for (int w = g * GW; w < (g + 1) * GW; ++w) {
          const u32 lo[4] = {pair<0>(word[m][0][w], p.bits), pair<0>(word[m][1][w], p.bits), pair<1>(word[m][0][w], p.bits), pair<1>(word[m][1][w], p.bits)};
          const u32 hi[4] = {pair<2>(word[m][0][w], p.bits), pair<2>(word[m][1][w], p.bits), pair<3>(word[m][0][w], p.bits), pair<3>(word[m][1][w], p.bits)};
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            mma(sum[t], lo, b[t][w][0], b[t][w][1]);
            mma(sum[t], hi, b[t][w][2], b[t][w][3]);
          }
        }
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) acc[m][t][x] = fmaf(scale[m][x >> 1][g], sum[t][x], acc[m][t][x]);
      }
  }

  // the warps' sums, then the cluster's
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int x = 0; x < 4; ++x) sums[warp][m * 16 + lr + (x >> 1) * 8][t * 8 + j * 2 + (x & 1)] = acc[m][t][x];
  __syncthreads();
  if (parts == 1) {
    for (int i = threadIdx.x; i < MT * 16 * RT * 8; i += kThreads) {
      const int n = i % (MT * 16), r = i / (MT * 16);
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) s += sums[w][n][r];
      if (r < p.R && n0 + n < p.N) p.out[(size_t)r * p.N + n0 + n] = s;
    }
    return;
  }
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  for (int i = threadIdx.x; i < MT * 16 * RT * 8; i += kThreads) {
    const int n = i % (MT * 16), r = i / (MT * 16);
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += sums[w][n][r];
    sums[0][n][r] = s;
  }
  cluster.sync();
  for (int i = part * kThreads + threadIdx.x; i < MT * 16 * RT * 8; i += parts * kThreads) {
    const int n = i % (MT * 16), r = i / (MT * 16);
    float s = 0.f;
    for (int q = 0; q < parts; ++q) s += *cluster.map_shared_rank(&sums[0][n][r], q);
    if (r < p.R && n0 + n < p.N) p.out[(size_t)r * p.N + n0 + n] = s;
  }
  cluster.sync();                      // no CTA leaves while others read its sums
}

template <int GW, int RT, int MT> int run_small(const W4Args &a, cudaStream_t s) {
  const int tiles = ceil_div(a.N, MT * 16), chunks = ceil_div(a.K, kChunk);
  int parts = 1;
  while (parts < 8 && tiles * parts < kMeasuredSMs && parts * kWarps < chunks) parts *= 2;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 1; at.val.clusterDim.y = parts; at.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles, parts); cfg.blockDim = dim3(kThreads); cfg.stream = s; cfg.attrs = &at; cfg.numAttrs = parts > 1;
  HSD_CUDA_OK(cudaLaunchKernelEx(&cfg, w4_small_kernel<GW, RT, MT>, a));
  hsd_count_launches(1);
  return hsd_launch_status();
}

// ---------------------------------------------------------------------------- tensor memory
constexpr int kStep = 128;             // k of a step: 64 bytes of codes of a row
constexpr int kTile = 128;             // weight rows
constexpr int kStageBytes = kTile * 64, kScaleBytes = kTile * 16;     // of codes; of the eight groups' scales that a step's are among
template <int RP> struct Tc {          // RP: rows of B (16, 32 or 64)
  static constexpr int WGS = RP == 16 ? 3 : 2, STAGES = RP == 16 ? 5 : RP == 32 ? 6 : 4, WORKERS = WGS * 4, THREADS = WGS * 160;
  static constexpr int ACT = RP * kStep * 2, STAGE = kStageBytes + ACT, WG_BYTES = STAGES * STAGE;     // codes, activations
  static constexpr int SCALES = WGS * WG_BYTES, BARS = SCALES + WGS * STAGES * kScaleBytes, SMEM = BARS + 512 + 1024;
};

struct W4TcArgs {
  CUtensorMap codes, scale_map;
  const __nv_bfloat16 *a, *scales;
  unsigned char *staged;               // activations of every step as they lie in shared memory
  float *out, *parts;
  int R, K, N, groups, steps;          // steps of a tile
  int total, line;                     // steps of all tiles; stretches they are divided over at most
  int mapped;                          // the scales have a tensor map
  u32 bits;                            // kCodeBits
  // Stretch w is [first(w), first(w + 1)); step x belongs to stretch of(x).
  __device__ __forceinline__ int first(int w) const { return total < line ? min(w, total) : (int)((long long)w * total / line); }
  __device__ __forceinline__ int of(int x) const { return total < line ? x : (int)((((long long)x + 1) * line - 1) / total); }
  // A stretch's sums of a tile that it does not hold whole: slot 0 where it begins inside of it, else 1; [row][weight row].
  __device__ __forceinline__ float *part(int w, int slot) const { return parts + ((size_t)w * 2 + slot) * R * kTile; }
};

// B: the descriptor's low word (address / 16); the high one says 8-row groups 1024 bytes apart, descriptor version, 128-byte swizzle.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_low, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tmov.b64 db, {%2, %5};\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_low), "r"(idesc), "r"(acc), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float *v) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr));
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Activations as the products read them: per step and 64 of k, RP rows (those past R zeros) of 128 bytes with the 128-byte swizzle,
// eight of k in a row in the order 0 4 1 5 2 6 3 7.  A thread has eight of k of a row.
template <int RP> __global__ void __launch_bounds__(128) w4_stage_kernel(const __grid_constant__ W4TcArgs p) {
  chain_wait();
  chain_next();
  const int x = blockIdx.x * 128 + threadIdx.x, step = x / (RP * (kStep / 8)), r = x / (kStep / 8) % RP, k8 = x % (kStep / 8), k = step * kStep + k8 * 8;
  if (step >= p.steps) return;
  const uint4 v = r < p.R && k < p.K ? __ldg(reinterpret_cast<const uint4 *>(p.a + (size_t)r * p.K + k)) : make_uint4(0, 0, 0, 0);
  *reinterpret_cast<uint4 *>(p.staged + (size_t)step * Tc<RP>::ACT + (k8 >> 3) * (RP * 128) + (r >> 3) * 1024 + (r & 7) * 128 + (((k8 & 7) ^ (r & 7)) << 4)) =
      make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
}

// G: group; RP: rows of B; RC: of them read back (8, or RP).
template <int G, int RP, int RC>
__global__ void __launch_bounds__(Tc<RP>::THREADS, 1)
w4_kernel(const __grid_constant__ W4TcArgs p) {
  using C = Tc<RP>;
  constexpr int U = kStep / G, ACOLS = G / 2;         // units (groups) of a step; columns of A
  constexpr uint32_t WG_COLS = 2 * ACOLS + 2 * RP;
  static_assert(C::WGS * WG_COLS <= 512, "tensor memory");
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int warp = warp_index(), lane = threadIdx.x & 31, row = threadIdx.x & 127;
  const bool worker = warp < C::WORKERS;
  const int wg = worker ? warp >> 2 : warp - C::WORKERS;
  unsigned char *mine = smem + wg * C::WG_BYTES;
  unsigned char *scales = smem + C::SCALES + wg * C::STAGES * kScaleBytes;
  const uint32_t ring = smem_u32(mine), scale_ring = smem_u32(scales), bars = smem_u32(smem + C::BARS) + wg * 128;
  auto full = [&](int s) { return bars + s * 8; };
  auto done = [&](int b) { return bars + 64 + b * 8; };
  auto ready = [&](int b) { return bars + 80 + b * 8; };
  volatile int *abort_flag = reinterpret_cast<int *>(smem + C::BARS + 384 + wg * 4);
  u32 *slot = reinterpret_cast<u32 *>(smem + C::BARS + 400);
  if (worker && row == 0) {
    for (int s = 0; s < C::STAGES; ++s) mbar_init(full(s), 1);
    mbar_init(ready(0), 4);
    mbar_init(ready(1), 4);
    mbar_init(done(0), 1);
    mbar_init(done(1), 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) tmem_alloc(smem_u32(slot), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *slot + wg * WG_COLS, lanes = (uint32_t)((warp & 3) * 32) << 16;
  const uint32_t idesc = umma_idesc_bf16(RP);
  chain_wait();
  chain_next();

  const int w = wg * (int)gridDim.x + (int)blockIdx.x, begin = p.first(w), n = p.first(w + 1) - begin;
  int tile = begin / p.steps, s = begin - tile * p.steps;
  if (n > 0 && !worker) {
    // ---------------------------------------------------------------- codes, products
    // (Every operation between two units' products counts: the workers wait for this warp, and it shares its issue slots with three of
    // theirs.  Addresses and descriptors go on by constants.)
    const bool issuer = elect_one();
    const uint32_t bytes = C::STAGE + (p.mapped ? kScaleBytes : 0);
    int ask_s = s, ask_stage = 0, ask_y = tile * kTile;                // the next step to ask for
    auto ask = [&] {
      if (issuer) {
        const uint32_t bar = full(ask_stage), to = ring + ask_stage * C::STAGE;
        mbar_expect_tx(bar, bytes);
        tma_load_2d(to, &p.codes, ask_s * (kStep / 2), ask_y, bar);
        bulk_load(to + kStageBytes, p.staged + (size_t)(uint32_t)ask_s * C::ACT, C::ACT, bar);
        if (p.mapped) tma_load_2d(scale_ring + ask_stage * kScaleBytes, &p.scale_map, (ask_s * U & ~7) * 2, ask_y, bar);
      }
      if (++ask_stage == C::STAGES) ask_stage = 0;
      if (++ask_s == p.steps) { ask_s = 0; ask_y += kTile; }
    };
    for (int i = 0; i < min(C::STAGES, n); ++i) ask();
    const uint32_t desc0 = ((ring + kStageBytes) & 0x3FFFFu) >> 4 | 1u << 16, desc_end = desc0 + C::STAGES * (C::STAGE >> 4);
    uint32_t desc = desc0, b = 0, phase = 0;                           // of the unit: which half of tensor memory, its barriers' parity
    for (int i = 0; i < n; ++i) {
      const int units = min(U, p.groups - s * U);
#pragma unroll 1
      for (int u = 0; u < units; ++u) {
        // (the workers have seen this stage's codes and activations land before they say so; waits that give up go on, here and there)
        mbar_wait_warp(ready(b), phase, abort_flag);
        tc_fence_after();
        if (issuer) {
          const uint32_t d = tmem + 2 * ACOLS + b * RP, A0 = tmem + b * ACOLS, at = desc + (u * (G / 16) >> 2) * (RP * 8) + (u * (G / 16) & 3) * 2;
#pragma unroll
          for (int q = 0; q < G / 16; ++q) umma_ts(d, A0 + q * 8, at + (q >> 2) * (RP * 8) + (q & 3) * 2, idesc, q > 0);        // 16 of k: 32 bytes of a row of B
          umma_commit(done(b));
        }
        __syncwarp();
        // The stage of the step before is free when this one's first products are ready behind its last ones.
        if (u == 0 && i > 0 && i - 1 + C::STAGES < n) {
          mbar_wait_warp(done(b ^ 1), b ? phase : phase ^ 1, abort_flag);
          ask();
        }
        phase ^= b;
        b ^= 1;
      }
      if (++s == p.steps) s = 0;
      desc += C::STAGE >> 4;
      if (desc == desc_end) desc = desc0;
    }
  } else if (n > 0) {
    // ---------------------------------------------------------------- codes -> pairs -> tensor memory -> sums
    float acc[RC];
#pragma unroll
    for (int r = 0; r < RC; ++r) acc[r] = 0.f;
    // Units' sums are added two units later, when their products have long been over: the next two units' pairs are made meanwhile.
    int count = 0, pending = 0;        // units so far; those whose sums are not added yet
    float scale0 = 0.f, scale1 = 0.f;  // theirs, the older first
    auto fold = [&] {
      const int x = count - pending, b = x & 1;
      mbar_wait(done(b), (uint32_t)((x >> 1) & 1), abort_flag);
      __syncwarp();
      tc_fence_after();
      const uint32_t d = tmem + lanes + 2 * ACOLS + b * RP;
#pragma unroll
      for (int c = 0; c < RC; c += 16) {
        float v[16];
        if constexpr (RC == 8) tmem_ld8(d, v);
        else tmem_ld16(d + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int r = 0; r < (RC < 16 ? RC : 16); ++r) acc[c + r] = fmaf(scale0, v[r], acc[c + r]);
      }
      scale0 = scale1;
      --pending;
    };
    const unsigned short *row_scales = reinterpret_cast<const unsigned short *>(p.scales) + (size_t)min(tile * kTile + row, p.N - 1) * p.groups;
    bool from_start = s == 0;          // of the tile
    int stage = 0;
    uint32_t full_phase = 0;
    for (int i = 0; i < n; ++i) {
      const bool last_s = s + 1 == p.steps;
      const int units = min(U, p.groups - s * U);
      mbar_wait(full(stage), full_phase, abort_flag);
      __syncwarp();
      const unsigned char *codes = mine + stage * C::STAGE + row * 64;
      const unsigned short *stage_scales = reinterpret_cast<const unsigned short *>(scales + stage * kScaleBytes + row * 16) + (s * U & 7);
#pragma unroll 1
      for (int u = 0; u < units; ++u) {
        const int b = count & 1;
        const u32 scale = p.mapped ? stage_scales[u] : row_scales[s * U + u];
        const uint32_t A = tmem + lanes + b * ACOLS;
        constexpr int HALF = G < 64 ? G : 64;                          // 32 columns of pairs at once at most
#pragma unroll
        for (int h = 0; h < G / HALF; ++h) {
          u32 x[HALF / 2];
#pragma unroll
          for (int q = 0; q < HALF / 32; ++q) {
            const uint4 v = *reinterpret_cast<const uint4 *>(codes + (((u * (G / 32) + h * 2 + q) ^ (row >> 1 & 3)) << 4));
            const u32 word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              x[q * 16 + y * 4] = pair<0>(word[y], p.bits);
              x[q * 16 + y * 4 + 1] = pair<1>(word[y], p.bits);
              x[q * 16 + y * 4 + 2] = pair<2>(word[y], p.bits);
              x[q * 16 + y * 4 + 3] = pair<3>(word[y], p.bits);
            }
          }
          if (h == 0 && pending == 2) fold();                          // (the products that read this half of tensor memory before are over then)
#pragma unroll
          for (int q = 0; q < HALF / 32; ++q) tmem_st16u(A + h * 32 + q * 16, x + q * 16);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(ready(b));
        (pending == 0 ? scale0 : scale1) = __uint_as_float(scale << 16);
        ++pending;
        ++count;
      }
      if (++stage == C::STAGES) { stage = 0; full_phase ^= 1; }
      if (last_s || i + 1 == n) {
        while (pending > 0) fold();
        const bool whole = last_s && from_start;
        const int nr = tile * kTile + row;
        float *to = whole ? p.out + nr : p.part(w, from_start ? 1 : 0) + row;
        const size_t pitch = whole ? p.N : kTile;
#pragma unroll
        for (int r = 0; r < RC; ++r) {
          if (r < p.R && (!whole || nr < p.N)) to[r * pitch] = *abort_flag ? NAN : acc[r];
          acc[r] = 0.f;
        }
        from_start = true;
      }
      if (last_s) {
        s = 0;
        row_scales += (size_t)(min((tile + 1) * kTile + row, p.N - 1) - min(tile * kTile + row, p.N - 1)) * p.groups;
        ++tile;
      } else {
        ++s;
      }
    }
  }
  if (*abort_flag) {                   // copies in flight land before the shared memory goes away
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) {}
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_dealloc(*slot, 512);
}

// Tiles that no stretch holds whole: a thread a weight row, four rows of activations.
__global__ void __launch_bounds__(128) w4_join_kernel(const __grid_constant__ W4TcArgs p) {
  const int tile = blockIdx.x, r0 = blockIdx.y * 4, n = tile * kTile + threadIdx.x, x = tile * p.steps;
  const int w0 = p.of(x), w1 = p.of(x + p.steps - 1);
  chain_wait();
  chain_next();
  if (w0 == w1) return;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int w = w0; w <= w1; ++w) {
    const float *from = p.part(w, w == w0 ? 1 : 0) + threadIdx.x;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r0 + r < p.R) sum[r] += from[(r0 + r) * kTile];
  }
  if (n >= p.N) return;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (r0 + r < p.R) p.out[(size_t)(r0 + r) * p.N + n] = sum[r];
}

int w4_rp(int R) { return R <= 16 ? 16 : R <= 32 ? 32 : 64; }
int w4_line(int R) { return kMeasuredSMs * (w4_rp(R) == 16 ? Tc<16>::WGS : Tc<32>::WGS); }

template <int G, int RP, int RC> int run_tc(const W4TcArgs &a, cudaStream_t s) {
  static std::atomic<u64> done{0};
  const int status = hsd_smem_limit((const void *)w4_kernel<G, RP, RC>, Tc<RP>::SMEM, done);
  if (status) return status;
  HSD_CUDA_OK(hsd_launch(w4_stage_kernel<RP>, dim3(ceil_div(a.steps * RP * (kStep / 8), 128)), 128, 0, s, 0, true, a));
  HSD_CUDA_OK(hsd_launch(w4_kernel<G, RP, RC>, dim3(kMeasuredSMs), Tc<RP>::THREADS, Tc<RP>::SMEM, s, 0, true, a));
  HSD_CUDA_OK(hsd_launch(w4_join_kernel, dim3(ceil_div(a.N, kTile), ceil_div(a.R, 4)), 128, 0, s, 0, true, a));
  hsd_count_launches(3);
  return hsd_launch_status();
}
template <int G> int run_tc_rows(const W4TcArgs &a, cudaStream_t s) {
  return a.R <= 8 ? run_tc<G, 16, 8>(a, s) : a.R <= 16 ? run_tc<G, 16, 16>(a, s) : a.R <= 32 ? run_tc<G, 32, 32>(a, s) : run_tc<G, 64, 64>(a, s);
}

bool takes_small(int R, long long N, int K) { return false; }

}  // namespace
}  // namespace hsd

extern "C" size_t hsd_gemm_w4_workspace_bytes(int R, int N, int K, int group) {
  using namespace hsd;
  if (R <= 0 || R > 64 || N <= 0 || K <= 0 || K > (1 << 26) || (group != 32 && group != 64 && group != 128) || K % group) return 0;
  return (size_t)w4_line(R) * 2 * R * kTile * sizeof(float) + (size_t)ceil_div(K, kStep) * w4_rp(R) * kStep * 2;
}

extern "C" int hsd_gemm_w4(const void *A, int R, int K, const void *codes, const void *scales, int N, int group, float *out, void *workspace,
                           size_t workspace_bytes, void *stream) {
  using namespace hsd;
  if (!A || !codes || !scales || !out || !workspace || R <= 0 || R > 64 || N <= 0 || K <= 0) return HSD_E_INVALID_ARG;
  if ((group != 32 && group != 64 && group != 128) || K % group) return HSD_E_INVALID_ARG;
  if (K > (1 << 26) || (long long)ceil_div(N, kTile) * ceil_div(K, kStep) > (1 << 30)) return HSD_E_TOO_LARGE;
  if (((reinterpret_cast<uintptr_t>(A) | reinterpret_cast<uintptr_t>(codes) | reinterpret_cast<uintptr_t>(workspace)) & 15) || (reinterpret_cast<uintptr_t>(scales) & 1) ||
      (reinterpret_cast<uintptr_t>(out) & 3)) return HSD_E_INVALID_ARG;
  if (workspace_bytes < hsd_gemm_w4_workspace_bytes(R, N, K, group)) return HSD_E_WORKSPACE_TOO_SMALL;
  cudaStream_t s = (cudaStream_t)stream;
  const auto *a = static_cast<const __nv_bfloat16 *>(A), *sc = static_cast<const __nv_bfloat16 *>(scales);
  if (takes_small(R, N, K)) {
    const W4Args p = {a, static_cast<const uint8_t *>(codes), sc, out, R, K, N, K / group, kCodeBits};
    return group == 128 ? run_small<4, 1, 1>(p, s) : group == 64 ? run_small<2, 1, 1>(p, s) : run_small<1, 1, 1>(p, s);
  }
  W4TcArgs p = {};
  const int status = tc_make_byte_map(&p.codes, codes, N, K / 2, kTile, 64);
  if (status) return status;
  p.a = a; p.scales = sc; p.out = out; p.parts = static_cast<float *>(workspace);
  p.staged = static_cast<unsigned char *>(workspace) + (size_t)w4_line(R) * 2 * R * kTile * sizeof(float);
  p.R = R; p.K = K; p.N = N; p.groups = K / group;
  p.steps = ceil_div(K, kStep);
  p.total = ceil_div(N, kTile) * p.steps;
  p.line = w4_line(R);
  p.bits = kCodeBits;
  if (p.groups % 8 == 0 && reinterpret_cast<uintptr_t>(scales) % 16 == 0) {
    const int s2 = tc_make_byte_map(&p.scale_map, scales, N, (long long)p.groups * 2, kTile, 16);
    if (s2) return s2;
    p.mapped = 1;
  }
  return group == 128 ? run_tc_rows<128>(p, s) : group == 64 ? run_tc_rows<64>(p, s) : run_tc_rows<32>(p, s);
}
