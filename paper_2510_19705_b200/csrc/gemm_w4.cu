// Few-row products with 4-bit weights and group scales (hsd_gemm_w4): out[r, n] = sum_k A[r, k] (c[n, k] - 8) s[n, k / group].
// Bound by memory: half a byte a weight.  What stands between that and the products is making bf16 of the codes, eleven operations
// for the eight codes of a word: c less 8 is made from the bits (0x4300 | c is 128 + c in bf16, less 136: exact), a pair at a time, and
// the pairs are (0,4), (1,5), (2,6), (3,7) of a word; the order of k inside a product is free, so the activations are put in the same.
// A group's products are summed in the tensor cores' fp32, then scaled and added in fp32: no rounding to fewer bits anywhere.
// The codes go from shared memory to registers once, as the operand of mma.sync that has 16 weight rows; the activations are its columns,
// eight a tile, brought into the order of its fragments by w4_stage_kernel.  w4_kernel: a warp has 16 weight rows, a CTA 128, all at the
// same k, and both operands come through one ring (cp.async).  Tiles' steps (256 of k) stand in one line that is divided evenly over
// the CTAs, two on an SM; where a stretch ends inside a tile its sums go to the workspace and w4_join_kernel adds them in order.
// (Pairs through tensor memory for tcgen05.mma, 128 rows a warpgroup: 25 us for 9 x 28672 x 4096; its chains of codes, pairs, products
// and sums wait for one another, and three warpgroups an SM do not cover that.)
// w4_small_kernel: up to eight rows of most matrices.
#include <cooperative_groups.h>

#include "common.cuh"

namespace hsd {
namespace {

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

// Eight of k in the order of a word's pairs: 0 4 1 5 2 6 3 7.
__device__ __forceinline__ uint4 pairs_of(const uint4 &v) {
  return make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
}

// ---------------------------------------------------------------------------- small products
// Up to eight rows.  A CTA has 16 weight rows; its warps divide k (chunk by chunk in turn, so that together they read long pieces of a
// row), and where the matrix has few rows a cluster divides it once more.  Codes and activations are loaded straight into registers:
// few of these, so that many warps hide the loads.  GW: words of a lane in a group (group = 32 GW).
template <int GW>
__global__ void __launch_bounds__(kThreads)
w4_small_kernel(W4Args p) {
  constexpr int GROUPS = 4 / GW;       // of a chunk
  __shared__ float sums[kWarps][16][8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 3, lr = lane >> 2;
  const int parts = gridDim.y, part = blockIdx.y, n0 = blockIdx.x * 16;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  chain_wait();
  chain_next();

  const int chunks = (p.K + kChunk - 1) / kChunk;
  for (int c = part * kWarps + warp; c < chunks; c += parts * kWarps) {
    u32 word[2][4];
    float scale[2][GROUPS];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = min(n0 + h * 8 + lr, p.N - 1);                     // rows past the last are read as the last and not stored
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int k = c * kChunk + g * GW * 32 + j * GW * 8, group = c * GROUPS + g;
        const bool in = group < p.groups;
        const uint8_t *at = p.codes + ((size_t)n * p.K + k) / 2;
        u32 *w = &word[h][g * GW];
        if constexpr (GW == 4) {
          const uint4 v = __ldg(reinterpret_cast<const uint4 *>(at));
          w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else if constexpr (GW == 2) {
          const uint2 v = in ? __ldg(reinterpret_cast<const uint2 *>(at)) : make_uint2(0, 0);
          w[0] = v.x; w[1] = v.y;
        } else {
          w[0] = in ? __ldg(reinterpret_cast<const u32 *>(at)) : 0u;
        }
        scale[h][g] = in ? __bfloat162float(p.scales[(size_t)n * p.groups + group]) : 0.f;
      }
    }
    uint4 b[4];                        // activations of the lane's row and words, as pairs in the codes' order
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int k = c * kChunk + w / GW * GW * 32 + j * GW * 8 + w % GW * 8;
      b[w] = lr < p.R && k < p.K ? pairs_of(__ldg(reinterpret_cast<const uint4 *>(p.a + (size_t)lr * p.K + k))) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = g * GW; w < (g + 1) * GW; ++w) {
        const u32 lo[4] = {pair<0>(word[0][w], p.bits), pair<0>(word[1][w], p.bits), pair<1>(word[0][w], p.bits), pair<1>(word[1][w], p.bits)};
        const u32 hi[4] = {pair<2>(word[0][w], p.bits), pair<2>(word[1][w], p.bits), pair<3>(word[0][w], p.bits), pair<3>(word[1][w], p.bits)};
        mma(sum, lo, b[w].x, b[w].y);
        mma(sum, hi, b[w].z, b[w].w);
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[x] = fmaf(scale[x >> 1][g], sum[x], acc[x]);
    }
  }

  // the warps' sums, then the cluster's
#pragma unroll
  for (int x = 0; x < 4; ++x) sums[warp][lr + (x >> 1) * 8][j * 2 + (x & 1)] = acc[x];
  __syncthreads();
  const int n = threadIdx.x & 15, r = threadIdx.x >> 4;                // of the first 128 threads
  float total = 0.f;
  if (threadIdx.x < 128)
#pragma unroll
    for (int w = 0; w < kWarps; ++w) total += sums[w][n][r];
  if (parts > 1) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    if (threadIdx.x < 128) sums[0][n][r] = total;                      // (read by this thread alone so far)
    cluster.sync();
    if (part == 0 && threadIdx.x < 128) {
      total = 0.f;
      for (int q = 0; q < parts; ++q) total += *cluster.map_shared_rank(&sums[0][n][r], q);
    }
    cluster.sync();                    // no CTA leaves while others read its sums
  }
  if (part == 0 && threadIdx.x < 128 && r < p.R && n0 + n < p.N) p.out[(size_t)r * p.N + n0 + n] = total;
}

template <int GW> int run_small(const W4Args &a, cudaStream_t s) {
  const int tiles = ceil_div(a.N, 16), chunks = ceil_div(a.K, kChunk);
  int parts = 1;
  while (parts < 8 && tiles * parts < kMeasuredSMs && parts * kWarps < chunks) parts *= 2;
  cudaLaunchAttribute at[2] = {};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 1; at[1].val.clusterDim.y = parts; at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles, parts); cfg.blockDim = dim3(kThreads); cfg.stream = s; cfg.attrs = at; cfg.numAttrs = 1 + (parts > 1);
  HSD_CUDA_OK(cudaLaunchKernelEx(&cfg, w4_small_kernel<GW>, a));
  hsd_count_launches(1);
  return hsd_launch_status();
}

// ---------------------------------------------------------------------------- large products
constexpr int kStep = 256;             // k of a step: 128 bytes of codes of a row
constexpr int kWide = 8, kTile = kWide * 16;   // warps; weight rows
constexpr int kLine = 2 * kMeasuredSMs;         // CTAs, two on an SM
constexpr int kCodeBytes = kTile * 128;
template <int RT> struct Ring {                // stages of a step's codes and activations
  static constexpr int ACT = RT * 8 * kStep * 2, STAGE = kCodeBytes + ACT, STAGES = RT == 8 ? 2 : RT == 4 ? 3 : 4, SMEM = STAGES * STAGE;
};

struct W4Line {
  const __nv_bfloat16 *a, *scales;
  const uint8_t *codes;
  unsigned char *staged;               // activations of every step in the order of the fragments
  float *out, *parts;
  int R, K, N, groups, steps;          // steps of a tile
  int total;                           // steps of all tiles
  int eights;                          // a row's scales are whole aligned eights
  u32 bits;                            // kCodeBits
  // Stretch w (of kLine) is [first(w), first(w + 1)); step x belongs to stretch of(x).
  __device__ __forceinline__ int first(int w) const { return total < kLine ? min(w, total) : (int)((long long)w * total / kLine); }
  __device__ __forceinline__ int of(int x) const { return total < kLine ? x : (int)((((long long)x + 1) * kLine - 1) / total); }
  // A stretch's sums of a tile that it does not hold whole: slot 0 where it begins inside of it, else 1; [row][weight row].
  __device__ __forceinline__ float *part(int w, int slot) const { return parts + ((size_t)w * 2 + slot) * R * kTile; }
};

__device__ __forceinline__ void copy16(u32 to, const void *from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// 16-byte pieces of row r of a stage are permuted by this: reads of 4 bytes by 8 rows x 4 lanes, and of 16 by 2 rows x 4, meet no bank twice.
__device__ __forceinline__ int swizzle(int r) { return (r & 1) << 2 | (r >> 1 & 3); }
template <int GW> __device__ __forceinline__ void load_words(u32 *w, u32 at) {
  if constexpr (GW == 4) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
  else if constexpr (GW == 2) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
  else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
}

// Activations as a lane of w4_kernel takes them: per step, word of the step and tile of eight rows, 16 bytes a lane (its row's eight of k
// behind that word, in the order 0 4 1 5 2 6 3 7).  Rows past R and k past K are zeros.
__global__ void __launch_bounds__(128) w4_stage_kernel(W4Line p, int gw, int rt) {
  chain_wait();
  chain_next();
  const int x = blockIdx.x * 128 + threadIdx.x, lane = x & 31, t = (x >> 5) % rt, word = (x >> 5) / rt % 8, step = (x >> 5) / (rt * 8);
  if (step >= p.steps) return;
  const int r = t * 8 + (lane >> 2), k = step * kStep + word / gw * gw * 32 + (lane & 3) * gw * 8 + word % gw * 8;
  reinterpret_cast<uint4 *>(p.staged)[x] = r < p.R && k < p.K ? pairs_of(__ldg(reinterpret_cast<const uint4 *>(p.a + (size_t)r * p.K + k))) : make_uint4(0, 0, 0, 0);
}

// GW: words of a lane in a group (group = 32 GW); RT: tiles of eight activation rows.
template <int GW, int RT>
__global__ void __launch_bounds__(kWide * 32, 2)
w4_kernel(W4Line p) {
  constexpr int U = 8 / GW;            // groups of a step
  using R = Ring<RT>;
  constexpr int kStages = R::STAGES;
  extern __shared__ __align__(128) unsigned char smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 3, lr = lane >> 2;
  const u32 ring = (u32)__cvta_generic_to_shared(smem);
  chain_wait();
  chain_next();
  const int w = blockIdx.x, begin = p.first(w), n = p.first(w + 1) - begin;
  if (n <= 0) return;
  int tile = begin / p.steps, s = begin - tile * p.steps;

  // codes: lane i has piece i % 8 of rows i / 8, i / 8 + 4, ..; rows past the last are read as the last and not stored
  const int c = lane & 7, cr = lane >> 3;
  int ask_tile = tile, ask_s = s, ask_stage = 0;
  const uint8_t *from[4];
  auto rows_of = [&](int t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) from[i] = p.codes + (size_t)min(t * kTile + warp * 16 + i * 4 + cr, p.N - 1) * (p.K / 2) + c * 16;
  };
  rows_of(tile);
  auto ask = [&] {
    if (ask_s * kStep + c * 32 < p.K) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = i * 4 + cr;
        copy16(ring + ask_stage * R::STAGE + (warp * 16 + r) * 128 + ((c ^ swizzle(r)) << 4), from[i] + ask_s * (kStep / 2));
      }
    }
#pragma unroll
    for (int i = 0; i < R::ACT / 16 / (kWide * 32); ++i) {
      const int x = (i * kWide * 32 + threadIdx.x) * 16;
      copy16(ring + ask_stage * R::STAGE + kCodeBytes + x, p.staged + (size_t)ask_s * R::ACT + x);
    }
    if (++ask_stage == kStages) ask_stage = 0;
    if (++ask_s == p.steps) { ask_s = 0; rows_of(++ask_tile); }
  };
#pragma unroll 1
  for (int i = 0; i < kStages - 1; ++i) {
    if (i < n) ask();
    copies_end();
  }
  // scales of the lane's two rows: the eight groups' that the step's are the first of, the next eight on their way
  const __nv_bfloat16 *row_scales[2];
  uint4 now[2], next[2];
  auto scale_rows = [&](int t) {
#pragma unroll
    for (int h = 0; h < 2; ++h) row_scales[h] = p.scales + (size_t)min(t * kTile + warp * 16 + h * 8 + lr, p.N - 1) * p.groups;
  };
  auto fetch_eight = [&](int g) {
#pragma unroll
    for (int h = 0; h < 2; ++h) next[h] = __ldg(reinterpret_cast<const uint4 *>(row_scales[h] + g));
  };
  auto shift = [&] {                   // by a step's
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (U == 2) now[h] = make_uint4(now[h].y, now[h].z, now[h].w, 0);
      else if constexpr (U == 4) now[h] = make_uint4(now[h].z, now[h].w, 0, 0);
    }
  };
  int scale_tile = tile;
  scale_rows(tile);
  if (p.eights) fetch_eight(s * U & ~7);

  float acc[RT][4];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int x = 0; x < 4; ++x) acc[t][x] = 0.f;
  bool from_start = s == 0;            // of the tile
  int stage = 0;
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    copies_wait<kStages - 2>();
    __syncthreads();                   // (a step's copies are all warps', and so is the stage that is filled again)
    if (i + kStages - 1 < n) ask();
    copies_end();
    if (p.eights) {
      if (i == 0 || (s * U & 7) == 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) now[h] = next[h];
        if (i == 0)
          for (int x = (s * U & 7) / U; x > 0; --x) shift();
        int g = (s * U & ~7) + 8;
        if (g == p.groups) { g = 0; scale_rows(++scale_tile); }
        fetch_eight(g);                // (behind the last tile: its last row's again)
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const unsigned short *at = reinterpret_cast<const unsigned short *>(row_scales[h]) + s * U;
        u32 q[4] = {0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (s * U + u < p.groups) q[u / 2] |= (u32)at[u] << (u % 2 * 16);
        now[h] = make_uint4(q[0], q[1], q[2], q[3]);
      }
    }
    const uint4 *b_at = reinterpret_cast<const uint4 *>(smem + stage * R::STAGE + kCodeBytes) + lane;
    const u32 codes = ring + stage * R::STAGE + warp * 16 * 128;
    u32 word[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int g = 0; g < U; ++g) {
        const int r = h * 8 + lr, byte = g * GW * 16 + j * GW * 4;
        load_words<GW>(&word[h][g * GW], codes + r * 128 + (((byte >> 4) ^ swizzle(r)) << 4) + (byte & 15));
      }
#pragma unroll
    for (int g = 0; g < U; ++g) {
      float sum[RT][4], sum2[RT][4];   // of a word's two products each: half as long a chain
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) sum[t][x] = sum2[t][x] = 0.f;
#pragma unroll
      for (int q = g * GW; q < (g + 1) * GW; ++q) {
        uint4 b[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) b[t] = b_at[(q * RT + t) * 32];
        const u32 lo[4] = {pair<0>(word[0][q], p.bits), pair<0>(word[1][q], p.bits), pair<1>(word[0][q], p.bits), pair<1>(word[1][q], p.bits)};
        const u32 hi[4] = {pair<2>(word[0][q], p.bits), pair<2>(word[1][q], p.bits), pair<3>(word[0][q], p.bits), pair<3>(word[1][q], p.bits)};
#pragma unroll
        for (int t = 0; t < RT; ++t) mma(sum[t], lo, b[t].x, b[t].y);
#pragma unroll
        for (int t = 0; t < RT; ++t) mma(RT > 2 ? sum[t] : sum2[t], hi, b[t].z, b[t].w);
      }
      float scale[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32 two = g / 2 == 0 ? now[h].x : g / 2 == 1 ? now[h].y : g / 2 == 2 ? now[h].z : now[h].w;
        scale[h] = __uint_as_float(g % 2 ? two & 0xFFFF0000u : two << 16);
      }
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[t][x] = fmaf(scale[x >> 1], RT > 2 ? sum[t][x] : sum[t][x] + sum2[t][x], acc[t][x]);
    }
    if (p.eights) shift();
    if (++stage == kStages) stage = 0;
    const bool last = s + 1 == p.steps;
    if (last || i + 1 == n) {
      const bool whole = last && from_start;
      float *to = whole ? p.out + tile * kTile : p.part(w, from_start ? 1 : 0);
      const size_t pitch = whole ? p.N : kTile;
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int row = warp * 16 + lr + (x >> 1) * 8, r = t * 8 + j * 2 + (x & 1);
          if (r < p.R && tile * kTile + row < p.N) to[r * pitch + row] = acc[t][x];
          acc[t][x] = 0.f;
        }
      from_start = true;
    }
    if (last) {
      s = 0;
      ++tile;
      if (!p.eights) scale_rows(tile);
    } else {
      ++s;
    }
  }
  copies_wait<0>();
}

// Tiles that no stretch holds whole: a thread a weight row, four rows of activations.
__global__ void __launch_bounds__(kTile) w4_join_kernel(W4Line p) {
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

template <int GW, int RT> int run_line(const W4Line &a, cudaStream_t s) {
  static std::atomic<u64> done{0};
  const int status = hsd_smem_limit((const void *)w4_kernel<GW, RT>, Ring<RT>::SMEM, done);
  if (status) return status;
  HSD_CUDA_OK(hsd_launch(w4_stage_kernel, dim3(a.steps * RT * 2), 128, 0, s, 0, true, a, GW, RT));
  HSD_CUDA_OK(hsd_launch(w4_kernel<GW, RT>, dim3(kLine), kWide * 32, Ring<RT>::SMEM, s, 0, true, a));
  HSD_CUDA_OK(hsd_launch(w4_join_kernel, dim3(ceil_div(a.N, kTile), ceil_div(a.R, 4)), kTile, 0, s, 0, true, a));
  hsd_count_launches(3);
  return hsd_launch_status();
}
template <int GW> int run_line_rows(const W4Line &a, cudaStream_t s) {
  return a.R <= 8 ? run_line<GW, 1>(a, s) : a.R <= 16 ? run_line<GW, 2>(a, s) : a.R <= 32 ? run_line<GW, 4>(a, s) : run_line<GW, 8>(a, s);
}
int w4_tiles(int R) { return R <= 8 ? 1 : R <= 16 ? 2 : R <= 32 ? 4 : 8; }

// Up to eight rows: one launch of loads straight into registers, or the ring's three launches.  us of the one / the other, by the weights:
//   groups of 32, whose codes come in pieces of 4 bytes: 8192 x 4096, 1 / 8 rows 11.9 / 13.2 and 13.7 / 13.9; 11008 x 4096 16.9 / 14.3 and 19.6 / 15.3
//   groups of 64: 8192 x 8192 15.5 / 16.6 and 16.8 / 17.5; 20480 x 4096, 1 / 4 / 8 rows 17.6 / 17.9, 18.7 / 18.0, 21.6 / 18.3
//   groups of 128: 8192 x 8192, 1 / 8 rows 13.5 / 16.1 and 15.8 / 16.8; 20480 x 4096, 1 / 4 / 8 rows 16.6 / 17.5, 17.1 / 17.6, 21.1 / 18.0;
//     28672 x 4096, 1 / 4 rows 21.2 / 22.0 and 21.7 / 22.1; 128256 x 2048 45.8 / 39.7 and 47.1 / 40.1
// (Below the limits the ring was at most 0.8 us ahead, at 4096 x 14336 with one row.)
bool takes_small(int R, int N, int K, int group) {
  const long long weights = (long long)N * K;
  return R <= 8 && weights <= (group == 32 ? 40000000 : group == 128 && R <= 4 ? 120000000 : 70000000);
}

}  // namespace
}  // namespace hsd

extern "C" size_t hsd_gemm_w4_workspace_bytes(int R, int N, int K, int group) {
  using namespace hsd;
  if (R <= 0 || R > 64 || N <= 0 || K <= 0 || K > (1 << 27) || (group != 32 && group != 64 && group != 128) || K % group) return 0;
  return (size_t)kLine * 2 * R * kTile * sizeof(float) + (size_t)ceil_div(K, kStep) * w4_tiles(R) * 8 * kStep * 2;
}

extern "C" int hsd_gemm_w4(const void *A, int R, int K, const void *codes, const void *scales, int N, int group, float *out, void *workspace,
                           size_t workspace_bytes, void *stream) {
  using namespace hsd;
  if (!A || !codes || !scales || !out || !workspace || R <= 0 || R > 64 || N <= 0 || K <= 0) return HSD_E_INVALID_ARG;
  if ((group != 32 && group != 64 && group != 128) || K % group) return HSD_E_INVALID_ARG;
  if (N > 0x7FFFFF00 || K > (1 << 27) || (long long)ceil_div(N, kTile) * ceil_div(K, kStep) > (1 << 30)) return HSD_E_TOO_LARGE;
  if (((reinterpret_cast<uintptr_t>(A) | reinterpret_cast<uintptr_t>(codes) | reinterpret_cast<uintptr_t>(workspace)) & 15) || (reinterpret_cast<uintptr_t>(scales) & 1) ||
      (reinterpret_cast<uintptr_t>(out) & 3)) return HSD_E_INVALID_ARG;
  if (workspace_bytes < hsd_gemm_w4_workspace_bytes(R, N, K, group)) return HSD_E_WORKSPACE_TOO_SMALL;
  cudaStream_t s = (cudaStream_t)stream;
  const auto *a = static_cast<const __nv_bfloat16 *>(A), *sc = static_cast<const __nv_bfloat16 *>(scales);
  if (takes_small(R, N, K, group)) {
    const W4Args p = {a, static_cast<const uint8_t *>(codes), sc, out, R, K, N, K / group, kCodeBits};
    return group == 128 ? run_small<4>(p, s) : group == 64 ? run_small<2>(p, s) : run_small<1>(p, s);
  }
  W4Line p = {};
  p.codes = static_cast<const uint8_t *>(codes);
  p.a = a; p.scales = sc; p.out = out; p.parts = static_cast<float *>(workspace);
  p.staged = static_cast<unsigned char *>(workspace) + (size_t)kLine * 2 * R * kTile * sizeof(float);
  p.R = R; p.K = K; p.N = N; p.groups = K / group;
  p.steps = ceil_div(K, kStep);
  p.total = ceil_div(N, kTile) * p.steps;
  p.bits = kCodeBits;
  p.eights = p.groups % 8 == 0 && reinterpret_cast<uintptr_t>(scales) % 16 == 0;
  return group == 128 ? run_line_rows<4>(p, s) : group == 64 ? run_line_rows<2>(p, s) : run_line_rows<1>(p, s);
}
