// Few-row products with 4-bit weights and group scales (hsd_gemm_w4): out[r, n] = sum_k A[r, k] (c[n, k] - 8) s[n, k / group].
// Bound by memory (half a byte a weight) up to some 16 rows; the weights never leave registers: a lane loads 32 codes of a weight row
// and makes bf16 pairs of them (0x4300 | c is 128 + c in bf16, less 136: exact), which are its operands of mma.sync with 16
// weight rows as the tile's rows and the activations as its columns.  The order of k inside a product is free, so it is the
// order in which the codes lie in a word: pairs (0,4), (1,5), (2,6), (3,7), the activations permuted alike.
// A group's products are summed in the tensor core's fp32, then scaled and added in fp32: no rounding to fewer bits anywhere.
// A CTA has 16 weight rows; its warps divide k (chunk by chunk in turn, so that together they read long pieces of a row), and
// where the matrix has few rows a cluster divides it once more.  Partial sums are added in a fixed order.
#include <cooperative_groups.h>

#include "common.cuh"

namespace hsd {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kChunk = 128;            // k of a warp's step: 16 bytes of codes a lane

struct W4Args {
  const __nv_bfloat16 *a;
  const uint8_t *codes;
  const __nv_bfloat16 *scales;
  float *out;
  int R, K, N, groups;                 // groups of a row
};

__device__ __forceinline__ void mma(float *c, const u32 *a, u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Codes i and i + 4 of a word, less 8, as two bf16.
template <int I> __device__ __forceinline__ u32 pair(u32 word) {
  const u32 x = ((word >> (4 * I)) & 0x000F000Fu) | 0x43004300u, bias = 0x43084308u;
  const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&bias));
  return *reinterpret_cast<const u32 *>(&y);
}

// GW: words of a lane in a group (group = 32 GW); RT: tiles of 8 activation rows; MT: tiles of 16 weight rows.
template <int GW, int RT, int MT>
__global__ void __launch_bounds__(kThreads)
gemm_w4_kernel(W4Args p) {
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
          const u32 lo[4] = {pair<0>(word[m][0][w]), pair<0>(word[m][1][w]), pair<1>(word[m][0][w]), pair<1>(word[m][1][w])};
          const u32 hi[4] = {pair<2>(word[m][0][w]), pair<2>(word[m][1][w]), pair<3>(word[m][0][w]), pair<3>(word[m][1][w])};
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

template <int GW, int RT, int MT> int run(const W4Args &a, cudaStream_t s) {
  const int tiles = ceil_div(a.N, MT * 16), chunks = ceil_div(a.K, kChunk);
  int parts = 1;
  while (parts < 8 && tiles * parts < kMeasuredSMs && parts * kWarps < chunks) parts *= 2;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 1; at.val.clusterDim.y = parts; at.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles, parts); cfg.blockDim = dim3(kThreads); cfg.stream = s; cfg.attrs = &at; cfg.numAttrs = parts > 1;
  HSD_CUDA_OK(cudaLaunchKernelEx(&cfg, gemm_w4_kernel<GW, RT, MT>, a));
  hsd_count_launches(1);
  return hsd_launch_status();
}
template <int GW> int run_rows(const W4Args &a, cudaStream_t s) {
  return a.R <= 8 ? run<GW, 1, 1>(a, s) : a.R <= 16 ? run<GW, 2, 1>(a, s) : a.R <= 32 ? run<GW, 4, 1>(a, s) : run<GW, 8, 1>(a, s);
}

}  // namespace
}  // namespace hsd

extern "C" int hsd_gemm_w4(const void *A, int R, int K, const void *codes, const void *scales, int N, int group, float *out, void *stream) {
  using namespace hsd;
  if (!A || !codes || !scales || !out || R <= 0 || R > 64 || N <= 0 || K <= 0) return HSD_E_INVALID_ARG;
  if ((group != 32 && group != 64 && group != 128) || K % group) return HSD_E_INVALID_ARG;
  if (K > (1 << 28)) return HSD_E_TOO_LARGE;
  if (((reinterpret_cast<uintptr_t>(A) | reinterpret_cast<uintptr_t>(codes)) & 15) || (reinterpret_cast<uintptr_t>(scales) & 1) || (reinterpret_cast<uintptr_t>(out) & 3)) return HSD_E_INVALID_ARG;
  W4Args a = {static_cast<const __nv_bfloat16 *>(A), static_cast<const uint8_t *>(codes), static_cast<const __nv_bfloat16 *>(scales), out, R, K, N, K / group};
  cudaStream_t s = (cudaStream_t)stream;
  return group == 128 ? run_rows<4>(a, s) : group == 64 ? run_rows<2>(a, s) : run_rows<1>(a, s);
}
