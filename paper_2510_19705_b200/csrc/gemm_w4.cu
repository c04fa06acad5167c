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

struct W4Args {
  const __nv_bfloat16 *a;
  const uint8_t *codes;
  const __nv_bfloat16 *scales;
  float *out;
  int R, K, N, groups, steps;          // groups of a row; steps of k
};

__device__ __forceinline__ void mma(float *c, const u32 *a, u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
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
// Codes i and i + 4 of a word, less 8, as two bf16.
template <int I> __device__ __forceinline__ u32 pair(u32 word) {
  const u32 x = ((word >> (4 * I)) & 0x000F000Fu) | 0x43004300u, bias = 0x43084308u;
  const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&bias));
  return *reinterpret_cast<const u32 *>(&y);
}

// GW: words of a lane in a group (group = 32 GW); RT: tiles of 8 activation rows.
// A CTA has 128 weight rows, 16 a warp, and [k_lo, k_hi) of k.  A warp's codes come through a ring of its own (cp.async, kStep of k a
// stage: 128 bytes of each of 16 rows); the activations of kBlock of k are staged once for all warps, in the order of the fragments
// and twice buffered, the next block's on their way in registers.
constexpr int kStep = 256, kStages = 4, kRowsCta = kWarps * 16;
template <int RT> constexpr int kBlock = RT >= 4 ? 256 : 1024 / RT;    // of k, at most 16 KB of activations
template <int RT> constexpr int kActBytes = RT * 8 * kBlock<RT> * 2;
template <int RT> constexpr int kSmem = kWarps * kStages * 2048 + 2 * kActBytes<RT>;

template <int GW, int RT>
__global__ void __launch_bounds__(kThreads)
gemm_w4_kernel(W4Args p) {
  constexpr int GROUPS = kStep / (32 * GW), WORDS = kStep / 32;        // groups and words of a step
  constexpr int BLOCK = kBlock<RT>, PIECES = kActBytes<RT> / 16 / kThreads;
  extern __shared__ __align__(128) unsigned char smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 3, lr = lane >> 2;
  const int parts = gridDim.y, part = blockIdx.y, n0 = blockIdx.x * kRowsCta + warp * 16;
  const int k_lo = (int)((long long)p.steps * part / parts) * kStep, k_hi = min((int)((long long)p.steps * (part + 1) / parts) * kStep, p.K);
  const u32 ring = (u32)__cvta_generic_to_shared(smem) + warp * kStages * 2048;
  unsigned char *act = smem + kWarps * kStages * 2048;

  // codes: lane i has piece i % 8 of rows i / 8, i / 8 + 4, ..; rows past the last are read as the last and not stored
  const uint8_t *from[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) from[i] = p.codes + (size_t)min(n0 + i * 4 + (lane >> 3), p.N - 1) * (p.K / 2) + (lane & 7) * 16;
  auto copy = [&](int k, int stage) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = i * 4 + (lane >> 3), c = lane & 7;
      if (k + c * 32 < k_hi) copy16(ring + stage * 2048 + r * 128 + ((c ^ swizzle(r)) << 4), from[i] + k / 2);
    }
  };
  // activations: piece i of a block is k8 = i % (BLOCK / 8) of row i / (BLOCK / 8)
  uint4 next[PIECES];
  auto fetch = [&](int k) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int x = i * kThreads + threadIdx.x, r = x / (BLOCK / 8), at = k + x % (BLOCK / 8) * 8;
      next[i] = r < p.R && at < k_hi ? __ldg(reinterpret_cast<const uint4 *>(p.a + (size_t)r * p.K + at)) : make_uint4(0, 0, 0, 0);
    }
  };
  auto put = [&](int buffer) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int x = i * kThreads + threadIdx.x, r = x / (BLOCK / 8), k8 = x % (BLOCK / 8), q = k8 % 16;
      const int w = (q / (4 * GW)) * GW + q % GW, jj = q / GW % 4;     // the lane's word and quarter of a chunk of 128
      const uint4 v = next[i];
      *reinterpret_cast<uint4 *>(act + buffer * kActBytes<RT> + ((((k8 / 16) * 4 + w) * RT * 8 + r) * 4 + jj) * 16) =
          make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
    }
  };

  float acc[RT][4];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int x = 0; x < 4; ++x) acc[t][x] = 0.f;
  fetch(k_lo);
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    copy(k_lo + i * kStep, i);
    copies_end();
  }
  const __nv_bfloat16 *scales[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) scales[h] = p.scales + (size_t)min(n0 + h * 8 + lr, p.N - 1) * p.groups;
  float scale[2][GROUPS];              // of the next step
  auto fetch_scales = [&](int k) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int i = k / (32 * GW) + g;
        scale[h][g] = i < p.groups && k < k_hi ? __bfloat162float(scales[h][i]) : 0.f;
      }
  };
  fetch_scales(k_lo);
  put(0);
  __syncthreads();

  int stage = 0, buffer = 0;
  for (int k0 = k_lo; k0 < k_hi; k0 += BLOCK) {
    const bool more = k0 + BLOCK < k_hi;
    if (more) fetch(k0 + BLOCK);
    for (int k = k0; k < min(k0 + BLOCK, k_hi); k += kStep) {
      copies_wait<kStages - 2>();
      __syncwarp();
      copy(k + (kStages - 1) * kStep, (stage + kStages - 1) % kStages);
      copies_end();
      float s[2][GROUPS];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) s[h][g] = scale[h][g];
      fetch_scales(k + kStep);
      u32 word[2][WORDS];
      const u32 codes = ring + stage * 2048;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          const int r = h * 8 + lr, byte = g * GW * 16 + j * GW * 4;
          load_words<GW>(&word[h][g * GW], codes + r * 128 + (((byte >> 4) ^ swizzle(r)) << 4) + (byte & 15));
        }
      const unsigned char *b0 = act + buffer * kActBytes<RT> + (k - k0) / 8 * RT * 8 * 16 + (lr * 4 + j) * 16;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        float sum[RT][4];
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) sum[t][x] = 0.f;
#pragma unroll
        for (int w = g * GW; w < (g + 1) * GW; ++w) {
          const u32 lo[4] = {pair<0>(word[0][w]), pair<0>(word[1][w]), pair<1>(word[0][w]), pair<1>(word[1][w])};
          const u32 hi[4] = {pair<2>(word[0][w]), pair<2>(word[1][w]), pair<3>(word[0][w]), pair<3>(word[1][w])};
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const uint4 b = *reinterpret_cast<const uint4 *>(b0 + (w * RT * 8 + t * 8) * 64);
            mma(sum[t], lo, b.x, b.y);
            mma(sum[t], hi, b.z, b.w);
          }
        }
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) acc[t][x] = fmaf(s[x >> 1][g], sum[t][x], acc[t][x]);
      }
      stage = (stage + 1) % kStages;
    }
    if (more) put(buffer ^ 1);
    buffer ^= 1;
    __syncthreads();
  }
  copies_wait<0>();

  if (parts == 1) {                    // a lane's eight output rows of a tile lie N apart, its two weight rows 8
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int n = n0 + lr + (x >> 1) * 8, r = t * 8 + j * 2 + (x & 1);
        if (r < p.R && n < p.N) p.out[(size_t)r * p.N + n] = acc[t][x];
      }
    return;
  }
  // the cluster's sums
  __syncthreads();
  float *sums = reinterpret_cast<float *>(smem);       // [RT * 8][kRowsCta]
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int x = 0; x < 4; ++x) sums[(t * 8 + j * 2 + (x & 1)) * kRowsCta + warp * 16 + lr + (x >> 1) * 8] = acc[t][x];
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  for (int i = part * kThreads + threadIdx.x; i < p.R * kRowsCta; i += parts * kThreads) {
    const int n = blockIdx.x * kRowsCta + i % kRowsCta;
    float s = 0.f;
    for (int q = 0; q < parts; ++q) s += *cluster.map_shared_rank(sums + i, q);
    if (n < p.N) p.out[(size_t)(i / kRowsCta) * p.N + n] = s;
  }
  cluster.sync();                      // no CTA leaves while others read its sums
}

template <int GW, int RT> int run(W4Args a, cudaStream_t s) {
  static std::atomic<u64> done{0};
  const int status = hsd_smem_limit((const void *)gemm_w4_kernel<GW, RT>, kSmem<RT>, done);
  if (status) return status;
  const int tiles = ceil_div(a.N, kRowsCta);
  a.steps = ceil_div(a.K, kStep);
  int parts = 1;
  while (parts < 8 && tiles * parts < 2 * kMeasuredSMs && parts * 2 <= a.steps) parts *= 2;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 1; at.val.clusterDim.y = parts; at.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles, parts); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = kSmem<RT>; cfg.stream = s; cfg.attrs = &at; cfg.numAttrs = parts > 1;
  HSD_CUDA_OK(cudaLaunchKernelEx(&cfg, gemm_w4_kernel<GW, RT>, a));
  hsd_count_launches(1);
  return hsd_launch_status();
}
template <int GW> int run_rows(const W4Args &a, cudaStream_t s) {
  return a.R <= 8 ? run<GW, 1>(a, s) : a.R <= 16 ? run<GW, 2>(a, s) : a.R <= 32 ? run<GW, 4>(a, s) : run<GW, 8>(a, s);
}

}  // namespace
}  // namespace hsd

extern "C" int hsd_gemm_w4(const void *A, int R, int K, const void *codes, const void *scales, int N, int group, float *out, void *stream) {
  using namespace hsd;
  if (!A || !codes || !scales || !out || R <= 0 || R > 64 || N <= 0 || K <= 0) return HSD_E_INVALID_ARG;
  if ((group != 32 && group != 64 && group != 128) || K % group) return HSD_E_INVALID_ARG;
  if (K > (1 << 28)) return HSD_E_TOO_LARGE;
  if (((reinterpret_cast<uintptr_t>(A) | reinterpret_cast<uintptr_t>(codes)) & 15) || (reinterpret_cast<uintptr_t>(scales) & 1) || (reinterpret_cast<uintptr_t>(out) & 3)) return HSD_E_INVALID_ARG;
  W4Args a = {static_cast<const __nv_bfloat16 *>(A), static_cast<const uint8_t *>(codes), static_cast<const __nv_bfloat16 *>(scales), out, R, K, N, K / group, 0};
  cudaStream_t s = (cudaStream_t)stream;
  return group == 128 ? run_rows<4>(a, s) : group == 64 ? run_rows<2>(a, s) : run_rows<1>(a, s);
}
