// New rows into a paged key-value cache, queries and keys rotated on the way (hsd_kv_append).
//   (y_i, y_{i+h}) = (x_i cos - x_{i+h} sin, x_{i+h} cos + x_i sin), h = head_dim / 2, cos and sin of the row's position from the
// caller's table; values are copied.  The products and the sum are rounded to fp32 (none fused), the result once to the pool's type.
// A thread takes eight pairs of one head of one row (16 bytes of a bf16 pool at each of the two places).  The rows' positions and
// pages come first: a warp a row counts the row starts that do not lie behind it.
// Bound by memory for prompts, by the chain row -> position -> page -> store for a few rows, whose heads are divided over CTAs.
#include "paged.cuh"

namespace hsd {
namespace {

constexpr int kThreads = 256, kRows = 4;       // rows of a CTA at most (8191 rows of 48 heads of 128: 39 us, of 8 45, of 2 49)

struct AppendArgs {
  const unsigned char *qkv;
  long long row_bytes;
  const int32_t *row_starts, *kv_lens, *page_table;
  const float *rope;
  unsigned char *q_out;
  PoolView pool;
  int rows, batch, pages_per_seq, n_positions, nq, nkv;
  int cta_rows, parts;                          // rows of a CTA, CTAs that share them
  bool zeros;                                   // the queries of skipped rows become zeros
};

template <typename T> __device__ __forceinline__ void load8(const unsigned char *p, float *f);
template <> __device__ __forceinline__ void load8<float>(const unsigned char *p, float *f) {
  const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const unsigned char *p, float *f) {
  const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
  f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
  f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
  f[4] = __uint_as_float(v.z << 16); f[5] = __uint_as_float(v.z & 0xFFFF0000u);
  f[6] = __uint_as_float(v.w << 16); f[7] = __uint_as_float(v.w & 0xFFFF0000u);
}
template <typename T> __device__ __forceinline__ void store8(unsigned char *p, const float *f);
template <> __device__ __forceinline__ void store8<float>(unsigned char *p, const float *f) {
  reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ u32 pack(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const u32 *>(&v);
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(unsigned char *p, const float *f) {
  *reinterpret_cast<uint4 *>(p) = make_uint4(pack(f[0], f[1]), pack(f[2], f[3]), pack(f[4], f[5]), pack(f[6], f[7]));
}

template <typename TI, typename TO, int HD>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(AppendArgs a) {
  constexpr int UNITS = HD / 16, HALF = HD / 2;
  static_assert(kRows == 4, "rows of a piece are found by three comparisons");
  __shared__ int sh_pos[kRows];                 // -1: the row is skipped
  __shared__ long long sh_at[kRows];            // its place in a head of the pools, in bytes
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  chain_wait();
  chain_next();
  const int r0 = (blockIdx.x / a.parts) * a.cta_rows, part = blockIdx.x % a.parts, n_rows = min(a.cta_rows, a.rows - r0);
  if (warp < n_rows) {
    const int r = r0 + warp;
    int seq = r, first = r;
    if (a.row_starts) {
      seq = 0;
      for (int i0 = 0; i0 < a.batch; i0 += 32) {
        const int i = i0 + lane;
        const u32 behind = __ballot_sync(0xFFFFFFFFu, i < a.batch && a.row_starts[i + 1] <= r);
        seq += __popc(behind);
        if (behind != 0xFFFFFFFFu) break;
      }
      first = seq < a.batch ? a.row_starts[seq] : r + 1;
    }
    if (lane == 0) {
      int pos = -1;
      long long at = 0;
      if (seq < a.batch && first <= r) {
        const int len = a.kv_lens[seq];
        const long long p = (long long)len + (r - first);
        if (len >= 0 && p < a.n_positions && p < (long long)a.pages_per_seq * a.pool.page) {
          const int pg = a.page_table[(size_t)seq * a.pages_per_seq + p / a.pool.page];
          if (pg >= 0 && pg < a.pool.n_pages) {
            pos = (int)p;
            at = pg * a.pool.page_bytes + (p % a.pool.page) * a.pool.token_bytes;
          }
        }
      }
      sh_pos[warp] = pos;
      sh_at[warp] = at;
    }
  }
  __syncthreads();
  const int per_row = (a.nq + 2 * a.nkv) * UNITS;
  for (int u = part * kThreads + threadIdx.x; u < n_rows * per_row; u += a.parts * kThreads) {
    const int row = (u >= per_row) + (u >= 2 * per_row) + (u >= 3 * per_row), x = u - row * per_row;
    const int h = x / UNITS, i = x % UNITS * 8, pos = sh_pos[row];
    if (pos < 0) {
      if (a.zeros && h < a.nq) {
        const float zero[8] = {};
        unsigned char *to = a.q_out + (((size_t)(r0 + row) * a.nq + h) * HD + i) * sizeof(TO);
        store8<TO>(to, zero);
        store8<TO>(to + HALF * sizeof(TO), zero);
      }
      continue;
    }
    const unsigned char *src = a.qkv + (size_t)(r0 + row) * a.row_bytes + ((size_t)h * HD + i) * sizeof(TI);
    float lo[8], hi[8];
    load8<TI>(src, lo);
    load8<TI>(src + HALF * sizeof(TI), hi);
    if (h < a.nq + a.nkv) {
      float c[8], s[8];
      const unsigned char *t = reinterpret_cast<const unsigned char *>(a.rope + (size_t)pos * HD + i);
      load8<float>(t, c);
      load8<float>(t + HALF * 4, s);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = lo[e], y = hi[e];
        lo[e] = __fsub_rn(__fmul_rn(x, c[e]), __fmul_rn(y, s[e]));
        hi[e] = __fadd_rn(__fmul_rn(y, c[e]), __fmul_rn(x, s[e]));
      }
    }
    unsigned char *dst;
    if (h < a.nq) dst = a.q_out + ((size_t)(r0 + row) * a.nq + h) * HD * sizeof(TO);
    else if (h < a.nq + a.nkv) dst = a.pool.k + (h - a.nq) * a.pool.head_bytes + sh_at[row];
    else dst = a.pool.v + (h - a.nq - a.nkv) * a.pool.head_bytes + sh_at[row];
    store8<TO>(dst + i * sizeof(TO), lo);
    store8<TO>(dst + (HALF + i) * sizeof(TO), hi);
  }
}

template <typename TI, typename TO> int run(AppendArgs &a, int hd, cudaStream_t s) {
  const int per_row = (a.nq + 2 * a.nkv) * (hd / 16);
  // few rows: one a CTA and a row's heads over several, so that every thread has one piece; many rows: CTAs of up to kRows
  a.cta_rows = a.rows >= kRows * 2 * kMeasuredSMs ? kRows : 1;
  a.parts = a.cta_rows > 1 ? 1 : ceil_div(per_row, kThreads);
  const long long grid = (long long)ceil_div(a.rows, a.cta_rows) * a.parts;
  if (grid > 0x7FFFFFFFll) return HSD_E_TOO_LARGE;
  switch (hd) {
    case 32: HSD_CUDA_OK(hsd_launch(kv_append_kernel<TI, TO, 32>, dim3((unsigned)grid), kThreads, 0, s, 0, true, a)); break;
    case 64: HSD_CUDA_OK(hsd_launch(kv_append_kernel<TI, TO, 64>, dim3((unsigned)grid), kThreads, 0, s, 0, true, a)); break;
    default: HSD_CUDA_OK(hsd_launch(kv_append_kernel<TI, TO, 128>, dim3((unsigned)grid), kThreads, 0, s, 0, true, a)); break;
  }
  hsd_count_launches(1);
  return hsd_launch_status();
}

int append(const void *qkv, int qkv_dtype, int rows, long long row_stride, int n_q_heads, int n_kv_heads, int head_dim, const int32_t *row_starts,
           const int32_t *kv_lens, int batch, const int32_t *page_table, int pages_per_seq, const float *rope, int n_positions,
           const hsd_kv_pool *pool, void *q_out, bool zeros, cudaStream_t s) {
  if (!qkv || !kv_lens || !page_table || !rope || rows <= 0 || batch <= 0 || n_q_heads < 0 || n_positions <= 0) return HSD_E_INVALID_ARG;
  if ((n_q_heads > 0 && !q_out) || (qkv_dtype != HSD_F32 && qkv_dtype != HSD_BF16) || (!row_starts && rows != batch)) return HSD_E_INVALID_ARG;
  if (!words(row_starts, kv_lens, page_table)) return HSD_E_INVALID_ARG;
  AppendArgs a = {};
  const int status = pool_view(pool, n_kv_heads, head_dim, pages_per_seq, a.pool);
  if (status) return status;
  if ((long long)n_q_heads + 2ll * n_kv_heads > 65536) return HSD_E_TOO_LARGE;
  const int e = qkv_dtype == HSD_F32 ? 4 : 2;
  a.row_bytes = row_stride * e;
  if (row_stride < (long long)(n_q_heads + 2 * n_kv_heads) * head_dim || (a.row_bytes & 15)) return HSD_E_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(qkv) | reinterpret_cast<uintptr_t>(rope) | reinterpret_cast<uintptr_t>(q_out)) & 15) return HSD_E_INVALID_ARG;
  a.qkv = static_cast<const unsigned char *>(qkv);
  a.row_starts = row_starts; a.kv_lens = kv_lens; a.page_table = page_table; a.rope = rope;
  a.q_out = static_cast<unsigned char *>(q_out);
  a.rows = rows; a.batch = batch; a.pages_per_seq = pages_per_seq; a.n_positions = n_positions; a.nq = n_q_heads; a.nkv = n_kv_heads;
  a.zeros = zeros;
  if (qkv_dtype == HSD_F32) return pool->dtype == HSD_F32 ? run<float, float>(a, head_dim, s) : run<float, __nv_bfloat16>(a, head_dim, s);
  return pool->dtype == HSD_F32 ? run<__nv_bfloat16, float>(a, head_dim, s) : run<__nv_bfloat16, __nv_bfloat16>(a, head_dim, s);
}

}  // namespace
}  // namespace hsd

extern "C" int hsd_kv_append(const void *qkv, int qkv_dtype, int rows, long long row_stride, int n_q_heads, int n_kv_heads, int head_dim,
                             const int32_t *row_starts, const int32_t *kv_lens, int batch, const int32_t *page_table, int pages_per_seq,
                             const float *rope, int n_positions, const hsd_kv_pool *pool, void *q_out, void *stream) {
  return hsd::append(qkv, qkv_dtype, rows, row_stride, n_q_heads, n_kv_heads, head_dim, row_starts, kv_lens, batch, page_table, pages_per_seq, rope,
                     n_positions, pool, q_out, false, (cudaStream_t)stream);
}

extern "C" int hsd_kv_append_zeros(const void *qkv, int qkv_dtype, int rows, long long row_stride, int n_q_heads, int n_kv_heads, int head_dim,
                                   const int32_t *row_starts, const int32_t *kv_lens, int batch, const int32_t *page_table, int pages_per_seq,
                                   const float *rope, int n_positions, const hsd_kv_pool *pool, void *q_out, void *stream) {
  return hsd::append(qkv, qkv_dtype, rows, row_stride, n_q_heads, n_kv_heads, head_dim, row_starts, kv_lens, batch, page_table, pages_per_seq, rope,
                     n_positions, pool, q_out, true, (cudaStream_t)stream);
}
