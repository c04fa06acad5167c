// New rows into a paged key-value cache, queries and keys rotated on the way (hsd_kv_append), and normalised before it by head
// (hsd_kv_append_norm: x becomes x / sqrt(mean x^2 + eps) * gain).
//   (y_i, y_{i+h}) = (x_i cos - x_{i+h} sin, x_{i+h} cos + x_i sin), h = head_dim / 2, cos and sin of the row's position from the
// caller's table; values are copied.  The products and the sum are rounded to fp32 (none fused), the result once to the pool's type.
// A thread takes eight pairs of one head after the other of one row (16 bytes of a bf16 pool at each of the two places).  The rows' positions and
// pages come first: a warp a row counts the row starts that do not lie behind it.  The norm's sum of squares goes over the two to eight
// neighbouring threads of a head, from the values they hold anyway: nothing is read twice.
// Bound by memory for prompts, by the chain row -> position -> page -> store for a few rows, whose heads are divided over CTAs.
#include <math.h>
#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace hsd {
namespace {

constexpr int kThreads = 256, kCtasPerSm = 4;
constexpr int kRows = 8;                       // rows of a CTA at most

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
  const unsigned char *q_gain, *k_gain;         // norm: of a head's values, or null (1)
  float eps;
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
// Eight gains as they lie in memory (registers cost CTAs here).
template <typename T> struct Gain8;
template <> struct Gain8<float> {
  float f[8];
  __device__ __forceinline__ void load(const unsigned char *p) { load8<float>(p, f); }
  __device__ __forceinline__ void ones() {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 1.f;
  }
  __device__ __forceinline__ float get(int e) const { return f[e]; }
};
template <> struct Gain8<__nv_bfloat16> {
  u32 w[4];
  __device__ __forceinline__ void load(const unsigned char *p) {
    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  }
  __device__ __forceinline__ void ones() { w[0] = w[1] = w[2] = w[3] = 0x3F803F80u; }
  __device__ __forceinline__ float get(int e) const { return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16); }
};
template <> struct Gain8<void> {};
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

// 1 / sqrt(mean of a head's squares + eps), from the 16 values that each of its threads has.
template <int HD>
__device__ __forceinline__ float norm(float eps, const float *lo, const float *hi) {
  constexpr int UNITS = HD / 16;
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum = fmaf(lo[e], lo[e], fmaf(hi[e], hi[e], sum));
  const u32 head = ((1u << UNITS) - 1) << (threadIdx.x & 31 & ~(UNITS - 1));       // the head's threads go through the loop together
#pragma unroll
  for (int o = 1; o < UNITS; o <<= 1) sum += __shfl_xor_sync(head, sum, o);
  return __frsqrt_rn(__fadd_rn(sum * (1.f / HD), eps));
}

template <typename TI, typename TO, typename TG, int HD>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)        // (with the norm: 8191 rows of 48 heads of 128 41 us; three CTAs an SM 50, five, which spill, 49)
kv_append_kernel(AppendArgs a) {
  constexpr int UNITS = HD / 16, HALF = HD / 2;
  static_assert(kThreads % kRows == 0 && kThreads / kRows % UNITS == 0, "a row has whole heads' threads");
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
  // A thread has the same 16 places of one head after the other of a row: angles and gains stay in its registers.
  constexpr bool NORM = !std::is_void<TG>::value;
  const int row_threads = kThreads / a.cta_rows, row = threadIdx.x / row_threads, x = part * row_threads + threadIdx.x % row_threads;
  if (row >= n_rows) return;
  const int heads = a.nq + 2 * a.nkv, turned = a.nq + a.nkv, i = x % UNITS * 8, step = a.parts * row_threads / UNITS, pos = sh_pos[row];
  if (pos < 0) {
    if (!a.zeros) return;
    for (int h = x / UNITS; h < a.nq; h += step) {
      const float zero[8] = {};
      unsigned char *to = a.q_out + (((size_t)(r0 + row) * a.nq + h) * HD + i) * sizeof(TO);
      store8<TO>(to, zero);
      store8<TO>(to + HALF * sizeof(TO), zero);
    }
    return;
  }
  const unsigned char *src = a.qkv + (size_t)(r0 + row) * a.row_bytes + i * sizeof(TI);
  const long long at = sh_at[row];
  float c[8], s[8];
  Gain8<TG> g, g2;
  const unsigned char *t = reinterpret_cast<const unsigned char *>(a.rope + (size_t)pos * HD + i);
  load8<float>(t, c);
  load8<float>(t + HALF * 4, s);
  auto gains = [&](const unsigned char *from) {
    if constexpr (NORM) {
      g.ones();
      g2.ones();
      if (from) {
        g.load(from + i * sizeof(TG));
        g2.load(from + (i + HALF) * sizeof(TG));
      }
    }
  };
  // heads from .. to - 1, whose first has its place at dst, the others head_bytes apart
  auto run = [&](int &h, int to, unsigned char *dst, long long head_bytes, bool turn) {
    dst += h * head_bytes + i * sizeof(TO);
#pragma unroll 1
    for (; h < to; h += step, dst += step * head_bytes) {
      float lo[8], hi[8];
      load8<TI>(src + (size_t)h * HD * sizeof(TI), lo);
      load8<TI>(src + ((size_t)h * HD + HALF) * sizeof(TI), hi);
      if (turn) {
        if constexpr (NORM) {
          const float f = norm<HD>(a.eps, lo, hi);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            lo[e] = lo[e] * f * g.get(e);
            hi[e] = hi[e] * f * g2.get(e);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = lo[e], y = hi[e];
          lo[e] = __fsub_rn(__fmul_rn(x, c[e]), __fmul_rn(y, s[e]));
          hi[e] = __fadd_rn(__fmul_rn(y, c[e]), __fmul_rn(x, s[e]));
        }
      }
      store8<TO>(dst, lo);
      store8<TO>(dst + HALF * sizeof(TO), hi);
    }
  };
  int h = x / UNITS;
  gains(a.q_gain);
  run(h, a.nq, a.q_out + (size_t)(r0 + row) * a.nq * HD * sizeof(TO), HD * sizeof(TO), true);
  gains(a.k_gain);
  run(h, turned, a.pool.k + at - a.nq * a.pool.head_bytes, a.pool.head_bytes, true);
  run(h, heads, a.pool.v + at - turned * a.pool.head_bytes, a.pool.head_bytes, false);
}

template <typename TI, typename TO, typename TG> int run(AppendArgs &a, int hd, cudaStream_t s) {
  const int per_row = (a.nq + 2 * a.nkv) * (hd / 16);
  // As few rows a CTA as let all CTAs run at once, and few rows' heads divided over as many as do.  us against twice the rows a CTA: 48 heads of 128, 800
  // rows, two a CTA 4.9 / 6.1, 1184 6.7 / 8.1, 2368, four 13.4 / 15.9, 8191, eight 37.5 (four 38.3); 144 heads, 592 rows, one 11.1 / 12.8, 1184, two 18.3 /
  // 21.8, 2368, four 32.3 / 38.9; 200 rows, a row over two CTAs 4.9, over five, of which 592 run at once, 5.9.  With the norm likewise (1184 rows 7.7 / 9.5, 2368 14.5 / 17.7).
  constexpr int at_once = kCtasPerSm * kMeasuredSMs;
  a.cta_rows = a.rows <= at_once ? 1 : a.rows <= 2 * at_once ? 2 : a.rows <= 4 * at_once ? 4 : kRows;
  a.parts = a.cta_rows > 1 ? 1 : std::max(1, std::min(ceil_div(per_row, kThreads), at_once / a.rows));
  const long long grid = (long long)ceil_div(a.rows, a.cta_rows) * a.parts;
  if (grid > 0x7FFFFFFFll) return HSD_E_TOO_LARGE;
  switch (hd) {
    case 32: HSD_CUDA_OK(hsd_launch(kv_append_kernel<TI, TO, TG, 32>, dim3((unsigned)grid), kThreads, 0, s, 0, true, a)); break;
    case 64: HSD_CUDA_OK(hsd_launch(kv_append_kernel<TI, TO, TG, 64>, dim3((unsigned)grid), kThreads, 0, s, 0, true, a)); break;
    default: HSD_CUDA_OK(hsd_launch(kv_append_kernel<TI, TO, TG, 128>, dim3((unsigned)grid), kThreads, 0, s, 0, true, a)); break;
  }
  hsd_count_launches(1);
  return hsd_launch_status();
}
template <typename TG> int run_types(AppendArgs &a, int from, int to, int hd, cudaStream_t s) {
  if (from == HSD_F32) return to == HSD_F32 ? run<float, float, TG>(a, hd, s) : run<float, __nv_bfloat16, TG>(a, hd, s);
  return to == HSD_F32 ? run<__nv_bfloat16, float, TG>(a, hd, s) : run<__nv_bfloat16, __nv_bfloat16, TG>(a, hd, s);
}

struct Norm { const void *q_gain, *k_gain; int gain_dtype; float eps; };

int append(const void *qkv, int qkv_dtype, int rows, long long row_stride, int n_q_heads, int n_kv_heads, int head_dim, const int32_t *row_starts,
           const int32_t *kv_lens, int batch, const int32_t *page_table, int pages_per_seq, const float *rope, int n_positions,
           const hsd_kv_pool *pool, void *q_out, bool zeros, const Norm *norm, cudaStream_t s) {
  if (!qkv || !kv_lens || !page_table || !rope || rows <= 0 || batch <= 0 || n_q_heads < 0 || n_positions <= 0) return HSD_E_INVALID_ARG;
  if ((n_q_heads > 0 && !q_out) || (qkv_dtype != HSD_F32 && qkv_dtype != HSD_BF16) || (!row_starts && rows != batch)) return HSD_E_INVALID_ARG;
  if (!words(row_starts, kv_lens, page_table)) return HSD_E_INVALID_ARG;
  AppendArgs a = {};
  if (norm) {
    if ((norm->gain_dtype != HSD_F32 && norm->gain_dtype != HSD_BF16) || !(norm->eps >= 0.f) || isinf(norm->eps)) return HSD_E_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(norm->q_gain) | reinterpret_cast<uintptr_t>(norm->k_gain)) & 15) return HSD_E_INVALID_ARG;
    a.q_gain = static_cast<const unsigned char *>(norm->q_gain);
    a.k_gain = static_cast<const unsigned char *>(norm->k_gain);
    a.eps = norm->eps;
  }
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
  if (!norm) return run_types<void>(a, qkv_dtype, pool->dtype, head_dim, s);
  return norm->gain_dtype == HSD_F32 ? run_types<float>(a, qkv_dtype, pool->dtype, head_dim, s) : run_types<__nv_bfloat16>(a, qkv_dtype, pool->dtype, head_dim, s);
}

}  // namespace
}  // namespace hsd

extern "C" int hsd_kv_append(const void *qkv, int qkv_dtype, int rows, long long row_stride, int n_q_heads, int n_kv_heads, int head_dim,
                             const int32_t *row_starts, const int32_t *kv_lens, int batch, const int32_t *page_table, int pages_per_seq,
                             const float *rope, int n_positions, const hsd_kv_pool *pool, void *q_out, void *stream) {
  return hsd::append(qkv, qkv_dtype, rows, row_stride, n_q_heads, n_kv_heads, head_dim, row_starts, kv_lens, batch, page_table, pages_per_seq, rope,
                     n_positions, pool, q_out, false, nullptr, (cudaStream_t)stream);
}

extern "C" int hsd_kv_append_zeros(const void *qkv, int qkv_dtype, int rows, long long row_stride, int n_q_heads, int n_kv_heads, int head_dim,
                                   const int32_t *row_starts, const int32_t *kv_lens, int batch, const int32_t *page_table, int pages_per_seq,
                                   const float *rope, int n_positions, const hsd_kv_pool *pool, void *q_out, void *stream) {
  return hsd::append(qkv, qkv_dtype, rows, row_stride, n_q_heads, n_kv_heads, head_dim, row_starts, kv_lens, batch, page_table, pages_per_seq, rope,
                     n_positions, pool, q_out, true, nullptr, (cudaStream_t)stream);
}

extern "C" int hsd_kv_append_norm(const void *qkv, int qkv_dtype, int rows, long long row_stride, int n_q_heads, int n_kv_heads, int head_dim,
                                  const void *q_gain, const void *k_gain, int gain_dtype, float eps, const int32_t *row_starts,
                                  const int32_t *kv_lens, int batch, const int32_t *page_table, int pages_per_seq, const float *rope,
                                  int n_positions, const hsd_kv_pool *pool, int zeros, void *q_out, void *stream) {
  const hsd::Norm norm = {q_gain, k_gain, gain_dtype, eps};
  return hsd::append(qkv, qkv_dtype, rows, row_stride, n_q_heads, n_kv_heads, head_dim, row_starts, kv_lens, batch, page_table, pages_per_seq, rope,
                     n_positions, pool, q_out, zeros != 0, &norm, (cudaStream_t)stream);
}
