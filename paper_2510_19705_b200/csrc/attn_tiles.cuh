// What a warp does with a tile of keys and values of the caller's paged cache in shared memory (hsd_paged_attention, hsd_prefix_attention):
// copies, both products on mma.sync, the running softmax; in bf16 and fp32.
#pragma once
#include <math.h>

#include "paged.cuh"

namespace hsd {
namespace {

// Keys of a tile (8 KB of keys and values, 4 KB for heads of 32) and query heads of one pass over them at most.
template <typename T, int HD> struct Form {
  static constexpr int KEYS = (HD == 128 ? 16 : 32) / ((int)sizeof(T) / 2), HEADS = sizeof(T) == 4 ? 8 : 16;
};
template <typename T, int HD> struct Ring {
  static constexpr int ROW = HD * (int)sizeof(T), HALF = Form<T, HD>::KEYS * ROW, STAGE = 2 * HALF;    // keys, then values
  static constexpr int STAGES = 24576 / STAGE, BYTES = STAGE * STAGES;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void copy16(u32 to, const void *from, bool there) {       // zeros where there is nothing to read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void mma(float *c, const u32 *a, u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float *c, const u32 *a, u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x = part[0] + part[1] + part[2], all of it: the first 11 bits, the next 11, the last two (four operations; NaN stays NaN, as do infinities).
__device__ __forceinline__ void split3(float x, u32 *part) {
  part[0] = __float_as_uint(x) & 0xFFFFE000u;
  const float rest = x - __uint_as_float(part[0]);
  part[1] = __float_as_uint(rest) & 0xFFFFE000u;
  part[2] = __float_as_uint(rest - __uint_as_float(part[1]));
}
// x = high + mid to a last place: rounded to 11 bits, what is left rounded to 11 bits.  (For few numbers: the conversion has a quarter of the
// rate.)  What rounding would make infinite is cut off.
__device__ __forceinline__ void split2(float x, u32 &high, u32 &mid) {
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(high) : "f"(x));
  if (fabsf(x) > 3.4e38f) high = __float_as_uint(x) & 0xFFFFE000u;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(mid) : "f"(x - __uint_as_float(high)));
}
__device__ __forceinline__ float4 lds4(u32 at) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts4(u32 at, float4 v) {
  asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void ldsm4(u32 *r, u32 at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(u32 *r, u32 at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// Byte of 16-byte piece c of row r of a tile: permuted so that the pieces a quarter warp reads together lie in different banks.
template <typename T, int HD> __device__ __forceinline__ u32 piece(int r, int c) {
  if constexpr (sizeof(T) == 4) return r * (HD * 4) + ((c ^ ((r & 1) << 2) ^ (r & 6)) << 4);
  else if constexpr (HD == 32) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
  else return r * (HD * 2) + ((c ^ (r & 7)) << 4);
}
__device__ __forceinline__ long long divide(long long a, long long b) {          // (32 bits do nearly always, in a fourth of the time)
  return ((a | b) >> 31) == 0 ? (long long)((u32)a / (u32)b) : a / b;
}

// ---------------------------------------------------------------------------- bf16
// Two weights (at most 1) as three bf16 parts of each, all of their 24 bits.
__device__ __forceinline__ void split3(float x, float y, u32 *part) {
#pragma unroll
  for (int e = 0; e < 3; ++e) {
    const __nv_bfloat162 z = __floats2bfloat162_rn(x, y);
    part[e] = *reinterpret_cast<const u32 *>(&z);
    x -= __low2float(z);
    y -= __high2float(z);
  }
}
template <int HD, int H> struct Bf16Tile {     // H: 8 or 16 rows with queries
  using T = __nv_bfloat16;
  static constexpr int YS = H / 8, PRODUCTS = YS == 1 ? 2 : 3;         // with the values
  u32 qf[HD / 16][4];
  float o[HD / 8][2 * YS], m[2], l[2];
  int lane;

  // Queries of the lane's rows, lane / 4 and lane / 4 + 8; null: zeros.
  __device__ __forceinline__ void begin(const T *q0, const T *q1) {
    const int col = (lane & 3) * 2;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const T *q = x & 1 ? q1 : q0;
        qf[k][x] = (x & 1) < YS && q ? __ldg(reinterpret_cast<const u32 *>(q + k * 16 + col + (x >> 1) * 8)) : 0u;
      }
#pragma unroll
    for (int n = 0; n < HD / 8; ++n)
#pragma unroll
      for (int x = 0; x < 2 * YS; ++x) o[n][x] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  // there0, there1: keys of the tile that the lane's rows see.
  __device__ __forceinline__ void tile(float scale, u32 at, u32 there0, u32 there1) {
    constexpr int KB = Form<T, HD>::KEYS / 16;                         // blocks of 16 keys
    float s[2 * KB][4];
#pragma unroll
    for (int n = 0; n < 2 * KB; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) s[n][x] = 0.f;
    const int kr = (lane & 7) + ((lane >> 4) << 3), kc = (lane >> 3) & 1;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k)
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        u32 f[4];
        ldsm4(f, at + piece<T, HD>(b * 16 + kr, 2 * k + kc));
        mma(s[2 * b], qf[k], f[0], f[1]);
        mma(s[2 * b + 1], qf[k], f[2], f[3]);
      }
    const int col = (lane & 3) * 2;
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < 2 * KB; ++n)
#pragma unroll
      for (int x = 0; x < 2 * YS; ++x) {
        s[n][x] = ((x >> 1 ? there1 : there0) >> (n * 8 + col + (x & 1))) & 1 ? s[n][x] * scale : -INFINITY;
        mx[x >> 1] = fmaxf(mx[x >> 1], s[n][x]);
      }
    u32 w[KB][PRODUCTS][4];
    float f[2] = {1.f, 1.f};
    bool grown = false;
#pragma unroll
    for (int y = 0; y < YS; ++y) {
      mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xFFFFFFFFu, mx[y], 1));
      mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xFFFFFFFFu, mx[y], 2));
      const float n = fmaxf(m[y], mx[y]), ref = n > -INFINITY ? n : 0.f;
      f[y] = ex2(m[y] - ref);
      grown |= n > m[y];
      m[y] = n;
      l[y] *= f[y];
#pragma unroll
      for (int n2 = 0; n2 < 2 * KB; ++n2) {
        const float p0 = ex2(s[n2][2 * y] - ref), p1 = ex2(s[n2][2 * y + 1] - ref);
        l[y] += p0 + p1;
        u32 part[3];
        split3(p0, p1, part);
        if constexpr (YS == 1) {               // rows 8 to 15: the middle parts
          w[n2 / 2][0][n2 % 2 * 2] = part[0]; w[n2 / 2][0][n2 % 2 * 2 + 1] = part[1];
          w[n2 / 2][1][n2 % 2 * 2] = part[2]; w[n2 / 2][1][n2 % 2 * 2 + 1] = 0;
        } else {
#pragma unroll
          for (int e = 0; e < 3; ++e) w[n2 / 2][e][n2 % 2 * 2 + y] = part[e];
        }
      }
    }
    if (__any_sync(0xFFFFFFFFu, grown)) {
#pragma unroll
      for (int n = 0; n < HD / 8; ++n)
#pragma unroll
        for (int x = 0; x < 2 * YS; ++x) o[n][x] *= f[x >> 1];
    }
    const u32 v = at + Ring<T, HD>::HALF;
    const int vr = lane & 15, vc = lane >> 4;
#pragma unroll
    for (int n = 0; n < HD / 16; ++n) {
      float d[2][4];                           // of this tile alone
#pragma unroll
      for (int x = 0; x < 4; ++x) d[0][x] = d[1][x] = 0.f;
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        u32 x[4];
        ldsm4t(x, v + piece<T, HD>(b * 16 + vr, 2 * n + vc));
#pragma unroll
        for (int e = PRODUCTS - 1; e >= 0; --e) {                      // the small ones first
          mma(d[0], w[b][e], x[0], x[1]);
          mma(d[1], w[b][e], x[2], x[3]);
        }
      }
#pragma unroll
      for (int x = 0; x < 2 * YS; ++x) {
        o[2 * n][x] += YS == 1 ? d[0][x] + d[0][2 + x] : d[0][x];
        o[2 * n + 1][x] += YS == 1 ? d[1][x] + d[1][2 + x] : d[1][x];
      }
    }
  }
  static constexpr int SUMS = HD / 8 * 2 * YS;
  __device__ __forceinline__ void save(volatile float *to) const {
#pragma unroll
    for (int i = 0; i < SUMS; ++i) to[i] = o[i / (2 * YS)][i % (2 * YS)];
  }
  __device__ __forceinline__ void restore(const volatile float *from, bool row0, bool row1) {          // of the lane's rows that say so
#pragma unroll
    for (int i = 0; i < SUMS; ++i)
      if (i % (2 * YS) / 2 ? row1 : row0) o[i / (2 * YS)][i % (2 * YS)] = from[i];
  }
  __device__ __forceinline__ void total() {     // the sum of a row's weights, which four lanes have a share of each
#pragma unroll
    for (int y = 0; y < YS; ++y) {
      l[y] += __shfl_xor_sync(0xFFFFFFFFu, l[y], 1);
      l[y] += __shfl_xor_sync(0xFFFFFFFFu, l[y], 2);
    }
  }
  // The lane's sums, two columns at a time, and each row's m and l (of one of its lanes).
  template <class F> __device__ __forceinline__ void rows(F &&f) const {
#pragma unroll
    for (int y = 0; y < YS; ++y)
#pragma unroll
      for (int n = 0; n < HD / 8; ++n) f((lane >> 2) + 8 * y, n * 8 + (lane & 3) * 2, make_float2(o[n][2 * y], o[n][2 * y + 1]));
  }
  template <class F> __device__ __forceinline__ void stats(F &&f) const {
#pragma unroll
    for (int y = 0; y < YS; ++y)
      if ((lane & 3) == 0) f((lane >> 2) + 8 * y, m[y], l[y]);
  }
  // The result of `heads` rows to out (rows one after the other), or, where out is null, the sums to a part: rows, then m and l of each of `chunk`.
  __device__ __forceinline__ void end(T *out, float *part, int chunk, int heads) {
    const int col = (lane & 3) * 2;
    total();
#pragma unroll
    for (int y = 0; y < YS; ++y) {
      const int row = (lane >> 2) + 8 * y;
      if (row >= heads) continue;
      if (out) {
        const float inv = l[y] != 0.f ? 1.f / l[y] : 0.f;
#pragma unroll
        for (int n = 0; n < HD / 8; ++n)
          *reinterpret_cast<__nv_bfloat162 *>(out + row * HD + n * 8 + col) = __floats2bfloat162_rn(o[n][2 * y] * inv, o[n][2 * y + 1] * inv);
      } else {
#pragma unroll
        for (int n = 0; n < HD / 8; ++n) *reinterpret_cast<float2 *>(part + row * HD + n * 8 + col) = make_float2(o[n][2 * y], o[n][2 * y + 1]);
        if ((lane & 3) == 0) *reinterpret_cast<float2 *>(part + chunk * HD + row * 2) = make_float2(m[y], l[y]);
      }
    }
  }
};

// ---------------------------------------------------------------------------- fp32
// A lane's four values of a 16-byte piece are its k = j and j + 4 of two steps (keys) or its columns of four tiles (values): any order
// of k will do that both factors have, and of columns that the output is written in.
template <int HD> struct Fp32Tile {
  using T = float;
  u32 q[HD / 8][4];                            // rows 0 to 7 of the tile: the queries' high parts, rows 8 to 15: the rest
  float o[HD / 8][2], m, l;
  int lane;

  // Queries of the lane's row, lane / 4; null: zeros.
  __device__ __forceinline__ void begin(const T *from, const T *) {
    const int j = lane & 3;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) {
      const float4 x = from ? __ldg(reinterpret_cast<const float4 *>(from + i * 16 + j * 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
      split2(x.x, q[2 * i][0], q[2 * i][1]);
      split2(x.y, q[2 * i][2], q[2 * i][3]);
      split2(x.z, q[2 * i + 1][0], q[2 * i + 1][1]);
      split2(x.w, q[2 * i + 1][2], q[2 * i + 1][3]);
    }
#pragma unroll
    for (int n = 0; n < HD / 8; ++n) o[n][0] = o[n][1] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void tile(float scale, u32 at, u32 there, u32) {
    constexpr int KB = Form<T, HD>::KEYS / 8;                          // blocks of 8 keys
    const int r = lane >> 2, j = lane & 3;
    float p[KB][2], mx = -INFINITY;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      float s[3][2][4];                        // of each part of the keys; two chains of each
#pragma unroll
      for (int e = 0; e < 3; ++e)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[e][0][x] = s[e][1][x] = 0.f;
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        const float4 k = lds4(at + piece<T, HD>(b * 8 + r, i * 4 + j));
        const float x[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          u32 k0[3], k1[3];
          split3(x[2 * y], k0);
          split3(x[2 * y + 1], k1);
#pragma unroll
          for (int e = 0; e < 3; ++e) mma_tf32(s[e][y], q[2 * i + y], k0[e], k1[e]);
        }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float sum = 0.f;                       // the small ones first
#pragma unroll
        for (int e = 2; e >= 0; --e) sum += (s[e][0][2 + x] + s[e][1][2 + x]) + (s[e][0][x] + s[e][1][x]);
        p[b][x] = (there >> (b * 8 + 2 * j + x)) & 1 ? sum * scale : -INFINITY;
        mx = fmaxf(mx, p[b][x]);
      }
    }
    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
    const float n = fmaxf(m, mx), ref = n > -INFINITY ? n : 0.f, f = ex2(m - ref);
    const bool grown = n > m;
    m = n;
    l *= f;
    if (__any_sync(0xFFFFFFFFu, grown)) {
#pragma unroll
      for (int i = 0; i < HD / 8; ++i) { o[i][0] *= f; o[i][1] *= f; }
    }
    u32 w[KB][4];                              // k = j: key 2 j; k = j + 4: key 2 j + 1
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const float p0 = ex2(p[b][0] - ref), p1 = ex2(p[b][1] - ref);
      l += p0 + p1;
      split2(p0, w[b][0], w[b][1]);
      split2(p1, w[b][2], w[b][3]);
    }
    const u32 v = at + Ring<T, HD>::HALF;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) {
      float d[4][4];                           // of this tile alone
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int x = 0; x < 4; ++x) d[c][x] = 0.f;
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        const float4 v0 = lds4(v + piece<T, HD>(b * 8 + 2 * j, i * 8 + r)), v1 = lds4(v + piece<T, HD>(b * 8 + 2 * j + 1, i * 8 + r));
        const float x[4] = {v0.x, v0.y, v0.z, v0.w}, y[4] = {v1.x, v1.y, v1.z, v1.w};
        u32 x3[4][3], y3[4][3];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          split3(x[c], x3[c]);
          split3(y[c], y3[c]);
        }
#pragma unroll
        for (int e = 2; e >= 0; --e)
#pragma unroll
          for (int c = 0; c < 4; ++c) mma_tf32(d[c], w[b], x3[c][e], y3[c][e]);
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int x = 0; x < 2; ++x) o[4 * i + c][x] += d[c][x] + d[c][2 + x];
    }
  }
  static constexpr int SUMS = HD / 8 * 2;
  __device__ __forceinline__ void save(volatile float *to) const {
#pragma unroll
    for (int i = 0; i < SUMS; ++i) to[i] = o[i / 2][i % 2];
  }
  __device__ __forceinline__ void restore(const volatile float *from, bool row, bool) {
#pragma unroll
    for (int i = 0; i < SUMS; ++i)
      if (row) o[i / 2][i % 2] = from[i];
  }
  __device__ __forceinline__ void total() {
    l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
    l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
  }
  template <class F> __device__ __forceinline__ void rows(F &&f) const {        // column n of tile 4 i + c stands for 32 i + 4 n + c
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) f(lane >> 2, i * 32 + (lane & 3) * 8 + x * 4 + y * 2, make_float2(o[4 * i + 2 * y][x], o[4 * i + 2 * y + 1][x]));
  }
  template <class F> __device__ __forceinline__ void stats(F &&f) const {
    if ((lane & 3) == 0) f(lane >> 2, m, l);
  }
  __device__ __forceinline__ void end(T *out, float *part, int chunk, int heads) {
    const int r = lane >> 2, j = lane & 3;
    total();
    if (r >= heads) return;
    float *to = (out ? out : part) + r * HD;
    const float inv = !out ? 1.f : l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x)              // column n of tile 4 i + c stands for 32 i + 4 n + c
#pragma unroll
        for (int y = 0; y < 2; ++y)
          *reinterpret_cast<float2 *>(to + i * 32 + j * 8 + x * 4 + y * 2) = make_float2(o[4 * i + 2 * y][x] * inv, o[4 * i + 2 * y + 1][x] * inv);
    if (!out && j == 0) *reinterpret_cast<float2 *>(part + chunk * HD + r * 2) = make_float2(m, l);
  }
};

template <typename T, int HD, int H> struct TileOf { using type = Bf16Tile<HD, H>; };
template <int HD> struct TileOf<float, HD, 8> { using type = Fp32Tile<HD>; };

__device__ __forceinline__ void store4(float *to, float4 v) { *reinterpret_cast<float4 *>(to) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *to, float4 v) {
  reinterpret_cast<__nv_bfloat162 *>(to)[0] = __floats2bfloat162_rn(v.x, v.y);
  reinterpret_cast<__nv_bfloat162 *>(to)[1] = __floats2bfloat162_rn(v.z, v.w);
}

}  // namespace
}  // namespace hsd
