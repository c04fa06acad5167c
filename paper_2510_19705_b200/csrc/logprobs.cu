// Log probabilities of given tokens, with entropy, rank and the top alternatives of every row (hsd_token_logprobs).
//   m = max l, S = sum exp(l - m), T = sum exp(l - m) (l - m):  log p(x) = (l_x - m) - log S,  H = log S - T / S
// (both terms of H are >= 0: nothing cancels).  One read of the row: every thread keeps its own running (m, S, T), rescaled when
// its maximum grows, its count of tokens in front of the given one, and its maximum; the triples are merged at the end.
// The top tokens need no second read either, but for a few threads' shares of the row: the k-th largest of the maxima of
// groups of threads bounds the k-th largest token from below, so only threads whose own maximum reaches it can hold one of the k.
// Their shares (out of L2 or L1, a warp together on each) give the candidates, usually little more than k; a candidate's place is
// the number of candidates in front of it.  Order: larger logit first, lower id among equals, so the result does not
// depend on the order in which candidates were found.
// Rows with more candidates than fit (masses of equal logits: a mask's -inf) take select_slow().
// A CTA has a row, or (few rows, or long ones) a cluster has one: each CTA finds the sums and the top tokens of its part, the first
// one adds and merges them out of the others' shared memory.
// Bound by memory for many rows (and by issue slots not far behind: some seven operations a bf16 logit, of which what can be done two at a
// time is), by latency for few.
#include <cooperative_groups.h>
#include <math.h>

#include "common.cuh"

namespace hsd {
namespace {

constexpr int kMaxTop = 32;
template <int THREADS> constexpr int kCand = THREADS == 32 ? 256 : 1024;       // candidates that fit
constexpr float kLog2e = 1.4426950408889634f;

struct LogprobArgs {
  const void *logits;
  const int32_t *tokens;
  float *logprob, *entropy;
  int32_t *rank, *top_id;
  float *top_lp;
  int V, top;
};

__device__ __forceinline__ float max_nan(float a, float b) {           // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ u32 max_nan2(u32 a, u32 b) {
  u32 y;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}

template <typename T> struct Vec;      // 16 bytes of logits
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr u32 kNone = 0xFF80FF80u;                            // two -inf
  __device__ static void unpack(const uint4 &v, float *f) {
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
    f[4] = __uint_as_float(v.z << 16); f[5] = __uint_as_float(v.z & 0xFFFF0000u);
    f[6] = __uint_as_float(v.w << 16); f[7] = __uint_as_float(v.w & 0xFFFF0000u);
  }
  __device__ static uint4 pack(const float *f) {
    uint4 v;
    v.x = __float_as_uint(f[0]) >> 16 | (__float_as_uint(f[1]) & 0xFFFF0000u); v.y = __float_as_uint(f[2]) >> 16 | (__float_as_uint(f[3]) & 0xFFFF0000u);
    v.z = __float_as_uint(f[4]) >> 16 | (__float_as_uint(f[5]) & 0xFFFF0000u); v.w = __float_as_uint(f[6]) >> 16 | (__float_as_uint(f[7]) & 0xFFFF0000u);
    return v;
  }
  template <int U> __device__ static float largest(const uint4 *v) {
    u32 m = kNone;
#pragma unroll
    for (int u = 0; u < U; ++u) m = max_nan2(m, max_nan2(max_nan2(v[u].x, v[u].y), max_nan2(v[u].z, v[u].w)));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  }
  // How many are larger than x (or equal to it): at most 4 U a half, whole numbers in bf16.
  template <int U> __device__ static int front(const uint4 *v, float x, bool equal) {
    const __nv_bfloat162 t = __float2bfloat162_rn(x);
    __nv_bfloat162 n = __float2bfloat162_rn(0.f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const u32 w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 y = *reinterpret_cast<const __nv_bfloat162 *>(&w[i]);
        n = __hadd2(n, equal ? __hge2(y, t) : __hgt2(y, t));
      }
    }
    return (int)(__low2float(n) + __high2float(n));
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static constexpr u32 kNone = 0xFF800000u;
  __device__ static void unpack(const uint4 &v, float *f) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  __device__ static uint4 pack(const float *f) { return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])); }
  template <int U> __device__ static float largest(const uint4 *v) {
    float m = -INFINITY, f[N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      unpack(v[u], f);
      m = max_nan(m, max_nan(max_nan(f[0], f[1]), max_nan(f[2], f[3])));
    }
    return m;
  }
  template <int U> __device__ static int front(const uint4 *v, float x, bool equal) {
    int n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[N];
      unpack(v[u], f);
      n += equal ? (f[0] >= x) + (f[1] >= x) + (f[2] >= x) + (f[3] >= x) : (f[0] > x) + (f[1] > x) + (f[2] > x) + (f[3] > x);
    }
    return n;
  }
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A float as a whole number of the same order (-0 as +0), and a token's place in a row's order.
__device__ __forceinline__ u32 ordered(float x) {
  const u32 b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(u32 o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ u64 key_of(float x, int id) { return ((u64)ordered(x) << 32) | (u32)~id; }

// A CTA's part [lo, hi) of a row, in 16-byte pieces of the row's memory: piece i holds ids first + i * N .., of which those outside
// the part are not read.
template <typename T> struct Part {
  static constexpr int N = Vec<T>::N;
  const T *row;
  int lo, hi, first, pieces;
  __device__ Part(const T *row_, int lo_, int hi_) : row(row_), lo(lo_), hi(hi_) {
    const int off = (int)((reinterpret_cast<uintptr_t>(row + lo) & 15) / sizeof(T));
    first = lo - off;
    pieces = hi > lo ? (hi - first + N - 1) / N : 0;
  }
  __device__ __forceinline__ bool whole(int i) const { return first + i * N >= lo && first + (i + 1) * N <= hi; }
  // -inf where there is no token
  __device__ __forceinline__ uint4 read(int i) const {
    if (whole(i)) return __ldg(reinterpret_cast<const uint4 *>(row + first + (ptrdiff_t)i * N));
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int id = first + i * N + e;
      f[e] = id >= lo && id < hi ? to_f32(row[id]) : -INFINITY;
    }
    return Vec<T>::pack(f);
  }
  __device__ __forceinline__ void read(int i, float *f) const { Vec<T>::unpack(read(i), f); }
  __device__ __forceinline__ bool has(int i, int e) const {
    const int id = first + i * N + e;
    return id >= lo && id < hi;
  }
};

// Running sums of a thread relative to its own maximum m (never below the lowest finite value, so that -inf tokens weigh 0):
// s = sum 2^y, t = sum 2^y y with y = (l - m) log2(e), cut off at -200, where 2^y is 0.
struct Sums {
  float m = -3.402823466e38f, s = 0.f, t = 0.f;
  __device__ __forceinline__ void raise(float m2) {
    const float y = fmaxf((m - m2) * kLog2e, -200.f), f = ex2(y);
    t = f * fmaf(s, y, t);
    s *= f;
    m = m2;
  }
  __device__ __forceinline__ void merge(float m2, float s2, float t2) {
    Sums o;
    o.m = m2; o.s = s2; o.t = t2;
    const float n = fmaxf(m, m2);
    if (n > m) raise(n);
    if (n > o.m) o.raise(n);
    s += o.s;
    t += o.t;
  }
};

template <int THREADS> struct Shared {
  float group_max[128];
  int flagged[THREADS], n_flagged;     // threads whose pieces may hold one of the top tokens
  float m[THREADS / 32], s[THREADS / 32], t[THREADS / 32];
  int front[THREADS / 32];
  u64 cand[kCand<THREADS>];
  u64 list[kMaxTop];                   // the part's top tokens in order
  u64 top[kMaxTop];                    // the row's
  float4 sums;                         // the part's m (NaN: of no distribution), s, t; tokens in front
  float bound;
  int n_cand, warp_n[THREADS / 32];
};

// The k-th largest value of a part whose candidates did not fit, by bisection on ordered(): counts of the tokens above a value,
// each one pass.  Then the tokens above it (fewer than k) and, in ascending order until there are k, those equal to it.
template <typename T, int THREADS>
__device__ void select_slow(const Part<T> &p, int k, float bound, float top, Shared<THREADS> &sh) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u32 lo = ordered(bound), hi = ordered(top);                          // at least k tokens >= lo; fewer than k > hi
  u32 v = lo;
  for (int step = 0; step < 34 && lo < hi; ++step) {
    int n = 0;
    const float at = unordered(v);
    for (int i = threadIdx.x; i < p.pieces; i += THREADS) {
      float f[N];
      p.read(i, f);
#pragma unroll
      for (int e = 0; e < N; ++e) n += f[e] > at && p.has(i, e);
    }
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xFFFFFFFFu, n, o);
    __syncthreads();
    if (lane == 0) sh.warp_n[warp] = n;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < THREADS / 32; ++w) all += sh.warp_n[w];
    if (all < k) hi = v;
    else lo = v + 1;
    v = lo + (hi - lo) / 2;
  }
  const float kth = unordered(lo);
  __syncthreads();
  if (threadIdx.x == 0) sh.n_cand = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < p.pieces; i += THREADS) {
    float f[N];
    p.read(i, f);
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (f[e] > kth && p.has(i, e)) sh.cand[atomicAdd(&sh.n_cand, 1)] = key_of(f[e], p.first + i * N + e);
  }
  __syncthreads();
  int got = sh.n_cand;
  __syncthreads();
  for (int i0 = 0; i0 < p.pieces && got < k; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    float f[N];
    int n = 0;
    if (i < p.pieces) {
      p.read(i, f);
#pragma unroll
      for (int e = 0; e < N; ++e) n += f[e] == kth && p.has(i, e);
    }
    int upto = n;
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) sh.warp_n[warp] = upto;
    __syncthreads();
    int at = got + upto - n, all = 0;
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) at += sh.warp_n[w];
      all += sh.warp_n[w];
    }
    if (n > 0) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (f[e] == kth && p.has(i, e)) {
          if (at < k) sh.cand[at] = key_of(f[e], p.first + i * N + e);
          ++at;
        }
    }
    got = min(k, got + all);
    __syncthreads();
  }
  if (threadIdx.x == 0) sh.n_cand = got;
  __syncthreads();
}

// The part's k first tokens (fewer if it has fewer; the rest of the list is 0, which no token's key is) into sh.list.  v: the thread's
// pieces, if it has no others (`all_here`).
template <typename T, int THREADS, int U>
__device__ void select_top(const Part<T> &p, int k, float mine, const uint4 *v, bool all_here, Shared<THREADS> &sh) {
  constexpr int N = Vec<T>::N, LANES = THREADS > 128 ? THREADS / 128 : 1;                // threads of a group: 128 groups at most
  const int lane = threadIdx.x & 31;
  float g = mine;
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xFFFFFFFFu, g, o));
  if (threadIdx.x % LANES == 0) sh.group_max[threadIdx.x / LANES] = g;
  if (threadIdx.x == 0) sh.n_cand = sh.n_flagged = 0;
  __syncthreads();
  // Every warp for itself: the largest value of 16 bits that k of the groups' maxima reach, bit by bit.
  u32 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = i * 32 < THREADS ? ordered(sh.group_max[i * 32 + lane]) >> 16 : 0;
  u32 reached = 0;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const u32 at = reached | 1u << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += __popc(__ballot_sync(0xFFFFFFFFu, x[i] >= at));
    if (n >= k) reached = at;
  }
  const float bound = fmaxf(unordered(max(reached << 16, 0x007FFFFFu)), -INFINITY);      // (0x007FFFFF: -inf)
  const bool flagged = mine >= bound && (int)threadIdx.x < p.pieces;
  auto take = [&](const uint4 &x, int i) {
    float f[N];
    Vec<T>::unpack(x, f);
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (f[e] >= bound && p.has(i, e)) {
        const int at = atomicAdd(&sh.n_cand, 1);
        if (at < kCand<THREADS>) sh.cand[at] = key_of(f[e], p.first + i * N + e);
      }
  };
  if (all_here) {
    if (flagged)
#pragma unroll
      for (int u = 0; u < U; ++u)
        if ((int)threadIdx.x + u * THREADS < p.pieces) take(v[u], threadIdx.x + u * THREADS);
  } else {                             // the flagged threads' pieces once more, by all threads
    if (flagged) sh.flagged[atomicAdd(&sh.n_flagged, 1)] = threadIdx.x;
    __syncthreads();
    const int each = (p.pieces + THREADS - 1) / THREADS, n = sh.n_flagged * each;
    for (int x0 = threadIdx.x; x0 < n; x0 += THREADS * U) {
      uint4 y[U];
      int at[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = x0 + u * THREADS;
        at[u] = x < n ? sh.flagged[x / each] + x % each * THREADS : p.pieces;
        if (at[u] < p.pieces) y[u] = p.read(at[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at[u] < p.pieces) take(y[u], at[u]);
    }
  }
  __syncthreads();
  if (sh.n_cand > kCand<THREADS>) {
    float top = -INFINITY;
    for (int i = 0; i < min(THREADS, 128); ++i) top = fmaxf(top, sh.group_max[i]);
    select_slow<T, THREADS>(p, k, bound, top, sh);
  }
  const int n = sh.n_cand;
  if (threadIdx.x < kMaxTop && (int)threadIdx.x >= n) sh.list[threadIdx.x] = 0;
  for (int c = threadIdx.x; c < n; c += THREADS) {
    const u64 x = sh.cand[c];
    int place = 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) place += sh.cand[i] > x;
    if (place < k) sh.list[place] = x;
  }
  __syncthreads();
}

// A row's CTAs (blockIdx.y, a cluster where there are several).
// U: pieces of a thread at once.
template <typename T, int THREADS, int U>
__global__ void __launch_bounds__(THREADS, THREADS == 32 ? 24 : 1024 / THREADS)
logprobs_kernel(LogprobArgs a) {
  constexpr int N = Vec<T>::N;
  __shared__ __align__(16) Shared<THREADS> sh;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, parts = gridDim.y, part = blockIdx.y;
  const long long r = blockIdx.x;
  const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.V;
  const Part<T> p(row, (int)((long long)a.V * part / parts), (int)((long long)a.V * (part + 1) / parts));
  chain_wait();
  chain_next();
  const int tok = a.tokens[r];
  const bool given = tok >= 0 && tok < a.V;
  const float xt = given ? to_f32(row[tok]) : 0.f;

  Sums z;
  float mine = -INFINITY;
  int front = 0;
  float2 s2 = make_float2(0.f, 0.f), t2 = s2;                          // of z, even and odd tokens apart
  uint4 v[U];
  for (int i0 = threadIdx.x; i0 < p.pieces; i0 += THREADS * U) {
    if (i0 > 0 && i0 + (U - 1) * THREADS < p.pieces - 1) {             // no piece at an end of the part
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = __ldg(reinterpret_cast<const uint4 *>(p.row + p.first + (ptrdiff_t)(i0 + u * THREADS) * N));
    } else
#pragma unroll
    for (int u = 0; u < U; ++u)
      v[u] = i0 + u * THREADS < p.pieces ? p.read(i0 + u * THREADS) : make_uint4(Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone);
    mine = max_nan(mine, Vec<T>::template largest<U>(v));
    if (mine > z.m) {
      z.s = s2.x + s2.y; z.t = t2.x + t2.y;
      z.raise(mine);
      s2 = make_float2(z.s, 0.f); t2 = make_float2(z.t, 0.f);
    }
    // The given token's place behind the first of these.  (Ids past the row's end would not fit 32 bits in the largest vocabularies.)
    const int at = (given ? tok : -1) - (p.first + i0 * N);
    const bool one_side = at < 0 || at >= (U - 1) * THREADS * N + N;   // of the given token, as nearly all are
    if (one_side) front += Vec<T>::template front<U>(v, xt, at > 0 && xt > -INFINITY);
    const float2 minus = make_float2(-z.m, -z.m), scale = make_float2(kLog2e, kLog2e);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int u0 = u * THREADS * N;
      float f[N];
      Vec<T>::unpack(v[u], f);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        float2 y = __fmul2_rn(__fadd2_rn(make_float2(f[e], f[e + 1]), minus), scale);
        y.x = fmaxf(y.x, -200.f); y.y = fmaxf(y.y, -200.f);
        const float2 w = make_float2(ex2(y.x), ex2(y.y));
        s2 = __fadd2_rn(s2, w);
        t2 = __ffma2_rn(w, y, t2);
      }
      if (one_side) continue;
      if (u0 > at || u0 + N <= at) {                                   // (places without a token hold -inf)
        front += Vec<T>::template front<1>(v + u, xt, u0 < at && xt > -INFINITY);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) front += f[e] > xt || (xt > -INFINITY && f[e] == xt && u0 + e < at);
      }
    }
  }
  if (given && xt == -INFINITY) {      // among equals of -inf the lower ids count, and places without a token do not
    front = 0;
    for (int i = threadIdx.x; i < p.pieces; i += THREADS) {
      float f[N];
      p.read(i, f);
#pragma unroll
      for (int e = 0; e < N; ++e) front += p.has(i, e) && (f[e] > xt || p.first + i * N + e < tok);
    }
  }
  z.s = s2.x + s2.y; z.t = t2.x + t2.y;
  // the part's maximum, then sums relative to it: one rescaling a thread
  float m = z.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  if (__any_sync(0xFFFFFFFFu, !(mine < INFINITY))) m = NAN;            // a NaN or +inf: no distribution
  if (lane == 0) sh.m[warp] = m;
  __syncthreads();
  bool none = false;
  m = z.m;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    none |= !(sh.m[w] == sh.m[w]);
    m = fmaxf(m, sh.m[w]);
  }
  if (m > z.m) z.raise(m);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    z.s += __shfl_xor_sync(0xFFFFFFFFu, z.s, o);
    z.t += __shfl_xor_sync(0xFFFFFFFFu, z.t, o);
  }
  front = __reduce_add_sync(0xFFFFFFFFu, front);
  if (lane == 0) { sh.s[warp] = z.s; sh.t[warp] = z.t; sh.front[warp] = front; }
  if (a.top > 0 && !none) {
    select_top<T, THREADS, U>(p, a.top, mine, v, p.pieces <= THREADS * U, sh);
  } else {
    if (threadIdx.x < kMaxTop) sh.list[threadIdx.x] = 0;
    __syncthreads();
  }
  Sums all;
  all.m = m;
  front = 0;
  if (warp == 0) {                     // (the rest is the first warp's)
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      all.s += sh.s[w];
      all.t += sh.t[w];
      front += sh.front[w];
    }
  }
  if (parts > 1) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    if (threadIdx.x == 0) sh.sums = make_float4(none ? NAN : all.m, all.s, all.t, __int_as_float(front));
    cluster.sync();
    if (part == 0) {
      if (warp == 0) {
        Sums sum;
        none = false;
        front = 0;
        for (int q = 0; q < parts; ++q) {
          const float4 x = *cluster.map_shared_rank(&sh.sums, q);
          none |= !(x.x == x.x);
          sum.merge(x.x, x.y, x.z);
          front += __float_as_int(x.w);
        }
        all = sum;
      }
      if (a.top > 0) {                 // the parts' lists are in order: a token's place is the sum of its places in them
        for (int i = threadIdx.x; i < parts * a.top; i += THREADS) sh.cand[i] = *cluster.map_shared_rank(&sh.list[i % a.top], i / a.top);
        __syncthreads();
        for (int i = threadIdx.x; i < parts * a.top; i += THREADS) {
          const u64 x = sh.cand[i];
          int place = 0;
          for (int k = 0; k < parts * a.top; ++k) place += sh.cand[k] > x;
          if (place < a.top && x != 0) sh.top[place] = x;
        }
      }
    }
    cluster.sync();                    // no CTA leaves while the first one reads
    if (part > 0) return;
  }
  if (warp > 0) return;
  const u64 *list = parts > 1 ? sh.top : sh.list;
  const float log_s = logf(all.s);
  if (threadIdx.x == 0) {
    a.logprob[r] = none || !given ? NAN : all.s > 0.f ? xt - all.m - log_s : -INFINITY;
    a.entropy[r] = none ? NAN : all.s > 0.f ? log_s - 0.6931471805599453f * (all.t / all.s) : 0.f;
    a.rank[r] = none || !given ? -1 : front;
  }
  if ((int)threadIdx.x < a.top) {
    const u64 x = list[threadIdx.x];
    const float l = unordered((u32)(x >> 32));
    a.top_id[r * a.top + threadIdx.x] = none ? -1 : (int)~(u32)x;
    a.top_lp[r * a.top + threadIdx.x] = none ? NAN : all.s > 0.f ? l - all.m - log_s : -INFINITY;
  }
}

template <typename T, int THREADS, int U> int run_threads(const LogprobArgs &a, int rows, int parts, cudaStream_t s) {
  cudaLaunchAttribute at[2] = {};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 1; at[1].val.clusterDim.y = parts; at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(rows, parts); cfg.blockDim = dim3(THREADS); cfg.stream = s; cfg.attrs = at; cfg.numAttrs = 1 + (parts > 1);
  HSD_CUDA_OK(cudaLaunchKernelEx(&cfg, logprobs_kernel<T, THREADS, U>, a));
  hsd_count_launches(1);
  return hsd_launch_status();
}
// Many short rows take a warp each if few alternatives are asked for: bf16 with five, 3000 x 500 / 1461 / 2048 7.5 / 11.1 / 10.6 us (by 128 threads
// 17.0 / 20.4 / 20.2), 600 rows 4.9 / 6.6 / 6.4 (6.6 / 7.7 / 7.7; fp32 of 1461 6.1, 5.7), 300 rows 4.8 / 6.3 / 6.3 (4.9 / 5.1 / 5.1); with eight up to 0.7
// more; but with 20 600 rows take 6.4 / 10.0 / 10.3 (7.3 / 8.5 / 8.5), as the maxima of 32 lanes bound those badly.
// Rows that do not fill the GPU are divided into parts of 2048 tokens or more.  Long ones take CTAs of 512 threads with eight pieces at once:
// 700 x 131072 fp32 76 us (of 256 threads with four 109, divided among two / four such 93 / 100), 400 x 131072 bf16 36.7 (37.7), 300 x 70001 fp32 30.7 (28.7),
// but 576 x 32000 bf16 25.7 (16.1).
template <typename T> int run(const LogprobArgs &a, int rows, cudaStream_t s) {
  if (a.V <= 2048 && a.top <= 8 && rows >= 600) return run_threads<T, 32, 4>(a, rows, 1, s);
  if (a.V <= 4096) return run_threads<T, 128, 4>(a, rows, 1, s);
  int parts = 1;
  while (parts < 8 && (long long)rows * parts * 2 <= 4 * kMeasuredSMs && a.V / (parts * 2) >= 2048) parts *= 2;
  return a.V / parts >= 65536 ? run_threads<T, 512, 8>(a, rows, parts, s) : run_threads<T, 256, 4>(a, rows, parts, s);
}

}  // namespace
}  // namespace hsd

extern "C" int hsd_token_logprobs(const void *logits, int dtype, int rows, int vocab, const int32_t *tokens, int top, float *out_logprobs,
                                  float *out_entropy, int32_t *out_ranks, int32_t *out_top_tokens, float *out_top_logprobs, void *stream) {
  using namespace hsd;
  if (!logits || !tokens || !out_logprobs || !out_entropy || !out_ranks || rows <= 0 || vocab <= 0) return HSD_E_INVALID_ARG;
  if (dtype != HSD_F32 && dtype != HSD_BF16) return HSD_E_INVALID_ARG;
  if (top < 0 || top > kMaxTop || top > vocab || (top > 0 && (!out_top_tokens || !out_top_logprobs))) return HSD_E_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == HSD_F32 ? 4 : 2)) return HSD_E_INVALID_ARG;
  for (const void *x : {(const void *)tokens, (const void *)out_logprobs, (const void *)out_entropy, (const void *)out_ranks, (const void *)out_top_tokens, (const void *)out_top_logprobs})
    if (reinterpret_cast<uintptr_t>(x) % 4) return HSD_E_INVALID_ARG;
  if (vocab > 0x7FFFFF00) return HSD_E_TOO_LARGE;
  LogprobArgs a = {logits, tokens, out_logprobs, out_entropy, out_ranks, out_top_tokens, out_top_logprobs, vocab, top};
  return dtype == HSD_F32 ? run<float>(a, rows, (cudaStream_t)stream) : run<__nv_bfloat16>(a, rows, (cudaStream_t)stream);
}
