// Attention of one new token per sequence over the caller's paged cache (hsd_paged_attention).
//   o = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale q.k_j - m),  m = max_j scale q.k_j   over the sequence's keys j
// Bound by memory: every key and value is read once, for all query heads of its group.  The tiles (16 or 8 keys of one sequence
// and head) of the whole batch stand in one line, which is divided evenly over the warps, whatever the lengths are: the grid
// does not depend on them, and they are read on the device.  A warp streams its stretch through a ring of its own in shared memory
// (cp.async, no barrier between warps), across the borders of sequences and heads.  Where a stretch ends inside a sequence, the parts
// (m, sum, o) of its neighbours are added by the CTA, and where the CTA ends inside one, its part goes to the workspace and
// attn_join_kernel adds those in order.
// bf16: both products on mma.sync with the group's queries as the 16 rows of a tile (at 4 to 16 queries a key the tensor pipe is
// far from its limit); weights as bf16 high and low parts, so that only the final rounding is one of 8 bits.
// fp32: the products in fp32, four lanes a key for the scores, a lane a few columns for the output.
#include <math.h>

#include "paged.cuh"

namespace hsd {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kGrid = kMeasuredSMs;            // CTAs at most: fixed, as the workspace's size depends on it
constexpr int kMaxBatch = 4096;                // its tiles' prefix sums lie in shared memory
constexpr int kJoinWarps = 8;

struct DecodeArgs {
  const void *q;
  void *out;
  const int32_t *page_table, *kv_lens;
  float *parts;                                // of stretches (kGrid * kWarps), then of CTAs (two each)
  int4 *joins;                                 // per CTA: the item that it begins inside of, if it is the second with a part of it
  PoolView pool;
  float scale;                                 // times log2(e)
  int batch, nq, nkv, pages_per_seq;
  int group, chunk, chunks;                    // query heads of a key head; of them at once; times
};

template <typename T> struct Form;
template <> struct Form<__nv_bfloat16> { static constexpr int KEYS = 16, HEADS = 16; };        // query heads at once, at most
template <> struct Form<float> { static constexpr int KEYS = 8, HEADS = 8; };
template <typename T, int HD> struct Ring {
  static constexpr int ROW = HD * (int)sizeof(T), HALF = Form<T>::KEYS * ROW, STAGE = 2 * HALF;    // keys, then values
  static constexpr int STAGES = (sizeof(T) == 4 ? 16384 : 24576) / STAGE, BYTES = STAGE * STAGES;  // (fp32 has its queries beside it)
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
__device__ __forceinline__ void ldsm4(u32 *r, u32 at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(u32 *r, u32 at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// Byte of 16-byte piece c of row r of a tile: permuted so that the pieces a quarter warp reads together lie in different banks.
template <typename T, int HD> __device__ __forceinline__ u32 piece(int r, int c) {
  if constexpr (sizeof(T) == 4) return r * (HD * 4) + ((c ^ ((r & 1) << 2)) << 4);
  else if constexpr (HD == 32) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
  else return r * (HD * 2) + ((c ^ (r & 7)) << 4);
}

// The line of tiles: sequence b has as many for each of `items` (key head, chunk of query heads); before[b]: tiles of the
// sequences in front of b, per item; lens[b]: keys.
struct Line {
  const int *before, *lens;
  int batch, items, stretches;
  long long per;                               // tiles of a stretch
  // Stretches [first(c), first(c + 1)) are CTA c's: few of them lie on as many SMs, and no CTA without one stands between others.
  __device__ __forceinline__ int first(int cta) const { return stretches < kGrid ? min(cta, stretches) : cta * stretches / kGrid; }
  __device__ __forceinline__ int cta_of(long long tile) const {
    const int i = (int)(tile / per);
    return stretches < kGrid ? i : ((i + 1) * kGrid - 1) / stretches;
  }
};
// Lengths within the page table's room, and the prefix sums; all threads of the CTA.
template <int KEYS, int THREADS>
__device__ __forceinline__ Line make_line(const int32_t *kv_lens, int batch, long long room, int items, int *before, int *lens, int *warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int carry = 0;
  for (int b0 = 0; b0 < batch; b0 += THREADS) {
    const int b = b0 + threadIdx.x;
    const int len = b < batch ? (int)min((long long)max(kv_lens[b], 0), room) : 0, n = (len + KEYS - 1) / KEYS;
    int upto = n;
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    int front = carry;
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) front += warp_sum[w];
      carry += warp_sum[w];
    }
    if (b < batch) {
      before[b + 1] = front + upto;
      lens[b] = len;
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) before[0] = 0;
  __syncthreads();
  Line l;
  l.before = before; l.lens = lens; l.batch = batch; l.items = items;
  const long long total = (long long)carry * items, warps = kGrid * kWarps;
  l.per = max((total + warps - 1) / warps, 1ll);
  l.stretches = (int)((total + l.per - 1) / l.per);
  return l;
}

// A place on the line.
struct Place {
  int b, item, tile, tiles;                    // tiles: of the sequence
  __device__ __forceinline__ void find(const Line &l, long long at) {
    const int per_item = (int)(at / l.items);  // before[b] <= per_item < before[b + 1]
    int lo = 0, hi = l.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (l.before[mid] <= per_item) lo = mid;
      else hi = mid - 1;
    }
    b = lo;
    tiles = l.before[b + 1] - l.before[b];
    const long long rest = at - (long long)l.before[b] * l.items;
    item = (int)(rest / tiles);
    tile = (int)(rest % tiles);
  }
  __device__ __forceinline__ void next(const Line &l) {
    if (++tile == tiles) next_item(l);
  }
  __device__ __forceinline__ void next_item(const Line &l) {           // b == batch behind the last
    tile = 0;
    if (++item < l.items) return;
    item = 0;
    do ++b;
    while (b < l.batch && l.before[b + 1] == l.before[b]);
    if (b < l.batch) tiles = l.before[b + 1] - l.before[b];
  }
};

// A part: per head o [HD], behind all of them m and sum of each.
template <int HD> __device__ __forceinline__ float *part_at(float *parts, int chunk, int i) { return parts + (size_t)i * chunk * (HD + 2); }
// ... of a CTA: slot 0 of an item that it begins inside of, slot 1 of one that it begins and does not end.
template <int HD> __device__ __forceinline__ float *cta_part(float *parts, int chunk, int cta, int slot) { return part_at<HD>(parts, chunk, kGrid * kWarps + cta * 2 + slot); }

// ---------------------------------------------------------------------------- tiles into a warp's ring
// Pages are looked up 32 at a time, a lane one: those of the window that the tiles come from, and, loaded a window ahead, those of the
// next one (the sequence's next 32 pages, or the first of the item behind it).
template <typename T, int HD> struct Feeder {
  using R = Ring<T, HD>;
  static constexpr int KEYS = Form<T>::KEYS;
  const DecodeArgs &a;
  const Line &line;
  u32 ring;                                    // shared memory
  u32 *masks;                                  // per stage: keys of its tile that are there
  int lane;
  Place at, ahead;                             // tile that is copied next; item of the next window
  int base, ahead_base;                        // first page of the windows
  int pages, ahead_pages;                      // the lane's

  __device__ __forceinline__ int load(const Place &p, int from) const {
    const int i = from + lane;
    return p.b < line.batch && (long long)i * a.pool.page < line.lens[p.b] ? a.page_table[(size_t)p.b * a.pages_per_seq + i] : -1;
  }
  __device__ __forceinline__ void window_behind() {                    // of the one in `ahead`
    if (((long long)ahead_base + 32) * a.pool.page < line.lens[ahead.b]) ahead_base += 32;
    else { ahead.next_item(line); ahead_base = 0; }
    ahead_pages = load(ahead, ahead_base);
  }
  __device__ __forceinline__ void begin(const Place &from) {
    at = ahead = from;
    base = ahead_base = from.tile * KEYS / a.pool.page / 32 * 32;
    pages = load(at, base);
    window_behind();
  }
  __device__ __forceinline__ void copy(int stage) {
    const int key = at.tile * KEYS + lane, pg = key / a.pool.page;
    int rel = pg - base;
    // a tile has at most 16 pages, so they lie in this window and the next
    int id = __shfl_sync(0xFFFFFFFFu, pages, rel & 31);
    const int other = __shfl_sync(0xFFFFFFFFu, ahead_pages, rel & 31);
    if (rel >= 32) id = other;
    long long row = -1;                        // of key `lane`: its place in the pools, -1 without one
    if (lane < KEYS && key < line.lens[at.b] && id >= 0 && id < a.pool.n_pages)
      row = id * a.pool.page_bytes + (key - pg * a.pool.page) * a.pool.token_bytes + (at.item / a.chunks) * a.pool.head_bytes;
    const u32 to = ring + stage * R::STAGE;
    const u32 there = __ballot_sync(0xFFFFFFFFu, row >= 0);
    constexpr int PIECES = R::ROW / 16, AT_ONCE = 32 / PIECES;         // rows that the warp copies at once
    const int c = lane % PIECES;
#pragma unroll
    for (int i = 0; i < KEYS / AT_ONCE; ++i) {
      const int r = i * AT_ONCE + lane / PIECES;
      const long long off = __shfl_sync(0xFFFFFFFFu, row, r);
      const bool ok = off >= 0;
      const long long from = ok ? off + c * 16 : 0;
      copy16(to + piece<T, HD>(r, c), a.pool.k + from, ok);
      copy16(to + R::HALF + piece<T, HD>(r, c), a.pool.v + from, ok);
    }
    if (lane == 0) masks[stage] = there;
    at.next(line);
    if (at.tile == 0) {
      if (at.b >= line.batch) return;          // the line's end
      shift();
      const int h = at.item / a.chunks, q0 = h * a.group + at.item % a.chunks * a.chunk;     // the next item's queries into L1
      const unsigned char *q = static_cast<const unsigned char *>(a.q) + ((size_t)at.b * a.nq + q0) * HD * sizeof(T);
      if (lane * 128 < min(a.chunk, h * a.group + a.group - q0) * HD * (int)sizeof(T)) asm volatile("prefetch.global.L1 [%0];" ::"l"(q + lane * 128));
    } else if ((long long)at.tile * KEYS >= ((long long)base + 32) * a.pool.page) {
      shift();
    }
  }
  __device__ __forceinline__ void shift() {
    base = ahead_base;
    pages = ahead_pages;
    if (ahead.b < line.batch) window_behind();
  }
};

// ---------------------------------------------------------------------------- bf16
template <int HD, int H> struct Bf16Tile {     // H: 8 or 16 rows with queries
  using T = __nv_bfloat16;
  static constexpr int YS = H / 8;
  u32 qf[HD / 16][4];
  float o[HD / 8][4], m[2], l[2];
  int lane;

  // Rows of the tile: the chunk's query heads; rows without one are zeros.
  __device__ __forceinline__ void begin(const DecodeArgs &a, int b, int item) {
    const int h = item / a.chunks, c = item % a.chunks, heads = min(a.chunk, a.group - c * a.chunk);
    const T *q = static_cast<const T *>(a.q) + ((size_t)b * a.nq + (size_t)h * a.group + c * a.chunk) * HD;
    const int r = lane >> 2, col = (lane & 3) * 2;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int row = r + (x & 1) * 8;
        qf[k][x] = (x & 1) < YS && row < heads ? __ldg(reinterpret_cast<const u32 *>(q + row * HD + k * 16 + col + (x >> 1) * 8)) : 0u;
      }
#pragma unroll
    for (int n = 0; n < HD / 8; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[n][x] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  __device__ __forceinline__ void tile(const DecodeArgs &a, u32 at, u32 there) {
    float s[2][4];
#pragma unroll
    for (int x = 0; x < 4; ++x) s[0][x] = s[1][x] = 0.f;
    const int kr = (lane & 7) + ((lane >> 4) << 3), kc = (lane >> 3) & 1;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
      u32 f[4];
      ldsm4(f, at + piece<T, HD>(kr, 2 * k + kc));
      mma(s[0], qf[k], f[0], f[1]);
      mma(s[1], qf[k], f[2], f[3]);
    }
    const int col = (lane & 3) * 2;
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        s[n][x] = (there >> (n * 8 + col + (x & 1))) & 1 ? s[n][x] * a.scale : -INFINITY;
        mx[x >> 1] = fmaxf(mx[x >> 1], s[n][x]);
      }
    u32 hi[4] = {0, 0, 0, 0}, lo[4] = {0, 0, 0, 0};
    float f[2] = {1.f, 1.f};
#pragma unroll
    for (int y = 0; y < YS; ++y) {
      mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xFFFFFFFFu, mx[y], 1));
      mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xFFFFFFFFu, mx[y], 2));
      const float n = fmaxf(m[y], mx[y]);
      f[y] = n > -INFINITY ? ex2(m[y] - n) : 1.f;
      m[y] = n;
      const float ref = n > -INFINITY ? n : 0.f;
      l[y] *= f[y];
#pragma unroll
      for (int n2 = 0; n2 < 2; ++n2) {
        const float p0 = ex2(s[n2][2 * y] - ref), p1 = ex2(s[n2][2 * y + 1] - ref);
        l[y] += p0 + p1;
        const __nv_bfloat162 h2 = __floats2bfloat162_rn(p0, p1);
        const __nv_bfloat162 l2 = __floats2bfloat162_rn(p0 - __low2float(h2), p1 - __high2float(h2));
        hi[n2 * 2 + y] = *reinterpret_cast<const u32 *>(&h2);
        lo[n2 * 2 + y] = *reinterpret_cast<const u32 *>(&l2);
      }
    }
    if (__any_sync(0xFFFFFFFFu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
      for (int n = 0; n < HD / 8; ++n) {
        o[n][0] *= f[0]; o[n][1] *= f[0];
        o[n][2] *= f[1]; o[n][3] *= f[1];
      }
    }
    const u32 v = at + Ring<T, HD>::HALF;
    const int vr = lane & 15, vc = lane >> 4;
#pragma unroll
    for (int n = 0; n < HD / 16; ++n) {
      u32 b[4];
      ldsm4t(b, v + piece<T, HD>(vr, 2 * n + vc));
      mma(o[2 * n], hi, b[0], b[1]);
      mma(o[2 * n + 1], hi, b[2], b[3]);
      mma(o[2 * n], lo, b[0], b[1]);
      mma(o[2 * n + 1], lo, b[2], b[3]);
    }
  }
  __device__ __forceinline__ void end(const DecodeArgs &a, int b, int item, bool whole, float *part) {
    const int h = item / a.chunks, c = item % a.chunks, heads = min(a.chunk, a.group - c * a.chunk), col = (lane & 3) * 2;
    T *out = static_cast<T *>(a.out) + ((size_t)b * a.nq + (size_t)h * a.group + c * a.chunk) * HD;
#pragma unroll
    for (int y = 0; y < YS; ++y) {
      l[y] += __shfl_xor_sync(0xFFFFFFFFu, l[y], 1);
      l[y] += __shfl_xor_sync(0xFFFFFFFFu, l[y], 2);
      const int row = (lane >> 2) + 8 * y;
      if (row >= heads) continue;
      if (whole) {
        const float inv = l[y] != 0.f ? 1.f / l[y] : 0.f;
#pragma unroll
        for (int n = 0; n < HD / 8; ++n)
          *reinterpret_cast<__nv_bfloat162 *>(out + row * HD + n * 8 + col) = __floats2bfloat162_rn(o[n][2 * y] * inv, o[n][2 * y + 1] * inv);
      } else {
#pragma unroll
        for (int n = 0; n < HD / 8; ++n) *reinterpret_cast<float2 *>(part + row * HD + n * 8 + col) = make_float2(o[n][2 * y], o[n][2 * y + 1]);
        if ((lane & 3) == 0) *reinterpret_cast<float2 *>(part + a.chunk * HD + row * 2) = make_float2(m[y], l[y]);
      }
    }
  }
};

// ---------------------------------------------------------------------------- fp32
template <int HD, int H> struct Fp32Tile {     // H: queries at once; those past the chunk's are zeros
  using T = float;
  static constexpr int KEYS = 8, HEADS = H, COLS = HD / 32;
  float o[HEADS][COLS], m[HEADS], l[HEADS];
  float *q;                                    // the warp's queries in shared memory [HEADS][HD]
  int lane, heads;

  __device__ __forceinline__ void begin(const DecodeArgs &a, int b, int item) {
    const int h = item / a.chunks, c = item % a.chunks;
    heads = min(a.chunk, a.group - c * a.chunk);
    const float *from = static_cast<const float *>(a.q) + ((size_t)b * a.nq + (size_t)h * a.group + c * a.chunk) * HD;
    __syncwarp();
    for (int i = lane; i < H * HD; i += 32) q[i] = i < heads * HD ? from[i] : 0.f;
    __syncwarp();
#pragma unroll
    for (int g = 0; g < HEADS; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int e = 0; e < COLS; ++e) o[g][e] = 0.f;
    }
  }
  __device__ __forceinline__ void tile(const DecodeArgs &a, u32 at, u32 there) {
    const unsigned char *k = static_cast<const unsigned char *>(__cvta_shared_to_generic(at)), *v = k + Ring<T, HD>::HALF;
    const int key = lane >> 2, j = lane & 3;
    float s[HEADS];
#pragma unroll
    for (int g = 0; g < HEADS; ++g) s[g] = 0.f;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) {
      const float4 x = *reinterpret_cast<const float4 *>(k + piece<T, HD>(key, i * 4 + j));
#pragma unroll
      for (int g = 0; g < H; ++g) {
        const float4 y = *reinterpret_cast<const float4 *>(q + g * HD + (i * 4 + j) * 4);
        s[g] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s[g]))));
      }
    }
    const bool here = (there >> key) & 1;
    float f[H], mx[H];
#pragma unroll
    for (int d = 1; d < 4; d <<= 1)
#pragma unroll
      for (int g = 0; g < H; ++g) s[g] += __shfl_xor_sync(0xFFFFFFFFu, s[g], d);
#pragma unroll
    for (int g = 0; g < H; ++g) mx[g] = s[g] = here ? s[g] * a.scale : -INFINITY;
#pragma unroll
    for (int d = 4; d < 32; d <<= 1)
#pragma unroll
      for (int g = 0; g < H; ++g) mx[g] = fmaxf(mx[g], __shfl_xor_sync(0xFFFFFFFFu, mx[g], d));
#pragma unroll
    for (int g = 0; g < H; ++g) {
      const float n = fmaxf(m[g], mx[g]), ref = n > -INFINITY ? n : 0.f;
      f[g] = ex2(m[g] - ref);
      m[g] = n;
      s[g] = ex2(s[g] - ref);
      l[g] = fmaf(l[g], f[g], s[g]);           // of this lane's keys: added up at the end
#pragma unroll
      for (int e = 0; e < COLS; ++e) o[g][e] *= f[g];
    }
#pragma unroll
    for (int kk = 0; kk < KEYS; ++kk) {
      float x[COLS];
      const unsigned char *row = v + piece<T, HD>(kk, lane * COLS / 4) + (lane * COLS % 4) * 4;
      if constexpr (COLS == 4) { const float4 y = *reinterpret_cast<const float4 *>(row); x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w; }
      else if constexpr (COLS == 2) { const float2 y = *reinterpret_cast<const float2 *>(row); x[0] = y.x; x[1] = y.y; }
      else x[0] = *reinterpret_cast<const float *>(row);
#pragma unroll
      for (int g = 0; g < H; ++g) {
        const float p = __shfl_sync(0xFFFFFFFFu, s[g], kk * 4);
#pragma unroll
        for (int e = 0; e < COLS; ++e) o[g][e] = fmaf(p, x[e], o[g][e]);
      }
    }
  }
  __device__ __forceinline__ void end(const DecodeArgs &a, int b, int item, bool whole, float *part) {
    const int h = item / a.chunks, c = item % a.chunks;
    float *out = static_cast<float *>(a.out) + ((size_t)b * a.nq + (size_t)h * a.group + c * a.chunk) * HD;
#pragma unroll
    for (int g = 0; g < HEADS; ++g)
      if (g < heads) {
        float sum = l[g];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        const float inv = !whole ? 1.f : sum != 0.f ? 1.f / sum : 0.f;
        float *to = (whole ? out : part) + g * HD + lane * COLS;
#pragma unroll
        for (int e = 0; e < COLS; ++e) to[e] = o[g][e] * inv;
        if (!whole && lane == 0) *reinterpret_cast<float2 *>(part + a.chunk * HD + g * 2) = make_float2(m[g], sum);
      }
  }
};

template <typename T, int HD, int H> struct TileOf { using type = Bf16Tile<HD, H>; };
template <int HD, int H> struct TileOf<float, HD, H> { using type = Fp32Tile<HD, H>; };
template <typename T, int HD, int H> constexpr int kQueryBytes = sizeof(T) == 4 ? H * HD * 4 : 0;          // a warp's, in shared memory
template <typename T, int HD, int H> constexpr int smem_bytes(int batch) {
  return kWarps * (Ring<T, HD>::BYTES + kQueryBytes<T, HD, H>) + kWarps * Ring<T, HD>::STAGES * 4 + kWarps * 4 + (2 * batch + 1) * 4;
}

// What a warp's stretch leaves to its CTA.
enum { kHead = 1, kEnd = 2, kThrough = 4 };    // a part of an item from in front of it that ends in it; of one that runs on behind it; from in front too

template <typename T, int HD, int H>
__global__ void __launch_bounds__(kThreads, 1)
attn_decode_kernel(DecodeArgs a) {
  using R = Ring<T, HD>;
  constexpr int S = R::STAGES;
  static_assert(H * (HD + 2) * 4 <= R::BYTES, "a warp's last part takes its ring's place");
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int left[kWarps];                 // kHead, kEnd, kThrough
  __shared__ int2 left_item[kWarps];           // sequence and item of the part that runs on
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, cta = blockIdx.x;
  unsigned char *rest = smem + kWarps * (R::BYTES + kQueryBytes<T, HD, H>);
  u32 *masks = reinterpret_cast<u32 *>(rest) + warp * S;
  int *warp_sum = reinterpret_cast<int *>(rest) + kWarps * S, *before = warp_sum + kWarps, *lens = before + a.batch + 1;
  chain_wait();
  chain_next();
  const Line line = make_line<Form<T>::KEYS, kThreads>(a.kv_lens, a.batch, (long long)a.pages_per_seq * a.pool.page, a.nkv * a.chunks, before, lens, warp_sum);

  // sequences without a key: zeros
  for (int b = cta; b < a.batch; b += kGrid)
    if (before[b + 1] == before[b])
      for (int i = threadIdx.x; i < a.nq * HD; i += kThreads) static_cast<T *>(a.out)[(size_t)b * a.nq * HD + i] = T(0.f);

  const int s0 = line.first(cta), n_warps = line.first(cta + 1) - s0, me = s0 + warp;
  const long long total = (long long)before[a.batch] * line.items;
  int left_here = 0;
  if (warp < n_warps) {
    const long long from = me * line.per, n = min(line.per, total - from);
    typename TileOf<T, HD, H>::type t;
    t.lane = lane;
    if constexpr (sizeof(T) == 4) t.q = reinterpret_cast<float *>(smem + kWarps * R::BYTES) + warp * H * HD;
    Place at;
    at.find(line, from);
    Feeder<T, HD> feed = {a, line, (u32)__cvta_generic_to_shared(smem) + warp * R::BYTES, masks, lane};
    feed.begin(at);
#pragma unroll
    for (int i = 0; i < S - 1; ++i) {
      if (i < n) feed.copy(i);
      copies_end();
    }
    int stage = 0, fill = S - 1, first = at.tile;
    const Place start = at;
    t.begin(a, at.b, at.item);
    for (long long i = 0; i < n; ++i) {
      copies_wait<S - 2>();
      __syncwarp();
      if (i + S - 1 < n) feed.copy(fill);
      copies_end();
      t.tile(a, feed.ring + stage * R::STAGE, masks[stage]);
      if (++stage == S) stage = 0;
      if (++fill == S) fill = 0;
      const bool last = at.tile + 1 == at.tiles;
      if (last || i + 1 == n) {
        float *part = nullptr;
        if (!last) {
          left_here |= kEnd | (first > 0 ? kThrough : 0);
          if (lane == 0) left_item[warp] = make_int2(at.b, at.item);
          __syncwarp();                        // all lanes are done with the ring
          part = reinterpret_cast<float *>(smem + warp * R::BYTES);
        } else if (first > 0) {
          left_here |= kHead;
          part = part_at<HD>(a.parts, a.chunk, me);
        }
        t.end(a, at.b, at.item, part == nullptr, part);
      }
      if (i + 1 < n) {
        at.next(line);
        if (last) { first = 0; t.begin(a, at.b, at.item); }
      }
    }
    if (warp == 0 && lane == 0) {              // the item that this CTA begins inside of, told by the second CTA that has a part of it
      const long long begin = from - start.tile;
      int4 j = make_int4(0, 0, 0, 0);
      if (start.tile > 0 && line.cta_of(begin) == line.cta_of(from - 1)) j = make_int4(start.b * a.nq + start.item / a.chunks * a.group + start.item % a.chunks * a.chunk,
          min(a.chunk, a.group - start.item % a.chunks * a.chunk), line.cta_of(begin), line.cta_of(begin + start.tiles - 1));
      a.joins[cta] = j;
    }
  } else if (n_warps == 0 && threadIdx.x == 0) {
    a.joins[cta] = make_int4(0, 0, 0, 0);
  }
  if (lane == 0) left[warp] = left_here;
  __syncthreads();

  // Runs of parts of one item: from warp w0 (whose part runs on, or the first) to the one that ends it, or to the CTA's last.
  for (int w0 = 0; w0 < n_warps; ++w0) {
    const bool outside = w0 == 0 && (left[0] & (kHead | kThrough));       // it began in front of this CTA
    for (int turn = outside ? 0 : 1; turn < 2; ++turn) {
      if (turn == 1 && (!(left[w0] & kEnd) || (left[w0] & kThrough))) continue;
      int w1 = w0;
      bool ended = turn == 0 && (left[w0] & kHead);
      while (!ended && w1 + 1 < n_warps) {
        ++w1;
        ended = left[w1] & kHead;
      }
      const bool whole = turn == 1 && ended;
      const int2 it = turn == 1 ? left_item[w0] : make_int2(0, 0);
      const int heads = min(a.chunk, a.group - it.y % a.chunks * a.chunk);
      float *to = cta_part<HD>(a.parts, a.chunk, cta, turn);
      for (int i = threadIdx.x; i < (turn == 1 ? heads : a.chunk) * HD; i += kThreads) {
        const int g = i / HD;
        float m = -INFINITY, l = 0.f, o = 0.f;
        for (int w = w0; w <= w1; ++w) {
          const float *p = ended && w == w1 ? part_at<HD>(a.parts, a.chunk, s0 + w) : reinterpret_cast<const float *>(smem + w * R::BYTES);
          const float m2 = p[a.chunk * HD + 2 * g], n = fmaxf(m, m2), ref = n > -INFINITY ? n : 0.f, f = ex2(m - ref), f2 = ex2(m2 - ref);
          m = n;
          l = fmaf(l, f, p[a.chunk * HD + 2 * g + 1] * f2);
          o = fmaf(o, f, p[i] * f2);
        }
        if (whole) {
          const float y = l != 0.f ? o / l : 0.f;
          const size_t at = ((size_t)it.x * a.nq + (size_t)(it.y / a.chunks) * a.group + it.y % a.chunks * a.chunk) * HD + i;
          if constexpr (sizeof(T) == 4) static_cast<float *>(a.out)[at] = y;
          else static_cast<__nv_bfloat16 *>(a.out)[at] = __float2bfloat16_rn(y);
        } else {
          to[i] = o;
          if (i % HD == 0) { to[a.chunk * HD + 2 * g] = m; to[a.chunk * HD + 2 * g + 1] = l; }
        }
      }
    }
  }
}

// Adds the CTAs' parts of the item that CTA blockIdx.x told of, a CTA a query head.  Warps take parts in turn and add them in order,
// then the warps' sums are added in order.
template <typename T, int HD>
__global__ void __launch_bounds__(kJoinWarps * 32)
attn_join_kernel(DecodeArgs a) {
  constexpr int COLS = HD / 32;
  __shared__ float sh_o[kJoinWarps][HD], sh_m[kJoinWarps], sh_l[kJoinWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = blockIdx.y;
  chain_wait();
  chain_next();
  const int4 it = a.joins[blockIdx.x];         // first row of the output, heads, CTAs
  if (g >= it.y) return;
  float o[COLS], l = 0.f, m = -INFINITY;
#pragma unroll
  for (int e = 0; e < COLS; ++e) o[e] = 0.f;
#pragma unroll 4
  for (int c = it.z + warp; c <= it.w; c += kJoinWarps) {
    const float *p = cta_part<HD>(a.parts, a.chunk, c, c == it.z ? 1 : 0);
    const float2 ml = *reinterpret_cast<const float2 *>(p + a.chunk * HD + g * 2);
    const float n = fmaxf(m, ml.x), ref = n > -INFINITY ? n : 0.f, f = ex2(m - ref), f2 = ex2(ml.x - ref);
    m = n;
    l = fmaf(l, f, ml.y * f2);
#pragma unroll
    for (int e = 0; e < COLS; ++e) o[e] = fmaf(o[e], f, p[g * HD + lane * COLS + e] * f2);
  }
#pragma unroll
  for (int e = 0; e < COLS; ++e) sh_o[warp][lane * COLS + e] = o[e];
  if (lane == 0) { sh_m[warp] = m; sh_l[warp] = l; }
  __syncthreads();
  for (int i = threadIdx.x; i < HD; i += kJoinWarps * 32) {
    float top = -INFINITY, sum = 0.f, all = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, sh_m[w]);
    const float ref = top > -INFINITY ? top : 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
      const float f = ex2(sh_m[w] - ref);
      sum = fmaf(sh_o[w][i], f, sum);
      all = fmaf(sh_l[w], f, all);
    }
    const float y = all != 0.f ? sum / all : 0.f;
    const size_t at = ((size_t)it.x + g) * HD + i;
    if constexpr (sizeof(T) == 4) static_cast<float *>(a.out)[at] = y;
    else static_cast<__nv_bfloat16 *>(a.out)[at] = __float2bfloat16_rn(y);
  }
}

template <typename T, int HD, int H> int run(const DecodeArgs &a, cudaStream_t s) {
  static std::atomic<u64> done{0};
  const int status = hsd_smem_limit((const void *)attn_decode_kernel<T, HD, H>, smem_bytes<T, HD, H>(kMaxBatch), done);
  if (status) return status;
  HSD_CUDA_OK(hsd_launch(attn_decode_kernel<T, HD, H>, dim3(kGrid), kThreads, smem_bytes<T, HD, H>(a.batch), s, 0, true, a));
  HSD_CUDA_OK(hsd_launch(attn_join_kernel<T, HD>, dim3(kGrid, a.chunk), kJoinWarps * 32, 0, s, 0, true, a));
  hsd_count_launches(2);
  return hsd_launch_status();
}
template <typename T, int HD> int run_heads(const DecodeArgs &a, cudaStream_t s) {
  if constexpr (sizeof(T) == 2) return a.chunk <= 8 ? run<T, HD, 8>(a, s) : run<T, HD, 16>(a, s);
  else return a.chunk == 1 ? run<T, HD, 1>(a, s) : a.chunk == 2 ? run<T, HD, 2>(a, s) : a.chunk <= 4 ? run<T, HD, 4>(a, s) : run<T, HD, 8>(a, s);
}
template <typename T> int run_hd(const DecodeArgs &a, int hd, cudaStream_t s) {
  return hd == 32 ? run_heads<T, 32>(a, s) : hd == 64 ? run_heads<T, 64>(a, s) : run_heads<T, 128>(a, s);
}

}  // namespace
}  // namespace hsd

extern "C" size_t hsd_paged_attention_workspace_bytes(int n_q_heads, int n_kv_heads, int head_dim) {
  if (n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || (head_dim != 32 && head_dim != 64 && head_dim != 128)) return 0;
  const int group = n_q_heads / n_kv_heads, chunk = group < 16 ? group : 16;
  return (size_t)hsd::kGrid * (hsd::kWarps + 2) * chunk * (head_dim + 2) * sizeof(float) + hsd::kGrid * sizeof(int4);
}

extern "C" int hsd_paged_attention(const void *q, int batch, int n_q_heads, int n_kv_heads, int head_dim, const hsd_kv_pool *pool,
                                   const int32_t *page_table, int pages_per_seq, const int32_t *kv_lens, float scale, void *workspace,
                                   size_t workspace_bytes, void *out, void *stream) {
  using namespace hsd;
  if (!q || !page_table || !kv_lens || !out || !workspace || batch <= 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads) return HSD_E_INVALID_ARG;
  if (!(scale == scale) || isinf(scale)) return HSD_E_INVALID_ARG;
  DecodeArgs a = {};
  const int status = pool_view(pool, n_kv_heads, head_dim, pages_per_seq, a.pool);
  if (status) return status;
  if (batch > kMaxBatch || (long long)pages_per_seq * pool->page_size > (1ll << 33) / batch || n_q_heads > 65536) return HSD_E_TOO_LARGE;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(workspace)) & 15) return HSD_E_INVALID_ARG;
  if (workspace_bytes < hsd_paged_attention_workspace_bytes(n_q_heads, n_kv_heads, head_dim)) return HSD_E_WORKSPACE_TOO_SMALL;
  a.q = q; a.out = out; a.page_table = page_table; a.kv_lens = kv_lens; a.joins = static_cast<int4 *>(workspace);
  a.parts = reinterpret_cast<float *>(a.joins + kGrid);
  a.scale = scale * 1.4426950408889634f;
  a.batch = batch; a.nq = n_q_heads; a.nkv = n_kv_heads; a.pages_per_seq = pages_per_seq;
  a.group = n_q_heads / n_kv_heads;
  const int most = pool->dtype == HSD_F32 ? Form<float>::HEADS : Form<__nv_bfloat16>::HEADS;
  a.chunks = ceil_div(a.group, most);
  a.chunk = ceil_div(a.group, a.chunks);
  return pool->dtype == HSD_F32 ? run_hd<float>(a, head_dim, (cudaStream_t)stream) : run_hd<__nv_bfloat16>(a, head_dim, (cudaStream_t)stream);
}
