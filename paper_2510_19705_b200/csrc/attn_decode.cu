// Attention of one new token per sequence over the caller's paged cache (hsd_paged_attention).
//   o = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale q.k_j - m),  m = max_j scale q.k_j   over the sequence's keys j
// Bound by memory: every key and value is read once, for all query heads of its group.  The tiles (8 to 32 keys of one sequence
// and head) of the whole batch stand in one line, which is divided evenly over the warps, whatever the lengths are: the grid
// does not depend on them, and they are read on the device.  A warp streams its stretch through a ring of its own in shared memory
// (cp.async, no barrier between warps), across the borders of sequences and heads.  Where a stretch ends inside a sequence, the parts
// (m, sum, o) of its neighbours are added by the CTA, and where the CTA ends inside one, its part goes to the workspace and
// attn_join_kernel adds those in order.
// bf16: both products on mma.sync with the group's queries as the 16 rows of a tile (at 4 to 16 queries a key the tensor pipe is
// far from its limit); weights as three bf16 parts, all of their 24 bits, so that only the final rounding is one of 8 bits (up to 8 queries a
// key: two products, as rows 8 to 15 take the middle parts; more: three, 16 over 1 head of 128, 16 x 8200 keys, 29.2 us against 28.1 with 16 bits).
// fp32: both products on mma.sync in TF32: keys and values as three TF32 parts, which are all of their bits, queries and weights as two, which are
// theirs but for a last place, one above the other in the rows of a tile, so that three products take all pairs that count: the same tile
// of 8 queries for any group, where products in fp32 read every query again from shared memory for each key.  (Keys and values as two
// parts and no product of the low ones were 20 % less exact than fp32, and no faster: 16 x 8200 keys, 32 heads over 8 of 128, 239 us against
// 234.)  What lies below TF32's smallest number, 2^-136, is lost.
// The tensor cores' adders cut off: a chain of products loses up to 2^-23 of its sum a product (1.2e-4 of the output over 20000 keys
// a sequence when the chain was a stretch).  So no chain is longer than a tile; tiles' products are added in fp32, rounded to nearest.
#include "attn_tiles.cuh"

namespace hsd {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kGrid = kMeasuredSMs;            // CTAs at most: fixed, as the workspace's size depends on it
constexpr int kMaxBatch = 4096;                // its tiles' prefix sums lie in shared memory
constexpr int kJoinWarps = 16;

struct DecodeArgs {
  const void *q;
  void *out;
  const int32_t *page_table, *kv_lens;
  float *parts;                                // of stretches (kGrid * kWarps), then of CTAs (two each)
  int4 *joins;                                 // per CTA: the item that it begins inside of, if it is the second with a part of it
  PoolView pool;
  float scale;                                 // times log2(e)
  int batch, nq, nkv, pages_per_seq, page_shift;        // log2 of the page size, or -1
  int group, chunk, chunks;                    // query heads of a key head; of them at once; times
};

// The line of tiles: sequence b has as many for each of `items` (key head, chunk of query heads); before[b]: tiles of the
// sequences in front of b, per item; lens[b]: keys.
struct Line {
  const int *before, *lens;
  int batch, items, stretches;
  long long total, per;                        // tiles; of a stretch
  // Stretches [first(c), first(c + 1)) are CTA c's: few of them lie on as many SMs, and no CTA without one stands between others.
  __device__ __forceinline__ int first(int cta) const { return stretches < kGrid ? min(cta, stretches) : cta * stretches / kGrid; }
  __device__ __forceinline__ int cta_of(long long tile) const {
    const int i = (int)divide(tile, per);
    return stretches < kGrid ? i : ((i + 1) * kGrid - 1) / stretches;
  }
};
// Lengths within the page table's room, and the prefix sums; all threads of the CTA.
template <int KEYS, int THREADS>
__device__ __forceinline__ Line make_line(const int32_t *kv_lens, int batch, long long room, int items, int *before, int *lens, int *warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int carry = 0;
  if (batch <= 32) {                           // every warp for itself: all of them write the same
    const int len = lane < batch ? (int)min((long long)max(kv_lens[lane], 0), room) : 0, n = (len + KEYS - 1) / KEYS;
    int upto = n;
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += x;
    }
    carry = __shfl_sync(0xFFFFFFFFu, upto, 31);
    if (lane < batch) {
      before[lane + 1] = upto;
      lens[lane] = len;
    }
    if (lane == 0) before[0] = 0;
    __syncwarp();
  } else for (int b0 = 0; b0 < batch; b0 += THREADS) {
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
    if (threadIdx.x == 0) before[0] = 0;
    __syncthreads();
  }
  Line l;
  l.before = before; l.lens = lens; l.batch = batch; l.items = items;
  const long long total = (long long)carry * items, warps = kGrid * kWarps;
  l.total = total;
  l.per = max(divide(total + warps - 1, warps), 1ll);
  l.stretches = (int)divide(total + l.per - 1, l.per);
  return l;
}

// A place on the line.
struct Place {
  int b, item, tile, tiles;                    // tiles: of the sequence
  __device__ __forceinline__ void find(const Line &l, long long at) {
    const int per_item = (int)divide(at, l.items);  // before[b] <= per_item < before[b + 1]
    int lo = 0, hi = l.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (l.before[mid] <= per_item) lo = mid;
      else hi = mid - 1;
    }
    b = lo;
    tiles = l.before[b + 1] - l.before[b];
    const long long rest = at - (long long)l.before[b] * l.items;
    item = (int)divide(rest, tiles);
    tile = (int)(rest - (long long)item * tiles);
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
  static constexpr int KEYS = Form<T, HD>::KEYS, PIECES = R::ROW / 16, AT_ONCE = 32 / PIECES;          // rows that the warp copies at once
  static_assert(32 % KEYS == 0, "a tile lies in one window");
  const DecodeArgs &a;
  const Line &line;
  u32 ring;                                    // shared memory
  u32 *masks;                                  // per stage: keys of its tile that are there
  int lane;
  Place at, ahead;                             // tile that is copied next; item of the next window
  int base, ahead_base;                        // first page of the windows
  int pages, ahead_pages;                      // the lane's
  int len;                                     // of the sequence
  long long head, mine;                        // the head's place in the pools; the lane's in the rows that are copied at once

  __device__ __forceinline__ int page_of(int key) const { return a.page_shift >= 0 ? key >> a.page_shift : key / a.pool.page; }
  __device__ __forceinline__ void item_begins() {
    len = line.lens[at.b];
    head = (at.item / a.chunks) * a.pool.head_bytes;
  }
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
    base = ahead_base = page_of(from.tile * KEYS) / 32 * 32;
    pages = load(at, base);
    window_behind();
    mine = lane / PIECES * a.pool.token_bytes + lane % PIECES * 16;
    item_begins();
  }
  // Place in the pools of a key of the tile, -1 without one.
  __device__ __forceinline__ long long place(int key, bool wanted) const {
    // a window's 32 pages are a multiple of 32 tokens, tiles are 8, 16 or 32 at multiples of their size: none lies in two windows
    const int pg = page_of(key), id = __shfl_sync(0xFFFFFFFFu, pages, (pg - base) & 31);
    return wanted && key < len && id >= 0 && id < a.pool.n_pages ? id * a.pool.page_bytes + (key - pg * a.pool.page) * a.pool.token_bytes + head : -1;
  }
  __device__ __forceinline__ void copy(int stage) {
    const u32 to = ring + stage * R::STAGE;
    const int key0 = at.tile * KEYS, rest = len - key0, c = lane % PIECES;
    u32 there;
    if (a.pool.page % 8 == 0) {                // eight keys in one page: lane b has the place of the b-th eight
      const long long p = place(key0 + 8 * (lane & 3), lane < KEYS / 8);
      there = 0;
#pragma unroll
      for (int b = 0; b < KEYS / 8; ++b) {
        const long long block = __shfl_sync(0xFFFFFFFFu, p, b);
        there |= block >= 0 ? 0xFFu << (8 * b) : 0u;
#pragma unroll
        for (int i = 0; i < 8 / AT_ONCE; ++i) {
          const int r = b * 8 + i * AT_ONCE + lane / PIECES;
          const bool ok = block >= 0 && r < rest;
          const long long from = ok ? block + i * AT_ONCE * a.pool.token_bytes + mine : 0;
          copy16(to + piece<T, HD>(r, c), a.pool.k + from, ok);
          copy16(to + R::HALF + piece<T, HD>(r, c), a.pool.v + from, ok);
        }
      }
      if (rest < 32) there &= (1u << rest) - 1;
    } else {                                   // lane i has the place of key i
      const long long p = place(key0 + lane, lane < KEYS);
      there = __ballot_sync(0xFFFFFFFFu, p >= 0);
#pragma unroll
      for (int i = 0; i < KEYS / AT_ONCE; ++i) {
        const int r = i * AT_ONCE + lane / PIECES;
        const long long row = __shfl_sync(0xFFFFFFFFu, p, r);
        const bool ok = row >= 0;
        const long long from = ok ? row + c * 16 : 0;
        copy16(to + piece<T, HD>(r, c), a.pool.k + from, ok);
        copy16(to + R::HALF + piece<T, HD>(r, c), a.pool.v + from, ok);
      }
    }
    if (lane == 0) masks[stage] = there;
    at.next(line);
    if (at.tile == 0) {
      if (at.b >= line.batch) return;          // the line's end
      shift();
      item_begins();
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

template <typename T, int HD> constexpr int smem_bytes(int batch) {
  return kWarps * Ring<T, HD>::BYTES + kWarps * Ring<T, HD>::STAGES * 4 + kWarps * 4 + (2 * batch + 1) * 4;
}

// Row of q and the output that an item's first query head has.
__device__ __forceinline__ size_t first_row(const DecodeArgs &a, int b, int item) {
  return (size_t)b * a.nq + (size_t)(item / a.chunks) * a.group + item % a.chunks * a.chunk;
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
  unsigned char *rest = smem + kWarps * R::BYTES;
  u32 *masks = reinterpret_cast<u32 *>(rest) + warp * S;
  int *warp_sum = reinterpret_cast<int *>(rest) + kWarps * S, *before = warp_sum + kWarps, *lens = before + a.batch + 1;
  chain_wait();
  chain_next();
  const Line line = make_line<Form<T, HD>::KEYS, kThreads>(a.kv_lens, a.batch, (long long)a.pages_per_seq * a.pool.page, a.nkv * a.chunks, before, lens, warp_sum);

  // sequences without a key: zeros
  for (int b = cta; b < a.batch; b += kGrid)
    if (before[b + 1] == before[b])
      for (int i = threadIdx.x; i < a.nq * HD; i += kThreads) static_cast<T *>(a.out)[(size_t)b * a.nq * HD + i] = T(0.f);

  const int s0 = line.first(cta), n_warps = line.first(cta + 1) - s0, me = s0 + warp;
  int left_here = 0;
  if (warp < n_warps) {
    const long long from = me * line.per, n = min(line.per, line.total - from);
    typename TileOf<T, HD, H>::type t;
    t.lane = lane;
    Place at;
    at.find(line, from);
    Feeder<T, HD> feed = {a, line, (u32)__cvta_generic_to_shared(smem) + warp * R::BYTES, masks, lane};
    feed.begin(at);
    int stage = 0, fill = 0, first = at.tile;
    const Place start = at;
#pragma unroll 1
    for (; fill < S - 1; ++fill) {             // (not unrolled: short calls wait for their instructions)
      if (fill < n) feed.copy(fill);
      copies_end();
    }
    auto begin = [&] {                         // rows of the tile: the chunk's query heads
      const int c = at.item % a.chunks, heads = min(a.chunk, a.group - c * a.chunk), r = lane >> 2;
      const T *q = static_cast<const T *>(a.q) + first_row(a, at.b, at.item) * HD + r * HD;
      t.begin(r < heads ? q : nullptr, r + 8 < heads ? q + 8 * HD : nullptr);
    };
    begin();
    for (long long i = 0; i < n; ++i) {
      copies_wait<S - 2>();
      __syncwarp();
      if (i + S - 1 < n) feed.copy(fill);
      copies_end();
      if (++fill == S) fill = 0;
      t.tile(a.scale, feed.ring + stage * R::STAGE, masks[stage], masks[stage]);
      if (++stage == S) stage = 0;
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
        t.end(part ? nullptr : static_cast<T *>(a.out) + first_row(a, at.b, at.item) * HD, part, a.chunk, min(a.chunk, a.group - at.item % a.chunks * a.chunk));
      }
      if (i + 1 < n) {
        at.next(line);
        if (last) { first = 0; begin(); }
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

  // Runs of parts of one item: from the first warp, if it begins inside of an item (run 0), or one whose part begins there and runs on,
  // to the warp that ends it, or to the CTA's last.
  u32 heads_of = 0, ends = 0, through = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    heads_of |= (left[w] & kHead) ? 1u << w : 0u;
    ends |= (left[w] & kEnd) ? 1u << w : 0u;
    through |= (left[w] & kThrough) ? 1u << w : 0u;
  }
  u32 runs = (ends & ~through) << 1 | ((heads_of | through) & 1u);     // bit 0: run 0, bit w + 1: from warp w
  // a run for each warp, or for two, four or all of them where there are few
  const int n_runs = __popc(runs), share = n_runs == 1 ? kWarps : n_runs == 2 ? kWarps / 2 : n_runs <= 4 ? kWarps / 4 : 1;
  const int thread = threadIdx.x % (share * 32);
  for (int r = 0; runs; ++r, runs &= runs - 1) {
    if (r % (kWarps / share) != warp / share) continue;
    const int run = __ffs(runs) - 1, w0 = max(run - 1, 0);
    const u32 behind = heads_of & ~(run == 0 ? 0u : (2u << w0) - 1);   // warps that may end it
    const bool ended = behind != 0, whole = run > 0 && ended;
    const int w1 = ended ? __ffs(behind) - 1 : n_warps - 1;
    const int2 it = run > 0 ? left_item[w0] : make_int2(0, 0);
    float *to = cta_part<HD>(a.parts, a.chunk, cta, run > 0);
    const int heads = run > 0 ? min(a.chunk, a.group - it.y % a.chunks * a.chunk) : a.chunk;
    for (int i = thread * 4; i < heads * HD; i += share * 128) {
      const int g = i / HD, stat = a.chunk * HD + 2 * g;
      float2 ml[kWarps];
      float4 o[kWarps];
      float m = -INFINITY, l = 0.f;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        ml[w] = make_float2(-INFINITY, 0.f);
        o[w] = sum;
        if (w >= w0 && w <= w1) {
          const float *p = ended && w == w1 ? part_at<HD>(a.parts, a.chunk, s0 + w) : reinterpret_cast<const float *>(smem + w * R::BYTES);
          ml[w] = *reinterpret_cast<const float2 *>(p + stat);
          o[w] = make_float4(p[i], p[i + 1], p[i + 2], p[i + 3]);
        }
        m = fmaxf(m, ml[w].x);
      }
      const float ref = m > -INFINITY ? m : 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = ex2(ml[w].x - ref);
        l = fmaf(ml[w].y, f, l);
        sum.x = fmaf(o[w].x, f, sum.x); sum.y = fmaf(o[w].y, f, sum.y); sum.z = fmaf(o[w].z, f, sum.z); sum.w = fmaf(o[w].w, f, sum.w);
      }
      if (whole) {
        const float inv = l != 0.f ? 1.f / l : 0.f;
        store4(static_cast<T *>(a.out) + ((size_t)it.x * a.nq + (size_t)(it.y / a.chunks) * a.group + it.y % a.chunks * a.chunk) * HD + i,
               make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
      } else {
        *reinterpret_cast<float2 *>(to + i) = make_float2(sum.x, sum.y);
        *reinterpret_cast<float2 *>(to + i + 2) = make_float2(sum.z, sum.w);
        if (i % HD == 0) *reinterpret_cast<float2 *>(to + stat) = make_float2(m, l);
      }
    }
  }
}

// Adds the CTAs' parts of the item that CTA blockIdx.x told of, a CTA a query head.  Warps take parts in turn, each at most kPerWarp, whose
// loads wait for nothing but the item's description, and add them in order; then the warps' sums are added in order.
constexpr int kPerWarp = (kGrid + kJoinWarps - 1) / kJoinWarps;
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
  auto part = [&](int c) -> const float * { return cta_part<HD>(a.parts, a.chunk, c, c == it.z ? 1 : 0); };
  const int mine = it.z + warp + lane * kJoinWarps;                    // the lane's part's statistics
  const bool there = lane < kPerWarp && mine <= it.w;
  const float2 ml = there ? *reinterpret_cast<const float2 *>(part(mine) + a.chunk * HD + g * 2) : make_float2(-INFINITY, 0.f);
  float x[kPerWarp][COLS];
#pragma unroll
  for (int k = 0; k < kPerWarp; ++k) {
    const int c = it.z + warp + k * kJoinWarps;
#pragma unroll
    for (int e = 0; e < COLS; ++e) x[k][e] = 0.f;
    if (c <= it.w) {
#pragma unroll
      for (int e = 0; e < COLS; ++e) x[k][e] = part(c)[g * HD + e * 32 + lane];
    }
  }
  float m = ml.x;
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  const float f = ex2(ml.x - (m > -INFINITY ? m : 0.f));
  float l = ml.y * f, o[COLS];
  for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, d);
#pragma unroll
  for (int e = 0; e < COLS; ++e) o[e] = 0.f;
#pragma unroll
  for (int k = 0; k < kPerWarp; ++k) {
    const float f2 = __shfl_sync(0xFFFFFFFFu, f, k);
#pragma unroll
    for (int e = 0; e < COLS; ++e) o[e] = fmaf(x[k][e], f2, o[e]);
  }
#pragma unroll
  for (int e = 0; e < COLS; ++e) sh_o[warp][e * 32 + lane] = o[e];
  if (lane == 0) { sh_m[warp] = m; sh_l[warp] = l; }
  __syncthreads();
  for (int i = threadIdx.x; i < HD; i += kJoinWarps * 32) {
    float top = -INFINITY, sum = 0.f, all = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, sh_m[w]);
    const float ref = top > -INFINITY ? top : 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
      const float f2 = ex2(sh_m[w] - ref);
      sum = fmaf(sh_o[w][i], f2, sum);
      all = fmaf(sh_l[w], f2, all);
    }
    const float y = all != 0.f ? sum / all : 0.f;
    const size_t at = ((size_t)it.x + g) * HD + i;
    if constexpr (sizeof(T) == 4) static_cast<float *>(a.out)[at] = y;
    else static_cast<__nv_bfloat16 *>(a.out)[at] = __float2bfloat16_rn(y);
  }
}

template <typename T, int HD, int H> int run(const DecodeArgs &a, cudaStream_t s) {
  static std::atomic<u64> done{0};
  const int status = hsd_smem_limit((const void *)attn_decode_kernel<T, HD, H>, smem_bytes<T, HD>(kMaxBatch), done);
  if (status) return status;
  HSD_CUDA_OK(hsd_launch(attn_decode_kernel<T, HD, H>, dim3(kGrid), kThreads, smem_bytes<T, HD>(a.batch), s, 0, true, a));
  HSD_CUDA_OK(hsd_launch(attn_join_kernel<T, HD>, dim3(kGrid, a.chunk), kJoinWarps * 32, 0, s, 0, true, a));
  hsd_count_launches(2);
  return hsd_launch_status();
}
template <typename T, int HD> int run_heads(const DecodeArgs &a, cudaStream_t s) {
  if constexpr (sizeof(T) == 2) if (a.chunk > 8) return run<T, HD, 16>(a, s);
  return run<T, HD, 8>(a, s);
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
  const float scale2 = scale * 1.4426950408889634f;
  if (!isfinite(scale2) || !words(page_table, kv_lens)) return HSD_E_INVALID_ARG;
  DecodeArgs a = {};
  const int status = pool_view(pool, n_kv_heads, head_dim, pages_per_seq, a.pool);
  if (status) return status;
  if (batch > kMaxBatch || (long long)pages_per_seq * pool->page_size > (1ll << 33) / batch || n_q_heads > 65536) return HSD_E_TOO_LARGE;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(workspace)) & 15) return HSD_E_INVALID_ARG;
  if (workspace_bytes < hsd_paged_attention_workspace_bytes(n_q_heads, n_kv_heads, head_dim)) return HSD_E_WORKSPACE_TOO_SMALL;
  a.q = q; a.out = out; a.page_table = page_table; a.kv_lens = kv_lens; a.joins = static_cast<int4 *>(workspace);
  a.parts = reinterpret_cast<float *>(a.joins + kGrid);
  a.scale = scale2;
  a.batch = batch; a.nq = n_q_heads; a.nkv = n_kv_heads; a.pages_per_seq = pages_per_seq;
  a.group = n_q_heads / n_kv_heads;
  a.page_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (pool->page_size == 1 << i) a.page_shift = i;
  const int most = pool->dtype == HSD_F32 ? Form<float, 128>::HEADS : Form<__nv_bfloat16, 128>::HEADS;
  a.chunks = ceil_div(a.group, most);
  a.chunk = ceil_div(a.group, a.chunks);
  return pool->dtype == HSD_F32 ? run_hd<float>(a, head_dim, (cudaStream_t)stream) : run_hd<__nv_bfloat16>(a, head_dim, (cudaStream_t)stream);
}
