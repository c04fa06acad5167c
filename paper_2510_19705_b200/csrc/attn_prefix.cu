// Attention of a batch whose sequences share a prefix, a few new tokens each (hsd_prefix_attention).
//   o_r = sum_j w_rj v_j / sum_j w_rj,  w_rj = exp(scale q_r.k_j - m_r)   over the prefix's keys and the row's own sequence's behind it
// The prefix's keys and values are read once for all rows, where attention by sequence reads them once for each.  The softmax is cut at
// the prefix's end: sums over the prefix with all rows as one set of queries, sums over a sequence's own keys with its rows, and a join
// (prefix_join_kernel) that adds the parts of each row and head.
//
// prefix_lane_kernel: the line of tiles of hsd_paged_attention, in which the prefix stands as one more sequence with all rows' queries in
// sets of 8 or 16; divided evenly over the warps of a grid of fixed size, whatever the lengths are.  Lengths, the prefix's too, are read
// on the device.  A part of an item goes to the place of its rows (one for the prefix, one for the own keys) from the CTA in which the
// item begins, and to a place of the CTA from those behind it.
#include "attn_prefix.cuh"
#include "attn_tiles.cuh"

namespace hsd {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32, kGrid = kPrefixGrid;
constexpr int kMaxBatch = 4096;                // its tiles' prefix sums lie in shared memory
constexpr int kMostChunk = 16;                 // queries of an item
constexpr int kAll = 0x7FFFFFFF;               // rows that are none see all positions

// A sequence's rows: the first and one past the last that the call has; how many its list names, and how many of those are in front of the first.
struct Rows { int x, y, n, front; };
__device__ __forceinline__ Rows rows_of(const PrefixArgs &a, int b) {
  if (!a.row_starts) return {b, b + 1, 1, 0};
  const int s0 = a.row_starts[b], s1 = a.row_starts[b + 1], r0 = min(max(s0, 0), a.rows);
  return {r0, min(max(s1, r0), a.rows), (int)min(max((long long)s1 - s0, 0ll), 0x7FFFFFFFll), s0 < 0 ? -s0 : 0};
}
__device__ __forceinline__ int seq_of(const PrefixArgs &a, int r) {            // -1, batch: rows without one
  if (!a.row_starts) return r;
  int lo = -1, hi = a.batch;                   // starts[lo] <= r < starts[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.row_starts[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo >= 0 && r < a.row_starts[lo + 1] ? lo : lo < 0 ? -1 : a.batch;
}
// What a sequence's rows see: the first of them the positions below `first` (each one behind it one more), own keys up to `end`.  A sequence
// that does not have the whole prefix has no keys: first < 0.
struct Seen { int first, end; };
__device__ __forceinline__ Seen seen_by(const PrefixArgs &a, const Lens &l, int b, const Rows &rows) {
  const int len = l.of(a, b), first = len - rows.n + 1;
  return first < l.prefix || rows.x == rows.y ? Seen{-1, 0} : Seen{first + rows.front, min(len, l.room)};
}

// The line of tiles.  Sequence 0 is the prefix, b + 1 the own keys of sequence b: tiles from `front` on (the own keys begin inside a tile).
struct Line {
  const int *before, *ends;                    // tiles times chunks of the sequences in front, per key head; keys end
  int seqs, nkv, stretches, front, prefix;
  long long total, per;                        // tiles; of a stretch
  __device__ __forceinline__ int first(int cta) const { return stretches < kGrid ? min(cta, stretches) : cta * stretches / kGrid; }
  __device__ __forceinline__ int cta_of(long long tile) const {
    const int i = (int)divide(tile, per);
    return stretches < kGrid ? i : ((i + 1) * kGrid - 1) / stretches;
  }
  template <int KEYS> __device__ __forceinline__ int tiles(int s) const { return (ends[s] + KEYS - 1) / KEYS - (s > 0 ? front : 0); }
};
template <int KEYS>
__device__ __forceinline__ Line make_line(const PrefixArgs &a, bool prefix, int *before, int *ends, int *warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Lens lens;
  lens.read(a);
  const int front = lens.prefix / KEYS, seqs = a.batch + 1;
  int carry = 0;
  for (int s0 = 0; s0 < seqs; s0 += kThreads) {
    const int s = s0 + threadIdx.x;
    int n = 0, end = 0;
    if (s == 0) {
      if (prefix) { end = lens.prefix; n = (end + KEYS - 1) / KEYS * ceil_div(a.rows * a.group, a.chunk); }
    } else if (s < seqs) {
      const Rows r = rows_of(a, s - 1);
      end = seen_by(a, lens, s - 1, r).end;
      if (end > lens.prefix) n = ((end + KEYS - 1) / KEYS - front) * ceil_div((r.y - r.x) * a.group, a.chunk);
    }
    int upto = n;
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    int in_front = carry;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) in_front += warp_sum[w];
      carry += warp_sum[w];
    }
    if (s < seqs) {
      before[s + 1] = in_front + upto;
      ends[s] = end;
    }
    if (threadIdx.x == 0) before[0] = 0;
    __syncthreads();
  }
  Line l;
  l.before = before; l.ends = ends; l.seqs = seqs; l.nkv = a.nkv; l.front = front; l.prefix = lens.prefix;
  const long long total = (long long)carry * a.nkv, warps = kGrid * kWarps;
  l.total = total;
  l.per = max(divide(total + warps - 1, warps), 1ll);
  l.stretches = (int)divide(total + l.per - 1, l.per);
  return l;
}

// A place on the line: item = key head times chunks + chunk, tile of the item.
template <int KEYS> struct Place {
  int s, item, tile, tiles, items;
  __device__ __forceinline__ void of_seq(const Line &l) {
    tiles = l.tiles<KEYS>(s);
    items = (l.before[s + 1] - l.before[s]) / tiles * l.nkv;
  }
  __device__ __forceinline__ void find(const Line &l, long long at) {
    const int per_head = (int)divide(at, l.nkv);                       // before[s] <= per_head < before[s + 1]
    int lo = 0, hi = l.seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (l.before[mid] <= per_head) lo = mid;
      else hi = mid - 1;
    }
    s = lo;
    of_seq(l);
    const long long rest = at - (long long)l.before[s] * l.nkv;
    item = (int)divide(rest, tiles);
    tile = (int)(rest - (long long)item * tiles);
  }
  __device__ __forceinline__ void next_item(const Line &l) {           // s == seqs behind the last
    tile = 0;
    if (++item < items) return;
    item = 0;
    do ++s;
    while (s < l.seqs && l.before[s + 1] == l.before[s]);
    if (s < l.seqs) of_seq(l);
  }
  __device__ __forceinline__ void next(const Line &l) {
    if (++tile == tiles) next_item(l);
  }
  __device__ __forceinline__ int first_key(const Line &l) const { return ((s > 0 ? l.front : 0) + tile) * KEYS; }
};

// The queries of an item: `n` of them, the first is query `v0` of the key head, counted over rows and, in them, over the head's group.
struct Queries {
  int head, v0, n, row0;                       // row0: the sequence's first row
  template <int KEYS> __device__ __forceinline__ void of(const PrefixArgs &a, const Place<KEYS> &p, int nkv) {
    const int chunks = p.items / nkv;
    head = p.item / chunks;
    Rows r = {0, a.rows, a.rows, 0};
    if (p.s > 0) r = rows_of(a, p.s - 1);
    row0 = r.x;
    v0 = (p.item - head * chunks) * a.chunk;
    n = min(a.chunk, (r.y - r.x) * a.group - v0);
  }
  __device__ __forceinline__ size_t at(const PrefixArgs &a, int i) const {      // row and head of q and the output
    const int v = v0 + i, r = v / a.group;
    return (size_t)(row0 + r) * a.nq + head * a.group + (v - r * a.group);
  }
};

// ---------------------------------------------------------------------------- tiles into a warp's ring
// Pages are looked up 32 at a time, a lane one: those of the window that the tiles come from, and, loaded a window ahead, those of the
// next one (the sequence's next 32 pages, or the first of the item behind it).
template <typename T, int HD> struct Feeder {
  using R = Ring<T, HD>;
  static constexpr int KEYS = Form<T, HD>::KEYS, PIECES = R::ROW / 16, AT_ONCE = 32 / PIECES;          // rows that the warp copies at once
  static_assert(32 % KEYS == 0, "a tile lies in one window");
  const PrefixArgs &a;
  const Line &line;
  u32 ring;                                    // shared memory
  u32 *masks;                                  // per stage: keys of its tile that are there
  int lane;
  Place<KEYS> at, ahead;                       // tile that is copied next; item of the next window
  int base, ahead_base;                        // first page of the windows
  int pages, ahead_pages;                      // the lane's
  int begin_key, end_key;                      // of the sequence
  long long head, mine;                        // the head's place in the pools; the lane's in the rows that are copied at once

  __device__ __forceinline__ int page_of(int key) const { return a.page_shift >= 0 ? key >> a.page_shift : key / a.pool.page; }
  __device__ __forceinline__ void item_begins() {
    end_key = line.ends[at.s];
    begin_key = at.s > 0 ? line.prefix : 0;
    head = at.item / (at.items / line.nkv) * a.pool.head_bytes;
  }
  __device__ __forceinline__ int load(const Place<KEYS> &p, int from) const {
    const int i = from + lane;
    if (p.s >= line.seqs || (long long)i * a.pool.page >= line.ends[p.s]) return -1;
    if (p.s == 0) return a.prefix_pages[i];
    return ((long long)i + 1) * a.pool.page <= line.prefix ? -1 : a.page_table[(size_t)(p.s - 1) * a.pages_per_seq + i];   // (whole pages below: not read)
  }
  __device__ __forceinline__ void window_behind() {                    // of the one in `ahead`
    if (((long long)ahead_base + 32) * a.pool.page < line.ends[ahead.s]) ahead_base += 32;
    else {
      ahead.next_item(line);
      ahead_base = ahead.s < line.seqs ? page_of(ahead.first_key(line)) / 32 * 32 : 0;
    }
    ahead_pages = load(ahead, ahead_base);
  }
  __device__ __forceinline__ void begin(const Place<KEYS> &from) {
    at = ahead = from;
    base = ahead_base = page_of(from.first_key(line)) / 32 * 32;
    pages = load(at, base);
    window_behind();
    mine = lane / PIECES * a.pool.token_bytes + lane % PIECES * 16;
    item_begins();
  }
  // Place in the pools of a key of the tile, -1 without one.
  __device__ __forceinline__ long long place(int key, bool wanted) const {
    // a window's 32 pages are a multiple of 32 tokens, tiles are 8, 16 or 32 at multiples of their size: none lies in two windows
    const int pg = page_of(key), id = __shfl_sync(0xFFFFFFFFu, pages, (pg - base) & 31);
    return wanted && key < end_key && id >= 0 && id < a.pool.n_pages ? id * a.pool.page_bytes + (key - pg * a.pool.page) * a.pool.token_bytes + head : -1;
  }
  __device__ __forceinline__ void copy(int stage) {
    const u32 to = ring + stage * R::STAGE;
    const int key0 = at.first_key(line), skip = begin_key - key0, rest = end_key - key0, c = lane % PIECES;
    u32 there;
    if (a.pool.page % 8 == 0) {                // eight keys in one page: lane b has the place of the b-th eight
      const long long p = place(key0 + 8 * (lane & 3), lane < KEYS / 8 && 8 * lane + 8 > skip);
      there = 0;
#pragma unroll
      for (int b = 0; b < KEYS / 8; ++b) {
        const long long block = __shfl_sync(0xFFFFFFFFu, p, b);
        there |= block >= 0 ? 0xFFu << (8 * b) : 0u;
#pragma unroll
        for (int i = 0; i < 8 / AT_ONCE; ++i) {
          const int r = b * 8 + i * AT_ONCE + lane / PIECES;
          const bool ok = block >= 0 && r < rest && r >= skip;
          const long long from = ok ? block + i * AT_ONCE * a.pool.token_bytes + mine : 0;
          copy16(to + piece<T, HD>(r, c), a.pool.k + from, ok);
          copy16(to + R::HALF + piece<T, HD>(r, c), a.pool.v + from, ok);
        }
      }
      if (rest < 32) there &= (1u << rest) - 1;
      if (skip > 0) there &= ~((1u << skip) - 1);
    } else {                                   // lane i has the place of key i
      const long long p = place(key0 + lane, lane < KEYS && lane >= skip);
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
      if (at.s >= line.seqs) return;           // the line's end
      shift();
      item_begins();
    } else if ((long long)at.first_key(line) >= ((long long)base + 32) * a.pool.page) {
      shift();
    }
  }
  __device__ __forceinline__ void shift() {
    base = ahead_base;
    pages = ahead_pages;
    if (ahead.s < line.seqs) window_behind();
  }
};

template <typename T, int HD> constexpr int smem_bytes(int batch) {
  return kWarps * Ring<T, HD>::BYTES + kWarps * Ring<T, HD>::STAGES * 4 + kWarps * 4 + (2 * (batch + 1) + 1) * 4;
}
__device__ __forceinline__ u32 below(int n) { return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1; }

// Of a tile that some rows see less of than others: whether one of the values that not all rows see (bits of `partly`) is not finite.
template <typename T, int HD> __device__ __forceinline__ bool not_finite(u32 values, u32 partly, int lane) {
  constexpr int PIECES = Ring<T, HD>::ROW / 16;
  bool bad = false;
  for (int i = lane; i < Form<T, HD>::KEYS * PIECES; i += 32) {
    if (!((partly >> (i / PIECES)) & 1)) continue;
    const float4 v = lds4(values + piece<T, HD>(i / PIECES, i % PIECES));
    const u32 w[4] = {__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= (w[e] & 0x7F800000u) == 0x7F800000u || (sizeof(T) == 2 && (w[e] & 0x7F80u) == 0x7F80u);
  }
  return __any_sync(0xFFFFFFFFu, bad);
}
template <typename T, int HD> __device__ __forceinline__ void zero_values(u32 values, int from, int lane) {
  constexpr int PIECES = Ring<T, HD>::ROW / 16;
  for (int i = from * PIECES + lane; i < Form<T, HD>::KEYS * PIECES; i += 32)
    sts4(values + piece<T, HD>(i / PIECES, i % PIECES), make_float4(0.f, 0.f, 0.f, 0.f));
  __syncwarp();
}

enum { kHead = 1, kEnd = 2, kThrough = 4 };    // a part of an item from in front of a stretch that ends in it; of one that runs on behind it; from in front too

template <typename T, int HD, int H>
__global__ void __launch_bounds__(kThreads, 1)
prefix_lane_kernel(PrefixArgs a, bool prefix) {        // prefix false: the kernel in front sums over the prefix
  using R = Ring<T, HD>;
  constexpr int S = R::STAGES, KEYS = Form<T, HD>::KEYS;
  static_assert(H * (HD + 2) * 4 <= R::BYTES, "a warp's last part takes its ring's place");
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int left[kWarps];                 // kHead, kEnd, kThrough
  __shared__ Place<KEYS> left_item[kWarps];    // place of the part that runs on (tile: its last)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, cta = blockIdx.x;
  unsigned char *rest_smem = smem + kWarps * R::BYTES;
  u32 *masks = reinterpret_cast<u32 *>(rest_smem) + warp * S;
  int *warp_sum = reinterpret_cast<int *>(rest_smem) + kWarps * S, *before = warp_sum + kWarps, *ends = before + a.batch + 2;
  // behind the call's own kernel, which began when all kernels in front of it were complete, the start need not wait
  if (prefix) chain_wait();
  chain_next();
  if (prefix && cta == 0 && threadIdx.x == 0) *a.status = 0;
  const Line line = make_line<KEYS>(a, prefix, before, ends, warp_sum);
  Lens lens;
  lens.read(a);
  const int cta_floats = a.chunk * (HD + 2);
  const size_t own = (size_t)a.rows * a.nq;    // rows of `first` in front of the own keys' parts

  const int s0 = line.first(cta), n_warps = line.first(cta + 1) - s0, me = s0 + warp;
  int left_here = 0;
  if (warp < n_warps) {
    const long long from = me * line.per, n = min(line.per, line.total - from);
    typename TileOf<T, HD, H>::type t;
    t.lane = lane;
    Place<KEYS> at;
    at.find(line, from);
    Feeder<T, HD> feed = {a, line, (u32)__cvta_generic_to_shared(smem) + warp * R::BYTES, masks, lane};
    feed.begin(at);
    int stage = 0, fill = 0, first = at.tile;
#pragma unroll 1
    for (; fill < S - 1; ++fill) {             // (not unrolled: short calls wait for their instructions)
      if (fill < n) feed.copy(fill);
      copies_end();
    }
    Queries qs;
    int lim[2], least;                         // positions that the lane's rows see (rows that are none: all); all rows
    auto begin = [&] {
      qs.of(a, at, line.nkv);
      const int sees = at.s > 0 ? seen_by(a, lens, at.s - 1, rows_of(a, at.s - 1)).first : line.prefix;
      const T *q[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int i = (lane >> 2) + 8 * y;
        const bool real = y < H / 8 && i < qs.n;
        q[y] = real ? static_cast<const T *>(a.q) + qs.at(a, i) * HD : nullptr;
        lim[y] = real && at.s > 0 ? sees + (qs.v0 + i) / a.group : kAll;
      }
      least = __reduce_min_sync(0xFFFFFFFFu, min(lim[0], lim[1]));
      t.begin(q[0], q[1]);
    };
    begin();
    for (long long i = 0; i < n; ++i) {
      copies_wait<S - 2>();
      __syncwarp();
      if (i + S - 1 < n) feed.copy(fill);
      copies_end();
      if (++fill == S) fill = 0;
      const int key0 = at.first_key(line);
      const u32 there = masks[stage], where = feed.ring + stage * R::STAGE;
      u32 th[2] = {there, there};
      int longest[2] = {-1, -1};
      bool in_turn = false;
      if (key0 + KEYS > least) {
        th[0] &= below(lim[0] - key0);         // (rows that are none see all)
        th[1] &= below(lim[1] - key0);
        const u32 partly = there & ~__reduce_and_sync(0xFFFFFFFFu, th[0] & th[1]);
        // A weight of 0 times a value that is not finite would be NaN in a row that does not see it.  Where there is one, rows go one limit
        // after the other, the longest first, with the values behind it made zeros, and the other rows' sums are put back.
        in_turn = partly && not_finite<T, HD>(where + R::HALF, partly, lane);
      }
      if (!in_turn) {
        t.tile(a.scale, where, th[0], th[1]);
      } else {
        volatile float old[decltype(t)::SUMS];                         // (in local memory: hardly ever used)
#pragma unroll
        for (int y = 0; y < 2; ++y) longest[y] = lim[y] == kAll ? -1 : min(max(lim[y] - key0, 0), KEYS);
        for (;;) {
          const int most = __reduce_max_sync(0xFFFFFFFFu, max(longest[0], longest[1]));
          if (most < 0) break;
          zero_values<T, HD>(where + R::HALF, most, lane);
          t.save(old);
          t.tile(a.scale, where, longest[0] == most ? th[0] : 0u, longest[1] == most ? th[1] : 0u);
          t.restore(old, longest[0] != most, longest[1] != most);
#pragma unroll
          for (int y = 0; y < 2; ++y)
            if (longest[y] == most) longest[y] = -1;
        }
      }
      if (++stage == S) stage = 0;
      const bool last = at.tile + 1 == at.tiles;
      if (last || i + 1 == n) {
        if (!last) {
          left_here |= kEnd | (first > 0 ? kThrough : 0);
          if (lane == 0) left_item[warp] = at;
          __syncwarp();                        // all lanes are done with the ring
          t.end(nullptr, reinterpret_cast<float *>(smem + warp * R::BYTES), a.chunk, qs.n);
        } else if (first > 0) {                // (its ring is in use: to the warp's place in memory, read by the CTA below)
          left_here |= kHead;
          t.end(nullptr, a.rest + (size_t)(kGrid + me) * cta_floats, a.chunk, qs.n);
        } else {
          t.total();
          t.rows([&](int row, int col, float2 v) {
            if (row < qs.n) *reinterpret_cast<float2 *>(a.first + ((at.s > 0 ? own : 0) + qs.at(a, row)) * HD + col) = v;
          });
          t.stats([&](int row, float m, float l) {
            if (row >= qs.n) return;
            const size_t to = (at.s > 0 ? own : 0) + qs.at(a, row);
            a.first_ml[to] = make_float2(m, l);
            a.more[to] = make_int4(0, 0, 0, 0);
          });
        }
      }
      if (i + 1 < n) {
        at.next(line);
        if (last) { first = 0; begin(); }
      }
    }
  }
  if (lane == 0) left[warp] = left_here;
  __syncthreads();

  // Runs of parts of one item: from the first warp, if it begins inside of an item (run 0), or one whose part begins there and runs on,
  // to the warp that ends it, or to the CTA's last.
  u32 heads_of = 0, stops = 0, through = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    heads_of |= (left[w] & kHead) ? 1u << w : 0u;
    stops |= (left[w] & kEnd) ? 1u << w : 0u;
    through |= (left[w] & kThrough) ? 1u << w : 0u;
  }
  u32 runs = (stops & ~through) << 1 | ((heads_of | through) & 1u);    // bit 0: run 0, bit w + 1: from warp w
  // a run for each warp, or for two, four or all of them where there are few
  const int n_runs = __popc(runs), share = n_runs == 1 ? kWarps : n_runs == 2 ? kWarps / 2 : n_runs <= 4 ? kWarps / 4 : 1;
  const int thread = threadIdx.x % (share * 32);
  for (int r = 0; runs; ++r, runs &= runs - 1) {
    if (r % (kWarps / share) != warp / share) continue;
    const int run = __ffs(runs) - 1, w0 = max(run - 1, 0);
    const u32 behind = heads_of & ~(run == 0 ? 0u : (2u << w0) - 1);   // warps that may end it
    const bool ended = behind != 0;
    const int w1 = ended ? __ffs(behind) - 1 : n_warps - 1;
    Queries qs = {0, 0, a.chunk, 0};
    size_t to_seq = 0;
    int more = 0;                              // CTAs behind this one that have a part of the item
    if (run > 0) {
      const Place<KEYS> it = left_item[w0];
      qs.of(a, it, line.nkv);
      to_seq = it.s > 0 ? own : 0;
      // the item's last tile: the warp's last tile is tile it.tile of it.tiles
      if (!ended) more = line.cta_of((long long)(s0 + w0 + 1) * line.per - 1 + (it.tiles - 1 - it.tile)) - cta;
    }
    float *to = a.rest + (size_t)cta * cta_floats;
    for (int i = thread * 4; i < qs.n * HD; i += share * 128) {
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
          const float *p = ended && w == w1 ? a.rest + (size_t)(kGrid + s0 + w) * cta_floats : reinterpret_cast<const float *>(smem + w * R::BYTES);
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
      if (run > 0) {
        const size_t row = to_seq + qs.at(a, g);
        store4(a.first + row * HD + i % HD, sum);
        if (i % HD == 0) {
          a.first_ml[row] = make_float2(m, l);
          a.more[row] = make_int4((cta + 1) * cta_floats + g * HD, (cta + 1) * cta_floats + stat, cta_floats, more);
        }
      } else {
        *reinterpret_cast<float2 *>(to + i) = make_float2(sum.x, sum.y);
        *reinterpret_cast<float2 *>(to + i + 2) = make_float2(sum.z, sum.w);
        if (i % HD == 0) *reinterpret_cast<float2 *>(to + stat) = make_float2(m, l);
      }
    }
  }
  if (!prefix) chain_wait();                   // the join waits for this kernel alone
}

// Adds a row and head's parts: those over the prefix, then those over the own keys.  A warp each, or, of few rows, eight warps each, which
// take the parts in turn.  Bound by the trips to memory that depend on one another, so all that can be asked for without an answer is asked
// for at once: first the lists, where the parts are, and the two first parts; then the others (rows and statistics), eight at a time.
constexpr int kJoinWarps = 8, kAtOnce = 8;
template <typename T, int HD, int W>
__global__ void __launch_bounds__(kJoinWarps * 32)
prefix_join_kernel(PrefixArgs a) {
  constexpr int COLS = HD / 32;
  struct alignas(COLS * 4) Cols { float v[COLS]; };
  __shared__ float sh_o[W > 1 ? kJoinWarps : 1][HD], sh_m[kJoinWarps], sh_l[kJoinWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, w = W > 1 ? warp : 0;
  const size_t at0 = W > 1 ? blockIdx.x : (size_t)blockIdx.x * kJoinWarps + warp, own = (size_t)a.rows * a.nq;
  chain_wait();
  chain_next();
  if (at0 >= own) return;                      // (W == 1: the warps are for themselves)
  const int row = (int)(at0 / a.nq);
  T *out = static_cast<T *>(a.out) + at0 * HD + lane * COLS;
  const int gave_up = *a.status;               // (final: both kernels in front are complete)
  const int4 more0 = a.more[at0], more1 = a.more[own + at0];           // (of parts that are not there: anything, and not used)
  const float2 ml0 = a.first_ml[at0], ml1 = a.first_ml[own + at0];
  const Cols o0 = *reinterpret_cast<const Cols *>(a.first + at0 * HD + lane * COLS), o1 = *reinterpret_cast<const Cols *>(a.first + (own + at0) * HD + lane * COLS);
  Lens lens;
  lens.read(a);
  const int b = seq_of(a, row);
  auto write = [&](const Cols &y) {
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
      if constexpr (sizeof(T) == 4) out[c] = y.v[c];
      else out[c] = __float2bfloat16_rn(y.v[c]);
    }
  };
  Cols sum = {};
  if (b < 0 || b >= a.batch) {
    if (a.zeros && w == 0) write(sum);
    return;
  }
  if (gave_up) {                               // parts may be missing, and where they would be may be anything
#pragma unroll
    for (int c = 0; c < COLS; ++c) sum.v[c] = NAN;
    if (w == 0) write(sum);
    return;
  }
  const Seen sees = seen_by(a, lens, b, rows_of(a, b));
  const bool has0 = sees.first >= 0 && lens.prefix > 0, has1 = sees.end > lens.prefix;
  float m = -INFINITY, l = 0.f;
  auto take = [&](float2 ml, const Cols &o) {  // one more part
    const float n = fmaxf(m, ml.x), ref = n > -INFINITY ? n : 0.f, f = ex2(m - ref), g = ex2(ml.x - ref);
    l = fmaf(l, f, ml.y * g);
#pragma unroll
    for (int c = 0; c < COLS; ++c) sum.v[c] = fmaf(sum.v[c], f, o.v[c] * g);
    m = n;
  };
  if (w == 0) {
    if (has0) take(ml0, o0);
    if (has1) take(ml1, o1);
  }
#pragma unroll 1
  for (int x = 0; x < 2; ++x) {
    const int4 more = x == 0 ? more0 : more1;
    const int n = (x == 0 ? has0 : has1) ? min(more.w, kGrid) : 0;
#pragma unroll 1
    for (int p0 = w; p0 < n; p0 += kAtOnce * W) {
      const int p = p0 + lane * W;             // the lane's part's statistics
      const float2 ml = lane < kAtOnce && p < n ? *reinterpret_cast<const float2 *>(a.rest + more.y + (size_t)p * more.z) : make_float2(-INFINITY, 0.f);
      Cols o[kAtOnce];
      const float *from = a.rest + more.x + (size_t)p0 * more.z + lane * COLS;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k, from += W * more.z) {
        o[k] = Cols{};
        if (p0 + k * W < n) o[k] = *reinterpret_cast<const Cols *>(from);
      }
      float top = ml.x;
      for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
      const float next = fmaxf(m, top), ref = next > -INFINITY ? next : 0.f, f = ex2(m - ref), g = ex2(ml.x - ref);
      float more_l = ml.y * g;
      for (int d = 16; d > 0; d >>= 1) more_l += __shfl_xor_sync(0xFFFFFFFFu, more_l, d);
      l = fmaf(l, f, more_l);
#pragma unroll
      for (int c = 0; c < COLS; ++c) sum.v[c] *= f;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const float gk = __shfl_sync(0xFFFFFFFFu, g, k);
#pragma unroll
        for (int c = 0; c < COLS; ++c) sum.v[c] = fmaf(o[k].v[c], gk, sum.v[c]);
      }
      m = next;
    }
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int c = 0; c < COLS; ++c) sh_o[warp][lane * COLS + c] = sum.v[c];
    if (lane == 0) { sh_m[warp] = m; sh_l[warp] = l; }
    __syncthreads();
    if (warp > 0) return;
    for (int k = 1; k < W; ++k) {
      Cols o;
#pragma unroll
      for (int c = 0; c < COLS; ++c) o.v[c] = sh_o[k][lane * COLS + c];
      take(make_float2(sh_m[k], sh_l[k]), o);
    }
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int c = 0; c < COLS; ++c) sum.v[c] *= inv;
  write(sum);
}

template <typename T, int HD, int H> int run(const PrefixArgs &a, bool tc, cudaStream_t s) {
  static std::atomic<u64> done{0};
  const int status = hsd_smem_limit((const void *)prefix_lane_kernel<T, HD, H>, smem_bytes<T, HD>(kMaxBatch), done);
  if (status) return status;
  HSD_CUDA_OK(hsd_launch(prefix_lane_kernel<T, HD, H>, dim3(kGrid), kThreads, smem_bytes<T, HD>(a.batch), s, 0, true, a, !tc));
  // eight warps a row and head while that leaves one CTA an SM at most
  const int outputs = a.rows * a.nq;
  if (outputs <= 2 * kGrid) HSD_CUDA_OK(hsd_launch(prefix_join_kernel<T, HD, kJoinWarps>, dim3(outputs), kJoinWarps * 32, 0, s, 0, true, a));
  else HSD_CUDA_OK(hsd_launch(prefix_join_kernel<T, HD, 1>, dim3(ceil_div(outputs, kJoinWarps)), kJoinWarps * 32, 0, s, 0, true, a));
  hsd_count_launches(2);
  return hsd_launch_status();
}
template <typename T, int HD> int run_chunk(PrefixArgs &a, bool tc, cudaStream_t s) {
  // queries of an item: eight, or sixteen where a sequence's rows have more
  const long long per_seq = (long long)ceil_div(a.rows, a.batch) * a.group;
  if constexpr (sizeof(T) == 2) if (per_seq > 8) { a.chunk = 16; return run<T, HD, 16>(a, tc, s); }
  a.chunk = 8;
  return run<T, HD, 8>(a, tc, s);
}
template <typename T> int run_hd(PrefixArgs &a, int hd, bool tc, cudaStream_t s) {
  return hd == 32 ? run_chunk<T, 32>(a, tc, s) : hd == 64 ? run_chunk<T, 64>(a, tc, s) : run_chunk<T, 128>(a, tc, s);
}

size_t align16(size_t n) { return (n + 15) / 16 * 16; }
struct Layout { size_t first, first_ml, more, rest, total; int tc_rest; };   // the status word in front
Layout layout(int rows, int n_q_heads, int hd) {
  const size_t n = 2 * (size_t)rows * n_q_heads;
  Layout l;
  l.first = 256;
  l.first_ml = l.first + n * hd * 4;
  l.more = align16(l.first_ml + n * 8);
  l.rest = (l.more + n * 16 + 255) / 256 * 256;
  l.tc_rest = kGrid * (kWarps + 1) * kMostChunk * (hd + 2);
  l.total = l.rest + ((size_t)l.tc_rest + prefix_tc_floats(hd)) * 4;
  return l;
}

}  // namespace
}  // namespace hsd

extern "C" size_t hsd_prefix_attention_workspace_bytes(int rows, int n_q_heads, int n_kv_heads, int head_dim) {
  if (rows <= 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || n_q_heads > 65536 || (long long)rows * n_q_heads > (1 << 26)) return 0;
  if (head_dim != 32 && head_dim != 64 && head_dim != 128) return 0;
  return hsd::layout(rows, n_q_heads, head_dim).total;
}

extern "C" int hsd_prefix_attention(const void *q, int rows, int n_q_heads, int n_kv_heads, int head_dim, const hsd_kv_pool *pool,
                                    const int32_t *page_table, int pages_per_seq, const int32_t *kv_lens, const int32_t *row_starts, int batch,
                                    const int32_t *prefix_pages, int n_prefix_pages, const int32_t *prefix_len, float scale, void *workspace,
                                    size_t workspace_bytes, int zeros, void *out, void *stream) {
  using namespace hsd;
  if (!q || !page_table || !kv_lens || !prefix_pages || !prefix_len || !out || !workspace || rows <= 0 || batch <= 0 || n_prefix_pages <= 0) return HSD_E_INVALID_ARG;
  if (n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || (!row_starts && rows != batch)) return HSD_E_INVALID_ARG;
  const float scale2 = scale * 1.4426950408889634f;
  if (!isfinite(scale2) || !words(page_table, kv_lens, row_starts) || !words(prefix_pages, prefix_len)) return HSD_E_INVALID_ARG;
  PrefixArgs a = {};
  const int status = pool_view(pool, n_kv_heads, head_dim, pages_per_seq, a.pool);
  if (status) return status;
  // tiles of 8 keys and sets of 8 queries, of all sequences and the prefix: below 2^31
  const long long room = (long long)pages_per_seq * pool->page_size, prefix_room = (long long)n_prefix_pages * pool->page_size, group = n_q_heads / n_kv_heads;
  if (batch > kMaxBatch || n_q_heads > 65536 || (long long)rows * n_q_heads > (1 << 26) || prefix_room > 0x7FFFFF00ll) return HSD_E_TOO_LARGE;
  const long long sets = rows * group / 8 + batch + 1;
  if ((sets * ((room > prefix_room ? room : prefix_room) / 8 + 2)) >> 31) return HSD_E_TOO_LARGE;
  if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) || (reinterpret_cast<uintptr_t>(workspace) & 255)) return HSD_E_INVALID_ARG;
  if (workspace_bytes < hsd_prefix_attention_workspace_bytes(rows, n_q_heads, n_kv_heads, head_dim)) return HSD_E_WORKSPACE_TOO_SMALL;
  const Layout l = layout(rows, n_q_heads, head_dim);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  a.q = q; a.out = out; a.page_table = page_table; a.kv_lens = kv_lens; a.prefix_pages = prefix_pages; a.prefix_len = prefix_len; a.row_starts = row_starts;
  a.status = reinterpret_cast<int *>(ws);
  a.first = reinterpret_cast<float *>(ws + l.first);
  a.first_ml = reinterpret_cast<float2 *>(ws + l.first_ml);
  a.more = reinterpret_cast<int4 *>(ws + l.more);
  a.rest = reinterpret_cast<float *>(ws + l.rest);
  a.scale = scale2;
  a.rows = rows; a.batch = batch; a.nq = n_q_heads; a.nkv = n_kv_heads; a.pages_per_seq = pages_per_seq; a.prefix_pages_n = n_prefix_pages;
  a.group = (int)group;
  a.zeros = zeros != 0;
  a.page_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (pool->page_size == 1 << i) a.page_shift = i;
  a.tc_rest = l.tc_rest;
  cudaStream_t s = (cudaStream_t)stream;
  bool tc = false;
  if (prefix_tc_takes(a, pool->dtype, head_dim)) {
    int launched = HSD_OK;
    tc = launch_prefix_tc(a, head_dim, s, launched);
    if (launched) return launched;
  }
  return pool->dtype == HSD_F32 ? run_hd<float>(a, head_dim, tc, s) : run_hd<__nv_bfloat16>(a, head_dim, tc, s);
}
