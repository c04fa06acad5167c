// Sums over a shared prefix for all rows of a batch, on tcgen05 with scores, weights and outputs in tensor memory (hsd_prefix_attention).
//
// An item is one key head and up to 2 x 128 queries (rows times the head's group, tiles A and B) over all keys of the prefix, in tiles of
// 64 keys; the items' tiles stand in one line, which is divided evenly over a CTA an SM, whatever the prefix's length is (it is read on the
// device).  Per key tile and query tile
//   S[128 x 64]   = Q K^T                      both operands in shared memory
//   P             = exp2(S c - m), thread = query, as three bf16 parts, all of its 24 bits: the high and middle ones overwrite S, the low ones go
//                   to shared memory (tensor memory is full at heads of 128)
//   T[128 x hd]   = P_lo V + P_mid V + P_hi V  fresh sums of this tile alone; V as it lies in the cache (MN-major)
//   O             = O f + T                    in fp32, in the softmax warps' registers
// The tensor cores' adders cut off: a chain of products loses up to 2^-23 of its sum a product.  So no chain is longer than a tile, and its small
// products come first.  With weights of 16 bits and chains of up to 2048 keys 64 x 8192 rows and keys took 54 us instead of 59, 100 x 40000 134 instead of 181, but
// 2.2e-3 and more of the bf16 outputs were not the nearest, against 1.1e-3 of the formula in fp32; now 0.35e-3.  (Three parts and chains of 512 keys,
// added in the workspace: 56 and 177 us, 1.0e-3.)
// Bound by the softmax warps and the way weights -> products -> sums -> next weights: at 100 x 40000 the tensor pipe is busy for 53 % of the time.
// The scores of 32 of a tile's 64 keys stay in registers from the maximum on, the others are read twice: registers hold O (16 more kept: 3 %
// slower, they spill).  What did not help: sixteen softmax warps, two a row (a barrier that has no limit); a quarter of the exponentials on the FMA
// pipe; the two query tiles' exponentials in turn; the next scores in front of the low parts' products; parts cut off instead of rounded.
// One issuing warp for both query tiles was a quarter slower.
// A short call waits for its instructions, first keys and the parts' way to memory.
// Two query tiles share every K and V tile; S has two buffers, so that the scores of the next key tile are ready when the weights of this one
// are.  m moves only when a row's maximum has passed it by 8; then O is rescaled.
// 384 threads: warps 0-3 / 4-7 = softmax of tile A / B, warp 8 = loader (TMA out of the pages, a lane a piece of a page; keys a tile in front of
// values), warps 9 / 10 = MMA issue of tile A / B, warp 11 none.  Every wait is bounded, and no waiter can be passed by (a parity wait sees a completion
// only until the next one) or come so late that it takes the one before the last for its own: k_full and v_full have their next loads behind k_free / v_free,
// which both issuers complete, in a piece without its query tile too, where an issuer waits for every key tile and lets it go; those their next MMAs behind
// the loader's tiles; s_full and pv_done theirs behind p_ready of the tile's four softmax warps, each of which waits for every tile's; q_ready its
// next queries behind q_free, which the commit behind a piece's last scores completes; p_ready its next weights behind the scores.  T is read before
// p_ready of the tile behind it; the low parts' buffer is free when the scores that use its buffer of S are there, as these are issued behind its products.
// Registers move once, right at the start, from the last four warps to the others; that wait ends as all four let theirs go without a condition.
#include <algorithm>
#include <type_traits>
#include "attn_prefix.cuh"
#include "gemm_tc.cuh"
#include "tc_ptx.cuh"

namespace hsd {
namespace {

using namespace ptx;

constexpr int kThreads = 384, kLoaderWarp = 8, kMmaWarp = 9;             // (two MMA warps, and one that fills up their warpgroup)
// Registers of a thread: at the launch, then of the softmax warps, which hold their rows' sums, and of the others.
constexpr int kRegs = 168, kRegsSoftmax = 224, kRegsOther = 56;
static_assert(256 * kRegsSoftmax + 128 * kRegsOther <= kThreads * kRegs, "registers come from the block's own");
constexpr int TK = 64, kSet = 256;                       // keys of a tile; queries of an item at most
constexpr int kQBlk = 128 * 128, kBlk = TK * 128;        // [128 queries][64 bf16] and [64 keys][64 bf16] blocks, 128-byte swizzle
constexpr int kMasks = 8;                                // (a mask outlives its keys' stage by two tiles at most)
constexpr int kLow = 128 * TK * 2;                       // the weights' low parts of a query tile, 128-byte swizzle

template <int HD> struct Cfg {
  static constexpr int NB = HD / 64;                     // 64-column blocks
  static constexpr int kStages = HD == 64 ? 4 : 3;
  static constexpr int kQTile = NB * kQBlk, kTile = NB * kBlk;
  static constexpr int kOffK = 2 * kQTile, kOffV = kOffK + kStages * kTile, kOffLow = kOffV + kStages * kTile, kOffMask = kOffLow + 4 * kLow;
  static constexpr int kOffBar = kOffMask + kMasks * 8, kSmem = kOffBar + 384 + 1024;
  static_assert(kSmem + 16 <= 232448, "a block's shared memory");
};
struct TcArgs {
  CUtensorMap k, v, q;
  PrefixArgs p;
  int box;                                               // tokens of a copy of keys
  int sets, per_set, per_tile;                           // items of a key head; rows (tokens) of each; of a query tile at most
};

constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo_k(uint32_t addr) { return ((addr & 0x3FFFFu) >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_lo_mn(uint32_t addr) { return ((addr & 0x3FFFFu) >> 4) | ((uint32_t)(kBlk >> 4) << 16); }
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(acc), "r"(kDescHi) : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tmov.b64 db, {%2, %5};\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(acc), "r"(kDescHi) : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ void tmem_st8u(uint32_t taddr, const unsigned *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}

// What a CTA has of the line: pieces of items, one after the other.
struct Pieces {
  int at, to, tiles, per, sets;                          // tiles of the line; of an item; of a CTA; items of a key head
  int head, set, t0, n;                                  // the piece: its item, first tile, tiles
  int item;
  __device__ __forceinline__ Pieces(const TcArgs &a, int prefix) {
    tiles = (prefix + TK - 1) / TK;
    sets = a.sets;
    const int total = tiles * sets * a.p.nkv;
    per = max((total + (int)gridDim.x - 1) / (int)gridDim.x, 1);
    at = min((int)blockIdx.x * per, total);
    to = min(at + per, total);
    n = 0;
  }
  __device__ __forceinline__ bool next() {
    at += n;
    if (at >= to) return false;
    item = at / tiles;
    head = item / sets;
    set = item - head * sets;
    t0 = at - item * tiles;
    n = min(tiles - t0, to - at);
    return true;
  }
  __device__ __forceinline__ int ctas_behind() const {   // that have a part of the piece's item
    return ((item + 1) * tiles - 1) / per - (int)blockIdx.x;
  }
};

template <int HD>
__global__ void __launch_bounds__(kThreads, 1) prefix_tc_kernel(const __grid_constant__ TcArgs a) {
  using C = Cfg<HD>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ uint32_t tmem_slot;
  __shared__ int sh_abort;
  volatile int *abort_flag = &sh_abort;
  const uint32_t s0 = smem_u32(smem), b0 = s0 + C::kOffBar;
  volatile uint64_t *masks = reinterpret_cast<volatile uint64_t *>(smem + C::kOffMask);
  constexpr int kStages = C::kStages;
  auto k_full = [&](int b) { return b0 + 8u * b; };
  auto k_free = [&](int b) { return b0 + 8u * (4 + b); };
  auto v_full = [&](int b) { return b0 + 8u * (8 + b); };
  auto v_free = [&](int b) { return b0 + 8u * (12 + b); };
  auto s_full = [&](int x, int b) { return b0 + 8u * (16 + 2 * x + b); };
  auto p_ready = [&](int x, int b) { return b0 + 8u * (20 + 2 * x + b); };
  auto pv_done = [&](int x) { return b0 + 8u * (24 + x); };
  auto q_ready = [&](int x) { return b0 + 8u * (26 + x); };
  auto q_free = [&](int x) { return b0 + 8u * (28 + x); };           // a piece's last scores
  const uint32_t v_land = b0 + 8u * 30;
  const int warp = warp_index(), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int b = 0; b < kStages; ++b) { mbar_init(k_full(b), 1); mbar_init(k_free(b), 2); mbar_init(v_full(b), 1); mbar_init(v_free(b), 2); }
    for (int x = 0; x < 2; ++x) {
      mbar_init(s_full(x, 0), 1); mbar_init(s_full(x, 1), 1); mbar_init(p_ready(x, 0), 4); mbar_init(p_ready(x, 1), 4);
      mbar_init(pv_done(x), 1); mbar_init(q_ready(x), 1); mbar_init(q_free(x), 1);
    }
    mbar_init(v_land, 1);
    sh_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) tmem_alloc(smem_u32(&tmem_slot), 512);
  chain_wait();
  chain_next();
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.p.status = 0;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  Lens lens;
  lens.read(a.p);
  auto tS = [&](int x) { return tmem + (uint32_t)(x * 128); };
  auto tO = [&](int x) { return tmem + 256u + (uint32_t)(x * HD); };
  auto low = [&](int x, int b) { return (uint32_t)(C::kOffLow + (2 * x + b) * kLow); };
  Pieces piece(a, lens.prefix);

  if (warp >= kLoaderWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == kLoaderWarp) {
      // ------------------------------------------------------------------ loader: lane i has the i-th piece of a tile's keys
      const int box = a.box, copies = TK / box, page = a.p.pool.page;
      bool ok = true;
      int kt = 0, tails = 0, pieces[2] = {0, 0};                       // tiles, pieces of each query tile so far
      auto wait = [&](uint32_t bar, uint32_t parity) { ok = mbar_wait_warp(bar, parity, abort_flag); return ok; };
      auto page_id = [&](int key) {                                    // n_pages, which reads as zeros, where there is none
        const int id = lane < copies && key < lens.prefix ? a.p.prefix_pages[key / page] : -1;
        return id >= 0 && id < a.p.pool.n_pages ? id : a.p.pool.n_pages;
      };
      while (ok && piece.next()) {
        int key = piece.t0 * TK + lane * box, id = page_id(key);
        const int row0 = piece.set * a.per_set, n_rows = min(a.per_set, a.p.rows - row0);
        for (int x = 0; x < 2 && x * a.per_tile < n_rows && ok; ++x) { // queries, of the whole tile's rows: those behind the last are not used
          if (!wait(q_free(x), (uint32_t)(pieces[x]++ & 1) ^ 1u)) break;
          if (lane == 0) mbar_expect_tx(q_ready(x), (uint32_t)(a.per_tile * a.p.group * 128 * C::NB));
          __syncwarp();
          if (lane < C::NB) tma_load_3d(s0 + x * C::kQTile + lane * kQBlk, &a.q, lane * 64, piece.head * a.p.group, row0 + x * a.per_tile, q_ready(x));
        }
        if (!ok) break;
        int of_v = 0, in_page_v = 0;                                   // the page and place in it of the values that come next
        bool tail_v = false;
        for (int j = 0; j <= piece.n; ++j) {                           // keys a tile in front of the values, whose place becomes free later
          const int of_k = id, in_page = key % page;
          const bool tail = j < piece.n && (piece.t0 + j + 1) * TK > lens.prefix;
          if (j < piece.n) {
            const int b = kt % kStages, k0 = (piece.t0 + j) * TK;
            const uint32_t there = __ballot_sync(0xFFFFFFFFu, id < a.p.pool.n_pages);
            key += TK;
            if (j + 1 < piece.n) id = page_id(key);                    // the next tile's, before the waits
            uint64_t mask = ~0ull;
            if (there != (copies == 32 ? ~0u : (1u << copies) - 1) || tail) {
              mask = 0;
              for (int i = 0; i < copies; ++i)
                if ((there >> i) & 1) mask |= (box == 64 ? ~0ull : (1ull << box) - 1) << (i * box);
              if (tail) mask &= (1ull << (lens.prefix - k0)) - 1;
            }
            if (!wait(k_free(b), (uint32_t)((kt / kStages) & 1) ^ 1u)) break;
            if (lane == 0) {
              masks[kt % kMasks] = mask;
              mbar_expect_tx(k_full(b), C::kTile);
            }
            __syncwarp();
            if (lane < copies) {
#pragma unroll
              for (int i = 0; i < C::NB; ++i)
                tma_load_4d(s0 + C::kOffK + b * C::kTile + i * kBlk + lane * box * 128, &a.k, i * 64, in_page, of_k, piece.head, k_full(b));
            }
            ++kt;
          }
          if (j > 0) {
            const int t = kt - (j < piece.n ? 2 : 1), b = t % kStages;
            if (!wait(v_free(b), (uint32_t)((t / kStages) & 1) ^ 1u)) break;
            const uint32_t lands = tail_v ? v_land : v_full(b);
            if (lane == 0) mbar_expect_tx(lands, C::kTile);
            __syncwarp();
            if (lane < copies) {
#pragma unroll
              for (int i = 0; i < C::NB; ++i)
                tma_load_4d(s0 + C::kOffV + b * C::kTile + i * kBlk + lane * box * 128, &a.v, i * 64, in_page_v, of_v, piece.head, lands);
            }
            if (tail_v) {                                              // values behind the prefix's end must be finite (P is 0 there)
              if (!wait(v_land, (uint32_t)(tails++ & 1))) break;
              const int r0 = lens.prefix - (piece.t0 + j - 1) * TK;
              for (int i = r0 * 8 * C::NB + lane; i < TK * 8 * C::NB; i += 32) {
                const int r = i / (8 * C::NB), c = i % (8 * C::NB);    // whole rows: the swizzle permutes within a row
                *reinterpret_cast<uint4 *>(smem + C::kOffV + b * C::kTile + (c >> 3) * kBlk + r * 128 + ((c & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) mbar_arrive(v_full(b));
            }
          }
          of_v = of_k;
          in_page_v = in_page;
          tail_v = tail;
        }
      }
      if (!ok) {                                                       // copies in flight land before the shared memory goes away
        const unsigned long long t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) {}
      }
    } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
      // ------------------------------------------------------------------ MMA issue of query tile x: a warp each, as an issuing thread stands
      // still while the pipe is full, and its waits and commits would leave the pipe empty
      const int x = warp - kMmaWarp;
      const bool issuer = elect_one();
      const uint32_t id1 = umma_idesc_bf16(TK), id2 = umma_idesc_bf16(HD) | (1u << 16);      // bit 16: B is MN-major
      bool ok = true;
      int kt = 0, st = 0, pieces = 0;                                  // key tiles, the query tile's key tiles and pieces so far
      while (ok && piece.next()) {
        const int n_rows = min(a.per_set, a.p.rows - piece.set * a.per_set), n = piece.n;
        if (x * a.per_tile >= n_rows) {                                // a query tile that there is not lets keys and values go as they come
          for (int j = 0; j < n && ok; ++j, ++kt) {
            const int b = kt % kStages;
            const uint32_t ph = (uint32_t)((kt / kStages) & 1);
            ok = mbar_wait_warp(k_full(b), ph, abort_flag);
            if (ok && lane == 0) mbar_arrive(k_free(b));
            ok = ok && mbar_wait_warp(v_full(b), ph, abort_flag);
            if (ok && lane == 0) mbar_arrive(v_free(b));
          }
          continue;
        }
        auto issue_s = [&](int j) {                                    // (the issuer only)
          const int b = (kt + j) % kStages, c = st + j;
          const uint32_t qb = desc_lo_k(s0 + x * C::kQTile), kb = desc_lo_k(s0 + C::kOffK + b * C::kTile), d = tS(x) + (uint32_t)((c & 1) * TK);
#pragma unroll
          for (int ks = 0; ks < HD / 16; ++ks)
            umma_ss(d, qb + (ks >> 2) * (kQBlk / 16) + (ks & 3) * 2, kb + (ks >> 2) * (kBlk / 16) + (ks & 3) * 2, id1, ks > 0 ? 1u : 0u);
          umma_commit(s_full(x, c & 1));
          umma_commit(k_free(b));
          if (j + 1 == n) umma_commit(q_free(x));
        };
        auto k_wait = [&](int j) { return mbar_wait_warp(k_full((kt + j) % kStages), (uint32_t)(((kt + j) / kStages) & 1), abort_flag); };
        ok = mbar_wait_warp(q_ready(x), (uint32_t)(pieces++ & 1), abort_flag);
        for (int j = 0; j < min(2, n) && ok; ++j) {                    // the first two key tiles' scores
          ok = k_wait(j);
          if (!ok) break;
          tc_fence_after();
          if (issuer) issue_s(j);
        }
        for (int j = 0; j < n && ok; ++j) {
          const int b = (kt + j) % kStages, c = st + j;
          const uint32_t vb = desc_lo_mn(s0 + C::kOffV + b * C::kTile);
          ok = mbar_wait_warp(v_full(b), (uint32_t)(((kt + j) / kStages) & 1), abort_flag);
          if (ok && j + 2 < n) ok = k_wait(j + 2);
          if (ok) ok = mbar_wait_warp(p_ready(x, c & 1), (uint32_t)((c >> 1) & 1), abort_flag);
          if (!ok) break;
          tc_fence_after();
          const uint32_t d = tO(x), p = tS(x) + (uint32_t)((c & 1) * TK);
          const uint32_t lows = desc_lo_k(s0 + low(x, c & 1));
          if (issuer) {                                                // sums of this tile alone, the small products first
#pragma unroll
            for (int ks = 0; ks < TK / 16; ++ks) umma_ss(d, lows + ks * 2, vb + ks * 128, id2, ks > 0 ? 1u : 0u);
#pragma unroll
            for (int ks = 0; ks < TK / 16; ++ks) umma_ts(d, p + ks * 16 + 8, vb + ks * 128, id2, 1u);
#pragma unroll
            for (int ks = 0; ks < TK / 16; ++ks) umma_ts(d, p + ks * 16, vb + ks * 128, id2, 1u);
            umma_commit(pv_done(x));
            umma_commit(v_free(b));
            if (j + 2 < n) issue_s(j + 2);                             // over P(j), after the products that read it
          }
        }
        kt += n;
        st += n;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // ------------------------------------------------------------------ softmax of query tile x: thread = query
    const int x = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lq = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t O = tO(x) + lq;
    const float sc = a.p.scale;
    const size_t cta_floats = (size_t)kSet * (HD + 2);
    bool ok = true;
    int kt = 0, st = 0;                                              // key tiles, this query tile's key tiles so far
    auto wait = [&](uint32_t bar, uint32_t parity) {                 // lane 0 waits, the warp takes one decision
      if (lane == 0) ok = mbar_wait(bar, parity, abort_flag);
      ok = __shfl_sync(0xFFFFFFFFu, ok ? 1 : 0, 0) != 0;
      if (ok) tc_fence_after();
      return ok;
    };
    while (ok && piece.next()) {
      const int row0 = piece.set * a.per_set + x * a.per_tile, n = piece.n;
      const int nq = min(min(a.per_set - x * a.per_tile, a.p.rows - row0), a.per_tile) * a.p.group;        // queries of the tile
      if (nq <= 0) { kt += n; continue; }
      const bool real = row < nq, busy = (warp & 3) * 32 < nq;       // (a warp without queries only keeps up)
      const int tok = row / a.p.group;
      const int at = (row0 + tok) * a.p.nq + piece.head * a.p.group + (row - tok * a.p.group);
      // the part's place: the item's, or the CTA's if the item begins in front of it
      float *const to = piece.t0 == 0 ? a.p.first : a.p.rest + a.p.tc_rest + blockIdx.x * cta_floats;
      const int to_row = piece.t0 == 0 ? at : x * 128 + row, reals = min(nq - (warp & 3) * 32, 32);
      bool next_ready = false;
      float m_ref = -INFINITY, l = 0.f, o[HD];                       // sums of the tiles so far, relative to m_ref
#pragma unroll
      for (int c = 0; c < HD; ++c) o[c] = 0.f;
      auto add = [&](float f) {                                      // a tile's products
        const float2 f2 = make_float2(f, f);
#pragma unroll
        for (int c0 = 0; c0 < HD; c0 += 32) {
          float y[32];
          tmem_ld32(O + (uint32_t)c0, y);
          tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const float2 z = __ffma2_rn(make_float2(y[c], y[c + 1]), f2, make_float2(o[c0 + c], o[c0 + c + 1]));
            o[c0 + c] = z.x;
            o[c0 + c + 1] = z.y;
          }
        }
      };
      for (int j = 0; j < n; ++j, ++kt, ++st) {
        const uint32_t S = tS(x) + lq + (uint32_t)((st & 1) * TK);
        if (!next_ready && !wait(s_full(x, st & 1), (uint32_t)((st >> 1) & 1))) break;
        tc_fence_after();
        next_ready = false;
        float f = 1.f;                                               // to the reference of this tile
        if (busy) {
          const uint64_t mask = masks[kt % kMasks];
          auto absent = [&](float *s, int c0, auto n) {
            if (mask == ~0ull) return;
            const uint32_t m = (uint32_t)(mask >> c0);
#pragma unroll
            for (int c = 0; c < n(); ++c)
              if (!((m >> c) & 1)) s[c] = -INFINITY;
          };
          float mx = -INFINITY, first[32];                           // the last keys first: the first ones' scores stay
#pragma unroll
          for (int c0 = TK - 32; c0 >= 0; c0 -= 32) {
            float top[2] = {-INFINITY, -INFINITY};
            tmem_ld32(S + (uint32_t)c0, first);
            tmem_ld_wait();
            absent(first, c0, std::integral_constant<int, 32>());
#pragma unroll
            for (int c = 0; c < 32; c += 2) top[(c >> 1) & 1] = max3(top[(c >> 1) & 1], first[c], first[c + 1]);
            mx = max3(mx, top[0], top[1]);
          }
          // the reference moves only when a row's maximum has passed it by more than 8 in log2 units
          const bool grow = (mx - m_ref) * sc > 8.f || (m_ref == -INFINITY && mx > -INFINITY);
          if (__any_sync(0xFFFFFFFFu, grow)) {
            const float m_new = grow ? mx : m_ref;
            if (m_ref > -INFINITY) f = ex2((m_ref - m_new) * sc);    // (sums without a key are zeros)
            l *= f;
            m_ref = m_new;
            if (j > 1) {
#pragma unroll
              for (int c = 0; c < HD; ++c) o[c] *= f;
            }
          }
          const float mneg = m_ref > -INFINITY ? -m_ref * sc : 0.f;
          float2 l2a = make_float2(0.f, 0.f), l2b = l2a;
          const float2 sc2 = make_float2(sc, sc), mneg2 = make_float2(mneg, mneg), minus = make_float2(-1.f, -1.f);
          uint8_t *const lows = smem + low(x, st & 1) + row * 128;
          // weights as three bf16 parts, all of their 24 bits: per 16 keys 8 columns of the high ones and 8 of the middle ones over their own
          // scores, the low ones to shared memory
#pragma unroll
          for (int c = 0; c < TK; c += 16) {
            float s[16];
            if (c < 32) {
#pragma unroll
              for (int e = 0; e < 16; ++e) s[e] = first[c + e];
            } else {
              tmem_ld16(S + (uint32_t)c, s);
              tmem_ld_wait();
              absent(s, c, std::integral_constant<int, 16>());
            }
            unsigned part[3][8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float2 t = __ffma2_rn(make_float2(s[2 * e], s[2 * e + 1]), sc2, mneg2);
              float2 p = make_float2(ex2(t.x), ex2(t.y));
              if (e & 1) l2b = __fadd2_rn(l2b, p);
              else l2a = __fadd2_rn(l2a, p);
#pragma unroll
              for (int i = 0; i < 3; ++i) {
                const __nv_bfloat162 w = __floats2bfloat162_rn(p.x, p.y);
                part[i][e] = *reinterpret_cast<const unsigned *>(&w);
                if (i < 2) p = __ffma2_rn(make_float2(__uint_as_float(part[i][e] << 16), __uint_as_float(part[i][e] & 0xFFFF0000u)), minus, p);
              }
            }
            tmem_st8u(S + (uint32_t)c, part[0]);
            tmem_st8u(S + (uint32_t)(c + 8), part[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
              *reinterpret_cast<uint4 *>(lows + (((c / 8 + h) ^ (row & 7)) << 4)) = make_uint4(part[2][4 * h], part[2][4 * h + 1], part[2][4 * h + 2], part[2][4 * h + 3]);
          }
          l += (l2a.x + l2a.y) + (l2b.x + l2b.y);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          // the next tile's scores are there by now, as a rule: looked at here, the answer costs nothing
          if (j + 1 < n) next_ready = mbar_test(s_full(x, (st + 1) & 1), (uint32_t)(((st + 1) >> 1) & 1));
          tmem_st_wait();
          next_ready = __all_sync(0xFFFFFFFFu, next_ready);
        }
        if (j > 0) {                                                 // the tile before: its products ran under these exponentials
          if (!wait(pv_done(x), (uint32_t)((st - 1) & 1))) break;
          if (busy) add(f);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready(x, st & 1));
      }
      if (!ok || !wait(pv_done(x), (uint32_t)((st - 1) & 1))) break;
      if (busy) {
        // To the part's place by way of tensor memory and the warp's rows of low parts that no product reads any more, so that a row's columns are written
        // by neighbouring lanes: 32 columns at a time, 16-byte pieces permuted within a row of 128.
        if (n > 1) {
          add(1.f);
#pragma unroll
          for (int c0 = 0; c0 < HD; c0 += 16) {
            unsigned y[16];
#pragma unroll
            for (int c = 0; c < 16; ++c) y[c] = __float_as_uint(o[c0 + c]);
            tmem_st16u(O + (uint32_t)c0, y);
          }
          tmem_st_wait();
        }
        float4 *const block = reinterpret_cast<float4 *>(smem + low(x, 0) + (warp & 3) * 32 * 128);
#pragma unroll 1
        for (int c0 = 0; c0 < HD; c0 += 32) {
          float y[32];
          tmem_ld32(O + (uint32_t)c0, y);
          tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < 8; ++c) block[lane * 8 + (c ^ (lane & 7))] = make_float4(y[4 * c], y[4 * c + 1], y[4 * c + 2], y[4 * c + 3]);
          __syncwarp();
#pragma unroll
          for (int k = 0; k < 8; ++k) {                              // four rows
            const int i = 4 * k + (lane >> 3);
            float4 *const p = reinterpret_cast<float4 *>(to + __shfl_sync(0xFFFFFFFFu, to_row, i) * (long long)HD + c0) + (lane & 7);
            if (i < reals) *p = block[i * 8 + ((lane & 7) ^ (i & 7))];
          }
          __syncwarp();
        }
      }
      if (real) {
        const float2 ml = make_float2(m_ref > -INFINITY ? m_ref * sc : -INFINITY, l);
        const size_t mine = a.p.tc_rest + blockIdx.x * cta_floats;
        if (piece.t0 == 0) {
          a.p.first_ml[at] = ml;
          a.p.more[at] = make_int4((int)(mine + cta_floats + (size_t)(x * 128 + row) * HD), (int)(mine + cta_floats + (size_t)kSet * HD + 2 * (x * 128 + row)),
                                   (int)cta_floats, piece.ctas_behind());
        } else {
          *reinterpret_cast<float2 *>(a.p.rest + mine + (size_t)kSet * HD + 2 * (x * 128 + row)) = ml;
        }
      }
      tc_fence_before();                                             // (O is read: the next piece's products come behind its weights)
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
  if (threadIdx.x == 0 && *abort_flag) atomicExch(a.p.status, 1);
}

// The split of registers holds for a kernel that is launched with kRegs a thread: with fewer the softmax warps would wait for registers that the
// block does not have.
template <int HD> bool registers_are_there() {
  static std::atomic<int> regs{0};
  if (regs.load(std::memory_order_relaxed) == 0) {
    cudaFuncAttributes at = {};
    if (cudaFuncGetAttributes(&at, (const void *)prefix_tc_kernel<HD>) != cudaSuccess) return false;
    regs.store(at.numRegs, std::memory_order_relaxed);
  }
  return regs.load(std::memory_order_relaxed) == kRegs;
}
template <int HD> int launch_t(const TcArgs &a, cudaStream_t s) {
  static std::atomic<u64> limits{0};
  const int limit = hsd_smem_limit((const void *)prefix_tc_kernel<HD>, Cfg<HD>::kSmem, limits);
  if (limit) return limit;
  HSD_CUDA_OK(hsd_launch(prefix_tc_kernel<HD>, dim3(kPrefixGrid), kThreads, Cfg<HD>::kSmem, s, 0, true, a));
  hsd_count_launches(1);
  return hsd_launch_status();
}

}  // namespace

// Whether the call's sums over the prefix go by this kernel or by the one whose warps take sets of 16 queries, whose start is shorter and which
// reads the prefix again for each set: by queries times keys (as many as the list has room for: the length itself is not known here) times the
// heads' columns.  us of the other / this one, 8 key heads of 128: 32 queries each over 2048 keys 19.5 / 22.2, 4096 28.4 / 25.3, 32768 157 / 66;
// 16 queries over 4096 19.2 / 24.3, 8192 28.8 / 29.6, 32768 84 / 65; 128 over 512 20.0 / 20.6, 1024 31.2 / 22.8.  2 of 64: 64 over 4096 13.3 / 16.3,
// 128 over 4096 19.2 / 17.0, 16 over 32768 18.5 / 23.5, 32 over 32768 28.0 / 23.8.
constexpr long long kEnoughWork = 90000000;
bool prefix_tc_takes(const PrefixArgs &a, int dtype, int hd) {
  const long long queries = (long long)a.rows * a.group, keys = (long long)a.prefix_pages_n * a.pool.page, tiles = (keys + TK - 1) / TK;
  return dtype == HSD_BF16 && (hd == 64 || hd == 128) && a.pool.page % 8 == 0 && a.scale > 0.f && a.group <= 64 && queries >= 16 &&
         queries * a.nkv * hd >= kEnoughWork / keys && (a.rows / (128 / a.group) + 1) * a.nkv * tiles < (1ll << 30);
}
size_t prefix_tc_floats(int hd) { return hd == 32 ? 0 : (size_t)kPrefixGrid * kSet * (hd + 2); }

bool launch_prefix_tc(const PrefixArgs &p, int hd, cudaStream_t s, int &status) {
  if (tc_init() || !(hd == 64 ? registers_are_there<64>() : registers_are_there<128>())) return false;
  TcArgs a;
  a.p = p;
  a.box = 8;
  while (a.box < TK && p.pool.page % (2 * a.box) == 0) a.box *= 2;
  a.per_tile = 128 / p.group;
  a.sets = ceil_div(p.rows, 2 * a.per_tile);
  a.per_set = ceil_div(p.rows, a.sets);
  const PoolView &v = p.pool;
  if (tc_make_map_rows(&a.q, p.q, hd, p.nq, p.rows, p.group, a.per_tile) ||
      tc_make_map_pool(&a.k, v.k, hd, v.page, v.n_pages, p.nkv, v.token_bytes, v.page_bytes, v.head_bytes, a.box) ||
      tc_make_map_pool(&a.v, v.v, hd, v.page, v.n_pages, p.nkv, v.token_bytes, v.page_bytes, v.head_bytes, a.box)) return false;
  status = hd == 64 ? launch_t<64>(a, s) : launch_t<128>(a, s);
  return true;
}

}  // namespace hsd
