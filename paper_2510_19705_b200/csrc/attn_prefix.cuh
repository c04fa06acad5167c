// Arguments of the kernels of hsd_prefix_attention, and the tensor-memory one's launch (attn_prefix_tc.cu).
#pragma once
#include "paged.cuh"

namespace hsd {

constexpr int kPrefixGrid = kMeasuredSMs;            // CTAs at most: fixed, as the workspace's size depends on it
struct PrefixArgs {
  const void *q;
  void *out;
  const int32_t *page_table, *kv_lens, *prefix_pages, *prefix_len, *row_starts;
  float *first;                                // sums of each part [2][rows][heads][HD]: over the prefix, over own keys, of the CTA that begins the item
  float2 *first_ml;                            // their m and l
  int4 *more;                                  // where the parts of the CTAs behind it are: o's and ml's float in `rest`, floats between two CTAs, how many
  float *rest;                                 // per CTA: a part of an item that begins in front of it, rows and their m and l
  int tc_rest;                                 // float of `rest` where the tensor-memory kernel's parts begin
  PoolView pool;
  float scale;                                 // times log2(e)
  int rows, batch, nq, nkv, pages_per_seq, prefix_pages_n, page_shift;   // log2 of the page size, or -1
  int group, chunk;                            // query heads of a key head; queries of an item at most
  bool zeros;                                  // rows without a sequence become zeros
  int *status;                                 // set if a bounded wait gave up
};

// What the device's lists say, within what there is room for.
struct Lens {
  int prefix, room;                            // keys of the prefix; positions that a sequence's pages have room for
  __device__ __forceinline__ void read(const PrefixArgs &a) {
    prefix = (int)min((long long)max(*a.prefix_len, 0), (long long)a.prefix_pages_n * a.pool.page);
    room = (int)((long long)a.pages_per_seq * a.pool.page);
  }
  __device__ __forceinline__ int of(const PrefixArgs &a, int b) const { return min(max(a.kv_lens[b], 0), max(room, prefix)); }
};

// Sums over the prefix on tensor memory: whether it takes the call, floats of `rest` that it needs behind `tc_rest`, and its launch (false: the
// pools' strides have no tensor map; nothing was launched).
bool prefix_tc_takes(const PrefixArgs &a, int dtype, int hd);
size_t prefix_tc_floats(int hd);
bool launch_prefix_tc(const PrefixArgs &a, int hd, cudaStream_t s, int &status);

}  // namespace hsd
