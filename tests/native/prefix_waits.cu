// Attention over a shared prefix as tests/test_gpu_operator_waits.py builds it: with a wait limit of a millisecond, and with copies of keys that
// bring half the bytes that their barriers count, so that the waits for them run out.
#define launch_prefix_tc launch_whole_prefix_tc
#include "../../paper_2510_19705_b200/csrc/attn_prefix_tc.cu"
#undef launch_prefix_tc

namespace hsd {
bool launch_prefix_tc(const PrefixArgs &p, int hd, cudaStream_t s, int &status) {
  TcArgs a = {};
  a.p = p;
  a.box = 16;
  a.per_tile = 128 / p.group;
  a.sets = ceil_div(p.rows, 2 * a.per_tile);
  a.per_set = ceil_div(p.rows, a.sets);
  const PoolView &v = p.pool;
  status = HSD_E_CUDA;
  if (v.page != 16 || tc_init() || !registers_are_there<64>() || !registers_are_there<128>()) return true;
  if (tc_make_map_rows(&a.q, p.q, hd, p.nq, p.rows, p.group, a.per_tile) ||
      tc_make_map_pool(&a.k, v.k, hd, v.page, v.n_pages, p.nkv, v.token_bytes, v.page_bytes, v.head_bytes, a.box / 2) ||
      tc_make_map_pool(&a.v, v.v, hd, v.page, v.n_pages, p.nkv, v.token_bytes, v.page_bytes, v.head_bytes, a.box)) return true;
  status = hd == 64 ? launch_t<64>(a, s) : launch_t<128>(a, s);
  return true;
}
}  // namespace hsd
