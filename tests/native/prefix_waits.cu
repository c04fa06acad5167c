// Attention over a shared prefix as tests/test_gpu_operator_waits.py builds it: with a wait limit of a millisecond, and its tensor-memory
// kernel without the warps that load and issue, so that the softmax warps' waits run out; nothing is in flight.
#define launch_prefix_tc launch_whole_prefix_tc
#include "../../paper_2510_19705_b200/csrc/attn_prefix_tc.cu"
#undef launch_prefix_tc

namespace hsd {
template <int HD> static int launch_without_loader(const TcArgs &a, cudaStream_t s) {
  if (cudaFuncSetAttribute((const void *)prefix_tc_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<HD>::kSmem) != cudaSuccess) return HSD_E_CUDA;
  prefix_tc_kernel<HD><<<kPrefixGrid, kLoaderWarp * 32, Cfg<HD>::kSmem, s>>>(a);
  return hsd_launch_status();
}
bool launch_prefix_tc(const PrefixArgs &p, int hd, cudaStream_t s, int &status) {
  TcArgs a = {};
  a.p = p;
  a.box = 8;
  a.per_tile = 128 / p.group;
  a.sets = ceil_div(p.rows, 2 * a.per_tile);
  a.per_set = ceil_div(p.rows, a.sets);
  status = hd == 64 ? launch_without_loader<64>(a, s) : launch_without_loader<128>(a, s);
  return true;
}
}  // namespace hsd
