// Products in 8-bit integers as tests/test_gpu_operator_waits.py builds them: with a wait limit of a millisecond, and with copies that bring
// fewer bytes than their barrier counts, so that the waits for them run out.
#include "../../paper_2510_19705_b200/csrc/gemm_w8.cu"

namespace hsd {
template <typename TO> static int without_data(W8Args a, const void *codes_a, const void *codes_w, int K, cudaStream_t s) {
  const int sms = sm_count();
  if (a.R <= 256) {
    const int S = split_of(a.N, a.KB, sms), n_tiles = ceil_div(a.N, a.tile_rows = tile_rows_of(a.N, S, sms)), grid = S > 1 ? n_tiles * S : n_tiles < sms ? n_tiles : sms;
    a.npad = ceil_div(a.R, 16) * 16;
    if (a.tile_rows < 16 || tc_make_map_bytes(&a.w, codes_w, a.N, K, a.tile_rows - 8) || tc_make_map_bytes(&a.a, codes_a, a.R, K, a.npad)) return HSD_E_CUDA;
    return tc_npad(a.R) == 16 ? run_stream<16, TO>(a, n_tiles, S, grid, s) : run_stream<256, TO>(a, n_tiles, S, grid, s);
  }
  a.tokens = 256;
  a.m_tiles = ceil_div(a.R, a.tokens);
  a.tiles = a.m_tiles * ceil_div(a.N, 2 * kTile);
  if (tc_make_map_bytes(&a.w, codes_w, a.N, K, kTile) || tc_make_map_bytes(&a.a, codes_a, a.R, K, a.tokens / 2 - 8)) return HSD_E_CUDA;
  if (cudaFuncSetAttribute((const void *)w8_pair_kernel<TO>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem) != cudaSuccess) return HSD_E_CUDA;
  w8_pair_kernel<TO><<<2 * std::min(sms / 2, a.tiles), kThreads, kPairSmem, s>>>(a);
  return hsd_launch_status();
}
}  // namespace hsd

// codes_a int8 [R, K], codes_w int8 [N, K]; status: a word of device memory
extern "C" int w8_without_data(const void *codes_a, const float *row_scales, int R, int K, const void *codes_w, const float *col_scales, int N, void *out,
                               int out_dtype, int *status, void *stream) {
  if (hsd::tc_init()) return HSD_E_UNSUPPORTED;
  hsd::W8Args a = {};
  a.row_scales = row_scales; a.col_scales = col_scales; a.out = out; a.R = R; a.N = N; a.KB = ceil_div(K, hsd::kBlock);
  a.status = status;
  return out_dtype == HSD_F32 ? hsd::without_data<float>(a, codes_a, codes_w, K, (cudaStream_t)stream) : hsd::without_data<__nv_bfloat16>(a, codes_a, codes_w, K, (cudaStream_t)stream);
}
