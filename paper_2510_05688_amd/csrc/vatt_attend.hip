// Attention over the tokens of listed blocks, or over all tokens of a quantised cache.
#include "vatt_attend.h"

namespace vatt {
namespace {

template <int D, int FMT, bool PAGED>
hipError_t launch_attend_f(const Plan& pl, const AttendArgs& A, hipStream_t st) {
  const dim3 grid(A.Hkv, A.splits * A.rounds, A.blocks ? pl.vbatch : pl.p.batch), merge(A.Hq, pl.vbatch), threads(kAttendThreads);
  if (A.blocks) {  // (one to eight vectors)
    if (pl.group <= 4) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kListedBlocks, 1, 3>), grid, threads, 0, st, A);
    else hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kListedBlocks, 1, 2>), grid, threads, 0, st, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attend_merge_kernel<D, FMT, PAGED, kListedBlocks>), merge, threads, 0, st, A);
    return hipGetLastError();
  } else if constexpr (FMT != VATT_KV_BF16) {
    const int vectors = pl.group * pl.q_len;
    if (vectors <= 5) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kAllTokens, 1, 3>), grid, threads, 0, st, A);
    else if (vectors <= 8) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kAllTokens, 1, 2>), grid, threads, 0, st, A);
    else if (vectors <= 16) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kAllTokens, 1, 1>), grid, threads, 0, st, A);
    else hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kAllTokens, 2, 1>), grid, threads, 0, st, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attend_merge_kernel<D, FMT, PAGED, kAllTokens>), merge, threads, 0, st, A);
    return hipGetLastError();
  } else {
    return hipErrorInvalidValue;  // (all tokens of a bf16 cache are dense_kernel's)
  }
}
template <int D, int FMT>
hipError_t launch_attend_d(const Plan& pl, const AttendArgs& A, hipStream_t st) {
  return pl.p.kv_layout == VATT_LAYOUT_PAGED ? launch_attend_f<D, FMT, true>(pl, A, st) : launch_attend_f<D, FMT, false>(pl, A, st);
}
template <int D>
hipError_t launch_attend_p(const Plan& pl, const AttendArgs& A, hipStream_t st) {
  if (pl.kv_format == VATT_KV_E4M3) return launch_attend_d<D, VATT_KV_E4M3>(pl, A, st);
  if (pl.kv_format == VATT_KV_E2M1) return launch_attend_d<D, VATT_KV_E2M1>(pl, A, st);
  return launch_attend_d<D, VATT_KV_BF16>(pl, A, st);
}

}  // namespace

hipError_t launch_attend(const Plan& pl, const void* q, const void* k, const void* v, const int32_t* block_table,
                         const int32_t* seq_lens, const int32_t* blocks, const int32_t* block_count, void* ws, float* out_o,
                         float* out_lse, hipStream_t st) {
  AttendArgs A = {};
  A.q = static_cast<const uint16_t*>(q);
  A.k = static_cast<const unsigned char*>(k);
  A.v = static_cast<const unsigned char*>(v);
  A.scale_off = (int64_t)kv_scale_offset(pl);
  A.seq_lens = seq_lens;
  A.blocks = blocks;
  A.block_count = block_count;
  A.out_o = out_o;
  A.out_lse = out_lse;
  A.M = row_map(pl, block_table);
  A.Hq = pl.p.n_q_heads;
  A.Hkv = pl.p.n_kv_heads;
  A.q_len = pl.q_len;
  A.capacity = block_list_capacity(pl);
  A.block_shift = pl.block_tokens ? 31 - __builtin_clz(pl.block_tokens) : 0;
  A.log2_scale = (float)((double)pl.sm_scale * 1.4426950408889634);
  const int vectors = blocks ? pl.group : pl.group * pl.q_len;
  A.rounds = vectors <= 16 ? 1 : (vectors + 31) / 32;
  // Four workgroups per CU in all, none with less than a unit of keys per wave at the longest; the partial sums fit the workspace.  Every
  // row gets as many, however long it is: with one long sequence among short ones a few workgroups have nearly all the work (one of 128K
  // tokens among 47 of 1000 in e4m3, 376 MB, 468 us; 2K to 32K evenly, 588 MB, 110).
  const int64_t rows = (int64_t)pl.vbatch * A.Hq, jobs = (int64_t)(blocks ? pl.vbatch : pl.p.batch) * A.Hkv * A.rounds;
  const int64_t longest = blocks ? (int64_t)A.capacity * pl.block_tokens : pl.p.n_max;
  int64_t splits = std::min<int64_t>((4 * pl.num_cus + jobs - 1) / jobs, (longest + kUnit * kAttendWaves - 1) / (kUnit * kAttendWaves));
  splits = std::min<int64_t>({splits, kSplitsMax, (int64_t)(pl.ws_bytes / (rows * (pl.p.head_dim + 2) * sizeof(float)))});
  A.splits = (int)std::max<int64_t>(splits, 1);
  A.part = static_cast<float*>(ws);
  A.part_ml = reinterpret_cast<float2*>(A.part + rows * A.splits * pl.p.head_dim);
  return pl.p.head_dim == 128 ? launch_attend_p<128>(pl, A, st) : launch_attend_p<64>(pl, A, st);
}

}  // namespace vatt
