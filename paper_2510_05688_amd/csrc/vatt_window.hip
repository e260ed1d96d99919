// Attention with few query vectors over the first tokens of a sequence and the last ones up to each query's own.
#include "vatt_attend.h"

namespace vatt {
namespace {

template <int D, int FMT, bool PAGED>
hipError_t launch_window_f(const AttendArgs& A, int batch, hipStream_t st) {
  const dim3 grid(A.Hkv, A.splits * A.rounds, batch), threads(kAttendThreads);
  const int vectors = A.Hq / A.Hkv * A.q_len;
  if (vectors <= 5) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kFirstAndWindow, 1, 3>), grid, threads, 0, st, A);
  else if (vectors <= 8) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kFirstAndWindow, 1, 2>), grid, threads, 0, st, A);
  else if (vectors <= 16) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kFirstAndWindow, 1, 1>), grid, threads, 0, st, A);
  else hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kFirstAndWindow, 2, 1>), grid, threads, 0, st, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attend_merge_kernel<D, FMT, PAGED, kFirstAndWindow>), dim3(A.Hq, batch * A.q_len), threads, 0, st, A);
  return hipGetLastError();
}
template <int D, int FMT>
hipError_t launch_window_d(const Plan& pl, const AttendArgs& A, hipStream_t st) {
  return pl.p.kv_layout == VATT_LAYOUT_PAGED ? launch_window_f<D, FMT, true>(A, pl.p.batch, st) : launch_window_f<D, FMT, false>(A, pl.p.batch, st);
}
template <int D>
hipError_t launch_window_p(const Plan& pl, const AttendArgs& A, hipStream_t st) {
  if (pl.kv_format == VATT_KV_E4M3) return launch_window_d<D, VATT_KV_E4M3>(pl, A, st);
  if (pl.kv_format == VATT_KV_E2M1) return launch_window_d<D, VATT_KV_E2M1>(pl, A, st);
  return launch_window_d<D, VATT_KV_BF16>(pl, A, st);
}

}  // namespace

hipError_t launch_window(const Plan& pl, const void* q, const void* k, const void* v, const int32_t* block_table, const int32_t* seq_lens,
                         int sink, int window, void* ws, float* out_o, float* out_lse, hipStream_t st) {
  AttendArgs A = {};
  A.q = static_cast<const uint16_t*>(q);
  A.k = static_cast<const unsigned char*>(k);
  A.v = static_cast<const unsigned char*>(v);
  A.scale_off = (int64_t)kv_scale_offset(pl);
  A.seq_lens = seq_lens;
  A.out_o = out_o;
  A.out_lse = out_lse;
  A.M = row_map(pl, block_table);
  A.Hq = pl.p.n_q_heads;
  A.Hkv = pl.p.n_kv_heads;
  A.q_len = pl.q_len;
  A.q_stride = (int64_t)A.Hq * pl.p.head_dim;
  A.log2_scale = (float)((double)pl.sm_scale * 1.4426950408889634);
  A.sink = std::min(sink, pl.p.n_max);
  A.window = std::min(window, pl.p.n_max);
  const int vectors = pl.group * pl.q_len;
  A.rounds = vectors <= 16 ? 1 : (vectors + 31) / 32;
  // Four workgroups per CU in all, none with less than a unit of keys per wave; the partial sums fit the workspace.
  const int64_t rows = (int64_t)pl.vbatch * A.Hq, jobs = (int64_t)pl.p.batch * A.Hkv * A.rounds;
  const int64_t longest = std::min<int64_t>(pl.p.n_max, (int64_t)A.sink + A.window + pl.q_len + 14);  // (whole groups of 8 at both ends)
  int64_t splits = std::min<int64_t>((4 * pl.num_cus + jobs - 1) / jobs, (longest + kUnit * kAttendWaves - 1) / (kUnit * kAttendWaves));
  splits = std::min<int64_t>({splits, kSplitsMax, (int64_t)(pl.ws_bytes / (rows * (pl.p.head_dim + 2) * sizeof(float)))});
  A.splits = (int)std::max<int64_t>(splits, 1);
  A.part = static_cast<float*>(ws);
  A.part_ml = reinterpret_cast<float2*>(A.part + rows * A.splits * pl.p.head_dim);
  return pl.p.head_dim == 128 ? launch_window_p<128>(pl, A, st) : launch_window_p<64>(pl, A, st);
}

}  // namespace vatt
