// Attention with few query vectors over the first tokens of a sequence and the last ones up to each query's own.
#include "vatt_attend.h"

namespace vatt {
namespace {

template <int D, int FMT, bool PAGED>
hipError_t launch_window_f(const AttendArgs& A, int batch, hipStream_t st) {
  const dim3 grid(A.Hkv, A.splits * A.rounds, batch), threads(kAttendThreads);
  const int vectors = A.Hq / A.Hkv * A.q_len;
  if (A.splits == 1) {
    const dim3 eight(8 * kWave);
    if (vectors <= 5) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kFirstAndWindow, 1, 3, 8, true>), grid, eight, 0, st, A);
    else if (vectors <= 8) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kFirstAndWindow, 1, 2, 8, true>), grid, eight, 0, st, A);
    else if (vectors <= 16) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kFirstAndWindow, 1, 1, 8, true>), grid, eight, 0, st, A);
    else hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, kFirstAndWindow, 2, 1, 8, true>), grid, eight, 0, st, A);
    return hipGetLastError();
  }
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

namespace {

// Workgroups that share out the tokens of a sequence.  One of eight waves, which writes the results, for up to 640 tokens (4 and 256, us: 1 x 8K
// 16.2 -> 11.6, 16 in e4m3 26.8 -> 13.2; 4 and 512 15.6 -> 14.7, 768 15.3 -> 16.3) and where there are jobs for all slots (64 sequences in e4m3, 4 and
// 2048 72 -> 62).  Else four of four waves, or what two slots per CU take, none with less than a unit of keys per wave (4 and 4096 with 2 / 4 / 8 / 16:
// 48 sequences in e4m3 89 / 93 / 102 / 116, 24 50 / 44 / 48 / 53, 16 in bf16 51 / 50 / 53 / 55).
int window_splits(const Plan& pl, int q_len, int64_t longest) {
  const int vectors = pl.group * q_len, rounds = vectors <= 16 ? 1 : (vectors + 31) / 32;
  const int64_t jobs = (int64_t)pl.p.batch * pl.p.n_kv_heads * rounds, slots = 2 * pl.num_cus;
  if (longest <= 640 || (jobs >= slots && longest <= 4608)) return 1;
  return (int)std::min<int64_t>({std::max<int64_t>(4, (slots + jobs - 1) / jobs), (longest + kUnit * kAttendWaves - 1) / (kUnit * kAttendWaves), kSplitsMax});
}

hipError_t launch_rows(const Plan& pl, AttendArgs& A, const void* q, const void* k, const void* v, const int32_t* block_table, int sink,
                       int window, int splits, void* ws, hipStream_t st) {
  A.q = static_cast<const uint16_t*>(q);
  A.k = static_cast<const unsigned char*>(k);
  A.v = static_cast<const unsigned char*>(v);
  A.scale_off = (int64_t)kv_scale_offset(pl);
  A.M = row_map(pl, block_table);
  A.Hq = pl.p.n_q_heads;
  A.Hkv = pl.p.n_kv_heads;
  A.log2_scale = (float)((double)pl.sm_scale * 1.4426950408889634);
  A.sink = std::min(sink, pl.p.n_max);
  A.window = std::min(window, pl.p.n_max);
  const int vectors = pl.group * A.q_len;
  A.rounds = vectors <= 16 ? 1 : (vectors + 31) / 32;
  A.splits = splits;
  A.part = static_cast<float*>(ws);
  A.part_ml = reinterpret_cast<float2*>(A.part + (int64_t)pl.p.batch * A.q_len * A.Hq * A.splits * pl.p.head_dim);
  return pl.p.head_dim == 128 ? launch_window_p<128>(pl, A, st) : launch_window_p<64>(pl, A, st);
}

}  // namespace

hipError_t launch_window(const Plan& pl, const void* q, const void* k, const void* v, const int32_t* block_table, const int32_t* seq_lens,
                         int sink, int window, void* ws, float* out_o, float* out_lse, hipStream_t st) {
  AttendArgs A = {};
  A.seq_lens = seq_lens;
  A.q_len = pl.q_len;
  A.q_stride = (int64_t)pl.p.n_q_heads * pl.p.head_dim;
  A.out_o = out_o;
  A.out_lse = out_lse;
  // (whole groups of 8 at both ends of the window; the partial sums fit the workspace)
  const int64_t longest = std::min<int64_t>(pl.p.n_max, (int64_t)std::min(sink, pl.p.n_max) + std::min(window, pl.p.n_max) + pl.q_len + 14);
  const int64_t fit = pl.ws_bytes / ((int64_t)pl.vbatch * pl.p.n_q_heads * (pl.p.head_dim + 2) * sizeof(float));
  const int splits = (int)std::max<int64_t>(1, std::min<int64_t>(window_splits(pl, pl.q_len, longest), fit));
  return launch_rows(pl, A, q, k, v, block_table, sink, window, splits, ws, st);
}

size_t few_workspace_bytes(const Plan& pl, int n_new) {
  const int splits = window_splits(pl, n_new, pl.p.n_max);  // (a window leaves no more)
  return splits == 1 ? 0 : (size_t)pl.p.batch * n_new * pl.p.n_q_heads * splits * (pl.p.head_dim + 2) * sizeof(float);
}

hipError_t launch_few(const Plan& pl, const void* q, int64_t q_stride, int n_new, const int32_t* first, const int32_t* new_lens, const void* k,
                      const void* v, const int32_t* block_table, int sink, int window, void* ws, bool bf16, void* out_o, float* out_lse,
                      hipStream_t st) {
  AttendArgs A = {};
  A.first = first;
  A.new_lens = new_lens;
  A.q_len = n_new;
  A.q_stride = q_stride;
  A.out_o = static_cast<float*>(out_o);
  A.out_lse = out_lse;
  A.out_bf16 = bf16;
  const int64_t seen = window > 0 ? (int64_t)std::min(sink, pl.p.n_max) + std::min(window, pl.p.n_max) + n_new + 14 : pl.p.n_max;
  const int splits = window_splits(pl, n_new, std::min<int64_t>(pl.p.n_max, seen));
  return launch_rows(pl, A, q, k, v, block_table, window > 0 ? sink : 0, window > 0 ? window : pl.p.n_max, splits, ws, st);
}

}  // namespace vatt
