// Attention with few query vectors over the first tokens of a sequence and the last ones up to each query's own.
#include "vatt_attend.h"

namespace vatt {
namespace {

template <int D, int FMT, bool PAGED>
hipError_t launch_window_f(const AttendArgs& A, hipStream_t st) {
  const int vectors = A.Hq / A.Hkv * A.q_len;
  if (A.workgroups == 0) {
    const dim3 grid(A.Hkv, A.rounds, A.batch), eight(8 * kWave);
    if (vectors <= 5) hipLaunchKernelGGL((window_kernel<D, FMT, PAGED, 1, 3>), grid, eight, 0, st, A);
    else if (vectors <= 8) hipLaunchKernelGGL((window_kernel<D, FMT, PAGED, 1, 2>), grid, eight, 0, st, A);
    else if (vectors <= 16) hipLaunchKernelGGL((window_kernel<D, FMT, PAGED, 1, 1>), grid, eight, 0, st, A);
    else hipLaunchKernelGGL((window_kernel<D, FMT, PAGED, 2, 1>), grid, eight, 0, st, A);
    return hipGetLastError();
  }
  const dim3 grid(A.workgroups), threads(kAttendThreads);
  if (vectors <= 5) hipLaunchKernelGGL((dealt_kernel<D, FMT, PAGED, 1, 3>), grid, threads, 0, st, A);
  else if (vectors <= 8) hipLaunchKernelGGL((dealt_kernel<D, FMT, PAGED, 1, 2>), grid, threads, 0, st, A);
  else if (vectors <= 16) hipLaunchKernelGGL((dealt_kernel<D, FMT, PAGED, 1, 1>), grid, threads, 0, st, A);
  else hipLaunchKernelGGL((dealt_kernel<D, FMT, PAGED, 2, 1>), grid, threads, 0, st, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attend_merge_kernel<D, FMT, PAGED, kFirstAndWindow>), dim3(A.Hq, A.batch * A.q_len), threads, 0, st, A);
  return hipGetLastError();
}
template <int D, int FMT>
hipError_t launch_window_d(const Plan& pl, const AttendArgs& A, hipStream_t st) {
  return pl.p.kv_layout == VATT_LAYOUT_PAGED ? launch_window_f<D, FMT, true>(A, st) : launch_window_f<D, FMT, false>(A, st);
}
template <int D>
hipError_t launch_window_p(const Plan& pl, const AttendArgs& A, hipStream_t st) {
  if (pl.kv_format == VATT_KV_E4M3) return launch_window_d<D, VATT_KV_E4M3>(pl, A, st);
  if (pl.kv_format == VATT_KV_E2M1) return launch_window_d<D, VATT_KV_E2M1>(pl, A, st);
  return launch_window_d<D, VATT_KV_BF16>(pl, A, st);
}

}  // namespace

namespace {

int window_rounds(const Plan& pl, int q_len) { return pl.group * q_len <= 16 ? 1 : (pl.group * q_len + 31) / 32; }
int64_t window_jobs(const Plan& pl, int q_len) { return (int64_t)pl.p.batch * pl.p.n_kv_heads * window_rounds(pl, q_len); }
// Workgroups that the tokens are dealt out to, two to a compute unit, and no more than the merge takes for one job; 0: every job has one of eight
// waves.  So it is for up to 640 tokens (4 and 256, us, shared by four / alone: 1 x 8K 16.2 / 11.6, 16 in e4m3 26.8 / 13.2; 4 and 512 15.6 / 14.7, 768
// 15.3 / 16.3), where there are jobs for all slots (64 sequences in e4m3, 4 and 2048 72 / 62), and with more sequences than a wave looks through.
int window_workgroups(const Plan& pl, int q_len, int64_t longest) {
  const int64_t slots = 2 * pl.num_cus;
  if (longest <= 640 || (window_jobs(pl, q_len) >= slots && longest <= 4608) || pl.p.batch > kDealtMost) return 0;
  return (int)std::min<int64_t>(slots, (int64_t)(kSplitsMax - 2) * pl.p.n_kv_heads * window_rounds(pl, q_len));
}
// Bytes of the partial sums (a workgroup's share ends inside a job, or a job ends inside a share) of `rows` vectors each, and of the jobs' list.
size_t window_part_bytes(const Plan& pl, int q_len, int workgroups, int rows) {
  const int64_t jobs = window_jobs(pl, q_len);
  return (size_t)(workgroups + jobs) * rows * (pl.p.head_dim + 2) * sizeof(float) + jobs * sizeof(int2);
}

hipError_t launch_rows(const Plan& pl, AttendArgs& A, const void* q, const void* k, const void* v, const int32_t* block_table, int sink,
                       int window, int workgroups, int slot_rows, void* ws, hipStream_t st) {
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
  A.batch = pl.p.batch;
  A.rounds = window_rounds(pl, A.q_len);
  A.slot_rows = slot_rows;
  A.workgroups = workgroups;
  A.part = static_cast<float*>(ws);
  A.slots = (int)(workgroups + window_jobs(pl, A.q_len));
  A.part_ml = reinterpret_cast<float2*>(A.part + (int64_t)A.slots * A.slot_rows * pl.p.head_dim);
  A.jobs = reinterpret_cast<int2*>(A.part_ml + (int64_t)A.slots * A.slot_rows);
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
  // (whole groups of 8 at both ends of the window)
  const int64_t longest = std::min<int64_t>(pl.p.n_max, (int64_t)std::min(sink, pl.p.n_max) + std::min(window, pl.p.n_max) + pl.q_len + 14);
  // The workspace is the plan's, which other calls size: sums of as many vectors as there are, not of 16, for which it has room in a part of the
  // workgroups only (us in so many / in all, one sequence in bf16, one query head per KV head: 8 KV heads and 4096 tokens, 118 of 512, 19.9 / 14.5, 8000,
  // 152, 21.5 / 17.7; one and 9000, 20 of 126, 16.2 / 15.6; but four and 16000, 111 of 504, 21.0 / 22.0).
  const int vectors = pl.group * pl.q_len, rows = vectors <= 16 ? vectors : 32;
  int workgroups = window_workgroups(pl, pl.q_len, longest);
  if (window_part_bytes(pl, pl.q_len, workgroups, rows) > pl.ws_bytes) {  // as many as there is room for (17 vectors of one KV head on 700 tokens: 102 of 126)
    const int64_t least = (int64_t)window_part_bytes(pl, pl.q_len, 0, rows), one = (int64_t)window_part_bytes(pl, pl.q_len, 1, rows) - least;
    workgroups = (int)std::max<int64_t>(((int64_t)pl.ws_bytes - least) / one, 0);
  }
  return launch_rows(pl, A, q, k, v, block_table, sink, window, workgroups, rows, ws, st);
}

namespace {
int few_slot_rows(const Plan& pl, int n_new) { return pl.group * n_new <= 16 ? 16 : 32; }
}  // namespace

size_t few_workspace_bytes(const Plan& pl, int n_new) {
  const int workgroups = window_workgroups(pl, n_new, pl.p.n_max);  // (a window leaves no more)
  return workgroups == 0 ? 0 : window_part_bytes(pl, n_new, workgroups, few_slot_rows(pl, n_new));
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
  const int workgroups = window_workgroups(pl, n_new, std::min<int64_t>(pl.p.n_max, seen));
  return launch_rows(pl, A, q, k, v, block_table, window > 0 ? sink : 0, window > 0 ? window : pl.p.n_max, workgroups, few_slot_rows(pl, n_new), ws,
                     st);
}

}  // namespace vatt
