// Blocks of tokens chosen by the upper bound of their scores that their summaries give.
#include "vatt_format.h"

namespace vatt {
namespace {

constexpr int kScoreThreads = 256, kChooseThreads = 512;

struct SelectBlocksArgs {
  const uint16_t* q;
  const uint16_t* summary;
  const int32_t* seq_lens;
  float* scores;  // [B * q_len][Hkv][n_blocks]
  int32_t* out_blocks;
  int32_t* out_count;
  int32_t* topk_idx;
  int32_t* topk_cnt;
  RowMap M;
  SelectParams sel;
  int Hq, Hkv, q_len, n_blocks, block_shift, head_blocks, capacity, k_max;
};

// How the blocks of a sequence of n tokens divide: [0, lo) hold sink tokens, [hi, total) window tokens (or the newest one), `take`
// of those between are chosen.
struct BlockParts {
  int lo, hi, total, take;
};
__device__ __forceinline__ BlockParts block_parts(const SelectParams& p, int n, int shift) {
  const int c = 1 << shift;
  BlockParts b;
  b.total = (n + c - 1) >> shift;
  b.lo = (min(p.sink, n) + c - 1) >> shift;
  b.hi = max(n - max(p.window, 1), 0) >> shift;
  if (b.lo >= b.hi) b.lo = b.hi = b.total;
  const int k = p.topk_abs > 0 ? p.topk_abs : (int)floor(p.topk_frac * (double)n);
  b.take = min(k >> shift, b.hi - b.lo);
  return b;
}

__device__ __forceinline__ int tokens_seen(const int32_t* seq_lens, int seq, int n_max, int q_len, int t) {
  return max(min(max(seq_lens[seq], 1), n_max) - (q_len - 1 - t), 1);
}

// One lane per 8 columns, D / 8 lanes per block; sums in 64 bits.
template <int D, bool PAGED>
__global__ __launch_bounds__(kScoreThreads) void block_score_kernel(SelectBlocksArgs A) {
  constexpr int LPR = D / 8, TT = kScoreThreads / LPR;
  const int seq = blockIdx.y, at = blockIdx.x / A.Hkv, kvh = blockIdx.x - at * A.Hkv;
  const int tid = threadIdx.x, c = tid % LPR, blk = at * TT + tid / LPR, G = A.Hq / A.Hkv;
  const BlockParts last = block_parts(A.sel, tokens_seen(A.seq_lens, seq, A.M.n_max, A.q_len, A.q_len - 1), A.block_shift);
  if (blk >= last.hi) return;
  int64_t place;
  if constexpr (PAGED)
    place = ((int64_t)row_block<PAGED>(A.M, seq, blk << A.block_shift) * A.Hkv + kvh) * A.head_blocks + (blk & (A.head_blocks - 1));
  else
    place = ((int64_t)seq * A.Hkv + kvh) * A.head_blocks + blk;
  const uint4 hi = *reinterpret_cast<const uint4*>(A.summary + place * 2 * D + 8 * c);
  const uint4 lo = *reinterpret_cast<const uint4*>(A.summary + (place * 2 + 1) * D + 8 * c);
  const uint32_t hw[4] = {hi.x, hi.y, hi.z, hi.w}, lw[4] = {lo.x, lo.y, lo.z, lo.w};
  for (int t = 0; t < A.q_len; ++t) {
    float best = -INFINITY;
    for (int g = 0; g < G; ++g) {
      const uint4 qq = *reinterpret_cast<const uint4*>(A.q + (((int64_t)seq * A.q_len + t) * A.Hq + kvh * G + g) * D + 8 * c);
      const uint32_t qw[4] = {qq.x, qq.y, qq.z, qq.w};
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float q0 = bf16_lo(qw[i]), q1 = bf16_hi(qw[i]);
        s = fma((double)q0, (double)(q0 < 0.f ? bf16_lo(lw[i]) : bf16_lo(hw[i])), s);
        s = fma((double)q1, (double)(q1 < 0.f ? bf16_hi(lw[i]) : bf16_hi(hw[i])), s);
      }
      s += dpp_f64<0xB1>(s);
      s += dpp_f64<0x4E>(s);
      s += dpp_f64<0x141>(s);
      if constexpr (LPR == 16) s += dpp_f64<0x140>(s);
      const float f = (float)s;
      best = (f > best || f != f) ? f : best;
    }
    if (c == 0) A.scores[(((int64_t)seq * A.q_len + t) * A.Hkv + kvh) * A.n_blocks + blk] = best;
  }
}

// The `take` largest of a row of scores, ties to the lower block, and the list of all blocks taken; one workgroup per list.
// The threshold is found by a radix selection over the scores' order keys, 8 bits at a time.
__global__ __launch_bounds__(kChooseThreads) void choose_blocks_kernel(SelectBlocksArgs A) {
  constexpr int WAVES = kChooseThreads / kWave;
  extern __shared__ uint32_t keys[];  // of the blocks between sink and window, then the chosen ones
  __shared__ uint32_t hist[256];
  __shared__ uint32_t s_bin, s_left;
  __shared__ uint32_t s_eq[WAVES], s_in[WAVES];
  const int kvh = blockIdx.x, vb = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seq = seq_of_pair(vb, A.q_len), G = A.Hq / A.Hkv;
  const BlockParts P = block_parts(A.sel, tokens_seen(A.seq_lens, seq, A.M.n_max, A.q_len, vb - seq * A.q_len), A.block_shift);
  const int64_t row = (int64_t)vb * A.Hkv + kvh;
  const int count = P.hi - P.lo, tail = P.total - P.hi;
  int32_t* out = A.out_blocks + row * A.capacity;
  for (int i = tid; i < P.lo; i += kChooseThreads) out[i] = i;
  for (int i = tid; i < tail; i += kChooseThreads) out[P.lo + P.take + i] = P.hi + i;
  if (tid == 0) A.out_count[row] = P.lo + P.take + tail;
  if (P.take > 0) {
    const float* src = A.scores + row * A.n_blocks + P.lo;
    for (int i = tid; i < count; i += kChooseThreads) {
      const float f = src[i] + 0.f;  // (-0 becomes +0)
      keys[i] = f != f ? 0xffffffffu : float_order_key(f);
    }
    uint32_t prefix = 0, mask = 0, left = (uint32_t)P.take;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kChooseThreads) hist[i] = 0;
      __syncthreads();
      for (int i = tid; i < count; i += kChooseThreads)
        if ((keys[i] & mask) == prefix) atomicAdd(&hist[(keys[i] >> shift) & 255u], 1u);
      __syncthreads();
      if (wave == 0) {  // bins from the top, four per lane
        uint32_t h[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += h[i] = hist[255 - 4 * lane - i];
        uint32_t before = wave_inclusive_scan_u32(sum) - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < left && before + h[i] >= left) {
            s_bin = 255 - 4 * lane - i;
            s_left = left - before;
          }
          before += h[i];
        }
      }
      __syncthreads();
      prefix |= s_bin << shift;
      mask |= 255u << shift;
      left = s_left;
    }
    // in order of the blocks: everything above the threshold, and the first `left` equal to it
    uint32_t eq_before = 0, in_before = 0;
    for (int i0 = 0; i0 < count; i0 += kChooseThreads) {
      const int i = i0 + tid;
      const uint32_t key = i < count ? keys[i] : 0u;
      const bool eq = i < count && key == prefix;
      const uint64_t eqs = __ballot(eq), below = (1ull << lane) - 1;
      if (lane == 0) s_eq[wave] = (uint32_t)__popcll(eqs);
      __syncthreads();
      uint32_t eq_rank = eq_before + (uint32_t)__popcll(eqs & below);
      for (int w = 0; w < WAVES; ++w) {
        if (w < wave) eq_rank += s_eq[w];
        eq_before += s_eq[w];
      }
      const bool in = i < count && (key > prefix || (eq && eq_rank < left));
      const uint64_t ins = __ballot(in);
      if (lane == 0) s_in[wave] = (uint32_t)__popcll(ins);
      __syncthreads();
      uint32_t place = in_before + (uint32_t)__popcll(ins & below);
      for (int w = 0; w < WAVES; ++w) {
        if (w < wave) place += s_in[w];
        in_before += s_in[w];
      }
      if (in) {
        out[P.lo + place] = P.lo + i;
        keys[place] = (uint32_t)(P.lo + i);  // (place <= i: keys of this round and before)
      }
    }
    __syncthreads();
  }
  if (A.topk_idx) {
    const int tokens = P.take << A.block_shift;
    for (int g = 0; g < G; ++g) {
      const int64_t head = (int64_t)vb * A.Hq + kvh * G + g;
      int32_t* dst = A.topk_idx + head * A.k_max;
      for (int i = tid; i < tokens; i += kChooseThreads)
        dst[i] = ((int)keys[i >> A.block_shift] << A.block_shift) + (i & ((1 << A.block_shift) - 1));
      if (tid == 0) A.topk_cnt[head] = tokens;
    }
  }
}

}  // namespace

hipError_t launch_select_blocks(const Plan& pl, const void* q, const void* summary, const int32_t* block_table, const int32_t* seq_lens,
                                void* ws, int32_t* out_blocks, int32_t* out_count, int32_t* topk_idx, int32_t* topk_cnt, hipStream_t st) {
  SelectBlocksArgs A = {};
  A.q = static_cast<const uint16_t*>(q);
  A.summary = static_cast<const uint16_t*>(summary);
  A.seq_lens = seq_lens;
  A.scores = reinterpret_cast<float*>(static_cast<char*>(ws) + pl.off_scores);
  A.out_blocks = out_blocks;
  A.out_count = out_count;
  A.topk_idx = topk_idx;
  A.topk_cnt = topk_cnt;
  A.M = row_map(pl, block_table);
  A.sel = pl.sel;
  A.Hq = pl.p.n_q_heads;
  A.Hkv = pl.p.n_kv_heads;
  A.q_len = pl.q_len;
  A.n_blocks = (pl.p.n_max + pl.block_tokens - 1) / pl.block_tokens;
  A.block_shift = 31 - __builtin_clz(pl.block_tokens);
  A.head_blocks = pl.p.kv_layout == VATT_LAYOUT_PAGED ? pl.p.page_size / pl.block_tokens : A.n_blocks;
  A.capacity = block_list_capacity(pl);
  A.k_max = pl.k_max;
  const int per = kScoreThreads / (pl.p.head_dim / 8);
  const dim3 grid((A.n_blocks + per - 1) / per * A.Hkv, pl.p.batch);
  const bool paged = pl.p.kv_layout == VATT_LAYOUT_PAGED;
  if (pl.p.head_dim == 128) {
    if (paged) hipLaunchKernelGGL((block_score_kernel<128, true>), grid, dim3(kScoreThreads), 0, st, A);
    else hipLaunchKernelGGL((block_score_kernel<128, false>), grid, dim3(kScoreThreads), 0, st, A);
  } else {
    if (paged) hipLaunchKernelGGL((block_score_kernel<64, true>), grid, dim3(kScoreThreads), 0, st, A);
    else hipLaunchKernelGGL((block_score_kernel<64, false>), grid, dim3(kScoreThreads), 0, st, A);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(choose_blocks_kernel, dim3(A.Hkv, pl.vbatch), dim3(kChooseThreads), A.n_blocks * sizeof(uint32_t), st, A);
  return hipGetLastError();
}

}  // namespace vatt
