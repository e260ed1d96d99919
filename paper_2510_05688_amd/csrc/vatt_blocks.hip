// Blocks of tokens chosen by the upper bound of their scores that their summaries give.
#include <algorithm>

#include "vatt_format.h"

namespace vatt {
namespace {

constexpr int kScoreThreads = 256, kScoreTile = 16 * kScoreThreads / kWave;  // blocks that a workgroup scores at a time

struct SelectBlocksArgs {
  const uint16_t* q;
  const uint16_t* summary;
  const int32_t* seq_lens;
  float* scores;  // [B * q_len][Hkv][score_stride]
  float* errors;  // [B * q_len][Hkv][score_splits]: how far scores may be off
  int32_t* out_blocks;
  int32_t* out_count;
  int32_t* topk_idx;
  int32_t* topk_cnt;
  RowMap M;
  SelectParams sel;
  int Hq, Hkv, q_len, n_blocks, score_stride, score_splits, block_shift, head_blocks, capacity, k_max;
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

__device__ __forceinline__ int tokens_seen_of(int n, int n_max, int q_len, int t) { return max(min(max(n, 1), n_max) - (q_len - 1 - t), 1); }
__device__ __forceinline__ int tokens_seen(const int32_t* seq_lens, int seq, int n_max, int q_len, int t) {
  return tokens_seen_of(seq_lens[seq], n_max, q_len, t);
}

__device__ __forceinline__ float top_of(float a, float b) { return (a > b || a != a) ? a : b; }  // (NaN where one is)

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4_t product(const uint4& a, const uint4& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t where_negative(uint32_t w, bool negative) {  // the halves of a bf16 pair of that sign, 0 for the others
  const uint32_t below = ((w >> 15) & 1u) * 0xffffu | ((w >> 31) & 1u) * 0xffff0000u;
  return w & (negative ? below : ~below);
}
__device__ __forceinline__ uint4 where_negative(const uint4& w, bool negative) {
  return make_uint4(where_negative(w.x, negative), where_negative(w.y, negative), where_negative(w.z, negative), where_negative(w.w, negative));
}
__device__ __forceinline__ uint4 magnitudes(const uint4& w) {
  return make_uint4(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu, w.z & 0x7fff7fffu, w.w & 0x7fff7fffu);
}

// Upper bounds of the blocks' scores to fp32 accuracy, and how far they may be off: the choice has to be the exact one, and
// choose_blocks_kernel works out the few blocks near the threshold in 64 bits.
// sum_c q_c (q_c < 0 ? low_c : top_c) = max(q, 0) . top + min(q, 0) . low is two products on the matrix cores, 16 blocks x 16 query vectors
// at a time (operand lane l: row or column l % 16, eight columns of the head); the same with magnitudes bounds the error.  A sum of 2 d
// products in any order, every addition off by at most 2^-23 of the magnitudes so far, is off by at most 2 d 2^-23 of the sum of all
// magnitudes; 2^-23 more covers the rounding of the exact sum to 32 bits.  (2^-100: products below the normal range.)
// What bounds it: the summaries' bytes, which are read again for every 16 query vectors of a KV head.  12 sequences of 8K - 128K tokens on pages,
// 213 MB of summaries, 39 us = 5.4 TB/s; all scores in 64 bits on the vector units took 58 (they were busy 85 % of the time).  Whole
// call on 8 x 64K, 134 MB: up to 16 vectors 32 - 34 us, 20 vectors 56, 40 vectors 77.
template <int D, bool PAGED>
__global__ __launch_bounds__(kScoreThreads) void block_score_kernel(SelectBlocksArgs A) {
  constexpr int S = D / 32, TILE = kScoreTile;
  constexpr float kError = (2 * D + 1) * 1.1920929e-7f * 1.01f;
  __shared__ float s_error[kScoreThreads / kWave][16];
  const int seq = blockIdx.y, split = blockIdx.x / A.Hkv, kvh = blockIdx.x - split * A.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, g4 = lane >> 4;
  const int G = A.Hq / A.Hkv, vectors = G * A.q_len;
  const int end = block_parts(A.sel, tokens_seen(A.seq_lens, seq, A.M.n_max, A.q_len, A.q_len - 1), A.block_shift).hi;
  if (split * TILE >= end) return;
  // A wave loads whole rows, LPR lanes each, and turns them round in LDS: with a row's 64 bytes per lane group and load instead, as the
  // operands want them, 12 x 128K tokens (403 MB) take 76 us, so 64.
  constexpr int LPR = 2 * D / 8, RPI = kWave / LPR, LOADS = 16 / RPI;  // lanes per block (both ends), blocks per load, loads
  __shared__ uint4 s_tile[kScoreThreads / kWave][16 * (LPR + 1)];
  uint4* rows = s_tile[wave];
  uint4 part[LOADS];
  // (paged: lane i asks for the block-table entry of block i a tile ahead, so that no row waits for its entry)
  auto entry_of = [&](int tile) { return row_block<PAGED>(A.M, seq, min(tile + wave * 16 + i16, end - 1) << A.block_shift); };
  auto load = [&](int tile, int entry) {
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int nth = u * RPI + lane / LPR, blk = min(tile + wave * 16 + nth, end - 1);
      int64_t place;
      if constexpr (PAGED) place = ((int64_t)__shfl(entry, nth) * A.Hkv + kvh) * A.head_blocks + (blk & (A.head_blocks - 1));
      else place = ((int64_t)seq * A.Hkv + kvh) * A.head_blocks + blk;
      part[u] = load_stream_16(A.summary + place * 2 * D + lane % LPR * 8);
    }
  };
  for (int v0 = 0; v0 < vectors; v0 += 16) {
    load(split * TILE, entry_of(split * TILE));
    int entry = entry_of(split * TILE + A.score_splits * TILE);
    const int v = min(v0 + i16, vectors - 1), t = v / G;  // (columns beyond the last vector repeat it)
    uint4 up[S], down[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const uint4 q = *reinterpret_cast<const uint4*>(A.q + (((int64_t)seq * A.q_len + t) * A.Hq + kvh * G + v % G) * D + s * 32 + g4 * 8);
      up[s] = where_negative(q, false);
      down[s] = where_negative(q, true);
    }
    const int64_t out_row = ((int64_t)seq * A.q_len + t) * A.Hkv + kvh;
    float worst = 0.f;
    for (int tile = split * TILE; tile < end; tile += A.score_splits * TILE) {
      f32x4_t u = {0.f, 0.f, 0.f, 0.f}, e = u;
#pragma unroll
      for (int l = 0; l < LOADS; ++l) rows[(l * RPI + lane / LPR) * (LPR + 1) + lane % LPR] = part[l];
      const int next = tile + A.score_splits * TILE;
      if (next < end) load(next, entry);
      entry = entry_of(next + A.score_splits * TILE);
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const uint4 top = rows[i16 * (LPR + 1) + s * 4 + g4], low = rows[i16 * (LPR + 1) + LPR / 2 + s * 4 + g4];
        u = product(top, up[s], u);
        u = product(low, down[s], u);
        e = product(magnitudes(top), up[s], e);
        e = product(magnitudes(low), magnitudes(down[s]), e);
      }
      __builtin_amdgcn_wave_barrier();
      // result lane l: vector l % 16, blocks 4 (l / 16) .. + 3; the largest over a KV head's vectors of one query token
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (G > 1) u[r] = top_of(dpp_f32<0xB1>(u[r]), u[r]);
        if (G > 2) u[r] = top_of(dpp_f32<0x4E>(u[r]), u[r]);
        if (G > 4) u[r] = top_of(dpp_f32<0x141>(u[r]), u[r]);
        const float x = e[r] * kError + 7.9e-31f;
        worst = x < INFINITY && fabsf(u[r]) < INFINITY ? fmaxf(worst, x) : INFINITY;
      }
      const int blk = tile + wave * 16 + 4 * g4;
      if (v0 + i16 < vectors && i16 % G == 0 && blk < end)
        *reinterpret_cast<float4*>(A.scores + out_row * A.score_stride + blk) = make_float4(u[0], u[1], u[2], u[3]);
    }
    worst = fmaxf(worst, __shfl_xor(worst, 16));
    worst = fmaxf(worst, __shfl_xor(worst, 32));
    if (G > 1) worst = fmaxf(worst, dpp_f32<0xB1>(worst));
    if (G > 2) worst = fmaxf(worst, dpp_f32<0x4E>(worst));
    if (G > 4) worst = fmaxf(worst, dpp_f32<0x141>(worst));
    __syncthreads();
    if (lane < 16) s_error[wave][lane] = worst;
    __syncthreads();
    if (tid < 16 && v0 + i16 < vectors && i16 % G == 0) {
#pragma unroll
      for (int w = 0; w < kScoreThreads / kWave; ++w) worst = fmaxf(worst, s_error[w][i16]);
      A.errors[out_row * A.score_splits + split] = worst;
    }
  }
}

// A block's bound in 64 bits, rounded to 32, by D / 8 lanes with 8 columns each; in all of them.
template <int D, bool PAGED>
__device__ __forceinline__ float exact_bound(const SelectBlocksArgs& A, int seq, int64_t vb, int kvh, int blk, int c) {
  const int G = A.Hq / A.Hkv;
  int64_t place = (int64_t)seq * A.Hkv + kvh;
  if constexpr (PAGED) place = (int64_t)row_block<PAGED>(A.M, seq, blk << A.block_shift) * A.Hkv + kvh;
  place = place * A.head_blocks + (PAGED ? blk & (A.head_blocks - 1) : blk);
  const uint4 top = *reinterpret_cast<const uint4*>(A.summary + place * 2 * D + 8 * c);
  const uint4 low = *reinterpret_cast<const uint4*>(A.summary + (place * 2 + 1) * D + 8 * c);
  const uint32_t tw[4] = {top.x, top.y, top.z, top.w}, lw[4] = {low.x, low.y, low.z, low.w};
  float best = -INFINITY;
  for (int g0 = 0; g0 < G; g0 += 4) {  // (four heads' rows under way at a time; beyond the last one it is repeated)
    uint4 q[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) q[g] = *reinterpret_cast<const uint4*>(A.q + (vb * A.Hq + kvh * G + min(g0 + g, G - 1)) * D + 8 * c);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint32_t qw[4] = {q[g].x, q[g].y, q[g].z, q[g].w};
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float q0 = bf16_lo(qw[i]), q1 = bf16_hi(qw[i]);
        s = fma((double)q0, (double)(q0 < 0.f ? bf16_lo(lw[i]) : bf16_lo(tw[i])), s);
        s = fma((double)q1, (double)(q1 < 0.f ? bf16_hi(lw[i]) : bf16_hi(tw[i])), s);
      }
      s += dpp_f64<0xB1>(s);
      s += dpp_f64<0x4E>(s);
      s += dpp_f64<0x141>(s);
      if constexpr (D == 128) s += dpp_f64<0x140>(s);
      best = top_of((float)s, best);
    }
  }
  return best;
}

// Exclusive sums over the threads of a workgroup, and the sum of all; to be called by all of them.  Two places take turns, so that one barrier
// a call is enough: a place is written again only after the barrier of the call between.
template <int THREADS>
struct Sums {
  uint32_t (*place)[THREADS / kWave];
  int turn = 0;
  __device__ __forceinline__ uint32_t before(uint32_t v, uint32_t& total) {
    const uint32_t incl = wave_inclusive_scan_u32(v);
    const int wave = threadIdx.x >> 6;
    uint32_t* s = place[turn & 1];
    ++turn;
    if ((threadIdx.x & 63) == 63) s[wave] = incl;
    __syncthreads();
    uint32_t below = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) {
      if (w < wave) below += s[w];
      total += s[w];
    }
    return below + incl - v;
  }
};

// The key that `left` of the marked scores of a workgroup are above or at, and how many of those at it count: a radix selection, 8 bits at
// a time.  key, marked: KPT per thread.
template <int THREADS, int KPT, int BINS>
__device__ __forceinline__ uint32_t threshold_key(const uint32_t (&key)[KPT], const bool (&marked)[KPT], uint32_t& left, uint32_t (&hist)[BINS],
                                                  Sums<THREADS>& sums, uint32_t& s_bin, uint32_t& s_left) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0, mask = 0, all;
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    for (int i = tid; i < 256; i += THREADS) hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < KPT; ++j)
      if (marked[j] && (key[j] & mask) == prefix) atomicAdd(&hist[(key[j] >> shift) & 255u], 1u);
    __syncthreads();
    const uint32_t mine = tid < 256 ? hist[255 - tid] : 0u;
    const uint32_t above = sums.before(mine, all);
    if (above < left && above + mine >= left) {
      s_bin = 255 - tid;
      s_left = left - above;
    }
    __syncthreads();
    prefix |= s_bin << shift;
    mask |= 255u << shift;
    left = s_left;
  }
  return prefix;
}

__device__ __forceinline__ uint32_t score_key(float f) {  // (-0 counts as +0, NaN is on top)
  f += 0.f;
  return f != f ? 0xffffffffu : float_order_key(f);
}

// The `take` blocks of a row with the largest bounds, ties to the lower block, and the list of all blocks taken; one workgroup per list, KPT
// neighbouring scores per thread in registers.
// With scores off by at most E and T the take-th largest of them, everything above T + 2 E is in and everything below T - 2 E is out:
// the take-th largest exact value lies within E of T.  Those between, a few where scores spread at all, get their bound in 64 bits and are
// ranked by it.
// T: its bin comes from one histogram over equal steps between the least and the largest finite score (bins of the bits, which a radix
// selection would begin with, hold nearly all scores of a row together, and their LDS atomics then wait for each other: 28.8 us for
// 96 rows of up to 8192 blocks); the few scores in that bin are ranked against each other.  Where one bin holds many (equal scores, or one
// far from all others), and where many lie between, a radix selection takes its place.
// What bounds it: a chain of some 14 barriers and three memory round trips; 96 rows of up to 8192 blocks 10.9 us, 8 of 2048 7.0, of which the
// bounds in 64 bits are 2.
template <int D, bool PAGED, int THREADS, int KPT>
__global__ __launch_bounds__(THREADS) void choose_blocks_kernel(SelectBlocksArgs A) {
  constexpr int WAVES = THREADS / kWave, BINS = 1024, PER = BINS / THREADS, MOST = 256, LPR = D / 8;
  static_assert(PER * THREADS == BINS && THREADS >= MOST && KPT % 4 == 0, "whole shares");
  __shared__ uint32_t hist[BINS], s_sums[2][WAVES], s_lo[WAVES], s_hi[WAVES];
  Sums<THREADS> sums = {s_sums};
  __shared__ float s_off[WAVES];
  __shared__ uint32_t s_bin, s_left, s_inside, s_filled, s_edge;
  __shared__ uint32_t c_key[MOST], c_blk[MOST], chosen_bit[THREADS * KPT / 32];
  __shared__ uint16_t list[THREADS * KPT];
  const int kvh = blockIdx.x, vb = blockIdx.y, tid = threadIdx.x, wave = tid >> 6;
  const int seq = seq_of_pair(vb, A.q_len), G = A.Hq / A.Hkv;
  const int64_t row = (int64_t)vb * A.Hkv + kvh;
  float f[KPT], off = 0.f;
#pragma unroll
  for (int j = 0; j < KPT; j += 4) {
    const int i = tid * KPT + j;  // (asked for without waiting for the sequence's length: what nobody wrote is not looked at)
    const float4 x = i < A.score_stride ? *reinterpret_cast<const float4*>(A.scores + row * A.score_stride + i) : make_float4(0.f, 0.f, 0.f, 0.f);
    f[j] = x.x; f[j + 1] = x.y; f[j + 2] = x.z; f[j + 3] = x.w;
  }
  const float first_error = tid < A.score_splits ? A.errors[row * A.score_splits + tid] : 0.f;
  const int n_seq = A.seq_lens[seq];
  const BlockParts P = block_parts(A.sel, tokens_seen_of(n_seq, A.M.n_max, A.q_len, vb - seq * A.q_len), A.block_shift);
  int32_t* out = A.out_blocks + row * A.capacity;
  const int tail = P.total - P.hi;
  for (int i = tid; i < P.lo; i += THREADS) out[i] = i;
  for (int i = tid; i < tail; i += THREADS) out[P.lo + P.take + i] = P.hi + i;
  if (tid == 0) A.out_count[row] = P.lo + P.take + tail;
  if (P.take > 0) {
    // (the score kernel's workgroups that had blocks, up to the last query token's)
    const int last = block_parts(A.sel, tokens_seen_of(n_seq, A.M.n_max, A.q_len, A.q_len - 1), A.block_shift).hi;
    const int parts = min(A.score_splits, (last + kScoreTile - 1) / kScoreTile);
    if (tid < parts) off = first_error;
    uint32_t key[KPT], lo = 0xffffffffu, hi = 0u, all;
    bool ours[KPT];
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      ours[j] = tid * KPT + j >= P.lo && tid * KPT + j < P.hi;
      key[j] = score_key(f[j]);
      if (ours[j] && fabsf(f[j]) < INFINITY) {
        lo = min(lo, key[j]);
        hi = max(hi, key[j]);
      }
    }
    lo = wave_min_u32(lo);
    hi = wave_max_u32(hi);
    off = wave_max(off);
    if ((tid & 63) == 0) {
      s_lo[wave] = lo;
      s_hi[wave] = hi;
      s_off[wave] = off;
    }
    for (int i = tid; i < BINS; i += THREADS) hist[i] = 0;
    for (int i = tid; i < THREADS * KPT / 32; i += THREADS) chosen_bit[i] = 0;
    if (tid == 0) s_filled = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      lo = min(lo, s_lo[w]);
      hi = max(hi, s_hi[w]);
      off = fmaxf(off, s_off[w]);
    }
    // (no finite score, or a range that 32 bits do not hold: one bin)
    const float least = float_from_order_key(lo), span = float_from_order_key(hi) - least;
    const float scale = lo < hi && span < INFINITY ? (float)(BINS - 1) / span : 0.f;
    int bin[KPT];
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      const float x = scale > 0.f && scale < INFINITY ? (f[j] - least) * scale : 0.f;
      bin[j] = x != x ? BINS - 1 : (int)fminf(fmaxf(x, 0.f), (float)(BINS - 1));
      if (ours[j]) atomicAdd(&hist[bin[j]], 1u);
    }
    __syncthreads();
    uint32_t h[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += h[i] = hist[BINS - 1 - (tid * PER + i)];
    uint32_t before = sums.before(sum, all);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (before < (uint32_t)P.take && before + h[i] >= (uint32_t)P.take) {
        s_bin = BINS - 1 - (tid * PER + i);
        s_left = (uint32_t)P.take - before;
        s_inside = h[i];
      }
      before += h[i];
    }
    __syncthreads();
    uint32_t edge;  // T's key
    if (s_inside <= MOST) {
      const int edge_bin = (int)s_bin, n = (int)s_inside;
      const uint32_t left = s_left;
#pragma unroll
      for (int j = 0; j < KPT; ++j)
        if (ours[j] && bin[j] == edge_bin) {
          const uint32_t at = atomicAdd(&s_filled, 1u);
          c_key[at] = key[j];
          c_blk[at] = tid * KPT + j;
        }
      __syncthreads();
      if (tid < n) {
        const uint32_t k = c_key[tid], b = c_blk[tid];
        uint32_t better = 0;
        for (int i = 0; i < n; ++i) better += c_key[i] > k || (c_key[i] == k && c_blk[i] < b);
        if (better == left - 1) s_edge = k;
      }
      __syncthreads();
      edge = s_edge;
    } else {
      uint32_t left = (uint32_t)P.take;
      edge = threshold_key<THREADS, KPT, BINS>(key, ours, left, hist, sums, s_bin, s_left);
    }
    const float T = float_from_order_key(edge), above = T + 2.f * off, below = T - 2.f * off;
    bool in[KPT], open[KPT];
    uint32_t sure = 0, unsure = 0;
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      in[j] = ours[j] && f[j] > above;
      open[j] = ours[j] && !in[j] && !(f[j] < below);  // (a NaN anywhere leaves everything open)
      sure += in[j];
      unsure += open[j];
    }
    uint32_t both;  // (at most 12288 each)
    uint32_t place = sums.before(unsure | sure << 16, both) & 0xffffu;
    const uint32_t n_open = both & 0xffffu;
    uint32_t left = (uint32_t)P.take - (both >> 16);  // of the open ones
    if (left < n_open) {
#pragma unroll
      for (int j = 0; j < KPT; ++j)
        if (open[j]) list[place++] = (uint16_t)(tid * KPT + j);
      __syncthreads();
      const bool few = n_open <= MOST;
      for (uint32_t i = tid / LPR; i < n_open; i += THREADS / LPR) {
        const int blk = list[i];
        const float x = exact_bound<D, PAGED>(A, seq, vb, kvh, blk, tid % LPR);
        if (tid % LPR == 0) {
          if (few) {
            c_key[i] = score_key(x);
            c_blk[i] = blk;
          } else {
            A.scores[row * A.score_stride + blk] = x;
          }
        }
      }
      __syncthreads();
      if (few) {
        if (tid < (int)n_open) {
          const uint32_t k = c_key[tid], b = c_blk[tid];
          uint32_t better = 0;
          for (uint32_t i = 0; i < n_open; ++i) better += c_key[i] > k || (c_key[i] == k && c_blk[i] < b);
          if (better < left) atomicOr(&chosen_bit[b / 32], 1u << (b & 31));
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < KPT; ++j) {
          const int i = tid * KPT + j;
          in[j] |= open[j] && (chosen_bit[i / 32] >> (i & 31) & 1u);
        }
      } else {
#pragma unroll
        for (int j = 0; j < KPT; ++j)
          if (open[j]) key[j] = score_key(A.scores[row * A.score_stride + tid * KPT + j]);
        const uint32_t least_key = threshold_key<THREADS, KPT, BINS>(key, open, left, hist, sums, s_bin, s_left);
        uint32_t equal = 0;
#pragma unroll
        for (int j = 0; j < KPT; ++j) equal += open[j] && key[j] == least_key;
        uint32_t rank = sums.before(equal, all);
#pragma unroll
        for (int j = 0; j < KPT; ++j) {
          const bool eq = open[j] && key[j] == least_key;
          in[j] |= open[j] && (key[j] > least_key || (eq && rank < left));
          rank += eq;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < KPT; ++j) in[j] |= open[j];
    }
    uint32_t count = 0;
#pragma unroll
    for (int j = 0; j < KPT; ++j) count += in[j];
    place = sums.before(count, all);
#pragma unroll
    for (int j = 0; j < KPT; ++j)
      if (in[j]) {
        out[P.lo + place] = tid * KPT + j;
        list[place++] = (uint16_t)(tid * KPT + j);
      }
    __syncthreads();
  }
  if (A.topk_idx) {
    const int tokens = P.take << A.block_shift, inner = (1 << A.block_shift) - 1;
    for (int g = 0; g < G; ++g) {
      const int64_t head = (int64_t)vb * A.Hq + kvh * G + g;
      int32_t* dst = A.topk_idx + head * A.k_max;
      for (int i = tid; i < tokens; i += THREADS) dst[i] = ((int)list[i >> A.block_shift] << A.block_shift) + (i & inner);
      if (tid == 0) A.topk_cnt[head] = tokens;
    }
  }
}

template <int D, bool PAGED>
hipError_t launch_select(const Plan& pl, const SelectBlocksArgs& A, hipStream_t st) {
  hipLaunchKernelGGL((block_score_kernel<D, PAGED>), dim3(A.score_splits * A.Hkv, pl.p.batch), dim3(kScoreThreads), 0, st, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(A.Hkv, pl.vbatch);
  static_assert(1024 * 12 * 16 >= kCapacityMax, "every row fits");
  if (A.n_blocks <= 256 * 8) hipLaunchKernelGGL((choose_blocks_kernel<D, PAGED, 256, 8>), grid, dim3(256), 0, st, A);
  else if (A.n_blocks <= 1024 * 8) hipLaunchKernelGGL((choose_blocks_kernel<D, PAGED, 1024, 8>), grid, dim3(1024), 0, st, A);
  else hipLaunchKernelGGL((choose_blocks_kernel<D, PAGED, 1024, 12>), grid, dim3(1024), 0, st, A);
  return hipGetLastError();
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
  A.score_stride = (A.n_blocks + 7) / 8 * 8;
  const int jobs = pl.p.batch * A.Hkv;
  A.score_splits = std::max(1, std::min((A.n_blocks + kScoreTile - 1) / kScoreTile, (8 * pl.num_cus + jobs - 1) / jobs));
  // (the region of the scores has a place for every token of every query head, these take one per block and some)
  A.errors = A.scores + (int64_t)pl.vbatch * A.Hkv * A.score_stride;
  const bool paged = pl.p.kv_layout == VATT_LAYOUT_PAGED;
  if (pl.p.head_dim == 128) return paged ? launch_select<128, true>(pl, A, st) : launch_select<128, false>(pl, A, st);
  return paged ? launch_select<64, true>(pl, A, st) : launch_select<64, false>(pl, A, st);
}

}  // namespace vatt
