// New rows into the cache (rotated, in the cache's format, with the summaries of the blocks they touch), and rows of it back.
#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "vatt_format.h"

namespace vatt {
namespace {

constexpr int kWriteThreads = 256;
constexpr int kAhead = 4;  // rows that a thread of the write kernel has under way (with two, 2 x 16K into e2m1 165 instead of 153 us)
// Tokens of a workgroup for the rows without summaries: as many heads' rows of a token as fit lie side by side, and the turns are made for so
// many tokens (us, 4 / 8 / 16 tokens: prompts of 2 x 16K into e2m1 151 / 153 / 155, of 4 x 0.3K - 2K out of a fused projection 34.4 /
// 29.3 / 30.1).
constexpr int kRowTokens = 8;

struct WriteArgs {
  const uint16_t* q;
  const uint16_t* k_new;
  const uint16_t* v_new;
  int64_t q_stride, k_stride, v_stride;
  const int32_t* first;
  const int32_t* new_lens;
  unsigned char* k;
  unsigned char* v;
  int64_t scale_off;
  uint16_t* summary;
  uint16_t* out_q;
  int32_t* out_lens;
  RowMap M;
  int n_new, Hq, Hkv;
  int block_shift, head_blocks;  // tokens per block; blocks per KV head of a sequence (contiguous) or of a page
  int k_jobs, k_groups, k_heads;       // workgroups with summaries per sequence, groups of KV heads, and KV heads of one
  int row_groups, q_groups, v_groups;  // the other rows: groups of heads, of them those of q and of V
  int row_passes, row_tokens_shift;    // passes of a workgroup over its heads, tokens of one
  int rot, pairs;
  double attention;
  double freq[64];
};

// sin and cos of a >= 0 in 64 bits, rounded to 32 with a factor: a minus the nearest multiple of pi / 2 (pi / 2 in two parts, whose own
// error is below 2^-100 of a; the two differences round by 2^-54 each), then the Taylor series to x^13 and x^12, whose next terms are
// below 2^-41 for |x| <= pi / 4.  a itself, a rounded product of position and frequency, is off by up to 2^-53 of it: 2^-35 at the
// furthest positions.
__device__ __forceinline__ float2 turn(double a, double factor) {
  const double k = rint(a * 0.63661977236758134308);
  const double x = fma(-k, 6.123233995736766036e-17, fma(-k, 1.57079632679489661923, a));
  const double x2 = x * x;
  double s = fma(x2, 1.0 / 6227020800.0, -1.0 / 39916800.0);
  s = fma(x2, s, 1.0 / 362880.0);
  s = fma(x2, s, -1.0 / 5040.0);
  s = fma(x2, s, 1.0 / 120.0);
  s = fma(x2, s, -1.0 / 6.0);
  s = fma(x * x2, s, x);
  double c = fma(x2, 1.0 / 479001600.0, -1.0 / 3628800.0);
  c = fma(x2, c, 1.0 / 40320.0);
  c = fma(x2, c, -1.0 / 720.0);
  c = fma(x2, c, 1.0 / 24.0);
  c = fma(x2, c, -0.5);
  c = fma(x2, c, 1.0);
  const int quarter = (int)k & 3;
  const double cs = (quarter & 1) ? s : c, sn = (quarter & 1) ? c : s;
  return make_float2((float)(factor * ((quarter == 1 || quarter == 2) ? -cs : cs)), (float)(factor * (quarter >= 2 ? -sn : sn)));
}

// (cos, sin) of the pairs of the positions from `base` on, `tokens` of them, as far as they lie in [first, end); by the whole
// workgroup, to be followed by a barrier.
template <int D>
__device__ __forceinline__ void make_turns(const WriteArgs& A, float2 (*turns)[D / 2], int base, int tokens, int first, int end) {
  // (the frequencies are read where the kernel's arguments lie)
  typedef const __attribute__((address_space(4))) double* Frequencies;
  const Frequencies freq = (Frequencies)((const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(WriteArgs, freq));
#pragma unroll 1
  for (int x = threadIdx.x; x < tokens * (D / 2); x += kWriteThreads) {
    const int i = x % (D / 2), t = x / (D / 2);
    if (i < A.rot / 2 && base + t >= first && base + t < end) turns[t][i] = turn((double)(base + t) * freq[i], A.attention);
  }
}

__device__ __forceinline__ uint4 load_part(const uint16_t* row, int c) { return *reinterpret_cast<const uint4*>(row + 8 * c); }
// The columns that a lane's 8 are rotated with in the layout of halves, from the lane of the row that has them.
template <int D>
__device__ __forceinline__ uint4 other_half(const WriteArgs& A, const uint4& own, int c) {
  const uint32_t w[4] = {own.x, own.y, own.z, own.w};
  uint32_t o[4];
  if (A.rot == D) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = D == 128 ? dpp_u32<0x128>(w[i]) : dpp_u32<0x1B>(dpp_u32<0x141>(w[i]));  // lane ^ 8; lane ^ 4
  } else {
    const int half = A.rot / 16, from = (int)(threadIdx.x & 63) - c + (c < half ? c + half : c < 2 * half ? c - half : c);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (uint32_t)__shfl((int)w[i], from);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// A lane's share of a token's turns: column i becomes own_i cos_i + partner_i sin_i, the sign of the sine included.  Columns that are not
// rotated have cos 1, partner 0 and sin -0, whose product -0 leaves every value as it is, -0 too.
struct LaneTurns {
  float cos[8], sin[8];
};
__device__ __forceinline__ LaneTurns lane_turns(const WriteArgs& A, const float2* turns, int c) {
  LaneTurns t;
  const bool lower = 8 * c < A.rot / 2, turned = 8 * c < A.rot;
  if (!turned) c = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 x = !turned ? make_float2(1.f, 0.f) : turns[A.pairs ? 4 * c + i / 2 : (lower ? 8 * c : 8 * c - A.rot / 2) + i];
    t.cos[i] = x.x;
    t.sin[i] = !turned || (A.pairs ? (i & 1) == 0 : lower) ? -x.y : x.y;
  }
  return t;
}
template <int D>
__device__ __forceinline__ void rotated(const WriteArgs& A, const uint4& own, int c, bool rotate, const LaneTurns& t, float (&y)[8]) {
  const uint32_t w[4] = {own.x, own.y, own.z, own.w};
  if (!rotate) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = bf16_lo(w[i]);
      y[2 * i + 1] = bf16_hi(w[i]);
    }
    return;
  }
  uint32_t o[4];
  if (A.pairs) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = w[i] << 16 | w[i] >> 16;
  } else {
    const uint4 other = other_half<D>(A, own, c);
    o[0] = other.x; o[1] = other.y; o[2] = other.z; o[3] = other.w;
  }
  const uint32_t turned = 8 * c < A.rot ? 0xffffffffu : 0u;  // (else nothing that 0 could make a NaN of)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = o[i] & turned;
    y[2 * i] = fmaf(bf16_lo(w[i]), t.cos[2 * i], bf16_lo(x) * t.sin[2 * i]);
    y[2 * i + 1] = fmaf(bf16_hi(w[i]), t.cos[2 * i + 1], bf16_hi(x) * t.sin[2 * i + 1]);
  }
}

__device__ __forceinline__ uint4 packed(const float (&y)[8]) {
  return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

// Columns 8 c .. of a row of K or V to the cache; what they stand for there comes back in bf16.  (All four lanes of a quad that share a
// scale are in the same row.)
template <int D, int FMT>
__device__ __forceinline__ uint4 store_row(unsigned char* buf, int64_t scale_off, const RowAt& at, int c, const float (&y)[8]) {
  unsigned char* dst = buf + at.row * kRowBytes<FMT, D> + c * (kRowBytes<FMT, D> / (D / 8));
  if constexpr (FMT == VATT_KV_BF16) {
    const uint4 x = packed(y);
    *reinterpret_cast<uint4*>(dst) = x;
    return x;
  } else {
    uint32_t byte;
    const Chunk<FMT> x = quantise<FMT>(y, byte);
    store_chunk<FMT>(dst, x);
    if ((c & 3) == 0) buf[scale_off + at.scales * (D / 32) + c / 4] = (unsigned char)byte;
    return chunk_bf16<FMT>(x, byte);
  }
}

// The larger (smaller) of two values; NaN where one is.
__device__ __forceinline__ float top_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float low_of(float a, float b) { return __builtin_elementwise_minimum(a, b); }

// The largest (smallest) over the 64 / LPR rows of a wave; lane l ends with columns lane_groups_column(l) and the next, as in add_lane_groups.
template <int LPR, class Pick>
__device__ __forceinline__ float2 pick_lane_groups(const float (&v)[8], Pick pick) {
  float half[4], two[2];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[c]), __float_as_uint(v[c + 4]), false, false);
    half[c] = pick(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(half[c]), __float_as_uint(half[c + 2]), false, false);
    two[c] = pick(__uint_as_float(r[0]), __uint_as_float(r[1]));
    if constexpr (LPR == 8) two[c] = pick(two[c], dpp_f32<0x128>(two[c]));  // row_ror:8
  }
  return make_float2(two[0], two[1]);
}

// Summaries of the blocks of one tile of tokens for `heads` KV heads from kvh0 on, whose new rows (from position `first` on; none with FILL)
// are written on the way.  One lane per 8 columns, D / 8 lanes per row, a pass over kWriteThreads / (D / 8) tokens at a time, head after
// head, the next row under way; the turns of a lane's columns stay in registers where a tile is one pass.
// The old rows of a block that is only begun are read again rather than taken from its summary: it then follows from the cache alone, also
// after a sequence was cut back.  That is up to 15 rows with blocks of 16, beside the row written.
template <int D, int FMT, bool PAGED, bool FILL>
__device__ __forceinline__ void summary_tile(const WriteArgs& A, int b, int kvh0, int heads, int tile_lo, int tile, int first, int end,
                                             float2 (*turns)[D / 2], float (*s_ends)[kWriteThreads / kWave][2][D]) {
  constexpr int LPR = D / 8, TT = kWriteThreads / LPR, WAVES = kWriteThreads / kWave;
  const int tid = threadIdx.x, c = tid % LPR, r = tid / LPR, lane = tid & 63, wave = tid >> 6;
  const int bs = 1 << A.block_shift, passes = tile / TT, items = heads * passes;
  struct Row {
    uint4 part;
    Chunk<FMT> code;
    uint32_t byte;
  };
  auto place = [&](int item) {
    const int h = passes == 1 ? item : item / passes, tok = tile_lo + (passes == 1 ? 0 : (item - h * passes) * TT) + r;
    return make_int2(kvh0 + h, tok);
  };
  auto load = [&](int item, int blk) {
    const int2 x = place(item);
    Row row = {};
    if (x.y >= end) return row;
    if (!FILL && x.y >= first) {
      row.part = load_part(A.k_new + ((int64_t)b * A.n_new + (x.y - first)) * A.k_stride + x.x * D, c);
    } else {
      const RowAt at = row_at<PAGED>(A.M, b, x.x, x.y, blk);
      row.code = load_chunk<FMT>(A.k + at.row * kRowBytes<FMT, D> + c * (kRowBytes<FMT, D> / LPR));
      if constexpr (FMT != VATT_KV_BF16) row.byte = A.k[A.scale_off + at.scales * (D / 32) + c / 4];
    }
    return row;
  };
  auto block_of = [&](int item) { return row_block<PAGED>(A.M, b, min(place(item).y, end - 1)); };
  float top[8], low[8];
  LaneTurns lt = {};
  int blk = block_of(0), buffer = 0;
  Row next = load(0, blk);
  for (int item = 0; item < items; ++item) {
    const int2 x = place(item);
    const int kvh = x.x, tok = x.y, p = passes == 1 ? 0 : item % passes;
    if (!FILL && A.rot > 0 && (passes > 1 || item == 0)) {
      if (item > 0) __syncthreads();
      make_turns<D>(A, turns, tile_lo + p * TT, TT, first, end);
      __syncthreads();
      lt = lane_turns(A, turns[r], c);
    }
    const Row row = next;
    const int row_blk = blk;
    if (item + 1 < items) {
      if (passes > 1) blk = block_of(item + 1);
      next = load(item + 1, blk);
    }
    if (p == 0 || bs <= TT) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        top[i] = -INFINITY;
        low[i] = INFINITY;
      }
    }
    if (tok < end) {
      uint4 v;
      if (!FILL && tok >= first) {
        float y[8];
        rotated<D>(A, row.part, c, A.rot > 0, lt, y);
        v = store_row<D, FMT>(A.k, A.scale_off, row_at<PAGED>(A.M, b, kvh, tok, row_blk), c, y);
      } else {
        v = chunk_bf16<FMT>(row.code, row.byte);
      }
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float z = (i & 1) ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
        top[i] = top_of(z, top[i]);
        low[i] = low_of(z, low[i]);
      }
    }
    if (p + 1 < passes && bs > TT) continue;  // the block goes on (a tile of several passes is one block)
    // (a wave's rows belong to one block; two places for the waves' extremes take turns, so that one barrier is enough)
    const float2 t2 = pick_lane_groups<LPR>(top, [](float a, float b) { return top_of(a, b); });
    const float2 l2 = pick_lane_groups<LPR>(low, [](float a, float b) { return low_of(a, b); });
    float(*ends)[2][D] = s_ends[buffer];
    buffer ^= 1;
    if (LPR == 16 || !(lane & 8)) {
      const int col = lane_groups_column<LPR>(lane);
      *reinterpret_cast<float2*>(&ends[wave][0][col]) = t2;
      *reinterpret_cast<float2*>(&ends[wave][1][col]) = l2;
    }
    __syncthreads();
    const int blocks = bs < TT ? TT / bs : 1, per = WAVES / blocks;
    if (tid < blocks * 2 * LPR) {
      const int which = (tid / LPR) & 1, k = tid / (2 * LPR), lo = tile_lo + k * bs;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = ends[k * per][which][8 * c + i];
      for (int w = 1; w < per; ++w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float z = ends[k * per + w][which][8 * c + i];
          y[i] = which == 0 ? top_of(z, y[i]) : low_of(z, y[i]);
        }
      }
      if (lo < end && lo + bs > first) {
        int64_t at;
        if constexpr (PAGED)
          at = ((int64_t)row_block<PAGED>(A.M, b, lo) * A.Hkv + kvh) * A.head_blocks + ((lo >> A.block_shift) & (A.head_blocks - 1));
        else
          at = ((int64_t)b * A.Hkv + kvh) * A.head_blocks + (lo >> A.block_shift);
        *reinterpret_cast<uint4*>(A.summary + (at * 2 + which) * D + 8 * c) = packed(y);
      }
    }
  }
}

// One launch for everything a write does.  The first k_jobs workgroups of a sequence each take a tile of whole blocks of some KV
// heads' K rows, with their summaries; the others take the remaining rows (q, V, and K without summaries), tokens of a tile times heads.
// Every workgroup's rows are of one kind, so that source, stride and rotation are scalars.
// What bounds it: prompts the bytes (2 x 16K tokens of 32 + 2 x 8 heads into e2m1, 707 MB, 152 us = 4.65 TB/s, a copy runs at 4.8; the vector
// units are busy 60 % of it), single tokens the chain first -> block-table entry -> old rows of the block -> its summary (4.1 us
// for one, 5.6 for 32).
template <int D, int FMT, bool PAGED>
__global__ __launch_bounds__(kWriteThreads) void write_kernel(WriteArgs A) {
  constexpr int LPR = D / 8, TT = kWriteThreads / LPR;
  __shared__ float2 turns[TT][D / 2];
  __shared__ float s_ends[2][kWriteThreads / kWave][2][D];
  const int b = blockIdx.y, tid = threadIdx.x, c = tid % LPR, r = tid / LPR;
  const int first = A.first[b];
  int end = first;
  if (first >= 0 && first < A.M.n_max) end = min(first + (A.new_lens ? min(max(A.new_lens[b], 0), A.n_new) : A.n_new), A.M.n_max);
  if (blockIdx.x == 0 && tid == 0 && A.out_lens) A.out_lens[b] = end;
  if (end <= first) return;
  int x = blockIdx.x;
  if (x < A.k_jobs) {
    const int tile = max(1 << A.block_shift, TT), at = x / A.k_groups, group = x - at * A.k_groups;
    const int tile_lo = (first / tile + at) * tile;
    if (tile_lo >= end) return;
    const int kvh0 = group * A.k_heads;
    summary_tile<D, FMT, PAGED, false>(A, b, kvh0, min(A.k_heads, A.Hkv - kvh0), tile_lo, tile, first, end, turns, s_ends);
    return;
  }
  x -= A.k_jobs;
  // groups of q heads, of KV heads for K (without summaries), of KV heads for V
  const int at = x / A.row_groups;
  int group = x - at * A.row_groups;
  const bool is_q = group < A.q_groups;
  if (!is_q) group -= A.q_groups;
  const bool is_v = !is_q && group >= A.row_groups - A.q_groups - A.v_groups;
  if (is_v) group -= A.row_groups - A.q_groups - A.v_groups;
  const bool turned = !is_v && A.rot > 0;
  const int tokens = 1 << A.row_tokens_shift, per_pass = TT >> A.row_tokens_shift;
  const int j0 = at << A.row_tokens_shift, t = r & (tokens - 1), tok = first + j0 + t;
  if (first + j0 >= end) return;
  const int heads = is_q ? A.Hq : A.Hkv, h0 = group * A.row_passes * per_pass;
  const int64_t src_row = (int64_t)b * A.n_new + j0 + t, stride = is_q ? A.q_stride : is_v ? A.v_stride : A.k_stride;
  int h = h0 + (r >> A.row_tokens_shift);
  const uint16_t* src = (is_q ? A.q : is_v ? A.v_new : A.k_new) + src_row * stride + h * D + 8 * c;
  uint16_t* dst = A.out_q + (src_row * A.Hq + h) * D + 8 * c;  // (q)
  const int left = min(A.row_passes, (heads - h + per_pass - 1) / per_pass);  // rows of this lane
  // kAhead heads' rows under way at a time; the turns of the lane's columns stay in registers.
  uint4 part[kAhead];
  auto load = [&](int p) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (tok < end && p + u < left) part[u] = *reinterpret_cast<const uint4*>(src + (p + u) * per_pass * D);
  };
  load(0);
  const int blk = is_q ? 0 : row_block<PAGED>(A.M, b, min(tok, end - 1));
  LaneTurns lt = {};
  if (turned) {
    make_turns<D>(A, turns, first + j0, tokens, first, end);
    __syncthreads();
    lt = lane_turns(A, turns[t], c);
  }
  if (tok >= end) return;
  for (int p = 0; p < left; p += kAhead) {
    if (p > 0) load(p);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (p + u >= left) break;
      float y[8];
      rotated<D>(A, part[u], c, turned, lt, y);
      if (is_q) *reinterpret_cast<uint4*>(dst + (p + u) * per_pass * D) = packed(y);
      else store_row<D, FMT>(is_v ? A.v : A.k, A.scale_off, row_at<PAGED>(A.M, b, h + (p + u) * per_pass, tok, blk), c, y);
    }
  }
}

// A tile of one KV head per workgroup, a pass over it at a time.  What bounds it: with blocks of 16 and 128 columns a thread has one row part
// under way (8 x 32K tokens, bf16, 604 MB, 155 us = 3.9 TB/s; blocks of 64, whose next pass is under way, 108 us = 5.1 TB/s; e4m3 on
// pages, 344 MB, 188 us).
template <int D, int FMT, bool PAGED>
__global__ __launch_bounds__(kWriteThreads) void summary_kernel(WriteArgs A) {
  constexpr int TT = kWriteThreads / (D / 8);
  __shared__ float s_ends[2][kWriteThreads / kWave][2][D];
  const int b = blockIdx.y, tile = max(1 << A.block_shift, TT);
  const int at = blockIdx.x / A.Hkv, kvh = blockIdx.x - at * A.Hkv;
  const int end = min(max(A.first[b], 0), A.M.n_max);
  if (at * tile >= end) return;
  summary_tile<D, FMT, PAGED, true>(A, b, kvh, 1, at * tile, tile, 0, end, nullptr, s_ends);
}

struct ReadArgs {
  const unsigned char* buf[2];
  uint16_t* out[2];
  int64_t scale_off;
  const int32_t* seq_lens;
  const int32_t* first;
  RowMap M;
  int n_rows;
};

// One lane per 8 columns of a row, kReadRows rows of a lane under way.  Bound by the bytes: 8 x 16K tokens of e2m1 at 64 columns, 340 MB, 59 us (5.7 TB/s);
// ragged 7 x 0.5K - 5K of e4m3 on pages, 119 MB, 26 (with one row of a lane
// 72 and 30).
constexpr int kReadRows = 4;
template <int D, int FMT, bool PAGED>
__global__ __launch_bounds__(kWriteThreads) void read_kernel(ReadArgs A) {
  constexpr int LPR = D / 8, TT = kWriteThreads / LPR;
  const int b = blockIdx.y, tid = threadIdx.x, c = tid % LPR, r = tid / LPR;
  const int at = blockIdx.x / A.M.Hkv, kvh = blockIdx.x - at * A.M.Hkv;
  const int first = A.first ? max(A.first[b], 0) : 0, end = min(max(A.seq_lens[b], 0), A.M.n_max);
  const int j0 = at * TT * kReadRows, rows = first < end ? min(A.n_rows, end - first) : 0;
  if (j0 >= rows) return;
  const unsigned char* buf = A.buf[blockIdx.z];
  int blk[kReadRows];
  Chunk<FMT> code[kReadRows];
  uint32_t byte[kReadRows];
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) blk[u] = row_block<PAGED>(A.M, b, first + min(j0 + u * TT + r, rows - 1));
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const RowAt row = row_at<PAGED>(A.M, b, kvh, first + min(j0 + u * TT + r, rows - 1), blk[u]);
    byte[u] = 0;
    if constexpr (FMT != VATT_KV_BF16) byte[u] = buf[A.scale_off + row.scales * (D / 32) + c / 4];
    code[u] = load_chunk<FMT>(buf + row.row * kRowBytes<FMT, D> + c * (kRowBytes<FMT, D> / LPR));
  }
  uint16_t* out = A.out[blockIdx.z] + ((int64_t)b * A.M.Hkv + kvh) * A.n_rows * D + 8 * c;
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const int j = j0 + u * TT + r;
    if (j < rows) *reinterpret_cast<uint4*>(out + (int64_t)j * D) = chunk_bf16<FMT>(code[u], byte[u]);
  }
}

// Calls f with the plan's head_dim, format and layout as constants.
template <class F>
hipError_t with_format(const Plan& pl, F f) {
  auto layout = [&](auto d, auto fmt) {
    return pl.p.kv_layout == VATT_LAYOUT_PAGED ? f(d, fmt, std::true_type{}) : f(d, fmt, std::false_type{});
  };
  auto format = [&](auto d) {
    if (pl.kv_format == VATT_KV_E4M3) return layout(d, std::integral_constant<int, VATT_KV_E4M3>{});
    if (pl.kv_format == VATT_KV_E2M1) return layout(d, std::integral_constant<int, VATT_KV_E2M1>{});
    return layout(d, std::integral_constant<int, VATT_KV_BF16>{});
  };
  return pl.p.head_dim == 128 ? format(std::integral_constant<int, 128>{}) : format(std::integral_constant<int, 64>{});
}

void set_blocks(const Plan& pl, WriteArgs& A) {
  A.block_shift = 31 - __builtin_clz(pl.block_tokens);
  A.head_blocks = pl.p.kv_layout == VATT_LAYOUT_PAGED ? pl.p.page_size / pl.block_tokens : (pl.p.n_max + pl.block_tokens - 1) / pl.block_tokens;
}

}  // namespace

hipError_t launch_write(const Plan& pl, const void* q, const void* k_new, const void* v_new, int64_t q_stride, int64_t k_stride,
                        int64_t v_stride, int n_new, const int32_t* first, const int32_t* new_lens, void* k, void* v,
                        const int32_t* block_table, void* summary, void* out_q, int32_t* out_lens, hipStream_t st) {
  WriteArgs A = {};
  A.q = static_cast<const uint16_t*>(q);
  A.k_new = static_cast<const uint16_t*>(k_new);
  A.v_new = static_cast<const uint16_t*>(v_new);
  A.q_stride = q_stride;
  A.k_stride = k_stride;
  A.v_stride = v_stride;
  A.first = first;
  A.new_lens = new_lens;
  A.k = static_cast<unsigned char*>(k);
  A.v = static_cast<unsigned char*>(v);
  A.scale_off = (int64_t)kv_scale_offset(pl);
  A.summary = static_cast<uint16_t*>(summary);
  A.out_q = static_cast<uint16_t*>(out_q);
  A.out_lens = out_lens;
  A.M = row_map(pl, block_table);
  A.n_new = n_new;
  A.Hq = pl.p.n_q_heads;
  A.Hkv = pl.p.n_kv_heads;
  A.rot = pl.rotary_dim;
  A.pairs = pl.rotary_pairs;
  A.attention = pl.rotary_attention;
  std::copy(pl.rotary_freq, pl.rotary_freq + 64, A.freq);
  const int tokens = kWriteThreads / (pl.p.head_dim / 8), batch = pl.p.batch;
  if (summary) {
    set_blocks(pl, A);
    const int tile = std::max(pl.block_tokens, tokens), tiles = (n_new + tile - 2) / tile + 1;
    A.k_heads = std::max(1, std::min({8, A.Hkv, (int)((int64_t)batch * tiles * A.Hkv / (8 * pl.num_cus))}));
    A.k_groups = (A.Hkv + A.k_heads - 1) / A.k_heads;
    A.k_jobs = tiles * A.k_groups;
  }
  while ((1 << A.row_tokens_shift) < std::min(n_new, kRowTokens)) ++A.row_tokens_shift;
  const int per_pass = tokens >> A.row_tokens_shift, tiles = (n_new + (1 << A.row_tokens_shift) - 1) >> A.row_tokens_shift;
  const int q_passes = out_q ? (A.Hq + per_pass - 1) / per_pass : 0, kv_passes = (A.Hkv + per_pass - 1) / per_pass;
  A.row_passes = std::max(1, std::min({8, std::max(q_passes, kv_passes), (int)((int64_t)batch * tiles * (q_passes + kv_passes) / (8 * pl.num_cus))}));
  A.q_groups = (q_passes + A.row_passes - 1) / A.row_passes;
  A.v_groups = (kv_passes + A.row_passes - 1) / A.row_passes;
  A.row_groups = A.q_groups + A.v_groups + (summary ? 0 : A.v_groups);
  const dim3 grid(A.k_jobs + tiles * A.row_groups, batch);
  return with_format(pl, [&](auto d, auto fmt, auto paged) {
    hipLaunchKernelGGL((write_kernel<d(), fmt(), paged()>), grid, dim3(kWriteThreads), 0, st, A);
    return hipGetLastError();
  });
}

hipError_t launch_block_summary(const Plan& pl, const void* k, const int32_t* block_table, const int32_t* seq_lens, void* summary,
                                hipStream_t st) {
  WriteArgs A = {};
  A.k = static_cast<unsigned char*>(const_cast<void*>(k));
  A.first = seq_lens;
  A.scale_off = (int64_t)kv_scale_offset(pl);
  A.summary = static_cast<uint16_t*>(summary);
  A.M = row_map(pl, block_table);
  A.Hkv = pl.p.n_kv_heads;
  set_blocks(pl, A);
  const int tile = std::max(pl.block_tokens, kWriteThreads / (pl.p.head_dim / 8));
  const dim3 grid((pl.p.n_max + tile - 1) / tile * A.Hkv, pl.p.batch);
  return with_format(pl, [&](auto d, auto fmt, auto paged) {
    hipLaunchKernelGGL((summary_kernel<d(), fmt(), paged()>), grid, dim3(kWriteThreads), 0, st, A);
    return hipGetLastError();
  });
}

hipError_t launch_read(const Plan& pl, const void* k, const void* v, const int32_t* block_table, const int32_t* seq_lens,
                       const int32_t* first, int n_rows, void* out_k, void* out_v, hipStream_t st) {
  ReadArgs A = {};
  int n = 0;
  if (out_k) {
    A.buf[n] = static_cast<const unsigned char*>(k);
    A.out[n++] = static_cast<uint16_t*>(out_k);
  }
  if (out_v) {
    A.buf[n] = static_cast<const unsigned char*>(v);
    A.out[n++] = static_cast<uint16_t*>(out_v);
  }
  A.scale_off = (int64_t)kv_scale_offset(pl);
  A.seq_lens = seq_lens;
  A.first = first;
  A.M = row_map(pl, block_table);
  A.n_rows = n_rows;
  const int tokens = kWriteThreads / (pl.p.head_dim / 8) * kReadRows;
  const dim3 grid((n_rows + tokens - 1) / tokens * A.M.Hkv, pl.p.batch, n);
  return with_format(pl, [&](auto d, auto fmt, auto paged) {
    hipLaunchKernelGGL((read_kernel<d(), fmt(), paged()>), grid, dim3(kWriteThreads), 0, st, A);
    return hipGetLastError();
  });
}

}  // namespace vatt
