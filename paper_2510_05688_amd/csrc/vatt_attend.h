// Attention with few query vectors: over the tokens of listed blocks, over all tokens of a quantised cache, or over the first tokens and a
// window.
#pragma once

#include <algorithm>

#include "vatt_format.h"

namespace vatt {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t lower_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

constexpr int kAttendThreads = 256, kAttendWaves = kAttendThreads / kWave;
constexpr int kUnit = 32;          // keys that a wave takes at a time
constexpr int kSlots = 1024;       // groups of 8 tokens that a workgroup looks up at a time
constexpr int kSplitsMax = 128;
constexpr int kAgainRows = 128;     // rows that are added up in one sum where a result is worked out again
constexpr int kNowhere = 0x7fffff00;  // token of a group that does not exist: beyond every sequence

// Which tokens: all of them, those of listed blocks, or the first `sink` and the last `window` up to each query's own.
enum { kAllTokens, kListedBlocks, kFirstAndWindow };

struct AttendArgs {
  const uint16_t* q;
  const unsigned char* k;
  const unsigned char* v;
  int64_t scale_off;
  const int32_t* seq_lens;
  const int32_t* blocks;
  const int32_t* block_count;
  float* part;     // [B * q_len * Hq][splits][d] or, dealt out, [slot_rows][slots][d]: sums of the weighted V rows
  float2* part_ml;  // the same without d: (max in units of log 2, sum of the weights); max -Inf: no token seen
  float* out_o;
  float* out_lse;
  RowMap M;
  int Hq, Hkv, q_len, splits, rounds, capacity, block_shift;
  float log2_scale;  // softmax scale / ln 2
  // kFirstAndWindow:
  int sink, window, out_bf16, batch;
  int2* jobs;                 // [rounds][Hkv][B]: the first of a job's places for sums, and how many it has
  int workgroups, slots, slot_rows;  // dealt out: workgroups at most, places for sums, vectors of each
  int64_t q_stride;         // elements between query tokens
  const int32_t* first;     // the first query token's position; nullptr: the q_len newest tokens of seq_lens
  const int32_t* new_lens;  // how many query tokens count; nullptr: all
};

// The query tokens of a sequence (kFirstAndWindow): the first one's position, and how many there are.  One at a position below 0 sees
// the first token.
struct QueryTokens {
  int first, count;
};
__device__ __forceinline__ QueryTokens query_tokens(const AttendArgs& A, int seq) {
  if (!A.first) return {min(max(A.seq_lens[seq], 1), A.M.n_max) - A.q_len, A.q_len};
  const int first = A.first[seq], count = A.new_lens ? min(max(A.new_lens[seq], 0), A.q_len) : A.q_len;
  if (first < 0 || first >= A.M.n_max) return {0, 0};
  return {first, min(count, A.M.n_max - first)};
}

// A list of tokens in groups of 8: how many groups, and the first token of each (kNowhere where there is none).
struct TokenList {
  const int32_t* blocks;
  int count, capacity, shift, n;  // n: tokens of the sequence that count
  int lo, sink, head, from;       // kFirstAndWindow: those from `lo` on and those below `sink`, in `head` groups and in those from `from` on
  __device__ __forceinline__ bool seen(int tok) const { return tok >= lo || tok < sink; }
};
// The tokens that are seen by queries of which the last sees n tokens and the first those from `lo` on.
template <int KIND>
__device__ __forceinline__ TokenList token_list(const AttendArgs& A, int vb, int kvh, int n, int lo = 0) {
  TokenList L = {nullptr, 0, A.capacity, A.block_shift, n, 0, 0, 0, 0};
  if constexpr (KIND == kListedBlocks) {
    const int64_t row = (int64_t)vb * A.Hkv + kvh;
    L.blocks = A.blocks + row * A.capacity;
    L.count = min(max(A.block_count[row], 0), A.capacity) << (A.block_shift - 3);
  } else if constexpr (KIND == kFirstAndWindow) {
    L.lo = lo;
    L.sink = A.sink;
    L.from = lo / 8;
    L.head = min((min(A.sink, lo) + 7) / 8, L.from);
    L.count = L.head + (n + 7) / 8 - L.from;
  } else {
    L.count = (n + 7) / 8;
  }
  return L;
}
// (an entry is read without waiting for the length of its list)
template <int KIND>
__device__ __forceinline__ int entry_of(const TokenList& L, int group) {
  return KIND == kListedBlocks ? L.blocks[min(group >> (L.shift - 3), L.capacity - 1)] : 0;
}
template <int KIND>
__device__ __forceinline__ int token_of(const TokenList& L, int group, int blk) {
  if (group >= L.count) return kNowhere;
  if constexpr (KIND == kFirstAndWindow) return (group < L.head ? group : group - L.head + L.from) * 8;
  if constexpr (KIND == kAllTokens) return group * 8;
  if ((uint32_t)blk > (uint32_t)(L.n - 1) >> L.shift) return kNowhere;
  // (nor is there a group behind the last token of the last block: a contiguous cache has no scales for it)
  const int tok = (blk << L.shift) + ((group << 3) & ((1 << L.shift) - 1));
  return tok < L.n ? tok : kNowhere;
}

// STREAM: read once.  All tokens' rows are with up to 32 query vectors per KV head (with more, every round of 32 reads them again, with the
// hint too: 4 x 32K in e4m3 with 32 vectors 70 us, with 64 111); those of lists may be in the lists of several query tokens (16 x 32K
// tokens in e4m3 192 us without the hint, 181 with it; lists of two query tokens, 12 x 4K - 64K, 29.0 without, 31.1 with).
template <bool STREAM>
__device__ __forceinline__ uint4 load_16(const unsigned char* p) {
  return STREAM ? load_stream_16(reinterpret_cast<const uint16_t*>(p)) : *reinterpret_cast<const uint4*>(p);
}
template <bool STREAM>
__device__ __forceinline__ uint2 load_8(const unsigned char* p) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  if constexpr (!STREAM) return *reinterpret_cast<const uint2*>(p);
  const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
  return make_uint2(x.x, x.y);
}

// The scale bytes of one row (d / 32 of them).
template <int D>
__device__ __forceinline__ uint32_t row_scales(const unsigned char* p) {
  if constexpr (D == 128) return *reinterpret_cast<const uint32_t*>(p);
  else return *reinterpret_cast<const uint16_t*>(p);
}

// The tokens of one list again for one head, by the whole workgroup: dot products, every row only where it is seen.
template <int D, int FMT, bool PAGED, int KIND, int WAVES>
__device__ __forceinline__ void attend_again(const AttendArgs& A, const uint16_t* q, int seq, int kvh, const TokenList& L, float (&s_acc)[WAVES][D],
                                             float (&s_m)[WAVES], float (&s_l)[WAVES]) {
  constexpr int LPR = D / 8, RPW = kWave / LPR;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane % LPR, rsub = lane / LPR;
  const uint4 qv = *reinterpret_cast<const uint4*>(q + sub * 8);
  const uint32_t qw[4] = {qv.x, qv.y, qv.z, qv.w};
  float m = -INFINITY, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  // (sums of up to kAgainRows rows are added up, not all rows one by one: see lrest)
  float l_now = 0.f, now[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  int rows = 0;
  auto add_now = [&]() {
    l += l_now;
    l_now = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      acc[j] += now[j];
      now[j] = 0.f;
    }
    rows = 0;
  };
  for (int64_t i = wave * RPW + rsub; i < (int64_t)L.count * 8; i += WAVES * RPW) {
    const int group = (int)(i >> 3), tok = token_of<KIND>(L, group, entry_of<KIND>(L, group)) + (int)(i & 7);
    if (tok >= L.n || (KIND == kFirstAndWindow && !L.seen(tok))) continue;
    const RowAt at = row_at<PAGED>(A.M, seq, kvh, tok, row_block<PAGED>(A.M, seq, tok));
    uint4 x[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const unsigned char* buf = y ? A.v : A.k;
      uint32_t byte = 0;
      if constexpr (FMT != VATT_KV_BF16) byte = buf[A.scale_off + at.scales * (D / 32) + sub / 4];
      x[y] = chunk_bf16<FMT>(load_chunk<FMT>(buf + at.row * kRowBytes<FMT, D> + sub * (kRowBytes<FMT, D> / LPR)), byte);
    }
    const uint32_t kw[4] = {x[0].x, x[0].y, x[0].z, x[0].w}, vw[4] = {x[1].x, x[1].y, x[1].z, x[1].w};
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) s += bf16_lo(kw[j]) * bf16_lo(qw[j]) + bf16_hi(kw[j]) * bf16_hi(qw[j]);
    s = group_sum<LPR>(s) * A.log2_scale;
    const float mnew = fmaxf(m, s), shift = mnew == -INFINITY ? -3.0e38f : mnew;
    const float alpha = m == -INFINITY ? 0.f : m == shift ? 1.f : __builtin_amdgcn_exp2f(m - shift);
    const float p = __builtin_amdgcn_exp2f(s - shift);
    m = shift;
    l *= alpha;
    l_now = l_now * alpha + p;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[2 * j] *= alpha;
      acc[2 * j + 1] *= alpha;
      now[2 * j] = now[2 * j] * alpha + p * bf16_lo(vw[j]);
      now[2 * j + 1] = now[2 * j + 1] * alpha + p * bf16_hi(vw[j]);
    }
    if (++rows == kAgainRows) add_now();
  }
  add_now();
  float all = m;
#pragma unroll
  for (int o = LPR; o < kWave; o <<= 1) all = fmaxf(all, __shfl_xor(all, o));
  const float f = m == -INFINITY ? 0.f : m == all ? 1.f : __builtin_amdgcn_exp2f(m - all);
  l *= f;
#pragma unroll
  for (int c = 0; c < 8; ++c) acc[c] *= f;
#pragma unroll
  for (int o = LPR; o < kWave; o <<= 1) {
    l += __shfl_xor(l, o);
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[c] += __shfl_xor(acc[c], o);
  }
  __syncthreads();
  if (rsub == 0) {
#pragma unroll
    for (int c = 0; c < 8; ++c) s_acc[wave][sub * 8 + c] = acc[c];
  }
  if (lane == 0) {
    s_m[wave] = all;
    s_l[wave] = l;
  }
  __syncthreads();
}

// N consecutive values of the output, from value `at` on, in the call's type.
template <int N>
__device__ __forceinline__ void store_row(const AttendArgs& A, int64_t at, const float (&x)[N]) {
  if (A.out_bf16) {
    uint16_t* out = reinterpret_cast<uint16_t*>(A.out_o) + at;
    if constexpr (N == 4) *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    else out[0] = (uint16_t)pack_bf16(x[0], x[0]);
  } else {
    if constexpr (N == 4) *reinterpret_cast<float4*>(A.out_o + at) = make_float4(x[0], x[1], x[2], x[3]);
    else A.out_o[at] = x[0];
  }
}

// Attention with the query vectors of a KV head on the matrix cores, 32 keys of a wave at a time:
//   S [keys x vectors] = K Q^T   and   O^T [d x vectors] += V^T P^T,   P = exp(S - m),
// both v_mfma_f32_16x16x32_bf16 (operand lane l: row or column l % 16, eight inner elements; result lane l: column l % 16, rows
// 4 (l / 16) .. + 3).  The result layout of S is the operand layout of P when lane group g = l / 16 takes keys 4 g + r and 16 + 4 g + r
// as inner elements r and 4 + r.
//   * Codes become bf16 in registers, exactly, with their scales.  Which columns of a row are inner elements of which step of the first
//     product is free as long as K and q agree: every lane loads 16 bytes of its row and takes the 8 to 32 values in them as one to
//     four steps.
//   * V is not transposed: a lane loads d / 16 columns of the eight rows of its group and pairs them by rows in registers.
//   * P goes in as three bf16 terms that add up to the fp32 value, so that the sums keep fp32 accuracy.  Where the vectors fill five columns at
//     most, their three terms are columns of one product (PACK 3); with up to eight, two of them are (PACK 2).
// The running maximum of a column moves only when a score passes it by more than kLazy.
// What bounds it: the rows' bytes.  All tokens of 16 x 32K in e4m3 (1.1 GB) take 170 to 180 us, by the clock (6.2 - 6.5 TB/s), where the
// same loads without the products and exponentials take 164; lists of 12 x 4K - 64K tokens with two queries each (98 MB in pieces of 2 KB, with scales of 64
// bytes apart from them) 28 us, loads alone 22.  Half or twice as many workgroups, three of them on a CU instead of two, and a least
// number of chunks for each made no difference or were slower.
// A workgroup's part of the work: chunks first, first + step, .. of a token list, at most `count` of them.
struct AttendPart {
  int z, kvh, round;  // sequence (kListedBlocks: sequence and query token), KV head, which vectors
  int first, step, count;
  int slot;    // where the sums go
  bool whole;  // kFirstAndWindow: these are all tokens, and the results are written
  QueryTokens queries;  // kFirstAndWindow
};
template <int D, int FMT, bool PAGED, int KIND, int NQT, int PACK, int WAVES>
__device__ __forceinline__ void attend_part(const AttendArgs& A, const AttendPart& part) {
  constexpr int kThreads = WAVES * kWave;
  constexpr int kChunk = 4 * WAVES;  // groups of 8 tokens that a workgroup takes at a time: a unit for each wave
  static_assert(WAVES == 4 || WAVES == 8, "see the end");
  constexpr bool LIST = KIND == kListedBlocks, RANGE = KIND == kFirstAndWindow;
  constexpr int S = D / 32;  // steps over a row of K
  constexpr int E = D / 16;  // values of a V row per lane = tiles over the head dimension
  constexpr int ROW = kRowBytes<FMT, D>;
  constexpr int KB = ROW / 4 < 16 ? ROW / 4 : 16, KL = ROW / 4 / KB;  // K: bytes per load, loads per lane and row
  constexpr int STEPS = S / KL;                                       // steps that one load holds
  constexpr int VB = ROW / 16;                                        // V: bytes per lane and row
  constexpr int VW = VB < 4 ? 1 : VB / 4;
  constexpr bool QUANT = FMT != VATT_KV_BF16;
  constexpr float kLazy = 8.0f;
  static_assert(PACK == 1 || NQT == 1, "packed terms are of one tile");

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, g4 = lane >> 4;
  const int kvh = part.kvh, round = part.round;
  const int G = A.Hq / A.Hkv, Q = A.q_len;
  const int seq = LIST ? seq_of_pair(part.z, Q) : part.z;
  QueryTokens T = {0, Q};
  if constexpr (RANGE) T = part.queries;
  const int n_seq = RANGE ? max(T.first + T.count, 1) : min(max(A.seq_lens[seq], 1), A.M.n_max);
  // LIST: the vectors are the heads of one query token; else those of all query tokens
  const int t0 = LIST ? part.z - seq * Q : 0, vectors = LIST ? G : T.count * G;
  const int n = LIST ? max(n_seq - (Q - 1 - t0), 1) : n_seq;
  const int c_base = round * 16 * NQT;
  if (RANGE && c_base >= vectors) return;
  const TokenList L = token_list<KIND>(A, part.z, kvh, n, RANGE ? max(max(T.first + 1, 1) - A.window, 0) : 0);

  __shared__ __align__(16) int s_tok[kSlots];
  __shared__ __align__(16) int s_at[kSlots];
  __shared__ float4 s_o[4][4][E / 4][kWave];
  __shared__ float s_m[4][16], s_l[4][16];
  // (with two tiles of vectors the queries stay in LDS: there are no registers for them)
  constexpr bool kQueriesInLds = NQT > 1;
  __shared__ uint4 s_q[kQueriesInLds ? NQT * S : 1][kWave];

  uint4 bq[kQueriesInLds ? 1 : NQT][S];
  int seen[NQT];
  int least = n;
#pragma unroll
  for (int nt = 0; nt < NQT; ++nt) {
    // (columns beyond the last vector repeat it and are not stored; with PACK > 1 they are its further terms)
    const int c = PACK > 1 ? i16 % vectors : min(c_base + nt * 16 + i16, vectors - 1);
    const int t = t0 + c / G, g = c % G;
    const uint16_t* src = RANGE ? A.q + ((int64_t)seq * Q + t) * A.q_stride + ((int64_t)kvh * G + g) * D
                                : A.q + (((int64_t)seq * Q + t) * A.Hq + (int64_t)kvh * G + g) * D;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const uint4 x = *reinterpret_cast<const uint4*>(src + (s / STEPS) * 4 * (STEPS * 8) + g4 * (STEPS * 8) + (s % STEPS) * 8);
      if constexpr (!kQueriesInLds) bq[nt][s] = x;
      else if (wave == 0) s_q[nt * S + s][lane] = x;  // (a barrier follows before the first unit)
    }
    seen[nt] = max(n_seq - ((RANGE ? T.count : Q) - 1 - t), 1);
  }
  if (!LIST) least = max(n_seq - ((RANGE ? T.count : Q) - 1), 1);
  const int last_lo = RANGE ? n - A.window : 0;  // the last query's window begins here

  // what a lane takes away from its weights before they are cut to bf16: nothing, their leading term, the leading two
  const int term = PACK > 1 ? i16 / vectors : 0;
  const uint32_t first_term = term >= 1 ? 0xffff0000u : 0u, second_term = PACK == 3 && term >= 2 ? 0xffff0000u : 0u;
  const uint32_t last_term = PACK == 2 && term == 1 ? 0xffffffffu : 0u;

  f32x4_t acc[NQT][E];
  // Running maxima of the scores in units of log 2, and sums of the weights, lrun + lrest: the 8 weights of a step are added up by themselves, and what
  // their sum loses when it is added to lrun goes to lrest.  One by one the weights of 170K keys of equal score would lose 1e-4 of their sum.
  float mrun[NQT], lrun[NQT], lrest[NQT];
  bool any[NQT];
#pragma unroll
  for (int nt = 0; nt < NQT; ++nt) {
    mrun[nt] = -INFINITY;
    lrun[nt] = lrest[nt] = 0.f;
    any[nt] = false;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[nt][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // Rows by groups of 8: paged, the group's place among all physical rows / 8; contiguous, its first token, behind a uniform base.
  const int page8 = A.M.page_shift - 3;
  const int64_t head = (int64_t)seq * A.Hkv + kvh;
  const unsigned char* k_base = A.k + (PAGED ? 0 : head * A.M.n_max * ROW);
  const unsigned char* v_base = A.v + (PAGED ? 0 : head * A.M.n_max * ROW);
  const unsigned char* ks_base = A.k + A.scale_off + (PAGED ? 0 : head * A.M.n_scales * (D / 32));
  const unsigned char* vs_base = A.v + A.scale_off + (PAGED ? 0 : head * A.M.n_scales * (D / 32));
  // (a contiguous cache may end inside a group of 8: no row behind the sequence's last one)
  auto row_of = [&](int slot, int r) {
    if constexpr (PAGED) return (uint64_t)(uint32_t)s_at[slot] * (uint32_t)(8 * ROW) + (uint32_t)(r * ROW);
    else return (uint32_t)(min(s_at[slot] + r, n_seq - 1) * ROW);
  };
  auto scales_of = [&](int slot, int r) {
    if constexpr (PAGED) return (uint64_t)(uint32_t)s_at[slot] * (uint32_t)(8 * (D / 32)) + (uint32_t)(r * (D / 32));
    else return (uint32_t)((s_at[slot] + r) * (D / 32));
  };
  uint32_t kr[2][KL][KB / 4], ks[2], vr[8][VW], vs[2][QUANT ? D / 32 : 1];
  auto load_k = [&](int s0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int slot = s0 + 2 * t + (i16 >> 3), r = i16 & 7;
      const unsigned char* p = k_base + (row_of(slot, r) + g4 * KB);
#pragma unroll
      for (int l = 0; l < KL; ++l) {
        if constexpr (KB == 16) {
          const uint4 x = load_16<!LIST>(p + l * 4 * KB);
          kr[t][l][0] = x.x; kr[t][l][1] = x.y; kr[t][l][2] = x.z; kr[t][l][3] = x.w;
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(p);
          kr[t][l][0] = x.x; kr[t][l][1] = x.y;
        }
      }
      if constexpr (QUANT) ks[t] = row_scales<D>(ks_base + scales_of(slot, r));
    }
  };
  auto load_v = [&](int s0) {
    auto row = [&](int j, const unsigned char* p) {
      if constexpr (VB == 16) {
        const uint4 x = load_16<!LIST>(p);
        vr[j][0] = x.x; vr[j][1] = x.y; vr[j][2] = x.z; vr[j][3] = x.w;
      } else if constexpr (VB == 8) {
        const uint2 x = load_8<!LIST>(p);
        vr[j][0] = x.x; vr[j][1] = x.y;
      } else if constexpr (VB == 4) {
        vr[j][0] = *reinterpret_cast<const uint32_t*>(p);
      } else {
        vr[j][0] = *reinterpret_cast<const uint16_t*>(p);
      }
    };
    const int half = (g4 & 1) * 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int slot = s0 + 2 * t + (g4 >> 1);
      if constexpr (PAGED) {  // (four rows of one page)
        const unsigned char* p = v_base + (row_of(slot, half) + i16 * VB);
#pragma unroll
        for (int j = 0; j < 4; ++j) row(4 * t + j, p + j * ROW);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) row(4 * t + j, v_base + (row_of(slot, half + j) + i16 * VB));
      }
    }
    if constexpr (QUANT) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {  // the scales of four rows, a whole number of words
        const unsigned char* p = vs_base + scales_of(s0 + 2 * t + (g4 >> 1), half);
        if constexpr (D == 128) {
          const uint4 x = *reinterpret_cast<const uint4*>(p);
          vs[t][0] = x.x; vs[t][1] = x.y; vs[t][2] = x.z; vs[t][3] = x.w;
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(p);
          vs[t][0] = x.x; vs[t][1] = x.y;
        }
      }
    }
  };

  auto group_of = [&](int i) { return (part.first + (i / kChunk) * part.step) * kChunk + i % kChunk; };
  const int entry0 = entry_of<KIND>(L, group_of(tid));
  const int chunks = (L.count + kChunk - 1) / kChunk, left = part.first < chunks ? (chunks - part.first + part.step - 1) / part.step : 0;
  const int mine = RANGE ? min(left, part.count) : left;
  for (int c0 = 0; c0 < mine; c0 += kSlots / kChunk) {
    const int c_n = min(kSlots / kChunk, mine - c0);
    if (c0 > 0) __syncthreads();
    for (int i = tid; i < c_n * kChunk; i += kThreads) {
      const int group = group_of(c0 * kChunk + i);
      const int tok = token_of<KIND>(L, group, c0 == 0 && i == tid ? entry0 : entry_of<KIND>(L, group)), safe = tok == kNowhere ? 0 : tok;
      s_tok[i] = tok;
      if constexpr (PAGED) s_at[i] = (int)((((uint32_t)row_block<PAGED>(A.M, seq, safe) * A.Hkv + kvh) << page8) + ((safe & ((1 << A.M.page_shift) - 1)) >> 3));
      else s_at[i] = safe;
    }
    __syncthreads();
    load_k(wave * 4);
    load_v(wave * 4);
    for (int c = 0; c < c_n; ++c) {
      const int s0 = c * kChunk + wave * 4;
      const bool more = c + 1 < c_n;
      int my = lane;
      if constexpr (kQueriesInLds) asm volatile("" : "+v"(my));  // (read again in every round, not kept)
      f32x4_t sc[NQT][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int nt = 0; nt < NQT; ++nt) sc[nt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < S; ++s) {
          uint4 ka;
          const uint32_t* w = kr[t][s / STEPS];
          if constexpr (FMT == VATT_KV_BF16) {
            ka = make_uint4(w[0], w[1], w[2], w[3]);
          } else {
            // (the scale group of the columns of this load and lane; a load spans 4 lanes' 8 STEPS columns each)
            const int group = ((s / STEPS) * 4 * STEPS * 8 + g4 * STEPS * 8 + (s % STEPS) * 8) / 32;
            const float scale = scale_of((ks[t] >> (8 * group)) & 255u);
            if constexpr (FMT == VATT_KV_E4M3) {
              const uint2 x = e4m3_to_bf16(w[(s % STEPS) * 2], scale), y = e4m3_to_bf16(w[(s % STEPS) * 2 + 1], scale);
              ka = make_uint4(x.x, x.y, y.x, y.y);
            } else {
              const uint32_t x = w[s % STEPS];
              ka = make_uint4(e2m1_to_bf16<0>(x, scale), e2m1_to_bf16<1>(x, scale), e2m1_to_bf16<2>(x, scale), e2m1_to_bf16<3>(x, scale));
            }
          }
#pragma unroll
          for (int nt = 0; nt < NQT; ++nt) {
            uint4 b;
            if constexpr (kQueriesInLds) b = s_q[nt * S + s][my];
            else b = bq[nt][s];
            sc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ka), __builtin_bit_cast(bf16x8_t, b), sc[nt][t], 0, 0, 0);
          }
        }
      }
      if (more) load_k(s0 + kChunk);
      const int4 tok = *reinterpret_cast<const int4*>(&s_tok[s0]);
      const int far = max(max(tok.x, tok.y), max(tok.z, tok.w)) + 8;
      bool edge = far > least;  // some column does not see all of the 32 keys
      if constexpr (RANGE) edge |= min(min(tok.x, tok.y), min(tok.z, tok.w)) < last_lo;
      // tokens of this lane's result rows: 4 g + r, then 16 + 4 g + r
      const int ta = ((g4 >> 1) ? tok.y : tok.x) + (g4 & 1) * 4, tb = ((g4 >> 1) ? tok.w : tok.z) + (g4 & 1) * 4;
      constexpr int TERMS = PACK == 3 ? 1 : PACK == 2 ? 2 : 3;  // second products that the weights take
      uint4 pb[NQT][TERMS];
#pragma unroll
      for (int nt = 0; nt < NQT; ++nt) {
        float s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = sc[nt][j >> 2][j & 3];
        if (edge) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int key = (j < 4 ? ta : tb) + (j & 3);
            bool ok = key < seen[nt];
            if constexpr (RANGE) ok = ok && (key >= seen[nt] - A.window || key < A.sink);
            s[j] = ok ? s[j] : -INFINITY;
            any[nt] |= ok;
          }
        } else {
          any[nt] = true;
        }
        float top = s[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
        top *= A.log2_scale;
        if (__ballot(top > mrun[nt] + kLazy)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float mnew = fmaxf(mrun[nt], top);
          const float alpha = mrun[nt] == mnew ? 1.f : __builtin_amdgcn_exp2f(mrun[nt] - mnew);
          mrun[nt] = mnew;
          lrun[nt] *= alpha;
          lrest[nt] *= alpha;
#pragma unroll
          for (int e = 0; e < E; ++e) acc[nt][e] *= alpha;
        }
        const float m = mrun[nt] == -INFINITY ? 0.f : mrun[nt];  // (so far every score is -Inf: weights 0)
        uint32_t w[TERMS][8];
        float step = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[j], A.log2_scale, -m));
          step += p;
          if constexpr (PACK > 1) {
            float r = p - __uint_as_float(__float_as_uint(p) & first_term);
            if constexpr (PACK == 3) r -= __uint_as_float(__float_as_uint(r) & second_term);
            w[0][j] = __float_as_uint(r);
            if constexpr (PACK == 2) w[1][j] = __float_as_uint(r - __uint_as_float(__float_as_uint(r) & 0xffff0000u)) & last_term;
          } else {
            const float r1 = p - __uint_as_float(__float_as_uint(p) & 0xffff0000u);
            const float r2 = r1 - __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
            w[0][j] = __float_as_uint(p);
            w[1][j] = __float_as_uint(r1);
            w[2][j] = __float_as_uint(r2);
          }
        }
        const float sum = lrun[nt] + step, of_step = sum - lrun[nt];
        lrest[nt] += (lrun[nt] - (sum - of_step)) + (step - of_step);
        lrun[nt] = sum;
#pragma unroll
        for (int x = 0; x < TERMS; ++x)
          pb[nt][x] = make_uint4(upper_halves(w[x][0], w[x][1]), upper_halves(w[x][2], w[x][3]), upper_halves(w[x][4], w[x][5]),
                                 upper_halves(w[x][6], w[x][7]));
      }
      float vscale[8];
      if constexpr (QUANT) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t w = D == 128 ? vs[j >> 2][(j & 3) % (D / 32)] : vs[j >> 2][(j & 3) / 2] >> (16 * (j & 1));
          vscale[j] = scale_of((w >> (8 * (i16 * E / 32))) & 255u);
        }
      }
#pragma unroll
      for (int x = 0; x < E / 2; ++x) {  // columns 2 x and 2 x + 1 of the lane
        uint32_t col[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if constexpr (FMT == VATT_KV_BF16) {
            col[j] = vr[j][x];
          } else if constexpr (FMT == VATT_KV_E4M3) {
            const uint2 y = e4m3_to_bf16(vr[j][x / 2], vscale[j]);
            col[j] = (x & 1) ? y.y : y.x;
          } else {
            col[j] = x == 0 ? e2m1_to_bf16<0>(vr[j][0], vscale[j]) : x == 1 ? e2m1_to_bf16<1>(vr[j][0], vscale[j])
                   : x == 2 ? e2m1_to_bf16<2>(vr[j][0], vscale[j]) : e2m1_to_bf16<3>(vr[j][0], vscale[j]);
          }
        }
        if (edge) {  // (rows that nobody sees: whatever lies there has no say)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int key = (j < 4 ? ta : tb) + (j & 3);
            col[j] = key < n && (!RANGE || L.seen(key)) ? col[j] : 0u;
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t a[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) a[j] = h ? upper_halves(col[2 * j], col[2 * j + 1]) : lower_halves(col[2 * j], col[2 * j + 1]);
          const uint4 va = make_uint4(a[0], a[1], a[2], a[3]);
#pragma unroll
          for (int nt = 0; nt < NQT; ++nt) {
#pragma unroll
            for (int y = TERMS - 1; y >= 0; --y)
              acc[nt][2 * x + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, va), __builtin_bit_cast(bf16x8_t, pb[nt][y]),
                                                                           acc[nt][2 * x + h], 0, 0, 0);
          }
        }
      }
      if (more) load_v(s0 + kChunk);
    }
  }

  // The waves' sums together, one 16-vector tile at a time, in the result layout (of eight waves the upper four's go to the lower four first):
  // wave w finishes rows 4 g + w.
  uint32_t odd = 0;  // vectors with an Inf or a NaN
#pragma unroll
  for (int nt = 0; nt < NQT; ++nt) {
    float l = lrun[nt] + lrest[nt];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    int saw = any[nt];
    saw |= __shfl_xor(saw, 16);
    saw |= __shfl_xor(saw, 32);
    // (a piece all of whose scores are -Inf is no piece without a token)
    float m_own = saw && mrun[nt] == -INFINITY ? -3.0e38f : mrun[nt];
    auto factor = [](float of, float m) { return of == -INFINITY ? 0.f : of == m ? 1.f : __builtin_amdgcn_exp2f(of - m); };
    __syncthreads();
    auto put = [&](int w) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int e = 0; e < E; e += 4)
          s_o[w][r][e / 4][lane] = make_float4(acc[nt][e][r], acc[nt][e + 1][r], acc[nt][e + 2][r], acc[nt][e + 3][r]);
      }
      if (g4 == 0) {
        s_m[w][i16] = m_own;
        s_l[w][i16] = l;
      }
    };
    if constexpr (WAVES == 8) {
      if (wave >= 4) put(wave - 4);
      __syncthreads();
      if (wave < 4) {
        const float m_other = s_m[wave][i16], m = fmaxf(m_own, m_other), f0 = factor(m_own, m), f1 = factor(m_other, m);
        l = l * f0 + s_l[wave][i16] * f1;
        m_own = m;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
          for (int e = 0; e < E; e += 4) {
            const float4 y = s_o[wave][r][e / 4][lane];
            acc[nt][e][r] = acc[nt][e][r] * f0 + y.x * f1;
            acc[nt][e + 1][r] = acc[nt][e + 1][r] * f0 + y.y * f1;
            acc[nt][e + 2][r] = acc[nt][e + 2][r] * f0 + y.z * f1;
            acc[nt][e + 3][r] = acc[nt][e + 3][r] * f0 + y.w * f1;
          }
        }
      }
      __syncthreads();
    }
    if (WAVES == 4 || wave < 4) put(wave);
    __syncthreads();
    float m = -INFINITY, fac[4];
    l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, s_m[w][i16]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      fac[w] = factor(s_m[w][i16], m);
      l += s_l[w][i16] * fac[w];
    }
    const int c = c_base + nt * 16 + i16;
    bool bad = false;
    if (c < vectors && (WAVES == 4 || wave < 4)) {
      const int t = t0 + c / G, g = c % G;
      const int64_t row = ((int64_t)seq * Q + t) * A.Hq + (int64_t)kvh * G + g;
      const int64_t place = RANGE ? (int64_t)(nt * 16 + i16) * A.slots + part.slot : row * A.splits + part.slot;
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
#pragma unroll
          for (int x = 0; x < PACK; ++x) {  // (the columns of a vector's terms)
            const float4 y = s_o[w][wave][e / 4][lane + x * vectors];
            o.x += y.x * fac[w];
            o.y += y.y * fac[w];
            o.z += y.z * fac[w];
            o.w += y.w * fac[w];
          }
        }
        if (RANGE && part.whole) {
          bad |= !(fabsf(o.x) + fabsf(o.y) + fabsf(o.z) + fabsf(o.w) < INFINITY);
          store_row<4>(A, row * D + E * (4 * g4 + wave) + e, {o.x / l, o.y / l, o.z / l, o.w / l});
        } else {
          *reinterpret_cast<float4*>(A.part + place * D + E * (4 * g4 + wave) + e) = o;
        }
      }
      if (wave == 0 && g4 == 0) {
        if (!RANGE || !part.whole) A.part_ml[place] = make_float2(m, l);
        else if (A.out_lse) A.out_lse[row] = m * 0.69314718055994530942f + logf(l);
      }
      bad |= !(l < INFINITY);
    }
    if (RANGE && part.whole) {
      const uint64_t there = __ballot(bad);
      odd |= (uint32_t)((there | there >> 16 | there >> 32 | there >> 48) & 0xffff) << (16 * nt);
    }
  }
  if (RANGE && part.whole) {
    // (see attend_merge_kernel)
    __syncthreads();
    if (lane == 0) s_tok[wave] = (int)odd;
    __syncthreads();
    odd = (uint32_t)__builtin_amdgcn_readfirstlane(s_tok[0] | s_tok[1] | s_tok[2] | s_tok[3]);
    if (__builtin_expect(odd == 0, 1)) return;
    __syncthreads();
    float(&s_acc)[WAVES][D] = *reinterpret_cast<float(*)[WAVES][D]>(&s_o[0][0][0][0]);
    float(&s_m2)[WAVES] = *reinterpret_cast<float(*)[WAVES]>(&s_m[0][0]);
    float(&s_l2)[WAVES] = *reinterpret_cast<float(*)[WAVES]>(&s_l[0][0]);
    while (odd) {
      const int c = c_base + __builtin_ctz(odd), t = c / G, h = kvh * G + c % G;
      odd &= odd - 1;
      const int n_t = max(T.first + t + 1, 1);
      attend_again<D, FMT, PAGED, KIND, WAVES>(A, A.q + ((int64_t)seq * Q + t) * A.q_stride + (int64_t)h * D, seq, kvh,
                                               token_list<KIND>(A, 0, kvh, n_t, max(n_t - A.window, 0)), s_acc, s_m2, s_l2);
      float m = s_m2[0], l = 0.f, a = 0.f;
      for (int w = 1; w < WAVES; ++w) m = fmaxf(m, s_m2[w]);
      for (int w = 0; w < WAVES; ++w) {
        if (s_m2[w] == -INFINITY) continue;
        const float f = s_m2[w] == m ? 1.f : __builtin_amdgcn_exp2f(s_m2[w] - m);
        l += s_l2[w] * f;
        if (tid < D) a += s_acc[w][tid] * f;
      }
      const int64_t row = ((int64_t)seq * Q + t) * A.Hq + h;
      if (tid < D) store_row<1>(A, row * D + tid, {a / l});
      if (tid == 0 && A.out_lse) A.out_lse[row] = m * 0.69314718055994530942f + logf(l);
      __syncthreads();
    }
  }
}

// All tokens and listed blocks: the chunks of a list go round the `splits` workgroups, so that which entries a workgroup looks up first does not
// depend on the length.
template <int D, int FMT, bool PAGED, int KIND, int NQT, int PACK>
__global__ __launch_bounds__(kAttendThreads, 2) void attend_kernel(AttendArgs A) {
  const int split = (int)blockIdx.y / A.rounds;
  attend_part<D, FMT, PAGED, KIND, NQT, PACK, kAttendWaves>(
      A, {(int)blockIdx.z, (int)blockIdx.x, (int)blockIdx.y - split * A.rounds, split, A.splits, INT32_MAX, split, false, {0, 0}});
}

// The first tokens and a window, one workgroup of eight waves for a sequence, KV head and 32 vectors.  Bound by round trips: lengths, page entries,
// rows, and the waves' sums in LDS (128 + 128 tokens of one sequence 8.1 us, with several workgroups and a merge 11.1).
template <int D, int FMT, bool PAGED, int NQT, int PACK>
__global__ __launch_bounds__(8 * kWave, 2) void window_kernel(AttendArgs A) {
  attend_part<D, FMT, PAGED, kFirstAndWindow, NQT, PACK, 8>(A, {(int)blockIdx.z, (int)blockIdx.x, (int)blockIdx.y, 0, 1, INT32_MAX, 0, true, query_tokens(A, blockIdx.z)});
}

// The same dealt out: the chunks of all sequences, one behind the other, KV head by KV head, in equal shares to the workgroups.  A job (sequence,
// KV head, vectors) that one workgroup has alone it finishes; the sums of the others are joined by the merge.  Lane l of a wave looks at
// sequences l, l + 64, ..  Bound by the rows' bytes and, at the beginning of every job, by the round trips to its first ones: 48 windows of 4096
// in e4m3, 406 MB, 84 us = 4.8 TB/s (equal splits of every sequence 90, with 768 and 1024 workgroups 103 and 93); one token for 32 x 1K - 16K in
// bf16 183 (equal splits 204).
constexpr int kDealtMost = kAttendThreads;  // sequences, one per thread
struct DealtSeq {
  int upto, own;  // chunks of the sequences of its wave up to and with this one, and its own
  QueryTokens queries;
};
struct Deal {
  const DealtSeq* seqs;
  int of_wave[kAttendWaves], total;  // chunks of a wave's sequences, and of all, of one KV head and set of vectors
  int share;                         // chunks of a workgroup; the last ones may have less, or nothing
  QueryTokens only;                  // of a batch of one, which needs no list
  __device__ __forceinline__ static int chunks_of(const AttendArgs& A, const QueryTokens& T) {
    constexpr int kChunk = 4 * kAttendWaves;
    if (T.count == 0) return 0;
    return (token_list<kFirstAndWindow>(A, 0, 0, max(T.first + T.count, 1), max(max(T.first + 1, 1) - A.window, 0)).count + kChunk - 1) / kChunk;
  }
  // By the whole workgroup.
  __device__ __forceinline__ Deal(const AttendArgs& A, DealtSeq (&s_seqs)[kDealtMost]) : seqs(s_seqs) {
    const int tid = threadIdx.x;
    total = 0;
    only = {0, 0};
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) of_wave[w] = 0;
    if (A.batch == 1) {
      only = query_tokens(A, 0);
      of_wave[0] = total = chunks_of(A, only);
    } else {
      if (A.batch > (tid & ~(kWave - 1))) {
        DealtSeq s = {0, 0, {0, 0}};
        if (tid < A.batch) {
          s.queries = query_tokens(A, tid);
          s.own = chunks_of(A, s.queries);
        }
        s.upto = (int)wave_inclusive_scan_u32((uint32_t)s.own);
        s_seqs[tid] = s;
      }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kAttendWaves; ++w) {
        if (A.batch > w * kWave) of_wave[w] = __builtin_amdgcn_readfirstlane(s_seqs[w * kWave + kWave - 1].upto);
        total += of_wave[w];
      }
    }
    // Rounded up: no share is smaller than all / workgroups, so that a job, `total` chunks at most, lies in at most workgroups / (Hkv * rounds) + 2
    // of them, which the merge can take.
    share = (total * A.Hkv * A.rounds + A.workgroups - 1) / A.workgroups;
  }
  __device__ __forceinline__ int begin(int w) const { return w * share; }
  __device__ __forceinline__ int owner(int x) const { return x / share; }
  struct Seq {
    int b, from, n;  // its first chunk, and how many
    QueryTokens queries;
  };
  __device__ __forceinline__ Seq seq(int b) const {
    if (only.count > 0) return {0, 0, total, only};
    const DealtSeq s = seqs[b];
    const int n = __builtin_amdgcn_readfirstlane(s.own);
    int from = __builtin_amdgcn_readfirstlane(s.upto) - n;
#pragma unroll
    for (int w = 0; w + 1 < kAttendWaves; ++w) from += b >= (w + 1) * kWave ? of_wave[w] : 0;
    return {b, from, n, {__builtin_amdgcn_readfirstlane(s.queries.first), __builtin_amdgcn_readfirstlane(s.queries.count)}};
  }
  // The sequence that has chunk x.
  __device__ __forceinline__ Seq find(int x) const {
    if (only.count > 0) return seq(0);
    int from = 0, w64 = 0, upto = 0;
#pragma unroll
    for (int w = 0; w + 1 < kAttendWaves; ++w) {
      upto += of_wave[w];
      if (x >= upto && upto < total) {
        from = upto;
        w64 = (w + 1) * kWave;
      }
    }
    return seq(w64 + __builtin_ctzll(__ballot(x < from + seqs[w64 + (threadIdx.x & 63)].upto)));
  }
};
template <int D, int FMT, bool PAGED, int NQT, int PACK>
__global__ __launch_bounds__(kAttendThreads, 2) void dealt_kernel(AttendArgs A) {
  __shared__ DealtSeq s_seqs[kDealtMost];
  const Deal deal(A, s_seqs);
  const int w = blockIdx.x, end = min(deal.begin(w + 1), deal.total * A.Hkv * A.rounds);
  for (int x = deal.begin(w); x < end;) {
    const int pair = x / deal.total;
    const Deal::Seq s = deal.find(x - pair * deal.total);
    const int job = pair * A.batch + s.b, job0 = pair * deal.total + s.from;
    if (x == job0 && threadIdx.x == 0) A.jobs[job] = make_int2(w + job, deal.owner(job0 + s.n - 1) - w + 1);
    const int first = x - pair * deal.total - s.from, count = min(s.n - first, end - x), round = pair / A.Hkv;
    attend_part<D, FMT, PAGED, kFirstAndWindow, NQT, PACK, kAttendWaves>(
        A, {s.b, pair - round * A.Hkv, round, first, 1, count, w + job, count == s.n, s.queries});
    x += count;
    if (x < end) __syncthreads();
  }
}

// Merge of a head's partial sums: bound by two dependent loads.  Every wave looks at all (max, sum) pairs, one or two per lane; the threads of
// a column take every PARTS-th partial sum each, the first ones asked for before it is known which count.
// A result with an Inf or a NaN is worked out again: the second product of attend_kernel gives every column every V row of a step, with
// weight 0 where the column does not see the token, and in three terms of which some are 0, so that a row with an Inf or a NaN makes a NaN
// where it has no say.
template <int D, int FMT, bool PAGED, int KIND>
__global__ __launch_bounds__(kAttendThreads) void attend_merge_kernel(AttendArgs A) {
  constexpr int PARTS = kAttendThreads / D, kAhead = 4;
  static_assert(kSplitsMax == 2 * kWave, "two pairs per lane");
  __shared__ float s_acc[kAttendWaves][D], s_m[kAttendWaves], s_l[kAttendWaves];
  const int h = blockIdx.x, tid = threadIdx.x, c = tid % D, part = tid / D, lane = tid & 63;
  const int64_t vb = blockIdx.y, head = vb * A.Hq + h;
  int splits = A.splits;
  int64_t place = head * A.splits;  // its partial sums
  const int seq = seq_of_pair((int)vb, A.q_len), t = (int)vb - seq * A.q_len;
  QueryTokens T = {0, A.q_len};
  if constexpr (KIND == kFirstAndWindow) {
    T = query_tokens(A, seq);
    const int G = A.Hq / A.Hkv, vector = t * G + h % G, round = vector / A.slot_rows;
    const int2 job = A.jobs[(round * A.Hkv + h / G) * A.batch + seq];
    if (t >= T.count || job.y == 1) return;  // (nothing to do, or done)
    splits = min(job.y, kSplitsMax);
    place = (int64_t)(vector - round * A.slot_rows) * A.slots + job.x;
  }
  const float2* ml = A.part_ml + place;
  const float* p = A.part + place * D + c;
  const float2 none = make_float2(-INFINITY, 0.f);
  const float2 x0 = lane < splits ? ml[lane] : none, x1 = kWave + lane < splits ? ml[kWave + lane] : none;
  float first[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) first[u] = p[min(part + u * PARTS, splits - 1) * D];
  float m = wave_max(fmaxf(x0.x, x1.x));
  // (pieces without a token, whose sums nobody wrote, do not count; one whose weight is 0 does, for the sake of an Inf or a NaN in it)
  auto counts = [](float2 x) { return x.x > -INFINITY; };
  auto weight_of = [&](float2 x) { return !counts(x) ? 0.f : x.x == m ? 1.f : __builtin_amdgcn_exp2f(x.x - m); };
  const float w0 = weight_of(x0), w1 = weight_of(x1);
  const uint64_t there0 = __ballot(counts(x0)), there1 = __ballot(counts(x1));
  float l = wave_sum_f32((counts(x0) ? x0.y * w0 : 0.f) + (counts(x1) ? x1.y * w1 : 0.f)), a = 0.f;
  auto weight = [&](int s) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(s < kWave ? w0 : w1), s & (kWave - 1))); };
  auto there = [&](int s) { return s < splits && ((s < kWave ? there0 : there1) >> (s & (kWave - 1)) & 1u); };
  const int wave_part = __builtin_amdgcn_readfirstlane(part);
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int s = wave_part + u * PARTS;
    if (there(s)) a += first[u] * weight(s);
  }
  for (int s0 = wave_part + kAhead * PARTS; s0 < splits; s0 += kAhead * PARTS) {
    float more[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) more[u] = p[min(s0 + u * PARTS, splits - 1) * D];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int s = s0 + u * PARTS;
      if (there(s)) a += more[u] * weight(s);
    }
  }
  s_acc[part][c] = a;
  const bool odd = __syncthreads_or(!(fabsf(a) < INFINITY) || !(l < INFINITY));
  a = 0.f;
#pragma unroll
  for (int x = 0; x < PARTS; ++x) a += s_acc[x][c];
  if (odd) {
    const int kvh = h / (A.Hq / A.Hkv);
    const uint16_t* q = A.q + head * D;
    int n, lo = 0;
    if constexpr (KIND == kFirstAndWindow) {
      n = max(T.first + t + 1, 1);
      lo = max(n - A.window, 0);
      q = A.q + vb * A.q_stride + (int64_t)h * D;
    } else {
      n = max(min(max(A.seq_lens[seq], 1), A.M.n_max) - (A.q_len - 1 - t), 1);
    }
    attend_again<D, FMT, PAGED, KIND, kAttendWaves>(A, q, seq, kvh, token_list<KIND>(A, (int)vb, kvh, n, lo), s_acc, s_m, s_l);
    m = s_m[0];
    for (int w = 1; w < kAttendWaves; ++w) m = fmaxf(m, s_m[w]);
    l = a = 0.f;
    for (int w = 0; w < kAttendWaves; ++w) {
      if (s_m[w] == -INFINITY) continue;
      const float f = s_m[w] == m ? 1.f : __builtin_amdgcn_exp2f(s_m[w] - m);
      l += s_l[w] * f;
      a += s_acc[w][c] * f;
    }
  }
  if (tid < D) {
    const float o = m == -INFINITY ? 0.f : a / l;
    if constexpr (KIND == kFirstAndWindow) store_row<1>(A, head * D + c, {o});
    else A.out_o[head * D + c] = o;
    if (tid == 0 && A.out_lse) A.out_lse[head] = m == -INFINITY ? -INFINITY : m * 0.69314718055994530942f + logf(l);
  }
}

}  // namespace
}  // namespace vatt
