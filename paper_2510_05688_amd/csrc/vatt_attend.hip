// Attention over the tokens of listed blocks, or over all tokens of a quantised cache.
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
constexpr int kChunk = 16;         // groups of 8 tokens that a workgroup takes at a time: a unit for each wave
constexpr int kSlots = 1024;       // groups of 8 tokens that a workgroup looks up at a time
constexpr int kSplitsMax = 128;
constexpr int kNowhere = 0x7fffff00;  // token of a group that does not exist: beyond every sequence

struct AttendArgs {
  const uint16_t* q;
  const unsigned char* k;
  const unsigned char* v;
  int64_t scale_off;
  const int32_t* seq_lens;
  const int32_t* blocks;  // nullptr: all tokens
  const int32_t* block_count;
  float* part;     // [B * q_len * Hq][splits][d]: sums of the weighted V rows
  float2* part_ml;  // [B * q_len * Hq][splits]: (max in units of log 2, sum of the weights); max -Inf: no token seen
  float* out_o;
  float* out_lse;
  RowMap M;
  int Hq, Hkv, q_len, splits, rounds, capacity, block_shift;
  float log2_scale;  // softmax scale / ln 2
};

// A list of tokens in groups of 8: how many groups, and the first token of each (kNowhere where there is none).
struct TokenList {
  const int32_t* blocks;
  int count, capacity, shift, n;  // n: tokens of the sequence that count
};
__device__ __forceinline__ TokenList token_list(const AttendArgs& A, int vb, int kvh, int n) {
  TokenList L = {nullptr, 0, A.capacity, A.block_shift, n};
  if (A.blocks) {
    const int64_t row = (int64_t)vb * A.Hkv + kvh;
    L.blocks = A.blocks + row * A.capacity;
    L.count = min(max(A.block_count[row], 0), A.capacity) << (A.block_shift - 3);
  } else {
    L.count = (n + 7) / 8;
  }
  return L;
}
// (an entry is read without waiting for the length of its list)
__device__ __forceinline__ int entry_of(const TokenList& L, int group) {
  return L.blocks ? L.blocks[min(group >> (L.shift - 3), L.capacity - 1)] : 0;
}
__device__ __forceinline__ int token_of(const TokenList& L, int group, int blk) {
  if (group >= L.count) return kNowhere;
  if (!L.blocks) return group * 8;
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
template <int D, int FMT, bool PAGED, bool LIST, int NQT, int PACK>
__global__ __launch_bounds__(kAttendThreads, 2) void attend_kernel(AttendArgs A) {
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
  const int kvh = blockIdx.x, split = (int)blockIdx.y / A.rounds, round = (int)blockIdx.y - split * A.rounds;
  const int G = A.Hq / A.Hkv, Q = A.q_len;
  const int seq = LIST ? seq_of_pair(blockIdx.z, Q) : blockIdx.z;
  const int n_seq = min(max(A.seq_lens[seq], 1), A.M.n_max);
  // LIST: the vectors are the heads of one query token; else those of all query tokens
  const int t0 = LIST ? (int)blockIdx.z - seq * Q : 0, vectors = LIST ? G : Q * G;
  const int n = LIST ? max(n_seq - (Q - 1 - t0), 1) : n_seq;
  const TokenList L = token_list(A, blockIdx.z, kvh, n);
  const int c_base = round * 16 * NQT;

  __shared__ __align__(16) int s_tok[kSlots];
  __shared__ __align__(16) int s_at[kSlots];
  __shared__ float4 s_o[kAttendWaves][4][E / 4][kWave];
  __shared__ float s_m[kAttendWaves][16], s_l[kAttendWaves][16];
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
    const uint16_t* src = A.q + (((int64_t)seq * Q + t) * A.Hq + (int64_t)kvh * G + g) * D;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const uint4 x = *reinterpret_cast<const uint4*>(src + (s / STEPS) * 4 * (STEPS * 8) + g4 * (STEPS * 8) + (s % STEPS) * 8);
      if constexpr (!kQueriesInLds) bq[nt][s] = x;
      else if (wave == 0) s_q[nt * S + s][lane] = x;  // (a barrier follows before the first unit)
    }
    seen[nt] = max(n_seq - (Q - 1 - t), 1);
  }
  if (!LIST) least = max(n_seq - (Q - 1), 1);

  // what a lane takes away from its weights before they are cut to bf16: nothing, their leading term, the leading two
  const int term = PACK > 1 ? i16 / vectors : 0;
  const uint32_t first_term = term >= 1 ? 0xffff0000u : 0u, second_term = PACK == 3 && term >= 2 ? 0xffff0000u : 0u;
  const uint32_t last_term = PACK == 2 && term == 1 ? 0xffffffffu : 0u;

  f32x4_t acc[NQT][E];
  float mrun[NQT], lrun[NQT];  // running maxima of the scores in units of log 2
  bool any[NQT];
#pragma unroll
  for (int nt = 0; nt < NQT; ++nt) {
    mrun[nt] = -INFINITY;
    lrun[nt] = 0.f;
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

  // The chunks of the list go round the workgroups, so that which entries a workgroup looks up first does not depend on the length.
  auto group_of = [&](int i) { return (split + (i / kChunk) * A.splits) * kChunk + i % kChunk; };
  const int entry0 = entry_of(L, group_of(tid));
  const int chunks = (L.count + kChunk - 1) / kChunk, mine = split < chunks ? (chunks - split + A.splits - 1) / A.splits : 0;
  for (int c0 = 0; c0 < mine; c0 += kSlots / kChunk) {
    const int c_n = min(kSlots / kChunk, mine - c0);
    if (c0 > 0) __syncthreads();
    for (int i = tid; i < c_n * kChunk; i += kAttendThreads) {
      const int group = group_of(c0 * kChunk + i);
      const int tok = token_of(L, group, c0 == 0 && i == tid ? entry0 : entry_of(L, group)), safe = tok == kNowhere ? 0 : tok;
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
      const bool edge = far > least;  // some column does not see all of the 32 keys
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
            const bool ok = (j < 4 ? ta : tb) + (j & 3) < seen[nt];
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
#pragma unroll
          for (int e = 0; e < E; ++e) acc[nt][e] *= alpha;
        }
        const float m = mrun[nt] == -INFINITY ? 0.f : mrun[nt];  // (so far every score is -Inf: weights 0)
        uint32_t w[TERMS][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[j], A.log2_scale, -m));
          lrun[nt] += p;
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
          for (int j = 0; j < 8; ++j) col[j] = (j < 4 ? ta : tb) + (j & 3) < n ? col[j] : 0u;
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

  // The waves' sums together, one 16-vector tile at a time, in the result layout: wave w finishes rows 4 g + w.
#pragma unroll
  for (int nt = 0; nt < NQT; ++nt) {
    float l = lrun[nt];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    int saw = any[nt];
    saw |= __shfl_xor(saw, 16);
    saw |= __shfl_xor(saw, 32);
    // (a piece all of whose scores are -Inf is no piece without a token)
    const float m_own = saw && mrun[nt] == -INFINITY ? -3.0e38f : mrun[nt];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int e = 0; e < E; e += 4)
        s_o[wave][r][e / 4][lane] = make_float4(acc[nt][e][r], acc[nt][e + 1][r], acc[nt][e + 2][r], acc[nt][e + 3][r]);
    }
    if (g4 == 0) {
      s_m[wave][i16] = m_own;
      s_l[wave][i16] = l;
    }
    __syncthreads();
    float m = -INFINITY, fac[kAttendWaves];
    l = 0.f;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, s_m[w][i16]);
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) {
      fac[w] = s_m[w][i16] == -INFINITY ? 0.f : s_m[w][i16] == m ? 1.f : __builtin_amdgcn_exp2f(s_m[w][i16] - m);
      l += s_l[w][i16] * fac[w];
    }
    const int c = c_base + nt * 16 + i16;
    if (c < vectors) {
      const int t = t0 + c / G, g = c % G;
      const int64_t place = (((int64_t)seq * Q + t) * A.Hq + (int64_t)kvh * G + g) * A.splits + split;
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) {
#pragma unroll
          for (int x = 0; x < PACK; ++x) {  // (the columns of a vector's terms)
            const float4 y = s_o[w][wave][e / 4][lane + x * vectors];
            o.x += y.x * fac[w];
            o.y += y.y * fac[w];
            o.z += y.z * fac[w];
            o.w += y.w * fac[w];
          }
        }
        *reinterpret_cast<float4*>(A.part + place * D + E * (4 * g4 + wave) + e) = o;
      }
      if (wave == 0 && g4 == 0) A.part_ml[place] = make_float2(m, l);
    }
  }
}

// The tokens of one list again for one head, by the whole workgroup: dot products, every row only where it is seen.
template <int D, int FMT, bool PAGED>
__device__ __forceinline__ void attend_again(const AttendArgs& A, int64_t vb, int h, int seq, int kvh, const TokenList& L, float (&s_acc)[kAttendWaves][D],
                                             float (&s_m)[kAttendWaves], float (&s_l)[kAttendWaves]) {
  constexpr int LPR = D / 8, RPW = kWave / LPR;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane % LPR, rsub = lane / LPR;
  const uint4 qv = *reinterpret_cast<const uint4*>(A.q + (vb * A.Hq + h) * D + sub * 8);
  const uint32_t qw[4] = {qv.x, qv.y, qv.z, qv.w};
  float m = -INFINITY, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int64_t i = wave * RPW + rsub; i < (int64_t)L.count * 8; i += kAttendWaves * RPW) {
    const int group = (int)(i >> 3), tok = token_of(L, group, entry_of(L, group)) + (int)(i & 7);
    if (tok >= L.n) continue;
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
    l = l * alpha + p;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[2 * j] = acc[2 * j] * alpha + p * bf16_lo(vw[j]);
      acc[2 * j + 1] = acc[2 * j + 1] * alpha + p * bf16_hi(vw[j]);
    }
  }
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

// Merge of a head's partial sums: bound by two dependent loads.  Every wave looks at all (max, sum) pairs, one or two per lane; the threads of
// a column take every PARTS-th partial sum each, the first ones asked for before it is known which count.
// A result with an Inf or a NaN is worked out again: the second product of attend_kernel gives every column every V row of a step, with
// weight 0 where the column does not see the token, and in three terms of which some are 0, so that a row with an Inf or a NaN makes a NaN
// where it has no say.
template <int D, int FMT, bool PAGED>
__global__ __launch_bounds__(kAttendThreads) void attend_merge_kernel(AttendArgs A) {
  constexpr int PARTS = kAttendThreads / D, kAhead = 4;
  static_assert(kSplitsMax == 2 * kWave, "two pairs per lane");
  __shared__ float s_acc[kAttendWaves][D], s_m[kAttendWaves], s_l[kAttendWaves];
  const int h = blockIdx.x, tid = threadIdx.x, c = tid % D, part = tid / D, lane = tid & 63;
  const int64_t vb = blockIdx.y, head = vb * A.Hq + h;
  const float2* ml = A.part_ml + head * A.splits;
  const float* p = A.part + head * A.splits * D + c;
  const float2 none = make_float2(-INFINITY, 0.f);
  const float2 x0 = lane < A.splits ? ml[lane] : none, x1 = kWave + lane < A.splits ? ml[kWave + lane] : none;
  float first[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) first[u] = p[min(part + u * PARTS, A.splits - 1) * D];
  float m = wave_max(fmaxf(x0.x, x1.x));
  // (pieces without a token, whose sums nobody wrote, do not count; one whose weight is 0 does, for the sake of an Inf or a NaN in it)
  auto counts = [](float2 x) { return x.x > -INFINITY; };
  auto weight_of = [&](float2 x) { return !counts(x) ? 0.f : x.x == m ? 1.f : __builtin_amdgcn_exp2f(x.x - m); };
  const float w0 = weight_of(x0), w1 = weight_of(x1);
  const uint64_t there0 = __ballot(counts(x0)), there1 = __ballot(counts(x1));
  float l = wave_sum_f32((counts(x0) ? x0.y * w0 : 0.f) + (counts(x1) ? x1.y * w1 : 0.f)), a = 0.f;
  auto weight = [&](int s) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(s < kWave ? w0 : w1), s & (kWave - 1))); };
  auto there = [&](int s) { return s < A.splits && ((s < kWave ? there0 : there1) >> (s & (kWave - 1)) & 1u); };
  const int wave_part = __builtin_amdgcn_readfirstlane(part);
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int s = wave_part + u * PARTS;
    if (there(s)) a += first[u] * weight(s);
  }
  for (int s0 = wave_part + kAhead * PARTS; s0 < A.splits; s0 += kAhead * PARTS) {
    float more[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) more[u] = p[min(s0 + u * PARTS, A.splits - 1) * D];
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
    const int kvh = h / (A.Hq / A.Hkv), seq = seq_of_pair((int)vb, A.q_len), t = (int)vb - seq * A.q_len;
    const int n = max(min(max(A.seq_lens[seq], 1), A.M.n_max) - (A.q_len - 1 - t), 1);
    attend_again<D, FMT, PAGED>(A, vb, h, seq, kvh, token_list(A, (int)vb, kvh, n), s_acc, s_m, s_l);
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
    A.out_o[head * D + c] = m == -INFINITY ? 0.f : a / l;
    if (tid == 0 && A.out_lse) A.out_lse[head] = m == -INFINITY ? -INFINITY : m * 0.69314718055994530942f + logf(l);
  }
}

template <int D, int FMT, bool PAGED>
hipError_t launch_attend_f(const Plan& pl, const AttendArgs& A, hipStream_t st) {
  const dim3 grid(A.Hkv, A.splits * A.rounds, A.blocks ? pl.vbatch : pl.p.batch), threads(kAttendThreads);
  if (A.blocks) {  // (one to eight vectors)
    if (pl.group <= 4) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, true, 1, 3>), grid, threads, 0, st, A);
    else hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, true, 1, 2>), grid, threads, 0, st, A);
  } else if constexpr (FMT != VATT_KV_BF16) {
    const int vectors = pl.group * pl.q_len;
    if (vectors <= 5) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, false, 1, 3>), grid, threads, 0, st, A);
    else if (vectors <= 8) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, false, 1, 2>), grid, threads, 0, st, A);
    else if (vectors <= 16) hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, false, 1, 1>), grid, threads, 0, st, A);
    else hipLaunchKernelGGL((attend_kernel<D, FMT, PAGED, false, 2, 1>), grid, threads, 0, st, A);
  } else {
    return hipErrorInvalidValue;  // (all tokens of a bf16 cache are dense_kernel's)
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attend_merge_kernel<D, FMT, PAGED>), dim3(A.Hq, pl.vbatch), dim3(kAttendThreads), 0, st, A);
  return hipGetLastError();
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
