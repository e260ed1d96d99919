// Attention of the new tokens of every sequence (a prompt, a piece of one, drafted tokens) over the cache that holds their rows.
#include <algorithm>

#include "vatt_format.h"

namespace vatt {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kChunkThreads = 256, kChunkWaves = kChunkThreads / kWave;
constexpr int kWaveRows = 32;                         // rows (query vectors) of a wave
constexpr int kTileRows = kWaveRows * kChunkWaves;    // ... of a workgroup
constexpr int kTileKeys = 64;
constexpr int kChunkSplitsMax = 64;

struct ChunkArgs {
  const uint16_t* q;
  int64_t q_stride;
  const unsigned char* k;
  const unsigned char* v;
  int64_t scale_off;
  const int32_t* first;
  const int32_t* new_lens;
  float* part;      // [B * n_new * Hq][splits][d]: sums of the weighted V rows
  float2* part_ml;  // [B * n_new * Hq][splits]: (max in units of log 2, sum of the weights); max -Inf: no token seen
  void* out_o;
  float* out_lse;
  RowMap M;
  int batch, Hq, Hkv, n_new, splits, sink, window;
  float log2_scale;  // softmax scale / ln 2
};

// The new tokens of a sequence: the first one's position, and how many count.
struct NewTokens {
  int first, count;
};
__device__ __forceinline__ NewTokens new_tokens(const ChunkArgs& A, int b) {
  const int first = A.first[b], want = A.new_lens ? min(max(A.new_lens[b], 0), A.n_new) : A.n_new;
  if (first < 0 || first >= A.M.n_max) return {0, 0};
  return {first, min(want, A.M.n_max - first)};
}

// Tiles of keys that the queries at positions p_lo .. p_hi see something of: those of the first tokens, then those from the first
// query's window on.
struct KeyTiles {
  int n_sink, from, count;
  __device__ __forceinline__ int at(int i) const { return i < n_sink ? i : i - n_sink + from; }
};
__device__ __forceinline__ KeyTiles key_tiles(const ChunkArgs& A, int p_lo, int p_hi) {
  KeyTiles T = {0, 0, 0};
  if (A.window > 0) {
    const int lo = max(p_lo - A.window + 1, 0);
    T.from = lo / kTileKeys;
    T.n_sink = min((min(A.sink, lo) + kTileKeys - 1) / kTileKeys, T.from);
  }
  T.count = T.n_sink + p_hi / kTileKeys + 1 - T.from;
  return T;
}

// Where 16-byte chunk c of row `row` lies in a tile in LDS.
template <int D>
__device__ __forceinline__ int k_place(int row, int c) {
  if constexpr (D == 128) return row * 256 + ((c ^ (row & 15)) << 4);
  else return row * 128 + ((c ^ ((row >> 1) & 7)) << 4);
}
template <int D>
__device__ __forceinline__ int v_place(int row, int c) {
  if constexpr (D == 128) return row * 256 + ((c ^ ((row & 3) << 2)) << 4);
  else return row * 128 + ((c ^ ((row & 2) << 1)) << 4);
}

template <bool BF16>
__device__ __forceinline__ void store_4(void* out, int64_t at, float a, float b, float c, float d) {
  if constexpr (BF16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
  else *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(a, b, c, d);
}

// One row again by one wave: dot products, every key only where it is seen.  (max, sum) and the lane's 8 columns (lane % (D / 8)).
template <int D, int FMT, bool PAGED>
__device__ __forceinline__ void row_again(const ChunkArgs& A, int b, int kvh, int64_t q_at, int p, const KeyTiles& T, int i0, int i1, float& m,
                                          float& l, float (&acc)[8]) {
  constexpr int LPR = D / 8, RPW = kWave / LPR;
  const int lane = threadIdx.x & 63, sub = lane % LPR, rsub = lane / LPR;
  const uint4 qv = *reinterpret_cast<const uint4*>(A.q + q_at + sub * 8);
  const uint32_t qw[4] = {qv.x, qv.y, qv.z, qv.w};
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  for (int i = i0; i < i1; ++i) {
    for (int r = rsub; r < kTileKeys; r += RPW) {
      const int tok = T.at(i) * kTileKeys + r;
      if (tok > p || (A.window > 0 && tok <= p - A.window && tok >= A.sink)) continue;
      const RowAt at = row_at<PAGED>(A.M, b, kvh, tok, row_block<PAGED>(A.M, b, tok));
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
      const float w = __builtin_amdgcn_exp2f(s - shift);
      m = shift;
      l = l * alpha + w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[2 * j] = acc[2 * j] * alpha + w * bf16_lo(vw[j]);
        acc[2 * j + 1] = acc[2 * j + 1] * alpha + w * bf16_hi(vw[j]);
      }
    }
  }
  float all = m;
#pragma unroll
  for (int o = LPR; o < kWave; o <<= 1) all = fmaxf(all, __shfl_xor(all, o));
  const float f = m == -INFINITY ? 0.f : m == all ? 1.f : __builtin_amdgcn_exp2f(m - all);
  l *= f;
#pragma unroll
  for (int c = 0; c < 8; ++c) acc[c] = m == -INFINITY ? 0.f : acc[c] * f;
#pragma unroll
  for (int o = LPR; o < kWave; o <<= 1) {
    l += __shfl_xor(l, o);
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[c] += __shfl_xor(acc[c], o);
  }
  m = all;
}

// Rows of a KV head: row r is query token r / G, head r % G of the group.  A workgroup takes 128 of them, a wave 32, over the key tiles
// of its split; the tiles go through LDS in bf16, the next one on its way in registers.
//   S^T [keys x rows] = K Q^T   and   O^T [d x rows] += V^T P^T,   P = exp(S - m),
// v_mfma_f32_32x32x16_bf16 (operand lane l: row or column l % 32, eight inner elements of half l / 32; result lane l: column l % 32,
// rows 8 (i / 4) + 4 (l / 32) + i % 4).  A row's scores lie in two lanes, and are the operand of the second product as they come when
// its inner elements j of half h are keys 4 h + j and 8 + 4 h + j - 4; V comes out of LDS transposed.
// TERMS 1 (output in bf16): P rounded to bf16, as the output is.  TERMS 3 (output in 32 bits): P as three bf16 terms that add up to the
// fp32 value.  The sums of P are of the unrounded values.
// The running maximum of a row moves only when a score passes it by more than kLazy.
template <int D, int FMT, bool PAGED, int TERMS>
__global__ __launch_bounds__(kChunkThreads, 2) void chunk_kernel(ChunkArgs A) {
  constexpr int S = D / 16;                        // steps of the first product
  constexpr int E = D / 32;                        // tiles over the head dimension
  constexpr int LPR = D / 8;                       // 16-byte chunks of a row in LDS
  constexpr int PASS = kChunkThreads / LPR;        // rows that the workgroup loads at a time
  constexpr int N = kTileKeys / PASS;
  constexpr int TILE = kTileKeys * D * 2;          // bytes
  constexpr float kLazy = 8.0f;
  constexpr bool BF16 = TERMS == 1;
  __shared__ __align__(256) unsigned char s_kv[2][2][TILE];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, col = lane & 31;
  const int pairs = A.batch * A.Hkv, rank = (int)blockIdx.x / pairs, pair = (int)blockIdx.x - rank * pairs;
  const int b = pair / A.Hkv, kvh = pair - b * A.Hkv, split = blockIdx.y;
  const int g_shift = 31 - __builtin_clz(A.Hq / A.Hkv), G = 1 << g_shift;
  const NewTokens New = new_tokens(A, b);
  const int rows = New.count << g_shift, tile = (rows + kTileRows - 1) / kTileRows - 1 - rank;  // (the longest first)
  if (tile < 0) return;

  const int r0 = tile * kTileRows;
  const int p_lo = New.first + (r0 >> g_shift), p_hi = New.first + ((min(r0 + kTileRows, rows) - 1) >> g_shift);
  const KeyTiles T = key_tiles(A, p_lo, p_hi);
  const int i0 = (int)((int64_t)T.count * split / A.splits), i1 = (int)((int64_t)T.count * (split + 1) / A.splits);

  // the wave's rows
  const int w0 = r0 + wave * kWaveRows;
  const bool active = w0 < rows;
  const int row = w0 + col, safe_row = min(row, rows - 1), t = safe_row >> g_shift;
  const int p = New.first + t, low = A.window > 0 ? p - A.window : -1;  // sees keys <= p that are > low or < sink
  const int wp_lo = New.first + (min(w0, rows - 1) >> g_shift), wp_hi = New.first + ((min(w0 + kWaveRows, rows) - 1) >> g_shift);
  const int64_t head = (int64_t)kvh * G + (safe_row & (G - 1));
  const int64_t q_at = ((int64_t)b * A.n_new + t) * A.q_stride + head * D;
  uint4 bq[S];
#pragma unroll
  for (int s = 0; s < S; ++s) bq[s] = *reinterpret_cast<const uint4*>(A.q + q_at + s * 16 + half * 8);

  // loads: thread tid has chunk tid % LPR of rows tid / LPR + PASS * n
  const int my_row = tid / LPR, my_chunk = tid % LPR;
  Chunk<FMT> rk[N], rv[N];
  uint32_t sk[N], sv[N];
  auto load = [&](int i) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int tok = min(T.at(i) * kTileKeys + my_row + PASS * n, p_hi);
      const RowAt at = row_at<PAGED>(A.M, b, kvh, tok, row_block<PAGED>(A.M, b, tok));
      const int64_t off = at.row * kRowBytes<FMT, D> + my_chunk * (kRowBytes<FMT, D> / LPR);
      rk[n] = load_chunk<FMT>(A.k + off);
      rv[n] = load_chunk<FMT>(A.v + off);
      sk[n] = sv[n] = 0;
      if constexpr (FMT != VATT_KV_BF16) {
        const int64_t so = A.scale_off + at.scales * (D / 32) + my_chunk / 4;
        sk[n] = A.k[so];
        sv[n] = A.v[so];
      }
    }
  };
  auto store = [&](int i, int buf) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int r = my_row + PASS * n;
      const bool there = T.at(i) * kTileKeys + r <= p_hi;
      *reinterpret_cast<uint4*>(&s_kv[buf][0][k_place<D>(r, my_chunk)]) = chunk_bf16<FMT>(rk[n], sk[n]);
      // (rows that nobody sees: whatever lies there has no say)
      const uint4 v = chunk_bf16<FMT>(rv[n], sv[n]);
      *reinterpret_cast<uint4*>(&s_kv[buf][1][v_place<D>(r, my_chunk)]) = there ? v : make_uint4(0, 0, 0, 0);
    }
  };

  f32x16_t acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[e][j] = 0.f;
  float mrun = -INFINITY, lrun = 0.f;
  bool any = false;

  if (i0 < i1) {
    load(i0);
    store(i0, 0);
  }
  __syncthreads();
  for (int i = i0; i < i1; ++i) {
    const int buf = (i - i0) & 1, k0 = T.at(i) * kTileKeys;
    if (i + 1 < i1) load(i + 1);
    const bool skip = !active || k0 > wp_hi || (A.window > 0 && k0 + kTileKeys - 1 <= wp_lo - A.window && k0 >= A.sink);
    if (!skip) {
      f32x16_t sc[2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int j = 0; j < 16; ++j) sc[x][j] = 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint4 a = *reinterpret_cast<const uint4*>(&s_kv[buf][0][k_place<D>(col, 2 * s + half) + x * 32 * D * 2]);
          sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, bq[s]), sc[x], 0, 0, 0);
        }
      }
      const bool edge = k0 + kTileKeys - 1 > wp_lo || (A.window > 0 && k0 <= wp_hi - A.window && k0 + kTileKeys > A.sink);
      if (edge) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int tok = k0 + x * 32 + 8 * (j / 4) + 4 * half + j % 4;
            const bool ok = tok <= p && (tok > low || tok < A.sink);
            sc[x][j] = ok ? sc[x][j] : -INFINITY;
            any |= ok;
          }
      } else {
        any = true;
      }
      float top = sc[0][0];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, sc[x][j]);
      top *= A.log2_scale;
      if (__ballot(top > mrun + kLazy)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mnew = fmaxf(mrun, top);
        const float alpha = mrun == mnew ? 1.f : __builtin_amdgcn_exp2f(mrun - mnew);
        mrun = mnew;
        lrun *= alpha;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= alpha;
      }
      const float m = mrun == -INFINITY ? 0.f : mrun;  // (so far every score is -Inf: weights 0)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          sc[x][j] = __builtin_amdgcn_exp2f(fmaf(sc[x][j], A.log2_scale, -m));
          lrun += sc[x][j];
        }
      uint4 pb[4][TERMS];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = sc[u / 2][8 * (u % 2) + j];
#pragma unroll
        for (int z = 0; z < TERMS; ++z) {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = pack_bf16(y[2 * j], y[2 * j + 1]);
          pb[u][z] = make_uint4(w[0], w[1], w[2], w[3]);
          if (z + 1 < TERMS) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              y[2 * j] -= bf16_lo(w[j]);
              y[2 * j + 1] -= bf16_hi(w[j]);
            }
          }
        }
      }
      typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
      const int l16 = lane & 15, c_half = (lane >> 4) & 1;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int r = 16 * u + 4 * half + (l16 >> 2), c = 4 * e + 2 * c_half + ((l16 & 3) >> 1);
          const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)&s_kv[buf][1][v_place<D>(r, c) + (l16 & 1) * 8]);
          const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)&s_kv[buf][1][v_place<D>(r + 8, c) + (l16 & 1) * 8]);
          const bf16x8_t va = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int z = TERMS - 1; z >= 0; --z)
            acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, __builtin_bit_cast(bf16x8_t, pb[u][z]), acc[e], 0, 0, 0);
        }
      }
    }
    if (i + 1 < i1) store(i + 1, buf ^ 1);
    __syncthreads();
  }
  if (!active) return;

  // A result with an Inf or a NaN is worked out again: the second product gives every row every V row of a tile, with weight 0 where
  // the row does not see the key (and in three terms of which some are 0), so that an Inf or a NaN has a say where it should have none.
  float l = lrun + __shfl_xor(lrun, 32);
  const bool saw = any || __shfl_xor((int)any, 32);
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int j = 0; j < 16; ++j) sum += fabsf(acc[e][j]);
  const uint64_t odd = __ballot(!(sum < INFINITY) || !(l < INFINITY));
  uint32_t again = (uint32_t)odd | (uint32_t)(odd >> 32);
  const int64_t out_row = ((int64_t)b * A.n_new + t) * A.Hq + head;
  const float m_own = saw && mrun == -INFINITY ? -3.0e38f : mrun;
  if (row < rows && !(again >> col & 1)) {
    if (A.splits == 1) {
      const float inv = 1.f / l;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          store_4<BF16>(A.out_o, out_row * D + 32 * e + 8 * x + 4 * half, acc[e][4 * x] * inv, acc[e][4 * x + 1] * inv, acc[e][4 * x + 2] * inv,
                        acc[e][4 * x + 3] * inv);
      if (A.out_lse && half == 0) A.out_lse[out_row] = m_own * 0.69314718055994530942f + logf(l);
    } else {
      const int64_t place = out_row * A.splits + split;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          store_4<false>(A.part, place * D + 32 * e + 8 * x + 4 * half, acc[e][4 * x], acc[e][4 * x + 1], acc[e][4 * x + 2], acc[e][4 * x + 3]);
      if (half == 0) A.part_ml[place] = make_float2(m_own, l);
    }
  }
  while (again) {
    const int c = __builtin_ctz(again);
    again &= again - 1;
    if (w0 + c >= rows) continue;
    const int64_t q_c = ((int64_t)b * A.n_new + ((w0 + c) >> g_shift)) * A.q_stride + ((int64_t)kvh * G + ((w0 + c) & (G - 1))) * D;
    const int64_t out_c = ((int64_t)b * A.n_new + ((w0 + c) >> g_shift)) * A.Hq + (int64_t)kvh * G + ((w0 + c) & (G - 1));
    float m, ls, a[8];
    row_again<D, FMT, PAGED>(A, b, kvh, q_c, New.first + ((w0 + c) >> g_shift), T, i0, i1, m, ls, a);
    if (lane >= LPR) continue;
    if (A.splits == 1) {
      const float inv = 1.f / ls;
      store_4<BF16>(A.out_o, out_c * D + lane * 8, a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv);
      store_4<BF16>(A.out_o, out_c * D + lane * 8 + 4, a[4] * inv, a[5] * inv, a[6] * inv, a[7] * inv);
      if (A.out_lse && lane == 0) A.out_lse[out_c] = m * 0.69314718055994530942f + logf(ls);
    } else {
      const int64_t place = out_c * A.splits + split;
      store_4<false>(A.part, place * D + lane * 8, a[0], a[1], a[2], a[3]);
      store_4<false>(A.part, place * D + lane * 8 + 4, a[4], a[5], a[6], a[7]);
      if (lane == 0) A.part_ml[place] = make_float2(m, ls);
    }
  }
}

// The splits' partial sums together: a wave per row.
template <int D, bool BF16>
__global__ __launch_bounds__(kChunkThreads) void chunk_merge_kernel(ChunkArgs A) {
  constexpr int C = D / kWave;
  static_assert(kChunkSplitsMax <= kWave, "a pair per lane");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = blockIdx.y;
  const int row = blockIdx.x * kChunkWaves + wave, t = row / A.Hq;
  if (t >= new_tokens(A, b).count) return;
  const int64_t out_row = (int64_t)b * A.n_new * A.Hq + row;
  const float2 ml = lane < A.splits ? A.part_ml[out_row * A.splits + lane] : make_float2(-INFINITY, 0.f);
  const float m = wave_max(ml.x);
  const bool counts = ml.x > -INFINITY;  // (a piece without a token, whose sums nobody wrote, does not)
  const float w = !counts ? 0.f : ml.x == m ? 1.f : __builtin_amdgcn_exp2f(ml.x - m);
  const float l = wave_sum_f32(counts ? ml.y * w : 0.f);
  const uint64_t there = __ballot(counts);
  float a[C];
#pragma unroll
  for (int c = 0; c < C; ++c) a[c] = 0.f;
  for (int s = 0; s < A.splits; ++s) {
    if (!(there >> s & 1)) continue;
    const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), s));
#pragma unroll
    for (int c = 0; c < C; ++c) a[c] += f * A.part[(out_row * A.splits + s) * D + lane * C + c];
  }
  const float inv = 1.f / l;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const float o = a[c] * inv;
    if constexpr (BF16) static_cast<uint16_t*>(A.out_o)[out_row * D + lane * C + c] = (uint16_t)pack_bf16(o, o);
    else static_cast<float*>(A.out_o)[out_row * D + lane * C + c] = o;
  }
  if (A.out_lse && lane == 0) A.out_lse[out_row] = m * 0.69314718055994530942f + logf(l);
}

template <int D, int FMT, bool PAGED, int TERMS>
hipError_t launch_chunk_t(const Plan& pl, const ChunkArgs& A, hipStream_t st) {
  const int ranks = (A.n_new * pl.group + kTileRows - 1) / kTileRows;
  hipLaunchKernelGGL((chunk_kernel<D, FMT, PAGED, TERMS>), dim3(ranks * A.batch * A.Hkv, A.splits), dim3(kChunkThreads), 0, st, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || A.splits == 1) return e;
  hipLaunchKernelGGL((chunk_merge_kernel<D, TERMS == 1>), dim3((A.n_new * A.Hq + kChunkWaves - 1) / kChunkWaves, A.batch), dim3(kChunkThreads), 0, st, A);
  return hipGetLastError();
}
template <int D, int FMT>
hipError_t launch_chunk_f(const Plan& pl, const ChunkArgs& A, bool bf16, hipStream_t st) {
  const bool paged = pl.p.kv_layout == VATT_LAYOUT_PAGED;
  if (bf16) return paged ? launch_chunk_t<D, FMT, true, 1>(pl, A, st) : launch_chunk_t<D, FMT, false, 1>(pl, A, st);
  return paged ? launch_chunk_t<D, FMT, true, 3>(pl, A, st) : launch_chunk_t<D, FMT, false, 3>(pl, A, st);
}
template <int D>
hipError_t launch_chunk_d(const Plan& pl, const ChunkArgs& A, bool bf16, hipStream_t st) {
  if (pl.kv_format == VATT_KV_E4M3) return launch_chunk_f<D, VATT_KV_E4M3>(pl, A, bf16, st);
  if (pl.kv_format == VATT_KV_E2M1) return launch_chunk_f<D, VATT_KV_E2M1>(pl, A, bf16, st);
  return launch_chunk_f<D, VATT_KV_BF16>(pl, A, bf16, st);
}

// Workgroups that share out a tile's keys: two per CU in all, none for less than four tiles of the capacity.
int chunk_splits(const Plan& pl, int n_new) {
  const int64_t tiles = (int64_t)pl.p.batch * pl.p.n_kv_heads * (((int64_t)n_new * pl.group + kTileRows - 1) / kTileRows);
  if (tiles >= pl.num_cus) return 1;
  const int64_t splits = (2 * pl.num_cus + tiles - 1) / tiles, most = (pl.p.n_max + 4 * kTileKeys - 1) / (4 * kTileKeys);
  return (int)std::min<int64_t>({splits, most, kChunkSplitsMax});
}

}  // namespace

bool chunk_fits(const Plan& pl, int n_new) {
  return (int64_t)pl.p.batch * pl.p.n_kv_heads * (((int64_t)n_new * pl.group + kTileRows - 1) / kTileRows) <= INT32_MAX / kChunkThreads;
}

size_t chunk_workspace_bytes(const Plan& pl, int n_new) {
  const int splits = chunk_splits(pl, n_new);
  return splits == 1 ? 0 : (size_t)pl.p.batch * n_new * pl.p.n_q_heads * splits * (pl.p.head_dim + 2) * sizeof(float);
}

hipError_t launch_chunk(const Plan& pl, const void* q, int64_t q_stride, int n_new, const int32_t* first, const int32_t* new_lens, const void* k,
                        const void* v, const int32_t* block_table, int sink, int window, void* ws, bool bf16, void* out_o, float* out_lse,
                        hipStream_t st) {
  ChunkArgs A = {};
  A.q = static_cast<const uint16_t*>(q);
  A.q_stride = q_stride;
  A.k = static_cast<const unsigned char*>(k);
  A.v = static_cast<const unsigned char*>(v);
  A.scale_off = (int64_t)kv_scale_offset(pl);
  A.first = first;
  A.new_lens = new_lens;
  A.out_o = out_o;
  A.out_lse = out_lse;
  A.M = row_map(pl, block_table);
  A.batch = pl.p.batch;
  A.Hq = pl.p.n_q_heads;
  A.Hkv = pl.p.n_kv_heads;
  A.n_new = n_new;
  A.splits = chunk_splits(pl, n_new);
  A.sink = std::min(sink, pl.p.n_max);
  A.window = std::min(window, pl.p.n_max);
  A.log2_scale = (float)((double)pl.sm_scale * 1.4426950408889634);
  A.part = static_cast<float*>(ws);
  A.part_ml = reinterpret_cast<float2*>(A.part + (size_t)A.batch * n_new * A.Hq * A.splits * pl.p.head_dim);
  return pl.p.head_dim == 128 ? launch_chunk_d<128>(pl, A, bf16, st) : launch_chunk_d<64>(pl, A, bf16, st);
}

}  // namespace vatt
