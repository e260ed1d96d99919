// Attention of the new tokens of every sequence (a prompt, a piece of one, drafted tokens) over the cache that holds their rows.
#include <algorithm>
#include <type_traits>

#include "vatt_format.h"

namespace vatt {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kChunkThreads = 256, kChunkWaves = kChunkThreads / kWave;
constexpr int kWaveRows = 32;                         // rows (query vectors) of a wave
constexpr int kTileShift = 7, kTileRows = 1 << kTileShift;  // ... of a workgroup
static_assert(kTileRows == kWaveRows * kChunkWaves, "32 rows of every wave");
constexpr int kTileKeys = 64;
constexpr int kPiecesMax = 64;      // pieces that a tile's keys are cut into at most
constexpr int kPieceLeast = 4;      // key tiles of a piece at least
constexpr int kRestLeast = 24;      // key tiles of a tile that is cut because it is over
constexpr float kOnePerUnit = 5000.f;  // key tiles in all below which there is one piece per compute unit, not two
// Key tiles whose weighted rows are added up in one sum where the output has 32 bits.  A matrix instruction cuts its sums off, 12 times a tile: rows
// of equal weight came out 2e-4 too small on 64K tokens and 7e-4 on 170K, so 1e-5 (with 32 tiles 8e-6, with 64 1.3e-5).  2K on 64K 3453 us in
// one sum, 3551 so (with 32 tiles 3655).  Output in bf16 has one term, 4 sums a tile, and half a step of 4e-3: one sum.
constexpr int kSumTiles = 48;
constexpr int kAgainTiles = 8;  // the same where a row is worked out again, whose sums are rounded
constexpr int kSteps = 8;           // of a tile's level, for the order (a power of two)
constexpr int kSeqsPerLane = 4, kSeqsMax = kSeqsPerLane * kWave;  // sequences that a wave looks through for its work

struct ChunkArgs {
  const uint16_t* q;
  int64_t q_stride;
  const unsigned char* k;
  const unsigned char* v;
  int64_t scale_off;
  const int32_t* first;
  const int32_t* new_lens;
  float* part;      // [pieces][kTileRows][d]: sums of the weighted V rows
  float2* part_ml;  // [pieces][kTileRows]: (max in units of log 2, sum of the weights); max -Inf: no token seen
  void* out_o;
  float* out_lse;
  RowMap M;
  int batch, Hq, Hkv, n_new, sink, window;
  int slots;  // workgroups that run at a time, two to a compute unit
  int room;   // pieces of one KV head that the workspace holds
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

__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane((int)wave_inclusive_scan_u32((uint32_t)v), kWave - 1); }

__device__ __forceinline__ uint64_t ones(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }  // the lowest n bits

// What a workgroup does: a tile of rows of one sequence and KV head, over one of `pieces` parts of its keys.
struct Work {
  int b, kvh, tile, piece, pieces, slot;  // slot: the piece's place in the workspace, for one KV head
};

// Pieces that the tiles of sequences are cut into.  total: key tiles of all tiles of one KV head, most: if each had as many as its sequence's last one.
// Tiles that are long beside what all work comes to per workgroup slot are cut into pieces of about that length, all tiles of a sequence into
// equally many; their sums are joined by the merge.  Where there is little to do one piece per compute unit is better than two, whose sums are twice
// the bytes: us with two / one (three calls at a time, as here below), 16 new tokens on 1 x 16K 33.8 / 29.3, 64 46.0 / 40.6, but 64 on 3 x 5K - 16K
// 66 / 85, 33 with groups of 8 49.0 / 60.4.  They are a little longer than an equal share, so that rounding leaves none over for which nobody is free (33
// with groups of 8 62.6 -> 49.0).
// (32-bit values, rounded the same way wherever this is worked out.)
struct Cut {
  float piece;  // key tiles; 0: nothing is cut
  float up = 0.5f;
  __device__ __forceinline__ Cut(const ChunkArgs& A, float total, float most, int longest) {
#pragma clang fp contract(off)
    const float share = total * A.Hkv / A.slots;
    const float at_once = 0.97f * (most * A.Hkv < kOnePerUnit ? A.slots / 2 : A.slots);
    piece = A.room > 0 && longest > 1.25f * share + 12.f ? fmaxf(most * A.Hkv / at_once, (float)kPieceLeast) : 0.f;
  }
  __device__ __forceinline__ int pieces(int last) const { return piece == 0.f ? 1 : max(min((int)(last / piece + up), kPiecesMax), 1); }
  // `cut` pieces of one KV head: where a few too many for the slots would wait for all others, twice as many of half the length, rounded down (700
  // new tokens on 32K, 176 tiles: three pieces each 503 us, five 411).
  __device__ __forceinline__ bool finer(const ChunkArgs& A, int cut) {
    if (cut * A.Hkv <= A.slots) return false;
    piece *= 0.5f;
    up = 0.f;
    return true;
  }
};

// Where nothing is long beside everybody's share, but the tiles leave a rest when the slots have been filled as often as they can be: the tiles of the
// rest, the last in the order, in equally many pieces each, which fill the slots once or twice (us whole / cut: 2304 new tokens on 32K, 576 tiles for
// 512 slots, 1384 / 1094, 2560 1412 / 1264, 256 on 9 x 8K 390 / 312, 32 on 72 x 4K 293 / 248; at 256 on 12 x 2K to 8K, 768 tiles, it would not pay, and
// is not done).  shortest: key tiles of the batch's shortest tile, from which the pieces are worked out for all, so that this is for sequences of about one
// length: with one of 300 tokens among them nothing is cut (9 x 8K and that one 378, 72 x 4K and that one 292).
struct Rest {
  int whole, pieces;  // tiles of a KV head before the rest
  __device__ __forceinline__ Rest(const ChunkArgs& A, int count, int shortest) : whole(count), pieces(1) {
    const int all = count * A.Hkv;
    if (A.room == 0 || shortest < kRestLeast || all <= A.slots) return;
    const int before = all / A.slots * A.slots / A.Hkv, rest = (count - before) * A.Hkv;
    if (rest == 0) return;
    // in units of a key tile of a workgroup that shares its unit: one alone takes 0.6; pieces cost 14 for every filling of the slots
    const int most = min(shortest / kPieceLeast, kPiecesMax), once = min(A.slots / rest, most), twice = min(2 * A.slots / rest, most);
    float least = 2 * rest <= A.slots ? 0.6f * shortest : (float)shortest;
    const float a = (float)shortest / (float)max(once, 1) + 14.f, b = 2.f * (float)shortest / (float)max(twice, 1) + 28.f;
    if (once > 1 && a < least) {
      least = a;
      pieces = once;
    }
    if (twice > 1 && b < least) pieces = twice;
    if (pieces > 1) whole = before;
  }
};

// A sequence's tiles: how many, and the key tiles of the first and the last one.
struct SeqTiles {
  int tiles, first, last;
  __device__ __forceinline__ SeqTiles(const ChunkArgs& A, int g_shift, const NewTokens& n) : tiles(0), first(0), last(0) {
    if (n.count == 0) return;
    const int tokens = kTileRows >> g_shift, end = n.first + n.count - 1;
    tiles = ((n.count << g_shift) + kTileRows - 1) / kTileRows;
    first = key_tiles(A, n.first, min(n.first + tokens - 1, end)).count;
    last = key_tiles(A, n.first + (tiles - 1) * tokens, end).count;
  }
};

// Which of `count` tiles, the longest first, item y is.  Where all run at once, two to a compute unit, a long one shares its unit with a short one.
__device__ __forceinline__ int order(const ChunkArgs& A, int y, int count) {
  const int half = A.slots / 2 / A.Hkv;
  return count * A.Hkv <= A.slots && y >= half && y < count ? count - 1 - (y - half) : y;
}

// The batch's work, as every wave sees it: lane l has sequences l, l + 64, ...  Pieces come first, then the tiles that are not cut, the longest
// first: what a tile costs goes by its place in the sequence, counted in tiles (its level).  In steps of an eighth of the highest level, within which a
// sequence's tiles are neighbours, so that they read its rows from L2 (level by level 32 x 512 new tokens on 4K 1474 us, so 994; 256 on 24 x 8K 1010
// and 790; ragged prompts the same within 1 %).
struct Batch {
  int tiles[kSeqsPerLane], pieces[kSeqsPerLane], level[kSeqsPerLane];
  int cut;    // pieces of one KV head in all
  int whole, rest;  // tiles that are not cut, and pieces of each of the others (1: there are none)

  __device__ __forceinline__ void read(const ChunkArgs& A, int g_shift) {
    const int lane = threadIdx.x & 63;
    int last[kSeqsPerLane];
    float total = 0.f, most = 0.f, shortest = 1e9f;
    int longest = 0, count = 0;
#pragma unroll
    for (int i = 0; i < kSeqsPerLane; ++i) {
      const int b = lane + i * kWave;
      tiles[i] = level[i] = last[i] = 0;
      pieces[i] = 1;
      if (i * kWave < A.batch && b < A.batch) {
        const NewTokens n = new_tokens(A, b);
        const SeqTiles t(A, g_shift, n);
        tiles[i] = t.tiles;
        level[i] = n.first >> (kTileShift - g_shift);
        last[i] = t.last;
        total += 0.5f * (float)(t.tiles * (t.first + t.last));
        most += (float)(t.tiles * t.last);
        longest = max(longest, t.last);
        count += t.tiles;
        if (t.tiles > 0) shortest = fminf(shortest, (float)t.first);
      }
    }
    cut = 0;
    whole = INT32_MAX;
    rest = 1;
    if (A.room == 0) return;
    Cut c(A, wave_sum_f32(total), wave_sum_f32(most), (int)wave_max((float)longest));
    if (c.piece == 0.f) {
      const Rest r(A, wave_total(count), (int)-wave_max(-shortest));
      if (r.pieces > 1) {
        whole = r.whole;
        rest = r.pieces;
        cut = (wave_total(count) - whole) * rest;
      }
      return;
    }
    auto cut_all = [&]() __attribute__((always_inline)) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < kSeqsPerLane; ++i) {
        pieces[i] = c.pieces(last[i]);
        if (pieces[i] > 1) n += tiles[i] * pieces[i];
      }
      cut = wave_total(n);
    };
    cut_all();
    if (c.finer(A, cut)) cut_all();
    if (cut > A.room) {  // (not reached: see chunk_pieces)
      cut = 0;
#pragma unroll
      for (int i = 0; i < kSeqsPerLane; ++i) pieces[i] = 1;
    }
  }
  // Tiles of whole sequences at a level or above it.
  __device__ __forceinline__ int above(int l) const {
    int n = 0;
#pragma unroll
    for (int i = 0; i < kSeqsPerLane; ++i) n += pieces[i] == 1 ? max(level[i] + tiles[i] - max(level[i], l), 0) : 0;
    return wave_total(n);
  }
  // Item y of one KV head; false where there is none.
  __device__ __forceinline__ bool find(const ChunkArgs& A, int y, Work& w) const {
    w.slot = y;
    w.piece = 0;
    w.pieces = 1;
    if (rest > 1) {
      if (y >= whole) {
        w.slot = y - whole;
        w.pieces = rest;
        y = w.slot / rest;
        w.piece = w.slot - y * rest;
        y += whole;
      }
    } else if (y < cut) {
      int before = 0;
#pragma unroll
      for (int i = 0; i < kSeqsPerLane; ++i) {
        const int mine = pieces[i] > 1 ? tiles[i] * pieces[i] : 0, upto = before + (int)wave_inclusive_scan_u32((uint32_t)mine);
        const uint64_t hit = __ballot(y >= upto - mine && y < upto);
        if (hit) {
          const int l = __builtin_ctzll(hit), from = __builtin_amdgcn_readlane(upto - mine, l);
          w.pieces = __builtin_amdgcn_readlane(pieces[i], l);
          w.b = l + i * kWave;
          w.tile = (y - from) / w.pieces;
          w.piece = y - from - w.tile * w.pieces;
          return true;
        }
        before = __builtin_amdgcn_readlane(upto, kWave - 1);
      }
      return false;
    } else {
      y -= cut;
    }
    int top = 0;
#pragma unroll
    for (int i = 0; i < kSeqsPerLane; ++i) top = max(top, level[i] + tiles[i]);
    const int step = ((int)wave_max((float)top) + kSteps - 1) / kSteps;
    int lo = 0, hi = kSteps;  // above(lo * step) > y >= above(hi * step)
    const int count = above(0);
    if (count <= y) return false;
    y = order(A, y, count);
#pragma unroll
    for (int x = 1; x < kSteps; x <<= 1) {
      const int mid = (lo + hi) / 2;
      if (above(mid * step) > y) lo = mid; else hi = mid;
    }
    y -= above(hi * step);
    int before = 0;
#pragma unroll
    for (int i = 0; i < kSeqsPerLane; ++i) {
      if (i * kWave >= A.batch) break;
      const int end = min(level[i] + tiles[i], hi * step), mine = pieces[i] == 1 ? max(end - max(level[i], lo * step), 0) : 0;
      const int upto = before + (int)wave_inclusive_scan_u32((uint32_t)mine);
      const uint64_t hit = __ballot(y >= upto - mine && y < upto);
      if (hit) {
        const int l = __builtin_ctzll(hit), last = __builtin_amdgcn_readlane(end - level[i], l) - 1;
        w.b = l + i * kWave;
        w.tile = last - (y - __builtin_amdgcn_readlane(upto - mine, l));
        return true;
      }
      before = __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return false;
  }
};

// Which 16-byte chunk of row `row` lies at place `pos` of the row in LDS, and where chunk c lies in a tile (the same exchange): 16 rows' chunks of
// one column, as K is read, lie in different banks, and so do the four rows by four chunks of V that are read transposed.
template <int D>
__device__ __forceinline__ int k_chunk(int row, int pos) { return D == 128 ? pos ^ (row & 15) : pos ^ ((row >> 1) & 7); }
template <int D>
__device__ __forceinline__ int v_chunk(int row, int pos) { return D == 128 ? pos ^ ((row & 3) << 2) : pos ^ ((row & 2) << 1); }
template <int D>
__device__ __forceinline__ int k_place(int row, int c) { return row * (2 * D) + (k_chunk<D>(row, c) << 4); }
template <int D>
__device__ __forceinline__ int v_place(int row, int c) { return row * (2 * D) + (v_chunk<D>(row, c) << 4); }

// 16 bytes per lane from global memory (a uniform address and a lane's offset) into LDS, the lanes' one behind the other from a uniform place on.
// In assembly, since the compiler lets every transposed read of LDS wait for all such loads; what it does not see has to be awaited by
// wait_loads.  (The result goes to LDS: there is no register that it could overwrite.  M0 is reserved, and nothing else here uses it.)
__device__ __forceinline__ void load_lds_16(const unsigned char* base, uint32_t off, unsigned char* dst) {
  typedef __attribute__((address_space(3))) unsigned char* Lds;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"((uint32_t)(uintptr_t)(Lds)dst), "v"(off), "s"(base) : "memory");
}
// Until this wave's loads into LDS are there (a barrier waits for the other waves').
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <bool BF16>
__device__ __forceinline__ void store_4(void* out, int64_t at, float a, float b, float c, float d) {
  if constexpr (BF16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
  else *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(a, b, c, d);
}

// One row again by one wave: dot products, every key only where it is seen.  (max, sum) and the lane's 8 columns (lane % (D / 8)).
// (Sums of kAgainTiles tiles are added up, not all rows one by one: see lrest.)
template <int D, int FMT, bool PAGED>
__device__ __forceinline__ void row_again(const ChunkArgs& A, int b, int kvh, int64_t q_at, int p, const KeyTiles& T, int i0, int i1, float& m,
                                          float& l, float (&acc)[8]) {
  constexpr int LPR = D / 8, RPW = kWave / LPR;
  const int lane = threadIdx.x & 63, sub = lane % LPR, rsub = lane / LPR;
  const uint4 qv = *reinterpret_cast<const uint4*>(A.q + q_at + sub * 8);
  const uint32_t qw[4] = {qv.x, qv.y, qv.z, qv.w};
  float l_now = 0.f, now[8];
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = now[j] = 0.f;
  auto add_now = [&]() {
    l += l_now;
    l_now = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      acc[j] += now[j];
      now[j] = 0.f;
    }
  };
  for (int i = i0; i < i1; ++i) {
    if ((i - i0) % kAgainTiles == 0) add_now();
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
      l *= alpha;
      l_now = l_now * alpha + w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[2 * j] *= alpha;
        acc[2 * j + 1] *= alpha;
        now[2 * j] = now[2 * j] * alpha + w * bf16_lo(vw[j]);
        now[2 * j + 1] = now[2 * j + 1] * alpha + w * bf16_hi(vw[j]);
      }
    }
  }
  add_now();
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

// This workgroup's work; false where there is none.  Neighbours have the same tile of all KV heads (workgroups go to the XCDs in turn: with a
// multiple of 8 KV heads a KV head's rows stay in one L2).
__device__ __forceinline__ bool find_work(const ChunkArgs& A, int g_shift, Work& w) {
  const int x = blockIdx.x;
  int y = x / A.Hkv;
  w.kvh = x - y * A.Hkv;
  if (A.batch == 1) {
    const NewTokens n = new_tokens(A, 0);
    const SeqTiles t(A, g_shift, n);
    w.b = 0;
    w.slot = y;
    w.piece = 0;
    Cut c(A, 0.5f * (float)(t.tiles * (t.first + t.last)), (float)(t.tiles * t.last), t.last);
    w.pieces = c.pieces(t.last);
    if (w.pieces > 1) {
      if (c.finer(A, w.pieces * t.tiles)) w.pieces = c.pieces(t.last);
      if (w.pieces * t.tiles > A.room) w.pieces = 1;
    }
    if (w.pieces > 1) {
      w.tile = y / w.pieces;
      w.piece = y - w.tile * w.pieces;
      return w.tile < t.tiles;
    }
    if (c.piece == 0.f) {
      const Rest r(A, t.tiles, t.first);
      if (y >= r.whole) {
        w.slot = y - r.whole;
        w.pieces = r.pieces;
        y = w.slot / r.pieces;
        w.piece = w.slot - y * r.pieces;
        y += r.whole;
      }
    }
    w.tile = t.tiles - 1 - order(A, y, t.tiles);
    return w.tile >= 0 && w.tile < t.tiles;
  }
  if (A.batch <= kSeqsMax) {
    Batch all;
    all.read(A, g_shift);
    return all.find(A, y, w);
  }
  // too many sequences to look through: sequence by sequence, whose tiles read the same rows, each beginning with another tile (short sequences leave
  // workgroups without work, and those with work should not all be on the same XCDs).  us with the tiles of a rank together / so: 256 new tokens on
  // 300 x 1K 1934 / 1301, 64 on 300 x 2K 984 / 759.
  const int most = ((A.n_new << g_shift) + kTileRows - 1) / kTileRows;
  w.slot = 0;
  w.b = y / most;
  const int rank = (y - w.b * most + w.b) % most;
  if (w.b >= A.batch) return false;
  w.tile = ((new_tokens(A, w.b).count << g_shift) + kTileRows - 1) / kTileRows - 1 - rank;
  w.piece = 0;
  w.pieces = 1;
  return w.tile >= 0;
}

// Rows of a KV head: row r is query token r / G, head r % G of the group.  A workgroup takes 128 of them, a wave 32, over the key tiles
// of its piece; the tiles go through LDS in bf16, two of K and two of V: while one is worked on, bf16 rows of the next one come straight into the
// other and codes into registers.
//   S^T [keys x rows] = K Q^T   and   O^T [d x rows] += V^T P^T,   P = exp(S - m),
// v_mfma_f32_32x32x16_bf16 (operand lane l: row or column l % 32, eight inner elements of half l / 32; result lane l: column l % 32,
// rows 8 (i / 4) + 4 (l / 32) + i % 4).  A row's scores lie in two lanes, and are the operand of the second product as they come when
// its inner elements j of half h are keys 4 h + j and 8 + 4 h + j - 4; V comes out of LDS transposed.
// TERMS 1 (output in bf16): P rounded to bf16, as the output is.  TERMS 3 (output in 32 bits): P as three bf16 terms that add up to the
// fp32 value.  The sums of P are of the unrounded values.
// The running maximum of a row moves only when a score passes it by more than kLazy (the sums are then at most 2^8 times larger, and fp32 has
// 2^127), so that the results so far are seldom multiplied.
// Bound by the matrix cores and the vector instructions beside them, at the clock that the power allows: 2048 tokens on 64K (group of 4, d 128,
// bf16) 2.01 ms, 1075 TFLOP/s of the 1232 that a large product reaches; the matrix cores are busy for 65 % of the cycles, no LDS bank conflicts.
// A tile of 64 keys takes a workgroup of a full compute unit 2 us (e4m3 2.2, output in 32 bits with d 64 2.5).
// 128 rows, since each row of K and V read from LDS then serves 32 rows of a wave and each loaded one 128; two workgroups per unit, since one's
// barriers are then the other's time (64 KB of LDS each).  The second product is made one tile late, so that the weights' exponentials have matrix
// instructions to run beside (2.38 -> 2.02 ms with the loads straight to LDS).
template <int D, int FMT, bool PAGED, int TERMS>
__global__ __launch_bounds__(kChunkThreads, 2) void chunk_kernel(ChunkArgs A) {
  constexpr int S = D / 16;                        // steps of the first product
  constexpr int E = D / 32;                        // tiles over the head dimension
  constexpr bool QUANT = FMT != VATT_KV_BF16;
  constexpr int TILE = kTileKeys * D * 2;          // bytes
  constexpr float kLazy = 8.0f;
  constexpr bool BF16 = TERMS == 1;
  constexpr int CARRY = BF16 ? 1 : 2;
  __shared__ __align__(256) unsigned char s_kv[4 * TILE];  // K, K, V, V

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, col = lane & 31;
  const int g_shift = 31 - __builtin_clz(A.Hq / A.Hkv), G = 1 << g_shift;
  Work W;
  if (!find_work(A, g_shift, W)) return;
  // (uniform values, as the compiler has to know)
  const int b = __builtin_amdgcn_readfirstlane(W.b), kvh = W.kvh, tile = __builtin_amdgcn_readfirstlane(W.tile);
  const int piece = __builtin_amdgcn_readfirstlane(W.piece), pieces = __builtin_amdgcn_readfirstlane(W.pieces);
  const NewTokens New = new_tokens(A, b);
  const int rows = New.count << g_shift;

  const int r0 = tile * kTileRows;
  const int p_lo = New.first + (r0 >> g_shift), p_hi = New.first + ((min(r0 + kTileRows, rows) - 1) >> g_shift);
  const KeyTiles T = key_tiles(A, p_lo, p_hi);
  const int i0 = T.count * piece / pieces, i1 = T.count * (piece + 1) / pieces;

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

  // The next rows of K and V on their way: bf16 straight into LDS, a 1 KB piece of whole rows per wave and instruction, the lanes' chunks of a
  // row in the order in which they lie there; codes through registers, 16 columns per lane.  A wave has rows 16 wave .. + 15 of a tile, in
  // two groups of 8 (of one page each).  Rows behind the last one that anybody sees are that one again.
  constexpr int ROW = kRowBytes<FMT, D>, LPR = D / 8, RPI = kWave / LPR, LPQ = D / 16, NQ = 16 * LPQ / kWave, QB = ROW / LPQ;
  uint32_t codes[2][NQ][QUANT ? QB / 4 : 1], scales[2][NQ];
  const int last_group = p_hi & ~7;
  struct Rows {
    RowAt at[2];
    int left[2];
  };
  auto block_of = [&](int i, int g) __attribute__((always_inline)) {
    return row_block<PAGED>(A.M, b, min(T.at(min(i, i1 - 1)) * kTileKeys + 16 * wave + 8 * g, last_group));
  };
  auto rows_of = [&](int i, const int (&blk)[2]) __attribute__((always_inline)) {
    Rows r;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int tok = min(T.at(i) * kTileKeys + 16 * wave + 8 * g, last_group);
      r.at[g] = row_at<PAGED>(A.M, b, kvh, tok, blk[g]);
      r.left[g] = p_hi - tok;
    }
    return r;
  };
  constexpr std::integral_constant<int, 0> K = {};
  constexpr std::integral_constant<int, 1> V = {};
  auto buffer = [&](auto kv, int parity) __attribute__((always_inline)) { return &s_kv[(2 * decltype(kv)::value + parity) * TILE]; };
  auto load = [&](auto which, const Rows& R, int parity) __attribute__((always_inline)) {
    constexpr int KV = decltype(which)::value;
    const unsigned char* src = KV ? A.v : A.k;
    if constexpr (!QUANT) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const unsigned char* base = src + R.at[g].row * ROW;
#pragma unroll
        for (int x = 0; x < 8 / RPI; ++x) {
          const int r = x * RPI + lane / LPR, row = 8 * g + r, pos = lane % LPR;
          const int c = KV ? v_chunk<D>(row, pos) : k_chunk<D>(row, pos);
          const uint32_t off = (uint32_t)(min(r, R.left[g]) * ROW + c * 16);
          load_lds_16(base, off, buffer(which, parity) + (16 * wave + 8 * g + x * RPI) * 2 * D);
        }
      }
    } else {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int row = n * (kWave / LPQ) + lane / LPQ, g = row >> 3, c = lane % LPQ;
        const int r = min(row & 7, g ? R.left[1] : R.left[0]);
        const unsigned char* p = src + (g ? R.at[1].row : R.at[0].row) * ROW + (r * ROW + c * QB);
        if constexpr (QB == 16) {
          const uint4 x = *reinterpret_cast<const uint4*>(p);
          codes[KV][n][0] = x.x; codes[KV][n][1] = x.y; codes[KV][n][2] = x.z; codes[KV][n][3] = x.w;
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(p);
          codes[KV][n][0] = x.x; codes[KV][n][1] = x.y;
        }
        scales[KV][n] = src[A.scale_off + (g ? R.at[1].scales : R.at[0].scales) * (D / 32) + (r * (D / 32) + c / 2)];
      }
    }
  };
  auto store = [&](auto which, int parity) __attribute__((always_inline)) {
    constexpr int KV = decltype(which)::value;
    if constexpr (QUANT) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int row = 16 * wave + n * (kWave / LPQ) + lane / LPQ, c = lane % LPQ;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          Chunk<FMT> x;
#pragma unroll
          for (int y = 0; y < QB / 8; ++y) x.w[y] = codes[KV][n][h * (QB / 8) + y];
          *reinterpret_cast<uint4*>(buffer(which, parity) + (KV ? v_place<D>(row, 2 * c + h) : k_place<D>(row, 2 * c + h))) = chunk_bf16<FMT>(x, scales[KV][n]);
        }
      }
    }
  };

  // V of keys between the first tokens and the window of the tile's first row, which nobody sees: 0, so that an Inf or a NaN there, as recycled pages may
  // hold, leaves no row to be worked out again (100 new tokens on 4 x 8K, window of 1000, hidden rows NaN: 2988 us without this, 37 with it).
  // A wave's own rows, before the others read them.
  const int hidden_end = A.window > 0 ? p_lo - A.window + 1 : 0;
  auto hide = [&](int i, int parity) __attribute__((always_inline)) {
    const int k0 = T.at(i) * kTileKeys, from = A.sink - k0, to = hidden_end - k0;
    if (max(from, 0) >= min(to, kTileKeys)) return;
    for (int x = lane; x < 16 * LPR; x += kWave) {
      const int row = 16 * wave + x / LPR;
      if (row >= from && row < to) *reinterpret_cast<uint4*>(buffer(V, parity) + row * (2 * D) + x % LPR * 16) = make_uint4(0, 0, 0, 0);
    }
  };

  f32x16_t acc[E], sc[2];
  uint4 pb[4][CARRY];  // the weights, in bf16 or in 32 bits, from one step to the next
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[e][j] = 0.f;
  // The sum of the weights so far is lrun + lrest: a tile's 32 weights of a lane are added up by themselves, and what their sum loses when it is added
  // to lrun goes to lrest.  Added one by one, the weights of 64K keys of equal score lose up to 5e-4 of their sum.
  float mrun = -INFINITY, lrun = 0.f, lrest = 0.f, ltile = 0.f;
  bool any = false;

  auto first_product = [&](int parity) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const uint4 a = *reinterpret_cast<const uint4*>(buffer(K, parity) + k_place<D>(col, 2 * s + half) + y * 32 * D * 2);
        f32x16_t zero;
#pragma unroll
        for (int j = 0; j < 16; ++j) zero[j] = 0.f;
        sc[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, bq[s]), s == 0 ? zero : sc[y], 0, 0, 0);
      }
    }
  };
  // Masks the scores, and moves the running maximum where one passes it by more than kLazy: true (for the wave) if so, and the factor that
  // the sums so far take.
  auto maximum = [&](int k0, float& alpha) __attribute__((always_inline)) {
    const bool edge = k0 + kTileKeys - 1 > wp_lo || (A.window > 0 && k0 <= wp_hi - A.window && k0 + kTileKeys > A.sink);
    if (edge) {
      // the tile's keys that the lane's row sees, a bit each; the lane's keys of a 32-bit half are 4 half + constants
      const uint64_t seen = ones(p - k0 + 1) & ~(ones(low - k0 + 1) & ~ones(A.sink - k0));
      any |= seen != 0;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const uint32_t bits = (uint32_t)(seen >> (32 * y)) >> (4 * half);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 8 * (j / 4) + j % 4, 1);
          sc[y][j] = __uint_as_float((__float_as_uint(sc[y][j]) & keep) | (0xff800000u & ~keep));  // (-Inf)
        }
      }
    } else {
      any = true;
    }
    float top = sc[0][0];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int j = 0; j < 16; ++j) top = fmaxf(top, sc[y][j]);
    top *= A.log2_scale;
    alpha = 1.f;
    if (!__ballot(top > mrun + kLazy)) return false;
    top = fmaxf(top, __shfl_xor(top, 32));
    const float mnew = fmaxf(mrun, top);
    alpha = mrun == mnew ? 1.f : __builtin_amdgcn_exp2f(mrun - mnew);
    mrun = mnew;
    lrun *= alpha;
    lrest *= alpha;
    return true;
  };
  auto weights = [&](int u, float m) __attribute__((always_inline)) {  // of the keys of step u of the second product
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      y[j] = __builtin_amdgcn_exp2f(fmaf(sc[u / 2][8 * (u % 2) + j], A.log2_scale, -m));
      ltile += y[j];
    }
    if constexpr (BF16) {
      pb[u][0] = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        pb[u][h] = make_uint4(__float_as_uint(y[4 * h]), __float_as_uint(y[4 * h + 1]), __float_as_uint(y[4 * h + 2]), __float_as_uint(y[4 * h + 3]));
    }
  };
  auto second_product = [&](int u, int parity) __attribute__((always_inline)) {
    typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
    const int l16 = lane & 15, c_half = (lane >> 4) & 1;
    uint4 term[TERMS];
    if constexpr (BF16) {
      term[0] = pb[u][0];
    } else {
      float y[8] = {__uint_as_float(pb[u][0].x), __uint_as_float(pb[u][0].y), __uint_as_float(pb[u][0].z), __uint_as_float(pb[u][0].w),
                    __uint_as_float(pb[u][1].x), __uint_as_float(pb[u][1].y), __uint_as_float(pb[u][1].z), __uint_as_float(pb[u][1].w)};
#pragma unroll
      for (int z = 0; z < TERMS; ++z) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j] = pack_bf16(y[2 * j], y[2 * j + 1]);
          y[2 * j] -= bf16_lo(w[j]);
          y[2 * j + 1] -= bf16_hi(w[j]);
        }
        term[z] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int r = 16 * u + 4 * half + (l16 >> 2), c = 4 * e + 2 * c_half + ((l16 & 3) >> 1);
      const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(buffer(V, parity) + v_place<D>(r, c) + (l16 & 1) * 8));
      const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(buffer(V, parity) + v_place<D>(r + 8, c) + (l16 & 1) * 8));
      const bf16x8_t va = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int z = TERMS - 1; z >= 0; --z)
        acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, __builtin_bit_cast(bf16x8_t, term[z]), acc[e], 0, 0, 0);
    }
  };

  // 32 bits: after kSumTiles tiles the sums go, added to those that went before, to the place of the row's result, at which they are relative to
  // maximum m_away; at the end they come back.
  float m_away = -INFINITY;
  bool away = false;  // (uniform)
  const int64_t out_row = ((int64_t)b * A.n_new + t) * A.Hq + head, place = ((int64_t)W.slot * A.Hkv + kvh) * kTileRows + wave * kWaveRows + col;
  auto add_away = [&](auto back) __attribute__((always_inline)) {
    if (row >= rows) return;
    float* at = (pieces == 1 ? static_cast<float*>(A.out_o) + out_row * D : A.part + place * D) + 4 * half;
    const float f = m_away == mrun ? 1.f : __builtin_amdgcn_exp2f(m_away - mrun);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float4* p = reinterpret_cast<float4*>(at + 32 * e + 8 * x);
        if (away) {
          const float4 y = *p;
          acc[e][4 * x] += y.x * f;
          acc[e][4 * x + 1] += y.y * f;
          acc[e][4 * x + 2] += y.z * f;
          acc[e][4 * x + 3] += y.w * f;
        }
        if constexpr (decltype(back)::value == 0) {
          *p = make_float4(acc[e][4 * x], acc[e][4 * x + 1], acc[e][4 * x + 2], acc[e][4 * x + 3]);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[e][4 * x + j] = 0.f;
        }
      }
  };
  auto put_away = [&]() __attribute__((always_inline)) {
    add_away(K);
    m_away = mrun;
    away = true;
  };

  // V is one tile behind K: the second product of tile i - 1 is made while the weights of tile i are, on the matrix cores and beside them.
  if (i0 < i1) {
    int blk[2] = {block_of(i0, 0), block_of(i0, 1)};
    Rows now = rows_of(i0, blk);
    load(K, now, 0);
    blk[0] = block_of(i0 + 1, 0);
    blk[1] = block_of(i0 + 1, 1);
    store(K, 0);
    wait_loads();
#pragma unroll
    for (int s = 0; s < S; ++s) asm volatile("" : "+v"(bq[s].x), "+v"(bq[s].y), "+v"(bq[s].z), "+v"(bq[s].w));
    __syncthreads();
    int parity = 0;
    auto step = [&](int i, auto begin) __attribute__((always_inline)) {
      constexpr bool FIRST = decltype(begin)::value == 1;
      const int other = parity ^ 1;
      load(V, now, parity);
      if (i + 1 < i1) {
        now = rows_of(i + 1, blk);
        load(K, now, other);
      }
      blk[0] = block_of(i + 2, 0);
      blk[1] = block_of(i + 2, 1);
      if (active) {
        first_product(parity);
        // (six reads of K ahead of the products)
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int x = 0; x < S; ++x) {
          __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        float alpha;
        const bool moved = maximum(T.at(i) * kTileKeys, alpha);
        const float m = mrun == -INFINITY ? 0.f : mrun;  // (so far every score is -Inf: weights 0)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if constexpr (!FIRST) second_product(u, other);
          weights(u, m);
        }
        const float sum = lrun + ltile, part = sum - lrun;
        lrest += (lrun - (sum - part)) + (ltile - part);
        lrun = sum;
        ltile = 0.f;
        // (made here, beside the products, not after the branch)
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int z = 0; z < CARRY; ++z) asm volatile("" : "+v"(pb[u][z].x), "+v"(pb[u][z].y), "+v"(pb[u][z].z), "+v"(pb[u][z].w));
        if (!FIRST && moved) {
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] *= alpha;
        }
      }
      store(V, parity);
      if (i + 1 < i1) store(K, other);
      wait_loads();
      hide(i, parity);
      __syncthreads();
      parity = other;
    };
    step(i0, V);
    for (int i = i0 + 1; i < i1;) {
      const int stop = BF16 ? i1 : min(i + kSumTiles, i1);
      for (; i < stop; ++i) step(i, K);
      if (!BF16 && active && i < i1) put_away();
    }
    if (active) {
#pragma unroll
      for (int u = 0; u < 4; ++u) second_product(u, parity ^ 1);
      if (!BF16 && away) add_away(V);
    }
  }
  if (!active) return;

  // A result with an Inf or a NaN is worked out again: the second product gives every row every V row of a tile, with weight 0 where
  // the row does not see the key (and in three terms of which some are 0), so that an Inf or a NaN has a say where it should have none.
  lrun += lrest;
  float l = lrun + __shfl_xor(lrun, 32);
  const bool saw = any || __shfl_xor((int)any, 32);
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int j = 0; j < 16; ++j) sum += fabsf(acc[e][j]);
  const uint64_t odd = __ballot(!(sum < INFINITY) || !(l < INFINITY));
  uint32_t again = (uint32_t)odd | (uint32_t)(odd >> 32);
  const float m_own = saw && mrun == -INFINITY ? -3.0e38f : mrun, inv = 1.f / l;
  // bf16: a row's two lanes change columns 8 x + 4 half .. + 3 of two groups for all 8 of one
  uint4 out16[BF16 ? E : 1][2];
  if constexpr (BF16) {
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint32_t w[2][2];
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int z = 0; z < 2; ++z) w[y][z] = pack_bf16(acc[e][8 * x + 4 * y + 2 * z] * inv, acc[e][8 * x + 4 * y + 2 * z + 1] * inv);
        const auto a = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false), b = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
        out16[e][x] = make_uint4(a[0], b[0], a[1], b[1]);
      }
  }
  if (row < rows && !(again >> col & 1)) {
    if (pieces == 1) {
      if constexpr (BF16) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int x = 0; x < 2; ++x)
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(A.out_o) + (out_row * D + 32 * e + 16 * x + 8 * half)) = out16[e][x];
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            store_4<false>(A.out_o, out_row * D + 32 * e + 8 * x + 4 * half, acc[e][4 * x] * inv, acc[e][4 * x + 1] * inv, acc[e][4 * x + 2] * inv,
                           acc[e][4 * x + 3] * inv);
      }
      if (A.out_lse && half == 0) A.out_lse[out_row] = m_own * 0.69314718055994530942f + logf(l);
    } else {
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
    if (pieces == 1) {
      const float inv = 1.f / ls;
      store_4<BF16>(A.out_o, out_c * D + lane * 8, a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv);
      store_4<BF16>(A.out_o, out_c * D + lane * 8 + 4, a[4] * inv, a[5] * inv, a[6] * inv, a[7] * inv);
      if (A.out_lse && lane == 0) A.out_lse[out_c] = m * 0.69314718055994530942f + logf(ls);
    } else {
      const int64_t place = ((int64_t)W.slot * A.Hkv + kvh) * kTileRows + wave * kWaveRows + c;
      store_4<false>(A.part, place * D + lane * 8, a[0], a[1], a[2], a[3]);
      store_4<false>(A.part, place * D + lane * 8 + 4, a[4], a[5], a[6], a[7]);
      if (lane == 0) A.part_ml[place] = make_float2(m, ls);
    }
  }
}

// The pieces' partial sums together, a row per wave at a time; the rows of a tile go round the workgroups of its pieces.  Bound by three dependent
// reads (the lengths, a row's maxima, its sums), 4 us; 10 where 33 tokens on 5K - 16K are cut into 236 pieces (16 MB).
template <int D, bool BF16>
__global__ __launch_bounds__(kChunkThreads) void chunk_merge_kernel(ChunkArgs A) {
  constexpr int C = D / kWave, kAhead = 8;
  static_assert(kPiecesMax <= kWave, "a pair per lane");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kvh = blockIdx.x % A.Hkv;
  const int part = blockIdx.y * kChunkWaves + wave, parts = gridDim.y * kChunkWaves;
  const int g_shift = 31 - __builtin_clz(A.Hq / A.Hkv);
  Batch all;
  all.read(A, g_shift);
  for (int y = blockIdx.x / A.Hkv; y < all.cut; y += gridDim.x / A.Hkv) {
    Work w;
    if (!all.find(A, all.rest > 1 ? all.whole + y : y, w)) return;
    const NewTokens New = new_tokens(A, w.b);
    // (the workgroups of all pieces share out the tile's rows)
    const int n = min((New.count << g_shift) - w.tile * kTileRows, kTileRows);
    for (int r = w.piece * parts + part; r < n; r += w.pieces * parts) {
      const int row = w.tile * kTileRows + r;
      const int64_t out_row = ((int64_t)w.b * A.n_new + (row >> g_shift)) * A.Hq + ((int64_t)kvh << g_shift) + (row & ((1 << g_shift) - 1));
      const int slot0 = (y - w.piece) * A.Hkv + kvh;
      auto place = [&](int s) { return (int64_t)(slot0 + s * A.Hkv) * kTileRows + r; };
      const float2 ml = lane < w.pieces ? A.part_ml[place(lane)] : make_float2(-INFINITY, 0.f);
      const float m = wave_max(ml.x);
      const bool counts = ml.x > -INFINITY;  // (a piece without a token, whose sums nobody wrote, does not)
      const float f = !counts ? 0.f : ml.x == m ? 1.f : __builtin_amdgcn_exp2f(ml.x - m);
      const float l = wave_sum_f32(counts ? ml.y * f : 0.f);
      const uint64_t there = __ballot(counts);
      float a[C];
#pragma unroll
      for (int c = 0; c < C; ++c) a[c] = 0.f;
      for (int s0 = 0; s0 < w.pieces; s0 += kAhead) {
        float x[kAhead][C];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
#pragma unroll
          for (int c = 0; c < C; ++c) x[u][c] = A.part[place(min(s0 + u, w.pieces - 1)) * D + lane * C + c];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          if (s0 + u >= w.pieces || !(there >> (s0 + u) & 1)) continue;
          const float g = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), s0 + u));
#pragma unroll
          for (int c = 0; c < C; ++c) a[c] += g * x[u][c];
        }
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
  }
}

// Tiles of all sequences if every new token counts.
int64_t chunk_tiles(const Plan& pl, int n_new) {
  return (int64_t)pl.p.batch * pl.p.n_kv_heads * (((int64_t)n_new * pl.group + kTileRows - 1) / kTileRows);
}
int chunk_slots(const Plan& pl) { return 2 * pl.num_cus; }
// Whether pieces can be wanted at all (the rule of Cut) for queries that see up to `keys` tokens; the merge is launched only then.  Of a batch the
// host knows too little.  fewer: fewer than n_new tokens may count.  Then every length can be wanted in pieces, and the launch for it, 2 to 15 us, is
// worth it beyond 32 key tiles (64 of 2048 tokens count, us in whole tiles / in pieces: on 4K 72 / 24, on 64K 1033 / 99; where all 4096 of a prompt
// count 165 / 167).
bool chunk_may_cut(const Plan& pl, int n_new, bool fewer, int64_t keys) {
  const double longest = (double)((keys + kTileKeys - 1) / kTileKeys), own = std::min((double)n_new / kTileKeys, longest);
  if (pl.p.batch > kSeqsMax || longest <= 12) return false;
  if (pl.p.batch > 1 || (fewer && longest > 32)) return true;
  // one sequence: a rest of tiles behind full slots, of some length; or its new tokens at the end of the capacity, or at its beginning (the rule is linear in between)
  const int64_t all = chunk_tiles(pl, n_new);
  if (all > chunk_slots(pl) && all % chunk_slots(pl) != 0 && std::min<int64_t>(pl.p.n_max - n_new, keys) / kTileKeys + 1 >= kRestLeast) return true;
  const double tiles = (double)all / chunk_slots(pl);
  return longest > 1.25 * tiles * (longest - own / 2) + 12 || own > 1.25 * tiles * own / 2 + 12;
}
// Pieces at most, so that what all tiles are cut into has room:
//   * A piece has 1 / 0.97 of an equal share of all tiles at their longest, `most`, for a slot each (Cut), so that all are 0.97 slots pieces long.  Two or
//     more to the nearest number are 4/3 of that at most: 1.3 slots.
//   * Only where these are more than the slots they are halved (Cut::finer): rounded down, 2 * 0.97 = 1.94 slots.
//   * Of a rest (Rest) there are two slots full.
//   * A tile of n key tiles has ceil(n / kPieceLeast) pieces at most: a piece is no shorter, and a halved one is longer too, since below kOnePerUnit
//     key tiles there is one piece for two slots, never more than the slots, and above it half a piece is 5000 / (2 * 0.97 slots) = 5.
int64_t chunk_pieces(const Plan& pl, int n_new, bool fewer, int64_t keys) {
  if (!chunk_may_cut(pl, n_new, fewer, keys)) return 0;
  const int64_t longest = (pl.p.n_max + kTileKeys - 1) / kTileKeys, each = std::min<int64_t>((longest + kPieceLeast - 1) / kPieceLeast, kPiecesMax);
  return std::min<int64_t>(2 * chunk_slots(pl), chunk_tiles(pl, n_new) * each);
}

template <int D, int FMT, bool PAGED, int TERMS>
hipError_t launch_chunk_t(const Plan& pl, const ChunkArgs& A, hipStream_t st) {
  const int64_t tiles = chunk_tiles(pl, A.n_new), pieces = (int64_t)A.room * A.Hkv;
  hipLaunchKernelGGL((chunk_kernel<D, FMT, PAGED, TERMS>), dim3((uint32_t)(tiles + pieces)), dim3(kChunkThreads), 0, st, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || A.room == 0) return e;
  // About a row per wave where a tile has few pieces (4 x 1K tokens, 32 new ones each, whole call 28.5 us with one workgroup per piece, 21.8 with
  // eight); one workgroup per piece where cuts are unlikely (with eight windowed prompts that are not cut take 147 us instead of 141).
  // No more than two times the compute units to a part (4 windowed chunks of 100 tokens, not cut, 28.2 us, with four times 30.3; 33 tokens on
  // 3 x 5K - 16K 49, with one time 54).
  const int64_t rows = std::min<int64_t>(kTileRows, (int64_t)A.n_new * pl.group), wgs = std::min<int64_t>(A.room, (2 * pl.num_cus + A.Hkv - 1) / A.Hkv);
  const int64_t parts = 2 * tiles >= pieces ? 1 : std::max<int64_t>(1, std::min<int64_t>(8, rows / kChunkWaves * tiles / pieces));
  hipLaunchKernelGGL((chunk_merge_kernel<D, TERMS == 1>), dim3((uint32_t)(wgs * A.Hkv), (uint32_t)parts), dim3(kChunkThreads), 0, st, A);
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

// Few query vectors per KV head go to the kernel of the decode steps, which reads the keys once for 32 of them.  Whole call, us, this kernel / that
// one: 28 vectors on 1K tokens 16.1 / 11.4, 16 on 16 x 16K 196 / 177 (e4m3 161 / 112), 32 on 16 x 16K 196 / 191 (e4m3 164 / 126), but 64 205 /
// 326 (e4m3 185 / 219).
bool chunk_is_few(const Plan& pl, int n_new) { return n_new * pl.group <= 32; }

}  // namespace

bool chunk_fits(const Plan& pl, int n_new) {
  return chunk_tiles(pl, n_new) + 2 * chunk_slots(pl) <= INT32_MAX / kChunkThreads;
}

size_t chunk_workspace_bytes(const Plan& pl, int n_new) {
  if (chunk_is_few(pl, n_new)) return few_workspace_bytes(pl, n_new);
  return (size_t)chunk_pieces(pl, n_new, true, pl.p.n_max) * kTileRows * (pl.p.head_dim + 2) * sizeof(float);
}

hipError_t launch_chunk(const Plan& pl, const void* q, int64_t q_stride, int n_new, const int32_t* first, const int32_t* new_lens, const void* k,
                        const void* v, const int32_t* block_table, int sink, int window, void* ws, bool bf16, void* out_o, float* out_lse,
                        hipStream_t st) {
  if (chunk_is_few(pl, n_new))
    return launch_few(pl, q, q_stride, n_new, first, new_lens, k, v, block_table, sink, window, ws, bf16, out_o, out_lse, st);
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
  A.slots = chunk_slots(pl);
  A.sink = std::min(sink, pl.p.n_max);
  A.window = std::min(window, pl.p.n_max);
  // (a window: its tiles and those of the first tokens, of which one more may be begun each, and those of a tile of rows)
  const int64_t seen = (int64_t)A.sink + A.window + kTileRows / pl.group + 2 * kTileKeys;
  const int64_t pieces = chunk_pieces(pl, n_new, new_lens != nullptr, A.window > 0 ? std::min<int64_t>(pl.p.n_max, seen) : pl.p.n_max);
  A.room = (int)(pieces / A.Hkv);
  A.log2_scale = (float)((double)pl.sm_scale * 1.4426950408889634);
  A.part = static_cast<float*>(ws);
  A.part_ml = reinterpret_cast<float2*>(A.part + (size_t)pieces * kTileRows * pl.p.head_dim);
  return pl.p.head_dim == 128 ? launch_chunk_d<128>(pl, A, bf16, st) : launch_chunk_d<64>(pl, A, bf16, st);
}

}  // namespace vatt
