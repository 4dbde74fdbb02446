// Attention of new tokens over a paged cache (include/paged_attn.h).
//
// Rows: the new tokens of a sequence times the query heads of a key/value head, 32 of them to a group (the columns of a 32 x 32 product), up to four groups to a block.  Units: a block of rows against
// kBlockKeys keys.  All units of a key/value head, sequence after sequence, are dealt to `shares` workgroups in equal shares, so that ragged lengths fill the chip evenly and one long sequence as well as
// many short ones.  A workgroup finds its share itself, from the lengths (a sum over the sequences: the host does not know them).  Inside it, its waves take tiles of 32 keys in turn, each with
// a softmax (maximum, sum, weighted values) of its own; what belongs to one block of rows is put together in LDS when the workgroup leaves it, and written, or, where the block's walk began in or goes on
// in another share, left in the workspace for join_kernel, which deals the rows of all such blocks to workgroups.
//
// A wave's tile: K from memory into the registers of the product K Q^T (no LDS: a key is read by one wave, once), V in whole rows through registers into LDS, from where it is read transposed; both are
// loaded one tile ahead (two ahead was slower).  Q lies in LDS, in the order in which lanes read it: in registers it left the compiler too few for the loads ahead (64 sequences of 3900 keys on average,
// 32/8 heads of 128: 259 -> 198 us).  Head dimension 256 would need 128 registers for the output and as many for a tile: there two waves share a tile, each with half of the dimensions, and add up
// their halves of the scores through LDS (32 sequences with up to 8 drafts, 16/4 heads: 293 -> 146 us then, 131 now).  More than 32 rows: the waves of a workgroup divide into groups of rows that load the same tile.
//
// Bound by memory: one token of 32/8 heads takes four operations for each byte of the cache, 32 rows 32.  Weights go into the product with V as two bf16 terms (one would leave the output with
// 2.4e-3 of itself in place of 1.7e-3), for e4m3 values, which float16 has, as one float16 term (2^-11).  Measured: 64 sequences as above 194 us, 5.4 TB/s; 8 of 32768 keys 197, 5.45; 8 of 131072
// keys of 8 bits 369, 5.8; one of 131072 keys of 8 bits with 40 rows 74, 3.6 TB/s: there vector units (48 % of the time) and matrix units (27 %) take turns.  What is short: a launch with one block of
// 60 keys takes 8 us, of which 2 until the first loads, 2.5 for them, 1 for the tile, 2 to put results together; cutting adds a launch of 4.4 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "../../include/paged_attn.h"
#include "kernels.hpp"
#include "operators.hpp"
#include "paged.hpp"
#include "paged_shares.hpp"
#include "tiles.hpp"

namespace chunk_attn {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRows = 32;               // rows of a block
constexpr int kTile = 32;               // keys of a tile
constexpr int kBlockKeys = kTile * kWaves;
constexpr int kMostShares = 2 * kCus;     // of a head
constexpr float kFloor = -3e38f;        // of a running maximum: what is masked (-inf) stays below it, so that no difference of two infinities is formed
// Weights are 2^(score - m) for an m that the largest score may exceed by kGrowth before it moves, to kBelow below that score (log2): weights that go into products as float16 (e4m3 values) then stay
// under 2^15, and what is flushed to zero is below 2^-32 of the largest.
constexpr float kGrowth = 15.f, kBelow = 7.f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnArgs {
  const __bf16* q;
  int64_t q_stride;
  const void *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *table, *kv_len, *q_start;
  __bf16* o;
  int64_t o_stride;
  float* lse;
  float* parts;   // two of each (share, head): the block of rows that came from the share before, and the one that goes on in the next
  int32_t* cuts;  // [shares][kCut]: the block of rows that begins in the share and goes on in the next
  int32_t num_seqs, total_q, heads, group, page_size, num_pages, max_pages, shares;
  int32_t most_subs;  // groups of rows that walk over the keys together, at most
  float scale_log2;
  Divide by_page, by_group, by_shares;
};
// First row of q of its sequence, its first row of the sequence's, how many rows, and in how many shares it lies.
enum { kCutSeqRow, kCutRow, kCutRows, kCutShares, kCut };

// Head dimension 256: a tile takes two waves, and LDS has no room for the queries of more groups.
template <int D>
constexpr int most_subs() { return D == 256 ? 1 : 4; }
template <int D>
constexpr int part_floats() { return kRows * (D + 2); }

// Sequence i, its numbers brought into their ranges.
static_assert(kRows == 1 << 5);
struct Sequence {
  int len, rows, first_row;  // tokens; rows of a key/value head; first row of q
  // groups of kRows rows that walk over the keys together: 1, 2 or 4 (`most` at most), as the logarithm
  __device__ int log_subs(int most) const { return rows <= kRows || most == 1 ? 0 : rows <= 2 * kRows ? 1 : 2; }
  __device__ int row_blocks(int most) const {
    const int log = 5 + log_subs(most);
    return (rows + (1 << log) - 1) >> log;
  }
  __device__ int key_blocks() const { return max(1, (int)(((unsigned)len + kBlockKeys - 1) / kBlockKeys)); }
  __device__ int units(int most) const { return row_blocks(most) * key_blocks(); }  // < 2^30 (check_desc)
};
__device__ __forceinline__ Sequence sequence_at(const AttnArgs& a, int i) {
  Sequence s;
  const int most = a.max_pages * a.page_size;
  s.len = min(max(a.kv_len[i], 0), most);
  const Rows r = rows_between(a.q_start[i], a.q_start[i + 1], a.total_q);
  s.first_row = r.first;
  s.rows = r.count * a.group;
  return s;
}

// A value that all lanes of a wave have, as one the compiler knows to be so.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// A barrier that what this wave wrote to LDS is there before, but that waits for no loads from memory.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  wg_barrier();
}
// The lowest n bits (none if n < 0, all if n > 31).
__device__ __forceinline__ unsigned first_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1; }

// 16 bytes of the cache.
__device__ __forceinline__ u32x4 load16(const char* p) { return *reinterpret_cast<const u32x4*>(p); }
// Eight e4m3 numbers as bf16, which has them all.
__device__ __forceinline__ bf16x8 widen8(unsigned a, unsigned b) {
  bf16x8 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const bf16x2 x = w & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w & 2 ? b : a, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w & 2 ? b : a, 1.f, false);
    r[2 * w] = x[0];
    r[2 * w + 1] = x[1];
  }
  return r;
}
// The same as float16, which has them all too, and weights to go with them in one term: half a step is 2^-11.
__device__ __forceinline__ f16x8 widen8_f16(unsigned a, unsigned b) {
  f16x8 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const f16x2 x = w & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w & 2 ? b : a, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w & 2 ? b : a, 1.f, false);
    r[2 * w] = x[0];
    r[2 * w + 1] = x[1];
  }
  return r;
}
// Whether one of the numbers in 16 bytes of the cache is infinite or none.
template <bool E4M3>
__device__ __forceinline__ bool some_not_finite(u32x4 x) {
  unsigned r = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    // an exponent of ones (e4m3: a NaN, all other bits ones), plus one in its last place, overflows into the bit above it
    if (E4M3) r |= ((x[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    else r |= ((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  }
  return r != 0;
}

// Bytes from row to row of V's tile in LDS: 64 bytes past a multiple of 256 (192: 64 short of it), so that the four rows of a transposed read lie on different banks.
template <int D>
constexpr int v_pitch() { return D == 96 ? 192 : D * 2 + 64; }

// Where the keys of a tile are: numbers of their pages and rows in them, of the first key of each half (HALVES: page_size is a multiple of 16, so that 16 keys lie on one page), or of this
// lane's key (col); bit k of `there`: key k lies on a page that is one.
template <bool HALVES>
struct Place {
  int number[2], row[2];
  unsigned there;
};
template <>
struct Place<false> {
  int number, row;
  unsigned there;
};

template <int D, bool E4M3, bool HALVES>
__global__ __launch_bounds__(kThreads, 2) void attn_kernel(const AttnArgs a) {
  constexpr int kBytes = E4M3 ? 1 : 2;                  // of a number in the cache
  constexpr int kParts = D == 256 ? 2 : 1, kSubs = most_subs<D>();
  constexpr int kOwn = D / kParts;                      // dimensions of a wave
  constexpr int kDims = kOwn / 32;                      // 32 dimensions of the output, or of the scores' sum, at a time
  constexpr int kPitch = v_pitch<kOwn>() / 2;           // elements
  constexpr int kRowBytes = D * kBytes, kOwnBytes = kOwn * kBytes;
  constexpr int kRowChunks = kOwnBytes / 16, kVChunks = kRowChunks / 2;  // 16-byte chunks of a wave's part of a row; of a tile, for each lane
  using Value = std::conditional_t<E4M3, _Float16, __bf16>;  // of V in LDS
  constexpr bool kEven = 64 % kRowChunks == 0;          // a wave's 16-byte loads are whole rows
  constexpr int kRowsApart = kEven ? 64 / kRowChunks : 0;
  // The n-th 16 bytes of a tile's V that a lane has: key, place in the row, place in LDS.
  struct Chunk {
    int row, in_row, in_lds;
    __device__ Chunk(int lane, int n) {
      row = kEven ? lane / kRowChunks + n * kRowsApart : (lane + 64 * n) / kRowChunks;
      in_row = kEven ? lane % kRowChunks : lane + 64 * n - row * kRowChunks;
      in_lds = (kEven ? lane / kRowChunks * kPitch + n * (kRowsApart * kPitch) : row * kPitch) + in_row * (16 / kBytes);
    }
  };
  struct Walk {
    __bf16 tiles[kWaves][kTile * kPitch];
    bf16x8 q[kSubs][D / 16][64];
    f32x4 partial[kParts == 2 ? kWaves : 1][kParts == 2 ? 4 : 1][kParts == 2 ? 64 : 1];  // scores of a wave's dimensions
  };
  __shared__ union __attribute__((aligned(16))) Pool {
    Walk walk;
    f32x4 values[kWaves][kDims * 4][64];  // the waves' results, when they are put together
    __device__ Pool() {}
  } pool;
  auto& tiles = pool.walk.tiles;
  auto& q = pool.walk.q;
  auto& partial = pool.walk.partial;
  __shared__ float maxima[kWaves][kRows], sums[kWaves][kRows];
  __shared__ uint32_t wave_units[kWaves];
  __shared__ int start_seq, start_unit;
  __shared__ Sequence in_lds[kThreads];  // where there are no more than threads

  const int head = blockIdx.x % a.heads, share = blockIdx.x / a.heads;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int part = wave % kParts;

  // ---- the share: units first .. last - 1 of all ----
  const int each = (a.num_seqs + kThreads - 1) / kThreads;
  const int seq0 = min((int)threadIdx.x * each, a.num_seqs), seq1 = min(seq0 + each, a.num_seqs);
  // (sums that stay at their largest: starts of rows that do not increase may make them too large, and the share is then of some of the units)
  uint32_t mine = 0;
  for (int i = seq0; i < seq1; ++i) {
    const Sequence s = sequence_at(a, i);
    if (each == 1) in_lds[i] = s;
    mine = sum_at_most(mine, s.units(a.most_subs));
  }
  const uint32_t up_to = wave_sum_up_to(mine);
  uint32_t before = (uint32_t)__shfl_up((int)up_to, 1);
  if (lane == 0) before = 0;
  if (lane == 63) wave_units[wave] = up_to;
  if (threadIdx.x == 0) start_seq = -1;
  __syncthreads();
  uint32_t all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before = sum_at_most(before, wave_units[w]);
    all = sum_at_most(all, wave_units[w]);
  }
  const int total = uniform((int)min(all, 1u << 30)), size = max(1, a.by_shares(total + a.shares - 1));
  const int first = (int)min((int64_t)share * size, (int64_t)total), last = min(first + size, total);
  if ((uint32_t)first >= before && (uint32_t)first < sum_at_most(before, mine)) {
    int at = first - (int)before, i = seq0;
    while (each > 1) {
      const int u = sequence_at(a, i).units(a.most_subs);
      if (at < u) break;
      at -= u;
      ++i;
    }
    start_seq = i;
    start_unit = at;
  }
  __syncthreads();
  int seq = uniform(start_seq), in_seq = uniform(start_unit);  // units of the sequence before the next
  if (threadIdx.x == 0 && head == 0) a.cuts[share * kCut + kCutRows] = 0;
  if (seq < 0 || first >= total) return;
  const float k_scale = E4M3 ? a.k_scale[head] : 1.f, v_scale = E4M3 ? a.v_scale[head] : 1.f;
  const float scale = a.scale_log2 * k_scale;
  const char *const k_base = (const char*)a.k + part * kOwnBytes, *const v_base = (const char*)a.v + part * kOwnBytes;

  for (int unit = first; unit < last;) {
    Sequence s = each == 1 ? in_lds[seq] : sequence_at(a, seq);
    s = Sequence{uniform(s.len), uniform(s.rows), uniform(s.first_row)};
    if (s.rows == 0 || in_seq >= s.units(a.most_subs)) {
      ++seq;
      in_seq = 0;
      continue;
    }
    const int key_blocks = s.key_blocks();
    const int row_block = in_seq < key_blocks ? 0 : (int)((unsigned)in_seq / (unsigned)key_blocks), block0 = in_seq - row_block * key_blocks;
    const int block1 = min(key_blocks, block0 + (last - unit));
    // rows of this lane's column
    // Waves: `part` of the dimensions, `sub` of the block's rows, and `team`, which takes every teams-th tile.  (Waves of one team load the same tile at about the same time, so that it
    // comes from memory once.)
    const int log_subs = s.log_subs(a.most_subs), subs = 1 << log_subs, sub = wave / kParts & (subs - 1), team = wave / kParts >> log_subs, teams = kWaves / kParts >> log_subs;
    const int row0 = min((row_block * subs + sub) * kRows, s.rows - 1);
    const int row = (row_block * subs + sub) * kRows + col;
    const bool live = row < s.rows;
    const int token = a.by_group(min(row, s.rows - 1)), q_row = s.first_row + token, q_head = head * a.group + min(row, s.rows - 1) - token * a.group;
    const int tokens = a.by_group(s.rows);
    const int seen = s.len - tokens + token + 1;  // keys that the row sees (none if <= 0)
    const int first_seen = s.len - tokens + a.by_group(row0) + 1;                               // of the first row,
    const int most_seen = max(0, s.len - tokens + a.by_group(min(row0 + kRows, s.rows) - 1) + 1);  // and of the last
    // operand B of K Q^T: in step 2 t + u, half h has dimensions 32 t + 16 h + 8 u .. + 7; the waves of a sub share the loads
    constexpr int kLoads = D / 16 / (kSubs == 1 ? kWaves : 1);  // at most
    bf16x8 own_q[kLoads];
    const int sharers = teams * kParts, first_q = team * kParts + part;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int n = i * sharers + first_q;
      if (n < D / 16) own_q[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const Loose8*>(a.q + (int64_t)q_row * a.q_stride + (int64_t)q_head * D + 16 * half + (n >> 1) * 32 + (n & 1) * 8));
    }
    f32x16 acc[kDims] = {};
    float m = kFloor, l = 0.f;

    // ---- the walk ----
    const int tile1 = min(block1 * kWaves, (int)(((unsigned)most_seen + kTile - 1) / kTile));
    const int32_t* const pages = a.table + (int64_t)seq * a.max_pages;
    u32x4 kr[kDims * kBytes], vr[kVChunks];
    Place<HALVES> at, next;
    auto find = [&](int tile) {
      Place<HALVES> r;
      if constexpr (HALVES) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = tile * kTile + 16 * h, page = a.by_page(min(key, most_seen - 1));
          r.number[h] = key < most_seen ? pages[page] : -1;
          r.row[h] = key - page * a.page_size;
        }
      } else {
        const int key = tile * kTile + col, page = a.by_page(min(key, most_seen - 1));
        r.number = key < most_seen ? pages[page] : -1;
        r.row = key - page * a.page_size;
      }
      return r;
    };
    // Starts the loads of a tile; afterwards at.there says which of its keys there are.
    auto load_tile = [&]() {
      if constexpr (HALVES) {
        int rows[2];
        bool ok[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int number = uniform(at.number[h]);
          ok[h] = number >= 0 && number < a.num_pages;
          rows[h] = ok[h] ? (number * a.heads + head) * a.page_size + at.row[h] : 0;
        }
        at.there = (ok[0] ? 0xffffu : 0u) | (ok[1] ? 0xffff0000u : 0u);
        const char* const p = k_base + (int64_t)(col & 16 ? rows[1] : rows[0]) * kRowBytes + (col & 15) * kRowBytes + half * (16 * kBytes);
#pragma unroll
        for (int t = 0; t < kDims; ++t)
#pragma unroll
          for (int u = 0; u < kBytes; ++u) kr[t * kBytes + u] = load16(p + t * (32 * kBytes) + u * 16);
        const char* const from[2] = {v_base + (int64_t)rows[0] * kRowBytes, v_base + (int64_t)rows[1] * kRowBytes};
#pragma unroll
        for (int n = 0; n < kVChunks; ++n) {
          // (where a wave's loads are whole rows, the n-th is of one half)
          const Chunk c(lane, n);
          if constexpr (kEven && kRowsApart <= 16) vr[n] = load16(from[n * kRowsApart / 16] + (unsigned)(lane / kRowChunks * kRowBytes + c.in_row * 16) + (n * kRowsApart % 16) * kRowBytes);
          else vr[n] = load16((c.row & 16 ? from[1] : from[0]) + (c.row & 15) * kRowBytes + c.in_row * 16);
        }
      } else {
        const bool ok = at.number >= 0 && at.number < a.num_pages;
        const int row = ok ? (at.number * a.heads + head) * a.page_size + at.row : 0;
        at.there = (unsigned)__ballot(ok);
        const char* const p = k_base + (int64_t)row * kRowBytes + half * (16 * kBytes);
#pragma unroll
        for (int t = 0; t < kDims; ++t)
#pragma unroll
          for (int u = 0; u < kBytes; ++u) kr[t * kBytes + u] = load16(p + t * (32 * kBytes) + u * 16);
#pragma unroll
        for (int n = 0; n < kVChunks; ++n) {
          const Chunk c(lane, n);
          vr[n] = load16(v_base + (int64_t)__shfl(row, c.row) * kRowBytes + c.in_row * 16);
        }
      }
    };
    __bf16* const v_tile = tiles[wave];
    int tile = block0 * kWaves + team;
    at = find(tile);
    next = find(tile + teams);
    load_tile();
    // queries to LDS, in the order in which the lanes read them (in registers they would leave too few for the loads ahead); the tiles' loads go on
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      if (i * sharers + first_q < D / 16) q[sub][i * sharers + first_q][lane] = live ? own_q[i] : bf16x8{};
    lds_barrier();
    // (waves that share a tile's dimensions all go on to the last tile of any, as they wait for each other)
    auto more = [&]() { return kParts == 1 ? tile < tile1 : tile - team < tile1; };
    auto step = [&]() {
      // bit k: key k of the tile is there and seen by a row of the block; is seen by this lane's row
      const unsigned keys = at.there & first_bits(most_seen - tile * kTile), visible = at.there & first_bits(seen - tile * kTile);
      const bool border = (tile + 1) * kTile > first_seen || at.there != 0xffffffffu;
      // V to LDS
      unsigned odd = 0;  // bit k: this lane has values of key k that are not finite
      if (border) {      // keys that no row sees are zeros
        const int first_row = kEven ? lane / kRowChunks : 0;
        const unsigned mine = keys >> first_row;
#pragma unroll
        for (int n = 0; n < kVChunks; ++n) {
          const int row = kEven ? n * kRowsApart : Chunk(lane, n).row;  // (less first_row)
          const bool there = mine & (1u << row);
#pragma unroll
          for (int e = 0; e < 4; ++e) vr[n][e] = there ? vr[n][e] : 0;
          odd |= some_not_finite<E4M3>(vr[n]) ? 1u << row : 0u;
        }
        odd <<= first_row;
      }
#pragma unroll
      for (int n = 0; n < kVChunks; ++n) {
        __bf16* const to = v_tile + Chunk(lane, n).in_lds;
        if constexpr (E4M3) {
          *reinterpret_cast<f16x8*>(to) = widen8_f16(vr[n][0], vr[n][1]);
          *reinterpret_cast<f16x8*>(to + 8) = widen8_f16(vr[n][2], vr[n][3]);
        } else {
          *reinterpret_cast<u32x4*>(to) = vr[n];
        }
      }
      // scores
      f32x16 score = {};
#pragma unroll
      for (int n = 0; n < 2 * kDims; ++n) {
        bf16x8 x;
        if constexpr (E4M3) x = n & 1 ? widen8(kr[n >> 1][2], kr[n >> 1][3]) : widen8(kr[n >> 1][0], kr[n >> 1][1]);
        else x = __builtin_bit_cast(bf16x8, kr[n]);
        score = mfma32(x, q[sub][part * 2 * kDims + n][lane], score);
      }
      // the next tile, and the page of the one after it (behind the last one: loads that nobody waits for, of a row that is there)
      at = next;
      load_tile();
      next = find(tile + 2 * teams);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (kParts == 2) {  // the other half of the dimensions
        wg_barrier();  // (the last tile's have been read: their sums were used)
#pragma unroll
        for (int g = 0; g < 4; ++g) partial[wave][g][lane] = f32x4{score[4 * g], score[4 * g + 1], score[4 * g + 2], score[4 * g + 3]};
        lds_barrier();
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 x = partial[wave ^ 1][g][lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) score[4 * g + e] += x[e];
        }
      }
      if (border) {
        const unsigned mine = visible >> (4 * half);
#pragma unroll
        for (int e = 0; e < 16; ++e) score[e] = mine & (1u << (8 * (e >> 2) + (e & 3))) ? score[e] : -INFINITY;
      }
      // softmax
      float top = score[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, score[e]);
      top = max_halves(top) * scale;
      if (__any(top > m + kGrowth)) {
        // (a row whose scores have not leaves its own where it is, so that no row's result depends on others)
        const float to = top > m + kGrowth ? top - kBelow : m, f = __builtin_amdgcn_exp2f(m - to);
        l *= f;
#pragma unroll
        for (int t = 0; t < kDims; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[t][e] *= f;
        m = to;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        score[e] = __builtin_amdgcn_exp2f(score[e] * scale - m);
        l += score[e];
      }
      // Values that are not finite, in keys that some rows do not see: zero times them is not zero.  Such values are added without the product, to the rows that see them, and leave it.
      if (border && __any(odd != 0)) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) odd |= __shfl_xor((int)odd, o);
#pragma unroll 1
        for (unsigned left = uniform((int)odd); left != 0; left &= left - 1) {
          const int key = __ffs((int)left) - 1;
          float weight = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (key - 4 * half == 8 * (e >> 2) + (e & 3)) weight = score[e];
          weight = __shfl(weight, col + 32 * (key >> 2 & 1));  // from the half that has the key
          const bool sees = visible >> key & 1;
#pragma unroll
          for (int t = 0; t < kDims; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const Value* const x = (const Value*)v_tile + key * kPitch + 32 * t + 8 * g + 4 * half;
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[t][4 * g + e] += sees && !(fabsf((float)x[e]) < INFINITY) ? weight * (float)x[e] : 0.f;
              __builtin_amdgcn_sched_barrier(0);
            }
          __builtin_amdgcn_wave_barrier();
          for (int i = lane; i < kOwn; i += 64)
            if (!(fabsf((float)((Value*)v_tile)[key * kPitch + i]) < INFINITY)) ((Value*)v_tile)[key * kPitch + i] = (Value)0.f;
          __builtin_amdgcn_wave_barrier();
        }
      }
      // the values' sums: weights as two bf16 terms, or one of float16
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        bf16x8 hi, lo;
        f16x8 one;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (E4M3) {
            one[e] = (_Float16)score[8 * st + e];
          } else {
            hi[e] = (__bf16)score[8 * st + e];
            lo[e] = (__bf16)(score[8 * st + e] - (float)hi[e]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        // lanes 4 e + c of a group of 16 address dimensions 4 c .. 4 c + 3 of its key e
        const __bf16* const from = v_tile + (16 * st + 4 * half + (lane >> 2 & 3)) * kPitch + (lane >> 4 & 1) * 16 + (lane & 3) * 4;
#pragma unroll
        for (int t = 0; t < kDims; ++t) {
          const s16x4 x = lds_read_tr(from + 32 * t), y = lds_read_tr(from + 32 * t + 8 * kPitch);
          const s16x8 v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
          if constexpr (E4M3) {
            acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, v), one, acc[t], 0, 0, 0);
          } else {
            acc[t] = mfma32(__builtin_bit_cast(bf16x8, v), hi, acc[t]);
            acc[t] = mfma32(__builtin_bit_cast(bf16x8, v), lo, acc[t]);
          }
        }
      }
      tile += teams;
    };
    while (more()) step();

    // ---- the waves' results together ----
    l = sum_halves(l);
    if (half == 0) {  // (a team's waves have the same)
      maxima[wave][col] = m;
      sums[wave][col] = l;
    }
    __syncthreads();  // (and no wave reads its tile any more)
    float top = kFloor, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; w += kParts)
      if ((w / kParts & (subs - 1)) == sub) top = fmaxf(top, maxima[w][col]);
#pragma unroll
    for (int w = 0; w < kWaves; w += kParts)
      if ((w / kParts & (subs - 1)) == sub) sum += sums[w][col] * __builtin_amdgcn_exp2f(maxima[w][col] - top);
    const float f = __builtin_amdgcn_exp2f(m - top);
#pragma unroll
    for (int t = 0; t < kDims; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g) pool.values[wave][4 * t + g][lane] = f32x4{acc[t][4 * g] * f, acc[t][4 * g + 1] * f, acc[t][4 * g + 2] * f, acc[t][4 * g + 3] * f};
    __syncthreads();
    // quarter u of the lane's row: dimensions 8 u + 4 half .. + 3 of the wave's; each team's wave sums up every teams-th
    const bool cut = block0 != 0 || block1 != key_blocks, some = sum > 0.f || sum != sum;
    float* const into = a.parts + (((int64_t)(share * 2 + (block0 == 0)) * a.heads + head) * a.most_subs + sub) * part_floats<D>();
    if (live) {
      const float inv = some ? v_scale / sum : 0.f;
      __bf16* const to = a.o + (int64_t)q_row * a.o_stride + (int64_t)q_head * D + part * kOwn + 4 * half;
      float* const to_part = into + col * D + part * kOwn + 4 * half;
      auto put = [&](auto number) {
        constexpr int TEAMS = decltype(number)::value;
#pragma unroll
        for (int i = 0; i < 4 * kDims / TEAMS; ++i) {
          const int u = i * TEAMS + team;
          f32x4 x = pool.values[sub * kParts + part][u][lane];
#pragma unroll
          for (int w = 1; w < TEAMS; ++w) x += pool.values[(w * subs + sub) * kParts + part][u][lane];
          struct __attribute__((packed, aligned(2))) Loose4 {
            bf16x4 x;
          };
          if (cut) *reinterpret_cast<f32x4*>(to_part + 8 * u) = x;
          else reinterpret_cast<Loose4*>(to + 8 * u)->x = pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
        }
      };
      if (teams == 4) put(std::integral_constant<int, 4>{});
      else if (teams == 2) put(std::integral_constant<int, 2>{});
      else put(std::integral_constant<int, 1>{});
      if (team == 0 && part == 0 && half == 0) {
        if (cut) {
          into[kRows * D + col] = top;
          into[kRows * D + kRows + col] = sum;
        } else if (a.lse) {
          a.lse[(int64_t)q_head * a.total_q + q_row] = some ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
        }
      }
    }
    if (cut && block0 == 0 && threadIdx.x == 0 && head == 0) {
      const int row = row_block * subs * kRows;
      a.cuts[share * kCut + kCutSeqRow] = s.first_row;
      a.cuts[share * kCut + kCutRow] = row;
      a.cuts[share * kCut + kCutRows] = min(subs * kRows, s.rows - row);
      a.cuts[share * kCut + kCutShares] = shares_of_block(unit, key_blocks, size, total);
    }
    __syncthreads();
    unit += block1 - block0;
    in_seq += block1 - block0;
  }
}

// Blocks of rows that were cut.  All their rows are dealt to the workgroups of a head: a row of few parts to a wave, of more to a workgroup.  The parts are joined in an order that
// their number alone gives.  Bound by latency: a chain of loads (cuts, statistics, parts) to a row.  Where all rows took a workgroup: head dimension 256, 32 sequences with drafts 9.9 -> 7.9 us; a whole call of 512
// sequences, e4m3, 106.8 -> 104.3, of 512 with up to 512 keys 32.2 -> 31.5.
constexpr int kFewParts = 16;
template <int D>
__global__ __launch_bounds__(kThreads) void join_kernel(const AttnArgs a, const int groups) {
  constexpr int kPer = (D + 63) / 64, kEach = kMostShares / kThreads, kEarly = 4;
  static_assert(kCut == 4 && kMostShares % 64 == 0 && kEarly * kWaves == kFewParts);
  __shared__ int4 cuts[kMostShares];
  __shared__ int starts[kMostShares];  // rows of the cuts before each
  __shared__ float factors[kMostShares], reduced[2][kWaves], values[kWaves][D];
  __shared__ int wave_rows[kWaves];
  const int head = blockIdx.x % a.heads, lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  int4 own[kEach];
  int mine = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int share = threadIdx.x * kEach + i;
    own[i] = share < a.shares ? reinterpret_cast<const int4*>(a.cuts)[share] : int4{};
    mine += own[i].z;
  }
  const int up_to = (int)wave_sum_up_to((uint32_t)mine);
  if (lane == 63) wave_rows[wave] = up_to;
  __syncthreads();
  int before = up_to - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += wave_rows[w];
    total += wave_rows[w];
  }
  if (blockIdx.x / a.heads >= total) return;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    cuts[threadIdx.x * kEach + i] = own[i];
    starts[threadIdx.x * kEach + i] = before;
    before += own[i].z;
  }
  __syncthreads();
  struct Row {
    int share, in_block, parts, q_row, q_head;
  };
  auto find = [&](int job) {
    int up_to = 0;
#pragma unroll
    for (int i = 0; i < kMostShares / 64; ++i) up_to += __popcll(__ballot(starts[i * 64 + lane] <= job));
    Row r;
    r.share = up_to - 1;  // (the last that begins at or before the row: those that have no rows come before)
    const int4 cut = cuts[r.share];
    r.in_block = job - starts[r.share];
    r.parts = uniform(cut.w);
    const int row = cut.y + r.in_block, token = a.by_group(row);
    r.q_row = cut.x + token;
    r.q_head = head * a.group + row - token * a.group;
    return r;
  };
  auto part_of = [&](const Row& r, int i) { return a.parts + (((int64_t)((r.share + i) * 2 + (i == 0)) * a.heads + head) * a.most_subs + r.in_block / kRows) * part_floats<D>(); };
  const float v_scale = a.v_scale ? a.v_scale[head] : 1.f;
  auto put_lse = [&](const Row& r, float top, float sum) {
    if (a.lse) a.lse[(int64_t)r.q_head * a.total_q + r.q_row] = sum > 0.f || sum != sum ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
  };

  for (int job = blockIdx.x / a.heads * kWaves + wave; job < total; job += groups * kWaves) {
    const Row r = find(job);
    if (r.parts > kFewParts) continue;
    const int col = r.in_block % kRows;
    const float* const own_part = part_of(r, min(lane, r.parts - 1)) + kRows * D + col;
    const float m = lane < r.parts ? own_part[0] : kFloor, l = lane < r.parts ? own_part[kRows] : 0.f;
    float x[kEarly][kPer];
    auto load = [&](int i, int slot) {
      const float* const p = part_of(r, min(i, r.parts - 1)) + col * D;
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[slot][e] = D % 64 == 0 || e * 64 + lane < D ? p[e * 64 + lane] : 0.f;
    };
#pragma unroll
    for (int j = 0; j < kEarly; ++j) load(j, j);  // (on their way while the factors are found)
    float top = m;
#pragma unroll
    for (int o = kFewParts / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float f = __builtin_amdgcn_exp2f(m - top), sum = lanes_sum<kFewParts>(l * f);
    float acc[kPer] = {};
    for (int i = 0; i < r.parts; i += kEarly) {
#pragma unroll
      for (int j = 0; j < kEarly; ++j)
        if (i + j < r.parts) {
          const float g = __shfl(f, i + j);
#pragma unroll
          for (int e = 0; e < kPer; ++e) acc[e] += x[j][e] * g;
        }
      if (i + kEarly < r.parts) {
#pragma unroll
        for (int j = 0; j < kEarly; ++j) load(i + kEarly + j, j);
      }
    }
    // (lanes 0 .. kFewParts - 1 have the sum)
    const float all = __shfl(sum, 0), inv = all > 0.f || all != all ? v_scale / all : 0.f;
    __bf16* const to = a.o + (int64_t)r.q_row * a.o_stride + (int64_t)r.q_head * D;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (D % 64 == 0 || e * 64 + lane < D) to[e * 64 + lane] = (__bf16)(acc[e] * inv);
    if (lane == 0) put_lse(r, top, sum);
  }

  for (int job = blockIdx.x / a.heads; job < total; job += groups) {
    const Row r = find(job);
    const int n = r.parts;
    if (n <= kFewParts) continue;
    const int col = r.in_block % kRows;
    float early[kEarly][kPer];  // the wave's first parts, on their way while the factors are found
#pragma unroll
    for (int j = 0; j < kEarly; ++j) {
      const float* const p = part_of(r, wave + j * kWaves) + col * D;
#pragma unroll
      for (int e = 0; e < kPer; ++e) early[j][e] = D % 64 == 0 || e * 64 + lane < D ? p[e * 64 + lane] : 0.f;
    }
    float ms[kEach], ls[kEach], top = kFloor;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int piece = threadIdx.x + i * kThreads;
      ms[i] = piece < n ? part_of(r, piece)[kRows * D + col] : kFloor;
      ls[i] = piece < n ? part_of(r, piece)[kRows * D + kRows + col] : 0.f;
      top = fmaxf(top, ms[i]);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) reduced[0][wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(reduced[0][0], reduced[0][1]), fmaxf(reduced[0][2], reduced[0][3]));
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const float f = __builtin_amdgcn_exp2f(ms[i] - top);
      factors[threadIdx.x + i * kThreads] = f;
      sum += ls[i] * f;
    }
    sum = lanes_sum<64>(sum);
    if (lane == 0) reduced[1][wave] = sum;
    __syncthreads();
    sum = (reduced[1][0] + reduced[1][1]) + (reduced[1][2] + reduced[1][3]);
    float acc[kPer] = {};
#pragma unroll
    for (int j = 0; j < kEarly; ++j) {
      const float f = factors[wave + j * kWaves];
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] += early[j][e] * f;
    }
#pragma unroll 8
    for (int i = wave + kEarly * kWaves; i < n; i += kWaves) {
      const float* const p = part_of(r, i) + col * D;
      const float f = factors[i];
#pragma unroll
      for (int e = 0; e < kPer; ++e)
        if (D % 64 == 0 || e * 64 + lane < D) acc[e] += p[e * 64 + lane] * f;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (D % 64 == 0 || e * 64 + lane < D) values[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    const float inv = sum > 0.f || sum != sum ? v_scale / sum : 0.f;
    for (int i = threadIdx.x; i < D; i += kThreads)
      a.o[(int64_t)r.q_row * a.o_stride + (int64_t)r.q_head * D + i] = (__bf16)(((values[0][i] + values[1][i]) + (values[2][i] + values[3][i])) * inv);
    if (threadIdx.x == 0) put_lse(r, top, sum);
    __syncthreads();
  }
}

// ---- host ----
// Units of a key/value head, at most.
int64_t most_units(const paged_attn_desc* d) {
  const int64_t rows = (int64_t)d->total_q * (d->num_q_heads / d->num_kv_heads);
  return std::min((int64_t)d->num_seqs + rows / kRows, std::max<int64_t>(rows, 1)) * (((int64_t)d->max_pages * d->page_size + kBlockKeys - 1) / kBlockKeys);
}
int check_desc(const paged_attn_desc* d) {
  if (!d || d->num_q_heads < 1 || d->num_kv_heads < 1 || d->num_seqs < 1 || d->total_q < 0 || d->page_size < 1 || d->num_pages < 1 || d->max_pages < 1 ||
      (d->cache_type != PAGED_CACHE_BF16 && d->cache_type != PAGED_CACHE_E4M3) || !finite_number(d->softmax_scale) || d->softmax_scale <= 0.f)
    return CHUNK_ATTN_INVALID_ARG;
  if (!paged_head_dim(d->head_dim) || d->num_q_heads % d->num_kv_heads != 0 || d->num_q_heads > PAGED_MAX_HEADS || d->num_seqs > PAGED_CACHE_MAX_REQUESTS ||
      d->page_size > PAGED_CACHE_MAX_PAGE_SIZE)
    return CHUNK_ATTN_UNSUPPORTED;
  // (products of three are formed of factors below 2^31 and 2^30)
  if ((int64_t)d->total_q * d->num_q_heads > INT32_MAX || (int64_t)d->max_pages * d->page_size > 1 << 30 ||
      (int64_t)d->num_pages * d->page_size > INT32_MAX / d->num_kv_heads || most_units(d) > 1 << 30)
    return CHUNK_ATTN_INVALID_ARG;
  return CHUNK_ATTN_OK;
}
// Workgroups for each key/value head: as many as two to a compute unit are, and no more than there can be shares.  All shares are equally long and a compute unit holds two (head dimension 64: three), so
// what is past two to each would begin when the first ones end: rounded down.  Not past half as many heads as that, where it would leave half of the places empty.  Rounded down / up, us, a query head to a
// key/value head of 128, bf16, 12000 to 134000 keys: 24 heads 291 / 329, 40 heads 254 / 291, 100 heads 283 / 314, 200 heads 312 / 319; 260 heads 430 / 348, 300 heads 570 / 464 (but 400 heads 461 / 484).
int count_shares(const paged_attn_desc* d) {
  const int64_t fill = (kMostShares + (d->num_kv_heads > kMostShares / 2 ? d->num_kv_heads - 1 : 0)) / d->num_kv_heads;
  return (int)std::max<int64_t>(1, std::min(fill, most_units(d)));
}
int count_subs(const paged_attn_desc* d) {
  const int64_t rows = (int64_t)d->total_q * (d->num_q_heads / d->num_kv_heads);
  return d->head_dim == 256 || rows <= kRows ? 1 : rows <= 2 * kRows ? 2 : 4;
}
size_t part_bytes(const paged_attn_desc* d) { return (size_t)count_shares(d) * count_subs(d) * 2 * d->num_kv_heads * kRows * (d->head_dim + 2) * sizeof(float); }
size_t need_bytes(const paged_attn_desc* d) { return part_bytes(d) + (size_t)count_shares(d) * kCut * sizeof(int32_t); }
bool aligned(const void* p, uintptr_t to) { return p && ((uintptr_t)p & (to - 1)) == 0; }

template <class F>
hipError_t by_dim(int d, F&& f) {
  switch (d) {
    case 64: return f(std::integral_constant<int, 64>{});
    case 96: return f(std::integral_constant<int, 96>{});
    case 128: return f(std::integral_constant<int, 128>{});
    default: return f(std::integral_constant<int, 256>{});
  }
}

}  // namespace
}  // namespace chunk_attn

extern "C" int paged_attn_validate(const paged_attn_desc* d) { return chunk_attn::check_desc(d); }

extern "C" int paged_attn_workspace_bytes(const paged_attn_desc* d, size_t* bytes) {
  const int rc = chunk_attn::check_desc(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (!bytes) return CHUNK_ATTN_INVALID_ARG;
  *bytes = chunk_attn::need_bytes(d);
  return CHUNK_ATTN_OK;
}

extern "C" int paged_attn_fwd(const paged_attn_desc* d, const void* q, int64_t q_stride, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                              const int32_t* table, const int32_t* kv_len, const int32_t* q_start, void* o, int64_t o_stride, float* lse, void* workspace, size_t workspace_bytes,
                              void* hip_stream) {
  using namespace chunk_attn;
  const int rc = check_desc(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (d->total_q == 0) return CHUNK_ATTN_OK;
  const int64_t row = (int64_t)d->num_q_heads * d->head_dim;
  const bool e4m3 = d->cache_type == PAGED_CACHE_E4M3;
  if (!aligned(q, 2) || !aligned(o, 2) || q_stride < row || o_stride < row || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(table, 4) || !aligned(kv_len, 4) ||
      !aligned(q_start, 4) || ((uintptr_t)lse & 3) != 0 || (e4m3 && (!aligned(k_scale, 4) || !aligned(v_scale, 4))) || !aligned(workspace, 256))
    return CHUNK_ATTN_INVALID_ARG;
  if (workspace_bytes < need_bytes(d)) return CHUNK_ATTN_WORKSPACE_TOO_SMALL;
  const int heads = d->num_kv_heads, group = d->num_q_heads / heads, shares = count_shares(d);
  const AttnArgs a{(const __bf16*)q, q_stride, k_cache, v_cache, e4m3 ? k_scale : nullptr, e4m3 ? v_scale : nullptr, table, kv_len, q_start, (__bf16*)o, o_stride, lse,
                   (float*)workspace, (int32_t*)((char*)workspace + part_bytes(d)), d->num_seqs, d->total_q, heads, group, d->page_size, d->num_pages, d->max_pages, shares, count_subs(d),
                   d->softmax_scale * kLog2e, Divide(d->page_size), Divide(group), Divide(shares)};
  const hipStream_t stream = (hipStream_t)hip_stream;
  const hipError_t e = by_dim(d->head_dim, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    const dim3 grid((unsigned)(shares * heads));
    auto with_pages = [&](auto halves) {
      constexpr bool HALVES = decltype(halves)::value;
      if (e4m3) hipLaunchKernelGGL((attn_kernel<D, true, HALVES>), grid, dim3(kThreads), 0, stream, a);
      else hipLaunchKernelGGL((attn_kernel<D, false, HALVES>), grid, dim3(kThreads), 0, stream, a);
    };
    if (d->page_size % 16 == 0) with_pages(std::true_type{});
    else with_pages(std::false_type{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || shares == 1) return e;
    // a workgroup for each row that may be cut, as long as that makes no more than eight of them to a compute unit
    const int64_t rows = std::min<int64_t>((int64_t)d->total_q * group, (int64_t)(shares - 1) * kRows * a.most_subs);
    const int groups = (int)std::max<int64_t>(1, std::min<int64_t>(rows, 8 * kCus / heads));
    hipLaunchKernelGGL((join_kernel<D>), dim3((unsigned)(groups * heads)), dim3(kThreads), 0, stream, a, groups);
    return hipGetLastError();
  });
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, "attention over a paged cache");
}
