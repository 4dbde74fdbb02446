// Linear attention with a decay for each head over the sequences of a chunk (include/chunk_linear.h): forward, backward, and one token at a time.
//
// A sequence is taken in blocks of 64 rows.  With S the state before a block of L rows, row i of the block is
//   o_i = scale (l^(i+1) q_i S + sum_(j<=i) l^(i-j) (q_i . k_j) v_j)        and the state behind it        S' = l^L S + sum_j l^(L-1-j) k_j^T v_j,
// four products of matrices.  A workgroup walks the blocks of a piece of a sequence with S in its accumulators: wave w owns columns 32 w .. 32 w + 31 of S and of the
// outputs.  All powers of l that occur have exponents >= 0, whatever the decay, and none of more than 64 rows' distance is formed inside a walk.
//
// The three gradients are the same walk with other tensors in the roles of q, k and v:
//   dq: (d_o, v, k), state S^T;   dv: (k, q, d_o) and dk: (v, d_o, q) backwards, from the last row to the first, over rows j >= i; their state is the gradient of S, or its transpose.
//   Backwards, R before a block (that is, behind its last row) gives   x_i = l^(L-1-i) q_i R + scale sum_(j>=i) l^(j-i) (q_i . k_j) v_j   and   R' = l^L R + scale sum_j l^(j+1) k_j^T v_j.
//
// Long sequences are cut into pieces so that there are enough workgroups.  A first kernel forms each piece's own sum of k^T v, a second one adds them up along the sequence, and the
// walks then start from there (forwards, with few pieces and small states, the walks add them up themselves: kDirect); states of pieces are float32 throughout.
//
// Accumulators as operands: an accumulator tile holds S[row][column = lane % 32], and the eight values of a lane in one half of it are what an MFMA operand wants of 16 rows, if
// only the rows are named accordingly (device_common.hpp, "C-order").  Here the rows of K^T are fed to the state's product in the order that makes the names come out as
// they are: transposed reads deliver column quads 0, 2, 1, 3.  Outputs are formed transposed (columns = tokens), so that the power of l a row is multiplied with is one
// value of a lane, and four neighbouring elements of an output row lie in a lane.
//
// Precision: an operand in bf16 that is not an input would be off by 2^-8, as much as the one rounding of a result, so it is a sum of bf16 terms, each a product of its own.  Two terms (2^-16) for the state and the
// weighted scores in an output's products (one each: root mean square error 2.3e-3 of the result where a single rounding leaves 1.7e-3, 11 - 13 % less time at head_dim 128: 8192 tokens of 32/32 with a state left
// 115 -> 131 us, 65536 packed of 32/8 389 -> 441, backward of 16384 326 -> 370) and for the weighted v_j in sums k_j^T (l^(L-1-j) v_j) that only become such an operand; three (24 bits) in sums and walks that go into a state or a
// state's gradient that is left, which is then as exact as float32 sums are.  At head_dim 128 the terms past the first are 38 of the 82 products of a wave in a block of one query head.
//
// Measured (us; head_dim 128 unless said).  Forward, 65536 tokens in 20 sequences, 32/8 heads: 440, of that the walk 355 (1.34 GB, 3.8 TB/s), the pieces' sums 70 and 12; 8192 tokens of 32/32
// with a state left 124 (walk 69 of 268 MB, sums 36 and 12), without one 110.  Backward, 16384 tokens of 32/8 in 8 sequences: 394, walk_back 180, dq's walk 101, sums 63 + 26 and 16 + 13.  Neither memory nor the
// matrix units are the bound of the walks: the latter are busy for 34 - 43 % of the cycles of compute units that have work, and waves wait for 40 % of theirs, on the chain of a step with two waves to a SIMD; 15 - 22 % of the units have no work
// (starts and unequal ends), and the clock is at 2.0 GHz, lower when calls follow each other.  head_dim 256: 8192 tokens of 16/16, forward 196, backward 496; its walks spill registers (61 - 167).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "../../include/chunk_linear.h"
#include "kernels.hpp"
#include "operators.hpp"
#include "tiles.hpp"

namespace chunk_attn {
namespace {

constexpr int kBlock = 64;       // rows of a block
constexpr int kLinearSegs = 144; // segments that travel with one launch

struct LinearSegs {
  int n;                      // segments, those that leave most rows beside their full pieces first
  int num_full, num_pieces;   // full pieces of these segments; all, the full ones first, then what is left of each segment that has something left
  int piece_rows;             // rows of a full piece, a multiple of kBlock
  int start[kLinearSegs], len[kLinearSegs], in[kLinearSegs], out[kLinearSegs];
  int full0[kLinearSegs];   // full pieces of the segments before
  int place0[kLinearSegs];  // place of its first piece's state in the workspace, where it has several
};
struct WalkArgs {
  const __bf16 *q, *k, *v;   // by role
  __bf16* o;
  const float* log_decay;
  const float* first;        // states that walks start from at the sequence's border (null: zeros), and that they leave there (null: not wanted), by slot
  float* last;
  float* inner;              // states of the pieces of cut sequences, [place][kv head][D][D]
  int heads, group;          // key/value heads; query heads to each
  float scale;
  int direct;                // whether walks add up the sums of the pieces before theirs themselves
};
static_assert(sizeof(LinearSegs) + sizeof(WalkArgs) <= 3900, "fits the kernel arguments");

struct Piece {
  int seg, index, pieces, row, rows;  // index among the segment's pieces; first row; rows
};
__device__ __forceinline__ Piece find_piece(const LinearSegs& s, int piece) {
  const int lane = threadIdx.x & 63;
  Piece p;
  if (piece < s.num_full) {
    int seg = -1;  // the last segment whose full pieces begin at or before this one
    for (int i = 0; i < s.n; i += 64) seg += __popcll(__ballot(i + lane < s.n && s.full0[min(i + lane, s.n - 1)] <= piece));
    p.seg = __builtin_amdgcn_readfirstlane(seg);
    p.index = piece - s.full0[p.seg];
  } else {
    p.seg = piece - s.num_full;
    p.index = s.len[p.seg] / s.piece_rows;
  }
  const int len = s.len[p.seg];
  p.pieces = (len + s.piece_rows - 1) / s.piece_rows;
  p.row = s.start[p.seg] + p.index * s.piece_rows;
  p.rows = min(s.piece_rows, len - p.index * s.piece_rows);
  return p;
}
// log2 of a head's decay.  The bound stands for -inf: l^0 is 1 and every other power 0.  A NaN stays one (told by its bits: a comparison, or the maximum alone, would lose it).
__device__ __forceinline__ float log2_decay(const float* log_decay, int h) {
  const float x = log_decay[h];
  return (__float_as_uint(x) & 0x7fffffffu) > 0x7f800000u ? x : fmaxf((float)((double)x * 1.4426950408889634), -1000.f);
}
__device__ __forceinline__ float power(float lg, int n) { return __builtin_amdgcn_exp2f(lg * (float)n); }

// Tiles in LDS are rows of D elements and a few more, so that an element's place is linear in its row and column (one address per lane and kind of read, the rest are constants) and neither 16-byte
// reads of 16 consecutive rows nor transposed reads of 4 rows x 32 bytes meet in a bank: the rows' stride in 16-byte units is odd, and 1 mod 16 apart.
constexpr int pitch(int cols) { return cols + (cols % 128 == 0 ? 24 : 8); }
constexpr size_t tile_bytes(int cols) { return (size_t)kBlock * pitch(cols) * 2; }

// A block's rows of one head in memory, as a buffer: reads of other rows give zeros and writes to them are dropped by the hardware, so that no access is behind a branch (the compiler can then
// count the ones in flight: with branches around the stores every step waited for the stores of the one before).
struct Rows {
  __amdgpu_buffer_rsrc_t buffer;
  int stride;  // bytes
  // `rows` rows of `bytes` bytes from `first` on
  __device__ __forceinline__ Rows(const void* first, int stride, int rows, int bytes)
      : buffer(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(first), 0, (rows - 1) * stride + bytes, 0x00027000)), stride(stride) {}
  __device__ __forceinline__ u32x4 load(int row, int byte) const { return __builtin_amdgcn_raw_buffer_load_b128(buffer, row * stride + byte, 0, 0); }
  __device__ __forceinline__ void store(int row, int byte, u32x4 x) const { __builtin_amdgcn_raw_buffer_store_b128(x, buffer, row * stride + byte, 0, 0); }
};

// A block's rows on their way to LDS, fetched ahead into registers.  Forwards a block of fewer rows stands at the end of its 64, behind `empty` rows of zeros: the weights of rows in the state are
// then the same in every block.
template <int D, int THREADS = 2 * D>
struct Tile {
  static constexpr int kChunks = D / 8, kThreads = THREADS, kEach = kBlock * kChunks / kThreads, kRowsApart = kThreads / kChunks;
  u32x4 x[kEach];
  __device__ __forceinline__ void fetch(const Rows& from, int empty) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = from.load((int)threadIdx.x % kThreads / kChunks + i * kRowsApart - empty, (int)threadIdx.x % kThreads % kChunks * 16);
  }
  __device__ __forceinline__ void store(lds_bf16* to) const {
    lds_bf16* const at = to + (int)threadIdx.x % kThreads / kChunks * pitch(D) + (int)threadIdx.x % kThreads % kChunks * 8;
#pragma unroll
    for (int i = 0; i < kEach; ++i) lds_store8(at + i * kRowsApart * pitch(D), __builtin_bit_cast(bf16x8, x[i]));
  }
};
// Operand of 32 rows (or columns) x 16 of the contraction along the row: lane l32 holds row0 + l32, eight elements from 16 step + 8 hh on.
template <int D>
__device__ __forceinline__ bf16x8 row_operand(const lds_bf16* tile, int row0, int step, int lane) {
  return lds_load8(tile + ((lane & 31) * pitch(D) + (lane >> 5) * 8) + (row0 * pitch(D) + 16 * step));
}
// Operand of 32 columns from col0 on x 16 rows from row0 on as the contraction.  SWAPPED: the column quads of each 16 in the order 0, 2, 1, 3.
template <int D, bool SWAPPED>
__device__ __forceinline__ bf16x8 column_operand(const lds_bf16* tile, int row0, int col0, int lane) {
  const int x = lane & 15, quad = x & 3;
  const lds_bf16* const at = tile + ((8 * (lane >> 5) + (x >> 2)) * pitch(D) + (lane & 16) + 4 * (SWAPPED ? (quad >> 1) | (quad & 1) << 1 : quad)) + (row0 * pitch(D) + col0);
  union {
    s16x4 half[2];
    bf16x8 all;
  } u;
  u.half[0] = lds_read_tr(at);
  u.half[1] = lds_read_tr(at + 4 * pitch(D));
  return u.all;
}

// x as a sum of bf16 terms, each the rounded rest of those before: two are good to 2^-16, three to float32.
template <int PARTS>
__device__ __forceinline__ void split(float (&x)[8], bf16x8 (&term)[PARTS]) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      term[p][e] = (__bf16)x[e];
      x[e] -= (float)term[p][e];
    }
}

// The state of a wave: D rows x 32 columns.
template <int D>
struct State {
  f32x16 t[D / 32];
  // rows of the state that registers 4 g + r of tile i stand for, for a lane of half hh
  static __device__ __forceinline__ int row(int i, int g, int hh) { return 32 * i + 16 * (g >> 1) + 8 * hh + 4 * (g & 1); }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) t[i] = f32x16{};
  }
  template <bool TRANSPOSED>
  __device__ __forceinline__ void load(const float* from, int col, int hh) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int r0 = row(i, g, hh);
        f32x4 x;
        if constexpr (TRANSPOSED) x = *reinterpret_cast<const f32x4*>(from + (int64_t)col * D + r0);
        else
          for (int r = 0; r < 4; ++r) x[r] = from[(int64_t)(r0 + r) * D + col];
#pragma unroll
        for (int r = 0; r < 4; ++r) t[i][4 * g + r] = x[r];
      }
  }
  __device__ __forceinline__ void store(float* to, int col, int hh) const {
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) to[(int64_t)(row(i, g, hh) + r) * D + col] = t[i][4 * g + r];
  }
  // As the waves hold it, [wave][tile][quad of rows][lane][4]: 16 bytes to a lane, next to its neighbours'.
  static __device__ __forceinline__ f32x4* own(float* state, int wave, int lane) { return reinterpret_cast<f32x4*>(state) + wave * (D / 8) * 64 + lane; }
  __device__ __forceinline__ void load_own(float* state, int wave, int lane) {
    const f32x4* const from = own(state, wave, lane);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 x = from[(4 * i + g) * 64];
#pragma unroll
        for (int r = 0; r < 4; ++r) t[i][4 * g + r] = x[r];
      }
  }
  __device__ __forceinline__ void store_own(float* state, int wave, int lane) const {
    f32x4* const to = own(state, wave, lane);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) to[(4 * i + g) * 64] = f32x4{t[i][4 * g], t[i][4 * g + 1], t[i][4 * g + 2], t[i][4 * g + 3]};
  }
  // by times it, and another one
  __device__ __forceinline__ void scale_and_add_own(float by, float* state, int wave, int lane) {
    const f32x4* const from = own(state, wave, lane);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 x = from[(4 * i + g) * 64];
#pragma unroll
        for (int r = 0; r < 4; ++r) t[i][4 * g + r] = t[i][4 * g + r] * by + x[r];
      }
  }
  __device__ __forceinline__ void scale(float by) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) t[i][e] *= by;
  }
  // operands of rows 16 step .. 16 step + 15 as the contraction: two bf16 terms
  __device__ __forceinline__ void operands(int step, bf16x8 (&term)[2]) const {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = t[step >> 1][8 * (step & 1) + e];
    split(x, term);
  }
  // adds k^T (w v) of 16 rows from row0 on: v's operand as it was read; element e's row weighs lead * base[e]
  template <int PARTS>
  __device__ __forceinline__ void add(const lds_bf16* k_tile, int row0, bf16x8 v, float lead, const float (&base)[8], int lane) {
    constexpr int kTiles = D / 32, kHalf = (kTiles + 1) / 2;
    bf16x8 kt[kTiles], part[PARTS];
    float x[8];
#pragma unroll
    for (int i = 0; i < kHalf; ++i) kt[i] = column_operand<D, true>(k_tile, row0, 32 * i, lane);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e] * (lead * base[e]);
    split(x, part);
#pragma unroll
    for (int i = kHalf; i < kTiles; ++i) kt[i] = column_operand<D, true>(k_tile, row0, 32 * i, lane);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int i = 0; i < kHalf; ++i) t[i] = mfma32(kt[i], part[p], t[i]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int i = kHalf; i < kTiles; ++i) t[i] = mfma32(kt[i], part[p], t[i]);
    __builtin_amdgcn_sched_barrier(0);
  }
};

// Weights of a block's rows in its state, l^(63 - j) or backwards (the gradient of S) scale * l^(j + 1) for row j = 16 s + 8 hh + e: lead[s] * base[e], both powers with exponents >= 0.
// Eights of rows that are not there in any block of a piece of fewer than 64 weigh nothing: a decay above 1 may have no float32 number for a power that no row needs, and that times a row of zeros is no zero.
template <bool REVERSE>
struct StateWeights {
  float base[8], lead[4];
  __device__ __forceinline__ StateWeights(float lg, float scale, int hh, int piece_rows) {
#pragma unroll
    for (int e = 0; e < 8; ++e) base[e] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(power(lg, REVERSE ? e : 7 - e))));
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int eight = REVERSE ? 16 * s + 8 * hh : 56 - 16 * s - 8 * hh;  // the least power of its rows, or one less
      lead[s] = eight >= piece_rows ? 0.f : REVERSE ? scale * power(lg, eight + 1) : power(lg, eight);
    }
  }
};

// Each piece's own k^T v into its place in the workspace, but for the one at the far end of its sequence, whose nobody needs, and for sequences of one piece.
template <int D, bool REVERSE, bool TRANSPOSED, int PARTS>
__device__ __forceinline__ void piece_states(const WalkArgs& a, const LinearSegs& segs, const Piece& p) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  lds_bf16* const ks = (lds_bf16*)smem;
  lds_bf16* const vs = ks + kBlock * pitch(D);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hh = lane >> 5;
  const int h = blockIdx.x % a.heads;
  const float lg = log2_decay(a.log_decay, h);
  const int group = REVERSE ? a.group : 1;
  const int64_t stride = (int64_t)a.heads * group * D;
  const StateWeights<REVERSE> weights(lg, a.scale, hh, p.rows);
  float* const place = a.inner + ((int64_t)(segs.place0[p.seg] + p.index) * a.heads + h) * D * D;
  const int col = 32 * wave + (lane & 31);
  State<D> s;
  const int from = REVERSE ? -1 : segs.in[p.seg];
  if (!REVERSE && D < 256 && a.direct && p.index == 0 && a.first && from >= 0) {
    // The state before the sequence goes into the first piece's sum, and into the last place, which no sum takes, for the first piece's walk (the slot may be where the last one's walk leaves its own).
    s.template load<TRANSPOSED>(a.first + ((int64_t)from * a.heads + h) * D * D, col, hh);
    s.store_own(place + (int64_t)(p.pieces - 1) * a.heads * D * D, wave, lane);
  } else {
    s.clear();
  }
  const int blocks = (p.rows + kBlock - 1) / kBlock, steps = blocks * group;
  Tile<D> kt, vt;
  auto fetch = [&](int step) {
    const int b = REVERSE ? blocks - 1 - step / group : step / group, g = step % group, rows = min(kBlock, p.rows - b * kBlock);
    const int64_t at = (int64_t)(p.row + b * kBlock) * stride + (h * group + g) * D;
    const int empty = REVERSE ? 0 : kBlock - rows;
    kt.fetch(Rows(a.k + at, 2 * (int)stride, rows, 2 * D), empty);
    vt.fetch(Rows(a.v + at, 2 * (int)stride, rows, 2 * D), empty);
  };
  fetch(0);
  for (int step = 0; step < steps; ++step) {
    __syncthreads();
    kt.store(ks);
    vt.store(vs);
    __syncthreads();
    if (step + 1 < steps) fetch(step + 1);
    if (step % group == 0) s.scale(power(lg, min(kBlock, p.rows - (REVERSE ? blocks - 1 - step / group : step / group) * kBlock)));
#pragma unroll
    for (int st = 0; st < 4; ++st) s.template add<PARTS>(ks, 16 * st, column_operand<D, false>(vs, 16 * st, 32 * wave, lane), weights.lead[st], weights.base, lane);
  }
  if constexpr (REVERSE) s.store(place, col, hh);
  else s.store_own(place, wave, lane);
}

template <int D, bool REVERSE, bool TRANSPOSED>
__global__ __launch_bounds__(2 * D, D < 256 ? 3 : 2) void piece_states_kernel(const WalkArgs a, const LinearSegs segs) {
  const Piece p = find_piece(segs, blockIdx.x / a.heads);
  if (p.index == (REVERSE ? 0 : p.pieces - 1)) return;  // (also where there is one piece)
  if (a.last && (REVERSE ? segs.in : segs.out)[p.seg] >= 0) piece_states<D, REVERSE, TRANSPOSED, 3>(a, segs, p);  // (the sum goes into a state that is left)
  else piece_states<D, REVERSE, TRANSPOSED, 2>(a, segs, p);
}

// Adds them up along each sequence: in the place of each piece's own, the state that it starts from.  (The first one's, too: the slot it comes from may be the one that
// the last piece's state goes to.)
template <int D, bool REVERSE, bool TRANSPOSED>
__global__ __launch_bounds__(256) void join_states_kernel(const WalkArgs a, const LinearSegs segs) {
  constexpr int elements = D * D;
  const int seg = blockIdx.y, h = blockIdx.x % a.heads;
  const int at = (int)(blockIdx.x / a.heads * 256 + threadIdx.x) * 4;
  const int len = segs.len[seg], pieces = (len + segs.piece_rows - 1) / segs.piece_rows;
  if (pieces == 1 || at >= elements) return;
  const float lg = log2_decay(a.log_decay, h);
  const int slot = REVERSE ? segs.out[seg] : segs.in[seg];
  f32x4 sum{};
  if (a.first && slot >= 0) {
    const float* const from = a.first + ((int64_t)slot * a.heads + h) * elements;
    if constexpr (REVERSE) {
      sum = *reinterpret_cast<const f32x4*>(from + at);
    } else {  // (forward places are in the waves' order)
      const int lane = at / 4 % 64, g = at / 256 % 4, i = at / 1024 % (D / 32), wave = at / (32 * D);
      const int col = 32 * wave + lane % 32, row = State<D>::row(i, g, lane / 32);
      if constexpr (TRANSPOSED) {
        sum = *reinterpret_cast<const f32x4*>(from + col * D + row);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[r] = from[(row + r) * D + col];
      }
    }
  }
  const float whole = power(lg, segs.piece_rows), first = REVERSE ? power(lg, len - (pieces - 1) * segs.piece_rows) : whole;
  const int64_t apart = (int64_t)a.heads * elements / 4 * (REVERSE ? -1 : 1);
  f32x4* x = reinterpret_cast<f32x4*>(a.inner + ((int64_t)segs.place0[seg] * a.heads + h) * elements + at) - (REVERSE ? (pieces - 1) * apart : 0);
  constexpr int kTogether = 8;  // states are loaded eight at a time: one after the other a sequence of 32 pieces took 20 us
  for (int n0 = 0; n0 < pieces; n0 += kTogether, x += kTogether * apart) {
    f32x4 own[kTogether];
#pragma unroll
    for (int n = 0; n < kTogether; ++n)
      if (n0 + n < pieces - 1) own[n] = x[n * apart];
#pragma unroll
    for (int n = 0; n < kTogether; ++n)
      if (n0 + n < pieces) {
        x[n * apart] = sum;
        if (n0 + n < pieces - 1) sum = sum * (n0 + n == 0 ? first : whole) + own[n];
      }
  }
}

// Four neighbouring elements of a row lie in either half of the wave (registers 4 g .. 4 g + 3 of an output tile are elements 8 g + 4 hh ..).  They are put together to 16 bytes of a lane, and then
// moved between the lanes of rows r and r + 16, so that each store takes the wave's 64 bytes of sixteen rows (half of them of all rows took the address unit twice as long).
__device__ __forceinline__ void store_rows(const Rows& to, int row0, int byte, const f32x16& o, int lane) {
  u32x4 x[2];
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    union {
      bf16x4 h;
      unsigned u[2];
    } even, odd;
    even.h = pack4(o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]);
    odd.h = pack4(o[4 * g + 4], o[4 * g + 5], o[4 * g + 6], o[4 * g + 7]);
    const u32x2 a = __builtin_amdgcn_permlane32_swap(even.u[0], odd.u[0], false, false), b = __builtin_amdgcn_permlane32_swap(even.u[1], odd.u[1], false, false);
    x[g / 2] = u32x4{a[0], b[0], a[1], b[1]};  // lane (row l32, hh): bytes 32 (g / 2) + 16 hh of its row's 64
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32x2 y = __builtin_amdgcn_permlane16_swap(x[0][i], x[1][i], false, false);
    x[0][i] = y[0];
    x[1][i] = y[1];
  }
  // x[0]: rows row0 .. + 15, x[1]: the sixteen behind them; lanes 0 - 15: bytes 0, 16 - 31: 32, 32 - 47: 16, 48 - 63: 48
  const int at = byte + (lane & 16) * 2 + (lane >> 5) * 16;
  to.store(row0 + (lane & 15), at, x[0]);
  to.store(row0 + 16 + (lane & 15), at, x[1]);
}

// ---- the three products of a step ----
constexpr int ahead(int d) { return d < 256 ? 2 : 1; }  // stages that operands are read ahead of their products (as far as there are registers)

// Weights of scores, times the scale of outputs, as a lane needs them: of a tile on the diagonal of the block, and of the one off it ([2][quad of columns][lane][4]);
// no weight for rows further apart than any two of the piece's.
constexpr int kNear = 2 * 16 * 64;
template <bool REVERSE, int THREADS>
__device__ __forceinline__ void score_weights(float lg, float scale, int piece_rows, lds_f32* near) {
  for (int i = threadIdx.x; i < kNear; i += THREADS) {
    const int l = i >> 2 & 63, j = 8 * (i >> 8 & 3) + 4 * (l >> 5) + (i & 3), far = (REVERSE ? j - (l & 31) : (l & 31) - j) + 32 * (i >> 10);
    near[i] = far >= 0 && far < piece_rows ? power(lg, far) * scale : 0.f;
  }
}
// Scores of rows i of q with rows j of k, in tiles of 32 x 32, only those with j <= i (backwards j >= i): 0: (0, 0), 1: the one off the diagonal, 2: (1, 1).  Formed transposed (a lane holds one row i
// and four columns j at a time), weighted, and written to LDS in two bf16 terms, the second ones' three tiles behind the first ones'.
constexpr int kScoreTile = 32 * pitch(32);
constexpr size_t kScoreBytes = 2 * 3 * kScoreTile * 2;
template <int D, bool REVERSE>
__device__ __forceinline__ void scores(int tile, const lds_bf16* qs, const lds_bf16* ks, const lds_f32* near, lds_bf16* ps, int lane) {
  const int ti = REVERSE ? tile >> 1 : (tile + 1) >> 1, tj = REVERSE ? (tile + 1) >> 1 : tile >> 1;
  constexpr int kSteps = D / 16;
  f32x16 c{}, c1{};  // (two sums, so that a product need not wait for the one before)
  bf16x8 kf[kSteps], qf[kSteps];
  auto read = [&](int st) {
    kf[st] = row_operand<D>(ks, 32 * tj, st, lane);
    qf[st] = row_operand<D>(qs, 32 * ti, st, lane);
  };
#pragma unroll
  for (int st = 0; st < ahead(D); ++st) read(st);
#pragma unroll
  for (int st = 0; st < kSteps; ++st) {
    if (st + ahead(D) < kSteps) read(st + ahead(D));
    __builtin_amdgcn_sched_barrier(0);
    f32x16& sum = D < 256 && st % 2 ? c1 : c;
    sum = mfma32(kf[st], qf[st], sum);
    __builtin_amdgcn_sched_barrier(0);
  }
  if constexpr (D < 256) c += c1;
  f32x4 w[4];
#pragma unroll
  for (int q4 = 0; q4 < 4; ++q4) w[q4] = lds_load4f(near + (tile == 1 ? 1024 : 0) + q4 * 256 + lane * 4);
  lds_bf16* const to = ps + ((lane & 31) * pitch(32) + 4 * (lane >> 5)) + tile * kScoreTile;
#pragma unroll
  for (int q4 = 0; q4 < 4; q4 += 2) {
    float x[8];
    bf16x8 term[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = c[4 * q4 + e] * w[q4 + e / 4][e % 4];
    split(x, term);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      *(__attribute__((address_space(3))) bf16x4*)(to + 3 * p * kScoreTile + 8 * q4) = __builtin_shufflevector(term[p], term[p], 0, 1, 2, 3);
      *(__attribute__((address_space(3))) bf16x4*)(to + 3 * p * kScoreTile + 8 * q4 + 8) = __builtin_shufflevector(term[p], term[p], 4, 5, 6, 7);
    }
  }
}
// What the state gives the wave's 32 columns, times each row's power of the decay and a scale.  Rows stand behind `empty` others.
template <int D, bool REVERSE>
__device__ __forceinline__ void state_outputs(const State<D>& s, const lds_bf16* qs, float lg, float scale, int rows, int empty, int lane, f32x16 (&o)[2]) {
  constexpr int kSteps = D / 16;
  bf16x8 qf[kSteps][2];
  auto read = [&](int st) {
    qf[st][0] = row_operand<D>(qs, 0, st, lane);
    qf[st][1] = row_operand<D>(qs, 32, st, lane);
  };
  o[0] = o[1] = f32x16{};
#pragma unroll
  for (int st = 0; st < ahead(D); ++st) read(st);
#pragma unroll
  for (int st = 0; st < kSteps; ++st) {
    if (st + ahead(D) < kSteps) read(st + ahead(D));
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 sb[2];
    s.operands(st, sb);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      o[0] = mfma32(sb[p], qf[st][0], o[0]);
      o[1] = mfma32(sb[p], qf[st][1], o[1]);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int i = 32 * half + (lane & 31) - empty;
    const float by = scale * power(lg, max(REVERSE ? rows - 1 - i : i + 1, 0));
#pragma unroll
    for (int e = 0; e < 16; ++e) o[half][e] *= by;
  }
}
// Adds what the scores give; leaves v's operands.
template <int D, bool REVERSE>
__device__ __forceinline__ void score_outputs(const lds_bf16* ps, const lds_bf16* vs, int col0, int lane, f32x16 (&o)[2], bf16x8 (&vop)[4]) {
  constexpr int kAhead = D < 128 ? 2 : 1;  // (two at 128 spill 36 registers: 65536 packed tokens 441 -> 455 us)
  bf16x8 pf[4][2][2];
  auto pair = [](int st, int half) { return REVERSE ? st >= 2 * half : st < 2 * half + 2; };
  auto read = [&](int st) {
    vop[st] = column_operand<D, false>(vs, 16 * st, col0, lane);
#pragma unroll
    for (int half = 0; half < 2; ++half)
      if (pair(st, half))
#pragma unroll
        for (int p = 0; p < 2; ++p)
          pf[st][half][p] = row_operand<32>(ps + (half + (st >> 1) + 3 * p) * kScoreTile, 0, st & 1, lane);
  };
#pragma unroll
  for (int st = 0; st < kAhead; ++st) read(st);
#pragma unroll
  for (int st = 0; st < 4; ++st) {
    if (st + kAhead < 4) read(st + kAhead);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int half = 0; half < 2; ++half)
        if (pair(st, half)) o[half] = mfma32(vop[st], pf[st][half][p], o[half]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The walk forwards: outputs, or dq.  A workgroup takes all query heads of its key/value head, one after the other in each block.  The next query head's rows are stored to LDS as soon as
// all waves are through with this one's, in the middle of its step, and those of the one after next fetched from then on; k and v of the next block are fetched while this one's query
// heads run.  Two workgroups share a compute unit (head_dim 128: 74 KB of LDS each).
template <int D, bool TRANSPOSED, int PARTS>
__device__ __forceinline__ void walk(const WalkArgs& a, const LinearSegs& segs, const Piece& p) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr int kTile = kBlock * pitch(D), kWaves = D / 32;
  constexpr bool kAheadOfBlock = D < 256;  // (at 256 the registers do not hold k and v of the next block as well)
  lds_bf16* const qs = (lds_bf16*)smem;
  lds_bf16* const ks = qs + kTile;
  lds_bf16* const vs = ks + kTile;
  lds_bf16* const ps = vs + kTile;  // weighted scores
  lds_f32* const near = (lds_f32*)(ps + kScoreBytes / 2);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hh = lane >> 5;
  const int h = blockIdx.x % a.heads;
  const float lg = log2_decay(a.log_decay, h);
  const int group = a.group;
  const int64_t q_stride = (int64_t)a.heads * group * D, kv_stride = (int64_t)a.heads * D;
  const int blocks = (p.rows + kBlock - 1) / kBlock;

  auto rows_of = [&](int n) { return min(kBlock, p.rows - n * kBlock); };
  auto q_rows = [&](const __bf16* t, int n, int g) {
    return Rows(t + (int64_t)(p.row + n * kBlock) * q_stride + (h * group + g) * D, 2 * (int)q_stride, rows_of(n), 2 * D);
  };
  Tile<D> qt, kt, vt;
  auto fetch_q = [&](int n, int g) { qt.fetch(q_rows(a.q, n, g), kBlock - rows_of(n)); };
  auto fetch_kv = [&](int n) {
    const int64_t at = (int64_t)(p.row + n * kBlock) * kv_stride + h * D;
    kt.fetch(Rows(a.k + at, 2 * (int)kv_stride, rows_of(n), 2 * D), kBlock - rows_of(n));
    vt.fetch(Rows(a.v + at, 2 * (int)kv_stride, rows_of(n), 2 * D), kBlock - rows_of(n));
  };
  // the query head `ahead` steps behind (n, g), if there is one
  auto fetch_q_ahead = [&](int n, int g, int ahead) {
    g += ahead;
    n += g / group;
    g %= group;
    if (n < blocks) fetch_q(n, g);
  };
  fetch_q(0, 0);
  fetch_kv(0);
  const int col = 32 * wave + (lane & 31);
  State<D> s;
  const int from = segs.in[p.seg];
  const bool direct = D < 256 && a.direct;
  if (p.pieces > 1 && (!direct || p.index > 0 || (a.first && from >= 0))) {
    const int64_t apart = (int64_t)a.heads * D * D;
    float* const sums = a.inner + segs.place0[p.seg] * apart + (int64_t)h * D * D;
    s.load_own(sums + (!direct ? p.index : p.index > 0 ? 0 : p.pieces - 1) * apart, wave, lane);
    if (direct) {
      const float whole = power(lg, segs.piece_rows);
      for (int i = 1; i < p.index; ++i) s.scale_and_add_own(whole, sums + i * apart, wave, lane);
    }
  } else if (p.pieces == 1 && a.first && from >= 0) s.template load<TRANSPOSED>(a.first + ((int64_t)from * a.heads + h) * D * D, col, hh);
  else s.clear();
  const StateWeights<false> weights(lg, 1.f, hh, p.rows);
  score_weights<false, 2 * D>(lg, a.scale, p.rows, near);
  wait_all_but<0>();  // (else the compiler has the loop wait for all loads wherever it uses the state)
  qt.store(qs);
  kt.store(ks);
  vt.store(vs);
  fetch_q_ahead(0, 0, 1);
  if (kAheadOfBlock && blocks > 1) fetch_kv(1);
  __syncthreads();

  for (int n = 0; n < blocks; ++n) {
    const int rows = rows_of(n), empty = kBlock - rows;
    for (int g = 0; g < group; ++g) {
      const bool last = g == group - 1;
      f32x16 o[2];
      bf16x8 vop[4];
      for (int tile = wave; tile < 3; tile += kWaves) scores<D, false>(tile, qs, ks, near, ps, lane);
      state_outputs<D, false>(s, qs, lg, a.scale, rows, empty, lane, o);
      __syncthreads();
      if (!last || n + 1 < blocks) {
        qt.store(qs);
        fetch_q_ahead(n, g, 2);
      }
      score_outputs<D, false>(ps, vs, 32 * wave, lane, o, vop);
      const Rows out = q_rows(a.o, n, g);
#pragma unroll
      for (int half = 0; half < 2; ++half) store_rows(out, 32 * half - empty, 64 * wave, o[half], lane);
      if (last) {
        s.scale(power(lg, rows));
#pragma unroll
        for (int st = 0; st < 4; ++st) s.template add<PARTS>(ks, 16 * st, D < 256 ? vop[st] : column_operand<D, false>(vs, 16 * st, 32 * wave, lane), weights.lead[st], weights.base, lane);
        if (n + 1 < blocks) {
          __syncthreads();
          if (!kAheadOfBlock) fetch_kv(n + 1);
          kt.store(ks);
          vt.store(vs);
          if (kAheadOfBlock && n + 2 < blocks) fetch_kv(n + 2);
        }
      }
      __syncthreads();
    }
  }
  if constexpr (PARTS == 3) s.store(a.last + ((int64_t)segs.out[p.seg] * a.heads + h) * D * D, col, hh);
}
template <int D, bool TRANSPOSED>
__global__ __launch_bounds__(2 * D, 2) void walk_kernel(const WalkArgs a, const LinearSegs segs) {
  const Piece p = find_piece(segs, blockIdx.x / a.heads);
  if constexpr (!TRANSPOSED) {  // (those leave none)
    if (a.last && segs.out[p.seg] >= 0 && p.index == p.pieces - 1) return walk<D, TRANSPOSED, 3>(a, segs, p);  // leaves its state
  }
  walk<D, TRANSPOSED, 2>(a, segs, p);
}

// The walk backwards: dv (q's role: k; k, v: q, d_o; the state R) and dk (v; d_o, q; R^T), both from the same tiles of q and d_o, which half of the waves take in one role and half in the other
// (head_dim 256, where their states do not fit the registers of one compute unit: a workgroup for each).  What all query heads hand to the key/value head adds up in the accumulators.  With two buffers
// (head_dim 96 and 128) the next query head's rows are stored while this one's are read.
struct BackArgs {
  const __bf16 *q, *k, *v, *d_o;
  __bf16 *dk, *dv;
  const float* log_decay;
  const float* first;
  float* last;
  float* inner;
  int heads, group;
  float scale;
  int only;  // where a workgroup has one role: the role of all of this launch, or -1: the two by turns
};
static_assert(sizeof(LinearSegs) + sizeof(BackArgs) <= 3900, "fits the kernel arguments");
template <int D>
struct Back {
  static constexpr int kRoles = D == 256 ? 1 : 2, kThreads = 2 * D * kRoles, kBuffers = D == 96 || D == 128 ? 2 : 1;
  static constexpr size_t smem = (kRoles + 2 * kBuffers) * tile_bytes(D) + kRoles * kScoreBytes + kNear * sizeof(float);
};
template <int D, int PARTS>
__device__ __forceinline__ void walk_back(const BackArgs& a, const LinearSegs& segs, const Piece& p, int h, int workgroup_role) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr int kTile = kBlock * pitch(D), kWaves = D / 32, kRoles = Back<D>::kRoles, kBuffers = Back<D>::kBuffers, kThreads = Back<D>::kThreads;
  const int lane = threadIdx.x & 63, hh = lane >> 5, wave = (threadIdx.x >> 6) % kWaves;
  const int role = __builtin_amdgcn_readfirstlane(kRoles == 2 ? (int)(threadIdx.x >> 6) / kWaves : workgroup_role);  // 0: dv, 1: dk
  lds_bf16* const own = (lds_bf16*)smem + (kRoles == 2 ? role * kTile : 0);  // k or v
  lds_bf16* const shared = (lds_bf16*)smem + kRoles * kTile;                 // q and d_o, by turns in two places
  lds_bf16* const ps = shared + 2 * kBuffers * kTile + (kRoles == 2 ? role * (int)kScoreBytes / 2 : 0);
  lds_f32* const near = (lds_f32*)((lds_bf16*)smem + (kRoles + 2 * kBuffers) * kTile + kRoles * (int)kScoreBytes / 2);
  const float lg = log2_decay(a.log_decay, h);
  const int group = a.group;
  const int64_t q_stride = (int64_t)a.heads * group * D, kv_stride = (int64_t)a.heads * D;
  const int blocks = (p.rows + kBlock - 1) / kBlock;

  auto rows_of = [&](int n) { return min(kBlock, p.rows - (blocks - 1 - n) * kBlock); };
  auto kv_rows = [&](const __bf16* t, int n) {
    return Rows(t + (int64_t)(p.row + (blocks - 1 - n) * kBlock) * kv_stride + h * D, 2 * (int)kv_stride, rows_of(n), 2 * D);
  };
  Tile<D, 2 * D> owned;
  Tile<D, kThreads> qt, dt;
  int next_block = 0, next_head = 0;  // what is fetched next
  auto fetch = [&] {
    if (next_block >= blocks) return;
    const int64_t at = (int64_t)(p.row + (blocks - 1 - next_block) * kBlock) * q_stride + (h * group + next_head) * D;
    qt.fetch(Rows(a.q + at, 2 * (int)q_stride, rows_of(next_block), 2 * D), 0);
    dt.fetch(Rows(a.d_o + at, 2 * (int)q_stride, rows_of(next_block), 2 * D), 0);
    if (++next_head == group) {
      next_head = 0;
      ++next_block;
    }
  };
  fetch();
  owned.fetch(kv_rows(role ? a.v : a.k, 0), 0);
  const int col = 32 * wave + (lane & 31), from = segs.out[p.seg];
  const bool given = a.first && from >= 0;
  State<D> s;
  if (p.pieces > 1 || given) {
    const float* const at = p.pieces > 1 ? a.inner + ((int64_t)(segs.place0[p.seg] + p.index) * a.heads + h) * D * D : a.first + ((int64_t)from * a.heads + h) * D * D;
    if (role) s.template load<true>(at, col, hh);
    else s.template load<false>(at, col, hh);
  } else {
    s.clear();
  }
  const StateWeights<true> weights(lg, a.scale, hh, p.rows);
  score_weights<true, kThreads>(lg, a.scale, p.rows, near);
  wait_all_but<0>();  // (as in the walk forwards)
  qt.store(shared);
  dt.store(shared + kTile);
  owned.store(own);
  constexpr bool kFetchAhead = D < 256;  // (at 256 the registers do not hold the next rows as well)
  if (kFetchAhead) {
    fetch();
    if (blocks > 1) owned.fetch(kv_rows(role ? a.v : a.k, 1), 0);
  }
  __syncthreads();

  int turn = 0;
  for (int n = 0; n < blocks; ++n) {
    const int rows = rows_of(n);
    f32x16 o[2];
    for (int g = 0; g < group; ++g) {
      const bool last = g == group - 1, more = !last || n + 1 < blocks;
      const lds_bf16* const ks = shared + (2 * turn + role) * kTile;  // dv: q, dk: d_o
      const lds_bf16* const vs = shared + (2 * turn + 1 - role) * kTile;
      bf16x8 vop[4];
      for (int tile = wave; tile < 3; tile += kWaves) scores<D, true>(tile, own, ks, near, ps, lane);
      if (g == 0) state_outputs<D, true>(s, own, lg, 1.f, rows, 0, lane, o);
      auto store_next = [&] {
        qt.store(shared + 2 * (turn ^ 1) * kTile);
        dt.store(shared + (2 * (turn ^ 1) + 1) * kTile);
        fetch();
      };
      __syncthreads();
      if (last && n + 1 < blocks) {
        if (!kFetchAhead) owned.fetch(kv_rows(role ? a.v : a.k, n + 1), 0);
        owned.store(own);
        if (kFetchAhead && n + 2 < blocks) owned.fetch(kv_rows(role ? a.v : a.k, n + 2), 0);
      }
      if (kBuffers == 2 && more && role == 0) store_next();  // (while the other half's products run, which stores when this half's run)
      score_outputs<D, true>(ps, vs, 32 * wave, lane, o, vop);
      if (last) {
        const Rows out = kv_rows(role ? a.dk : a.dv, n);
#pragma unroll
        for (int half = 0; half < 2; ++half) store_rows(out, 32 * half, 64 * wave, o[half], lane);
      }
      if (g == 0) s.scale(power(lg, rows));
#pragma unroll
      for (int st = 0; st < 4; ++st) s.template add<PARTS>(ks, 16 * st, D < 256 ? vop[st] : column_operand<D, false>(vs, 16 * st, 32 * wave, lane), weights.lead[st], weights.base, lane);
      if (kBuffers == 2 && more && role == 1) store_next();
      if (kBuffers == 1 && more) {
        __syncthreads();
        if (!kFetchAhead) fetch();
        qt.store(shared);
        dt.store(shared + kTile);
        if (kFetchAhead) fetch();
      }
      __syncthreads();
      if (kBuffers == 2) turn ^= 1;
    }
  }
  if (PARTS == 3 && role == 0) s.store(a.last + ((int64_t)segs.in[p.seg] * a.heads + h) * D * D, col, hh);
}
template <int D>
__global__ __launch_bounds__(Back<D>::kThreads, 2) void walk_back_kernel(const BackArgs a, const LinearSegs segs) {
  const bool turns = Back<D>::kRoles == 1 && a.only < 0;
  const int index = turns ? blockIdx.x / 2 : blockIdx.x, role = turns ? blockIdx.x % 2 : a.only;
  const Piece p = find_piece(segs, index / a.heads);
  if (a.last && segs.in[p.seg] >= 0 && p.index == 0) walk_back<D, 3>(a, segs, p, index % a.heads, role);  // leaves the gradient of a state
  else walk_back<D, 2>(a, segs, p, index % a.heads, role);
}

// ---- one token ----
struct StepArgs {
  const __bf16 *q, *k, *v;
  const float *log_decay, *states_in;
  float* states_out;
  const int32_t* slots;
  __bf16* o;
  int batch, num_states, heads, group;
  float scale;
};
constexpr int step_groups(int d) { return d == 96 ? 8 : 1024 / d; }  // groups of D / 4 threads; a group takes every step_groups-th row of the state
constexpr int step_threads(int d) { return d / 4 * step_groups(d); }
// A workgroup takes one row of the batch and one key/value head: a thread four columns of the state and every so many rows, up to sixteen of them loaded at once, before anything else; HEADS query
// heads at a time.  Bound by memory (the state, read and written).  STREAM: calls that read and write more than the last-level cache (256 MiB), that is states of more than 128 MiB, in place or not, pass it by.  What is
// better depends on what runs until the same states come again.  us, kept / streamed, 32 heads of 128, four sets of states in place by turns (a layer's states among others'): 32 MiB 13.4 / 11.8, 64 MiB
// 25 / 26, 96 MiB 44 / 36, 160 MiB 69 / 59, 256 MiB 107 / 93, 512 MiB 214 / 185; one set in place again and again: 64 MiB 23 / 23, 96 MiB 32 / 35, 160 MiB 51 / 59, 256 MiB 81 / 92, 512 MiB 216 / 184.  The rule keeps what
// is small, where either way may be a sixth ahead, and streams what the states of other layers would drive out of the cache.
constexpr int64_t kStreamBytes = (int64_t)256 << 20;
template <int D, int HEADS, bool STREAM>
__global__ __launch_bounds__(step_threads(D)) void step_kernel(const StepArgs a) {
  constexpr int kGroups = step_groups(D), kThreads = step_threads(D), kRows = D / kGroups, kAtOnce = kRows < 16 ? kRows : 16;
  __shared__ float ks[D], qs[HEADS][D], sums[HEADS][kGroups][D];
  __shared__ int next_row;
  const int h = blockIdx.x % a.heads, first = blockIdx.x / a.heads, slot = a.slots[first];
  if (slot < 0 || slot >= a.num_states) return;
  const int group = threadIdx.x / (D / 4), col = threadIdx.x % (D / 4) * 4;
  const int64_t at = ((int64_t)slot * a.heads + h) * D * D + group * D + col;
  const float* from = a.states_in + at;
  float* const to = a.states_out + at;
  auto load = [](const float* p) {
    const f32x4* const q = reinterpret_cast<const f32x4*>(p);
    return STREAM ? __builtin_nontemporal_load(q) : *q;
  };
  f32x4 x[kAtOnce];
  auto load_rows = [&](const float* p, int n0) {
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) x[n] = load(p + (n0 + n) * kGroups * D);
  };
  load_rows(from, 0);
  const float decay = power(log2_decay(a.log_decay, h), 1);
  int row = first;
  if (threadIdx.x == 0) next_row = a.batch;
  __syncthreads();
  // this workgroup runs all of the slot's rows if its own is the first of them
  bool mine = true;
  for (int i = threadIdx.x; i < a.batch; i += kThreads)
    if (a.slots[i] == slot) {
      if (i < first) mine = false;
      if (i > first) atomicMin(&next_row, i);
    }
  if (__syncthreads_or(!mine)) return;
  while (true) {
    const int64_t kv = ((int64_t)row * a.heads + h) * D;
    for (int i = threadIdx.x; i < D; i += kThreads) ks[i] = (float)a.k[kv + i];
    const bf16x4 v = *reinterpret_cast<const bf16x4*>(a.v + kv + col);
    for (int g0 = 0; g0 < a.group; g0 += HEADS) {
      const int heads = min(HEADS, a.group - g0);
      const int64_t q0 = (((int64_t)row * a.heads + h) * a.group + g0) * D;
      for (int i = threadIdx.x; i < heads * D; i += kThreads) qs[i / D][i % D] = (float)a.q[q0 + i];
      __syncthreads();
      float acc[HEADS][4] = {};
#pragma unroll 1
      for (int n0 = 0; n0 < kRows; n0 += kAtOnce) {
        if (n0 > 0 || g0 > 0 || row != first) load_rows(g0 == 0 ? from : to, n0);
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
          const int r = (n0 + n) * kGroups + group;
          if (g0 == 0) {
            const float kr = ks[r];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[n][e] = x[n][e] * decay + kr * (float)v[e];
            f32x4* const p = reinterpret_cast<f32x4*>(to + (n0 + n) * kGroups * D);
            if (STREAM) __builtin_nontemporal_store(x[n], p);
            else *p = x[n];
          }
#pragma unroll
          for (int g = 0; g < HEADS; ++g) {
            if (HEADS == 1 || g < heads) {
              const float qr = qs[g][r];
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[g][e] += qr * x[n][e];
            }
          }
        }
      }
#pragma unroll
      for (int g = 0; g < HEADS; ++g) *reinterpret_cast<f32x4*>(&sums[g][group][col]) = f32x4{acc[g][0], acc[g][1], acc[g][2], acc[g][3]};
      __syncthreads();
      for (int i = threadIdx.x; i < heads * D; i += kThreads) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) sum += sums[i / D][j][i % D];
        a.o[q0 + i] = (__bf16)(sum * a.scale);
      }
      __syncthreads();
    }
    row = next_row;  // the slot's next token
    if (row >= a.batch) return;
    from = to;
    __syncthreads();
    if (threadIdx.x == 0) next_row = a.batch;
    __syncthreads();
    for (int i = row + 1 + threadIdx.x; i < a.batch; i += kThreads)
      if (a.slots[i] == slot) atomicMin(&next_row, i);
    __syncthreads();
  }
}

// ---- host ----
bool head_dim_ok(int d) { return d == 64 || d == 96 || d == 128 || d == 256; }

int validate_linear(const chunk_linear_desc* d) {
  if (!d || d->num_q_heads < 1 || d->num_kv_heads < 1 || d->total < 1 || d->num_segments < 1 || d->num_states < 0 || !d->segments || !finite_number(d->scale) ||
      d->scale <= 0.f)
    return CHUNK_ATTN_INVALID_ARG;
  if (!head_dim_ok(d->head_dim) || d->num_q_heads % d->num_kv_heads != 0 || d->num_q_heads > CHUNK_LINEAR_MAX_HEADS) return CHUNK_ATTN_UNSUPPORTED;
  int64_t end = 0;
  for (int i = 0; i < d->num_segments; ++i) {
    const chunk_linear_seg& s = d->segments[i];
    if (s.len < 1 || s.start < end || (int64_t)s.start + s.len > d->total) return CHUNK_ATTN_BAD_SEGMENT;
    if (s.state_in < -1 || s.state_in >= d->num_states || s.state_out < -1 || s.state_out >= d->num_states) return CHUNK_ATTN_BAD_SEGMENT;
    end = (int64_t)s.start + s.len;
  }
  return CHUNK_ATTN_OK;
}

// Whether slots are used as they may be: no state_out twice; no state_in twice if `in_once`; if `in_place`, no state_out that is another segment's state_in.
int check_slots(const chunk_linear_desc* d, bool in_once, bool in_place) {
  try {
    std::vector<std::pair<int, int>> out, in;  // (slot, segment)
    for (int i = 0; i < d->num_segments; ++i) {
      if (d->segments[i].state_out >= 0) out.emplace_back(d->segments[i].state_out, i);
      if (d->segments[i].state_in >= 0) in.emplace_back(d->segments[i].state_in, i);
    }
    std::sort(out.begin(), out.end());
    std::sort(in.begin(), in.end());
    for (size_t i = 1; i < out.size(); ++i)
      if (out[i].first == out[i - 1].first) return CHUNK_ATTN_BAD_SEGMENT;
    for (size_t i = 1; in_once && i < in.size(); ++i)
      if (in[i].first == in[i - 1].first) return CHUNK_ATTN_BAD_SEGMENT;
    if (in_place) {
      size_t j = 0;
      for (const auto& o : out) {
        while (j < in.size() && in[j].first < o.first) ++j;
        for (size_t k = j; k < in.size() && in[k].first == o.first; ++k)
          if (in[k].second != o.second) return CHUNK_ATTN_BAD_SEGMENT;
      }
    }
  } catch (const std::bad_alloc&) {
    return CHUNK_ATTN_INVALID_ARG;
  }
  return CHUNK_ATTN_OK;
}

int pieces_of(int len, int rows) { return (len - 1) / rows + 1; }
int64_t count_places(const chunk_linear_desc* d, int rows) {
  int64_t n = 0;
  for (int i = 0; i < d->num_segments; ++i)
    if (d->segments[i].len > rows) n += pieces_of(d->segments[i].len, rows);
  return n;
}
size_t states_bytes(const chunk_linear_desc* d, int64_t n) { return (size_t)n * d->num_kv_heads * d->head_dim * d->head_dim * sizeof(float); }

// What a walk and the sums of its pieces' states take, in us, measured at head_dim 128: a workgroup's start, from zeros or from a state; a block's products for one query head and those it
// takes once, with few workgroups and with as many as the chip has places for (the memory is then the bound); a block in piece_states_kernel.
struct WalkCost {
  double start, start_cut, head[2], block[2], piece_block;
  int few, places;
};
// Rows of a piece: the estimate of all of it that ends first.  Fewer rows: more walks at once, and ends that leave fewer compute units without work; but more states to write, join and read, and k and v
// are read twice.  A launch takes as long as its work on the places it fills, or as the rounds of its full pieces.  us by rows of a piece (* chosen): 8192 tokens of 32/32 of 128, forward, 256: 133, *512: 110,
// 1024: 112, uncut: 428; 16384 in 8 sequences of 32/8, backward, 128: 447, 192: 388, *256: 394, 512: 401, 1024: 503, uncut: 2804; 32 sequences of 2000 of 32/8, backward, 512: 1185, 1024: 1079, *uncut: 942.  The other head
// dimensions go by the same figures; their own are within a tenth of the best cut.  64, 16384 tokens: 32/32, forward, 512: 99, 768: 90, *1024: 94, 2048: 125, backward, 512: 243, *1024: 228, 2048: 281; 16/4, forward, 64: 64, *128: 51,
// 256: 53, 512: 83, backward, 64: 144, *128: 116, 256: 122, 512: 193.  96, 8192 of 32/8: forward, 64: 72, *128: 59, 256: 55, 512: 83, backward, 64: 190, *128: 158, 256: 145, 512: 222.  256, 8192 of 16/16: forward, 256: 265,
// *512: 213, 1024: 296, backward, 256: 651, *512: 533, 1024: 602.
int piece_rows(const chunk_linear_desc* d, const WalkCost& c) {
  int longest = 0;
  int64_t blocks = 0;
  for (int i = 0; i < d->num_segments; ++i) {
    longest = std::max(longest, d->segments[i].len);
    blocks += (d->segments[i].len + kBlock - 1) / kBlock;
  }
  const int group = d->num_q_heads / d->num_kv_heads, all = (longest + kBlock - 1) / kBlock;
  const double heads = d->num_kv_heads;
  int best = 0;
  double best_us = 0;
  for (int m = 1, next = 2;; m = next, next = m < 4 ? m + 1 : m % 3 == 0 ? m / 3 * 4 : m / 2 * 3) {  // 1, 2, 3, 4, 6, 8, 12, 16, 24, ...
    m = std::min(m, all);
    const int rows = m * kBlock;
    int64_t full = 0, pieces = 0, places = 0, summed = 0;
    for (int i = 0; i < d->num_segments; ++i) {
      const int len = d->segments[i].len, n = pieces_of(len, rows);
      full += len / rows;
      pieces += n;
      if (n > 1) {
        places += n;
        summed += (int64_t)(n - 1) * m;
      }
    }
    const double filled = std::min<double>(pieces * heads, c.places), busy = std::min(1.0, std::max(0.0, (filled - c.few) / std::max(1, c.places - c.few)));
    const double block = c.block[0] + busy * (c.block[1] - c.block[0]) + group * (c.head[0] + busy * (c.head[1] - c.head[0]));
    const double start = places > 0 ? c.start_cut : c.start, piece = start + m * block;
    double us = std::max(std::max(((pieces - places) * c.start + places * c.start_cut + blocks * block) * heads / filled, piece), std::ceil(full * heads / c.places) * piece);
    if (places > 0) us += 12 + std::max(summed * heads / (2 * kCus), (double)m) * c.piece_block + states_bytes(d, places) * 2 / 5.5e6 + 0.06 * (all / m);
    if (best == 0 || us < best_us) {
      best = rows;
      best_us = us;
    }
    if (m == all || blocks / m * heads < 16) break;
  }
  return best;
}
int forward_rows(const chunk_linear_desc* d) { return piece_rows(d, {3, 9, {2.1, 3.4}, {1.5, 2.0}, 3.0, kCus, d->head_dim > 128 ? kCus : 2 * kCus}); }
int backward_rows(const chunk_linear_desc* d) {
  return piece_rows(d, {3, 9, {3.4, 3.4}, {1.0, 1.0}, 3.0 * (d->num_q_heads / d->num_kv_heads), kCus, d->head_dim > 128 ? kCus / 2 : kCus});
}

// Up to this many elements of sums before a piece its walk adds them up itself, which saves a launch.  us, added up by join_states_kernel / by the walks: four sequences of 128 - 512 tokens, 8 heads of 64
// (up to 8 pieces), 14.9 / 12.9; 8 of 2000, 8 heads of 64, 37.5 / 34.4; 16384 tokens, 32 heads of 64, 96 / 94; but 4096 tokens, 8 heads of 64 in 64 pieces 22.5 / 26.4, 16384 of 32/8 of 128
// in 64 125 / 154.  Not at head_dim 256, whose walks have no registers for it.
constexpr int kDirect = 5 * 128 * 128;

template <class F>
hipError_t by_dim(int d, F&& f) {
  using std::integral_constant;
  if (d == 64) return f(integral_constant<int, 64>{});
  if (d == 96) return f(integral_constant<int, 96>{});
  if (d == 128) return f(integral_constant<int, 128>{});
  return f(integral_constant<int, 256>{});
}

template <int D, bool REVERSE, bool TRANSPOSED>
hipError_t launch_piece_states(const WalkArgs& a, const LinearSegs& segs, hipStream_t stream) {
  constexpr size_t smem = 2 * tile_bytes(D);
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(&piece_states_kernel<D, REVERSE, TRANSPOSED>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((piece_states_kernel<D, REVERSE, TRANSPOSED>), dim3((unsigned)((REVERSE ? segs.num_pieces : segs.num_full) * a.heads)), dim3(2 * D), smem, stream, a, segs);
  if (!a.direct)
    hipLaunchKernelGGL((join_states_kernel<D, REVERSE, TRANSPOSED>), dim3((unsigned)(D * D / 1024 * a.heads), (unsigned)segs.n), dim3(256), 0, stream, a, segs);
  return hipGetLastError();
}
template <int D, bool TRANSPOSED>
hipError_t launch_walk(const WalkArgs& a, const LinearSegs& segs, hipStream_t stream) {
  constexpr size_t smem = 3 * tile_bytes(D) + kScoreBytes + kNear * sizeof(float);
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&walk_kernel<D, TRANSPOSED>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((walk_kernel<D, TRANSPOSED>), dim3((unsigned)(segs.num_pieces * a.heads)), dim3(2 * D), smem, stream, a, segs);
  return hipGetLastError();
}
// Forward sums and walks, of segments in at most `pieces` pieces.
template <int D, bool TRANSPOSED>
hipError_t launch_forward(WalkArgs a, const LinearSegs& segs, int pieces, hipStream_t stream) {
  a.direct = D < 256 && (pieces - 1) * D * D <= kDirect;
  const hipError_t e = pieces > 1 ? launch_piece_states<D, false, TRANSPOSED>(a, segs, stream) : hipSuccess;
  return e != hipSuccess ? e : launch_walk<D, TRANSPOSED>(a, segs, stream);
}
// Whether the gradient of some state is read and written in one place by the walks themselves.  (Cut sequences start from a copy in the workspace.)
bool in_place_uncut(const BackArgs& a, const LinearSegs& segs) {
  if (!a.last || a.last != a.first) return false;
  for (int i = 0; i < segs.n; ++i)
    if (segs.len[i] <= segs.piece_rows && segs.in[i] >= 0 && segs.in[i] == segs.out[i]) return true;
  return false;
}
template <int D>
hipError_t launch_walk_back(BackArgs a, const LinearSegs& segs, hipStream_t stream) {
  constexpr size_t smem = Back<D>::smem;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&walk_back_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (attr != hipSuccess) return attr;
  auto launch = [&](int roles, int only) {
    a.only = only;
    hipLaunchKernelGGL((walk_back_kernel<D>), dim3((unsigned)(segs.num_pieces * a.heads * roles)), dim3(Back<D>::kThreads), smem, stream, a, segs);
    return hipGetLastError();
  };
  if constexpr (Back<D>::kRoles == 1) {
    if (in_place_uncut(a, segs)) {  // dk's workgroups start from a gradient that dv's replace, and nothing says which of them run first: dk in a launch before
      const hipError_t e = launch(1, 1);
      return e != hipSuccess ? e : launch(1, 0);
    }
    return launch(2, -1);
  }
  return launch(1, -1);
}

// Goes through the segments, as many at a time as travel with a launch, with how many pieces any of them has.  Full pieces start first, the others in falling size: what starts last is short.
template <class F>
hipError_t for_segments(const chunk_linear_desc* d, int rows, F&& f) {
  std::vector<int> order;
  try {
    order.resize(d->num_segments);
  } catch (const std::bad_alloc&) {
    return hipErrorOutOfMemory;
  }
  for (int i = 0; i < d->num_segments; ++i) order[i] = i;
  std::sort(order.begin(), order.end(), [&](int a, int b) {
    const int x = d->segments[a].len % rows, y = d->segments[b].len % rows;
    return x != y ? x > y : a < b;
  });
  LinearSegs s;
  int64_t places = 0;
  for (int s0 = 0; s0 < d->num_segments; s0 += kLinearSegs) {
    s.n = std::min(kLinearSegs, d->num_segments - s0);
    s.piece_rows = rows;
    s.num_full = s.num_pieces = 0;
    int most = 1;
    for (int i = 0; i < s.n; ++i) {
      const chunk_linear_seg& x = d->segments[order[s0 + i]];
      s.start[i] = x.start;
      s.len[i] = x.len;
      s.in[i] = x.state_in;
      s.out[i] = x.state_out;
      s.full0[i] = s.num_full;
      s.place0[i] = (int)places;
      s.num_full += x.len / rows;
      s.num_pieces += x.len % rows != 0;
      if (x.len > rows) {
        places += pieces_of(x.len, rows);
        most = std::max(most, pieces_of(x.len, rows));
      }
    }
    s.num_pieces += s.num_full;
    const hipError_t e = f(s, most);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
bool aligned16(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (((uintptr_t)p & 15) != 0) return false;
  return true;
}

}  // namespace
}  // namespace chunk_attn

extern "C" int chunk_linear_validate(const chunk_linear_desc* d) {
  const int rc = chunk_attn::validate_linear(d);
  return rc != CHUNK_ATTN_OK ? rc : chunk_attn::check_slots(d, false, false);
}

extern "C" int chunk_linear_workspace_bytes(const chunk_linear_desc* d, size_t* fwd_bytes, size_t* bwd_bytes) {
  using namespace chunk_attn;
  const int rc = chunk_linear_validate(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (!fwd_bytes || !bwd_bytes) return CHUNK_ATTN_INVALID_ARG;
  *fwd_bytes = states_bytes(d, count_places(d, forward_rows(d)));
  *bwd_bytes = *fwd_bytes + states_bytes(d, count_places(d, backward_rows(d)));
  return CHUNK_ATTN_OK;
}

extern "C" int chunk_linear_fwd(const chunk_linear_desc* d, const void* q, const void* k, const void* v, const float* log_decay, const float* states_in, void* o,
                                float* states_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace chunk_attn;
  int rc = validate_linear(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (!q || !k || !v || !o || !log_decay || !aligned16({q, k, v, o, states_in, states_out}) || ((uintptr_t)log_decay & 3) != 0) return CHUNK_ATTN_INVALID_ARG;
  for (int i = 0; i < d->num_segments; ++i)
    if ((d->segments[i].state_in >= 0 && !states_in) || (d->segments[i].state_out >= 0 && !states_out)) return CHUNK_ATTN_INVALID_ARG;
  if ((rc = check_slots(d, false, states_in == states_out)) != CHUNK_ATTN_OK) return rc;
  const int rows = forward_rows(d);
  const size_t need = states_bytes(d, count_places(d, rows));
  if (need > 0) {
    if (!workspace || ((uintptr_t)workspace & 255) != 0) return CHUNK_ATTN_INVALID_ARG;
    if (workspace_bytes < need) return CHUNK_ATTN_WORKSPACE_TOO_SMALL;
  }
  WalkArgs a{(const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (__bf16*)o, log_decay, states_in, states_out, (float*)workspace, d->num_kv_heads,
             d->num_q_heads / d->num_kv_heads, d->scale};
  const hipStream_t stream = (hipStream_t)hip_stream;
  const hipError_t e = for_segments(d, rows, [&](const LinearSegs& segs, int pieces) {
    return by_dim(d->head_dim, [&](auto dim) {
      constexpr int D = decltype(dim)::value;
      return launch_forward<D, false>(a, segs, pieces, stream);
    });
  });
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, "linear attention forward");
}

extern "C" int chunk_linear_bwd(const chunk_linear_desc* d, const void* q, const void* k, const void* v, const float* log_decay, const float* states_in,
                                const void* d_o, const float* d_states_out, void* dq, void* dk, void* dv, float* d_states_in, void* workspace,
                                size_t workspace_bytes, void* hip_stream) {
  using namespace chunk_attn;
  int rc = validate_linear(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (!q || !k || !v || !d_o || !dq || !dk || !dv || !log_decay || !aligned16({q, k, v, d_o, dq, dk, dv, states_in, d_states_out, d_states_in}) ||
      ((uintptr_t)log_decay & 3) != 0)
    return CHUNK_ATTN_INVALID_ARG;
  for (int i = 0; i < d->num_segments; ++i)
    if (d->segments[i].state_in >= 0 && !states_in) return CHUNK_ATTN_INVALID_ARG;
  // (the slots of the gradients: read by state_out, written by state_in)
  if ((rc = check_slots(d, d_states_in != nullptr, d_states_in != nullptr && d_states_in == d_states_out)) != CHUNK_ATTN_OK) return rc;
  const int rows_q = forward_rows(d), rows_kv = backward_rows(d);
  const size_t need_q = states_bytes(d, count_places(d, rows_q)), need_kv = states_bytes(d, count_places(d, rows_kv));
  if (need_q + need_kv > 0) {
    if (!workspace || ((uintptr_t)workspace & 255) != 0) return CHUNK_ATTN_INVALID_ARG;
    if (workspace_bytes < need_q + need_kv) return CHUNK_ATTN_WORKSPACE_TOO_SMALL;
  }
  const __bf16 *bq = (const __bf16*)q, *bk = (const __bf16*)k, *bv = (const __bf16*)v, *bo = (const __bf16*)d_o;
  float* const inner_s = (float*)workspace;
  float* const inner_r = need_kv > 0 ? inner_s + need_q / sizeof(float) : nullptr;
  const int heads = d->num_kv_heads, group = d->num_q_heads / heads;
  const WalkArgs to_q{bo, bv, bk, (__bf16*)dq, log_decay, states_in, nullptr, inner_s, heads, group, d->scale};
  const WalkArgs r_states{nullptr, bq, bo, nullptr, log_decay, d_states_out, d_states_in, inner_r, heads, group, d->scale};
  const BackArgs to_kv{bq, bk, bv, bo, (__bf16*)dk, (__bf16*)dv, log_decay, d_states_out, d_states_in, inner_r, heads, group, d->scale, -1};
  const hipStream_t stream = (hipStream_t)hip_stream;
  hipError_t e = for_segments(d, rows_q, [&](const LinearSegs& segs, int pieces) {
    return by_dim(d->head_dim, [&](auto dim) {
      constexpr int D = decltype(dim)::value;
      return launch_forward<D, true>(to_q, segs, pieces, stream);
    });
  });
  if (e != hipSuccess) return report_hip(e, "linear attention backward, dq");
  e = for_segments(d, rows_kv, [&](const LinearSegs& segs, int pieces) {
    return by_dim(d->head_dim, [&](auto dim) {
      constexpr int D = decltype(dim)::value;
      const hipError_t e = pieces > 1 ? launch_piece_states<D, true, false>(r_states, segs, stream) : hipSuccess;
      return e != hipSuccess ? e : launch_walk_back<D>(to_kv, segs, stream);
    });
  });
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, "linear attention backward");
}

extern "C" int chunk_linear_step(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, const void* q, const void* k, const void* v,
                                 const float* log_decay, const float* states_in, float* states_out, int32_t num_states, const int32_t* slots, void* o, float scale,
                                 void* hip_stream) {
  using namespace chunk_attn;
  if (batch < 0 || num_q_heads < 1 || num_kv_heads < 1 || num_states < 0 || !finite_number(scale) || scale <= 0.f) return CHUNK_ATTN_INVALID_ARG;
  if (!head_dim_ok(head_dim) || num_q_heads % num_kv_heads != 0) return CHUNK_ATTN_UNSUPPORTED;
  if (batch == 0) return CHUNK_ATTN_OK;
  if (!q || !k || !v || !o || !log_decay || !slots || (num_states > 0 && (!states_in || !states_out)) || !aligned16({q, k, v, o, states_in, states_out}) ||
      (((uintptr_t)log_decay | (uintptr_t)slots) & 3) != 0 || (int64_t)batch * num_kv_heads >= 1 << 24)  // (threads of a launch: below 2^32)
    return CHUNK_ATTN_INVALID_ARG;
  const StepArgs a{(const __bf16*)q, (const __bf16*)k, (const __bf16*)v, log_decay, states_in, states_out, slots, (__bf16*)o, batch, num_states, num_kv_heads,
                   num_q_heads / num_kv_heads, scale};
  const hipError_t e = by_dim(head_dim, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    auto launch = [&](auto heads, auto stream) {
      hipLaunchKernelGGL((step_kernel<D, decltype(heads)::value, decltype(stream)::value>), dim3((unsigned)(batch * num_kv_heads)), dim3(step_threads(D)), 0, (hipStream_t)hip_stream, a);
    };
    auto with_heads = [&](auto heads) {
      if ((int64_t)batch * num_kv_heads * D * D * 8 > kStreamBytes) launch(heads, std::true_type{});
      else launch(heads, std::false_type{});
    };
    if (a.group == 1) with_heads(std::integral_constant<int, 1>{});
    else if (a.group <= 4) with_heads(std::integral_constant<int, 4>{});
    else with_heads(std::integral_constant<int, 8>{});
    return hipGetLastError();
  });
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, "linear attention step");
}
