// Linear attention with a decay for each head over the sequences of a chunk (include/chunk_linear.h): forward, backward, and one token at a time.
//
// A sequence is taken in blocks of 64 rows.  With S the state before a block of L rows, row i of the block is
//   o_i = l^(i+1) q_i S + sum_(j<=i) l^(i-j) (q_i . k_j) v_j        and the state behind it        S' = l^L S + sum_j l^(L-1-j) k_j^T v_j,
// four products of matrices.  A workgroup walks the blocks of a piece of a sequence with S in its accumulators: wave w owns columns 32 w .. 32 w + 31 of S and of the
// outputs.  All powers of l that occur have exponents >= 0, whatever the decay, and none of more than 64 rows' distance is formed inside a walk.
//
// The three gradients are the same walk with other tensors in the roles of q, k and v:
//   dq: (d_o, v, k), state S^T;   dv: (k, q, d_o) and dk: (v, d_o, q) backwards, from the last row to the first, over rows j >= i; their state is the gradient of S, or its transpose.
//   Backwards, R before a block (that is, behind its last row) gives   x_i = l^(L-1-i) q_i R + sum_(j>=i) l^(j-i) (q_i . k_j) v_j   and   R' = l^L R + sum_j l^(j+1) k_j^T v_j.
//
// Long sequences are cut into pieces so that there are enough workgroups.  A first kernel forms each piece's own sum of k^T v, a second one adds them up along the sequence, and the
// walks then start from there; states of pieces are float32 throughout.
//
// Accumulators as operands: an accumulator tile holds S[row][column = lane % 32], and the eight values of a lane in one half of it are what an MFMA operand wants of 16 rows, if
// only the rows are named accordingly (device_common.hpp, "C-order").  Here the rows of K^T are fed to the state's product in the order that makes the names come out as
// they are: transposed reads deliver column quads 0, 2, 1, 3.  Outputs are formed transposed (columns = tokens), so that the power of l a row is multiplied with is one
// value of a lane, and four neighbouring elements of an output row lie in a lane.
//
// Precision: k_j^T (l^(L-1-j) v_j) has the weighted v_j as a bf16 operand.  Rounded once it would leave states with 2^-9 relative error, so it is split into three bf16 terms
// (24 bits): the state is then as exact as float32 sums are, for three times its MFMAs (48 of 78 in a block at head_dim 128, where memory is the bound).  S and the weighted scores are
// rounded to bf16 once where they are operands of an output's product.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <new>
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
  int n, num_pieces, piece_rows;  // pieces of these segments; rows of a piece (a multiple of kBlock)
  int start[kLinearSegs], len[kLinearSegs], in[kLinearSegs], out[kLinearSegs];
  int piece0[kLinearSegs];  // first of its pieces among the launch's
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
  float first_scale, last_scale, scale;
};
static_assert(sizeof(LinearSegs) + sizeof(WalkArgs) <= 3900, "fits the kernel arguments");

struct Piece {
  int seg, index, pieces, row, rows;  // index among the segment's pieces; first row; rows
};
__device__ __forceinline__ Piece find_piece(const LinearSegs& s, int piece) {
  const int lane = threadIdx.x & 63;
  int seg = -1;
  for (int i = 0; i < s.n; i += 64) {
    const int j = min(i + lane, s.n - 1);
    seg += __popcll(__ballot(i + lane < s.n && s.piece0[j] <= piece));
  }
  Piece p;
  p.seg = __builtin_amdgcn_readfirstlane(seg);
  const int len = s.len[p.seg];
  p.pieces = (len + s.piece_rows - 1) / s.piece_rows;
  p.index = piece - s.piece0[p.seg];
  p.row = s.start[p.seg] + p.index * s.piece_rows;
  p.rows = min(s.piece_rows, len - p.index * s.piece_rows);
  return p;
}
// log2 of a head's decay.  The bound stands for -inf: l^0 is 1 and every other power 0.
__device__ __forceinline__ float log2_decay(const float* log_decay, int h) { return fmaxf((float)((double)log_decay[h] * 1.4426950408889634), -1000.f); }
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
template <int D>
struct Tile {
  static constexpr int kChunks = D / 8, kThreads = 2 * D, kEach = kBlock * kChunks / kThreads, kRowsApart = kThreads / kChunks;
  u32x4 x[kEach];
  __device__ __forceinline__ void fetch(const Rows& from, int empty) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = from.load((int)threadIdx.x / kChunks + i * kRowsApart - empty, (int)threadIdx.x % kChunks * 16);
  }
  __device__ __forceinline__ void store(lds_bf16* to) const {
    lds_bf16* const at = to + (int)threadIdx.x / kChunks * pitch(D) + (int)threadIdx.x % kChunks * 8;
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
  __device__ __forceinline__ void load(const float* from, int col, int hh, float by) {
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
        for (int r = 0; r < 4; ++r) t[i][4 * g + r] = x[r] * by;
      }
  }
  __device__ __forceinline__ void store(float* to, int col, int hh, float by) const {
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) to[(int64_t)(row(i, g, hh) + r) * D + col] = t[i][4 * g + r] * by;
  }
  __device__ __forceinline__ void scale(float by) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) t[i][e] *= by;
  }
  // operand of rows 16 step .. 16 step + 15 as the contraction
  __device__ __forceinline__ bf16x8 operand(int step) const {
    const f32x16& a = t[step >> 1];
    const int o = 8 * (step & 1);
    return pack8(a[o], a[o + 1], a[o + 2], a[o + 3], a[o + 4], a[o + 5], a[o + 6], a[o + 7]);
  }
  // adds k^T (w v) of 16 rows from row0 on: v's operand as it was read; element e's row weighs lead * base[e]
  template <int PARTS>
  __device__ __forceinline__ void add(const lds_bf16* k_tile, int row0, bf16x8 v, float lead, const float (&base)[8], int lane) {
    constexpr int kTiles = D / 32, kHalf = (kTiles + 1) / 2;
    bf16x8 kt[kTiles], part[PARTS];
#pragma unroll
    for (int i = 0; i < kHalf; ++i) kt[i] = column_operand<D, true>(k_tile, row0, 32 * i, lane);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x = (float)v[e] * (lead * base[e]);
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        part[p][e] = (__bf16)x;
        x -= (float)part[p][e];
      }
    }
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

// Weights of a block's rows in its state, l^(63 - j) or backwards l^(j + 1) for row j = 16 s + 8 hh + e: lead[s] * base[e], both powers with exponents >= 0.
template <bool REVERSE>
struct StateWeights {
  float base[8], lead[4];
  __device__ __forceinline__ StateWeights(float lg, int hh) {
#pragma unroll
    for (int e = 0; e < 8; ++e) base[e] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(power(lg, REVERSE ? e : 7 - e))));
#pragma unroll
    for (int s = 0; s < 4; ++s) lead[s] = power(lg, REVERSE ? 16 * s + 8 * hh + 1 : 56 - 16 * s - 8 * hh);
  }
};

// Each piece's own k^T v into its place in the workspace, but for the one at the far end of its sequence, whose nobody needs, and for sequences of one piece.
template <int D, bool REVERSE, int PARTS>
__global__ __launch_bounds__(2 * D, 2) void piece_states_kernel(const WalkArgs a, const LinearSegs segs) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  lds_bf16* const ks = (lds_bf16*)smem;
  lds_bf16* const vs = ks + kBlock * pitch(D);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hh = lane >> 5;
  const int h = blockIdx.x % a.heads;
  const Piece p = find_piece(segs, blockIdx.x / a.heads);
  if (p.index == (REVERSE ? 0 : p.pieces - 1)) return;
  const float lg = log2_decay(a.log_decay, h);
  const int group = REVERSE ? a.group : 1;
  const int64_t stride = (int64_t)a.heads * group * D;
  const StateWeights<REVERSE> weights(lg, hh);
  State<D> s;
  s.clear();
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
  s.store(a.inner + ((int64_t)(segs.place0[p.seg] + p.index) * a.heads + h) * D * D, 32 * wave + (lane & 31), hh, 1.f);
}

// Adds them up along each sequence: in the place of each piece's own, the state that it starts from.  (The first one's, too: the slot it comes from may be the one that
// the last piece's state goes to.)
template <bool REVERSE>
__global__ __launch_bounds__(256) void join_states_kernel(const WalkArgs a, const LinearSegs segs, int elements) {
  const int seg = blockIdx.y / a.heads, h = blockIdx.y % a.heads;
  const int at = (blockIdx.x * 256 + threadIdx.x) * 4;
  const int len = segs.len[seg], pieces = (len + segs.piece_rows - 1) / segs.piece_rows;
  if (pieces == 1 || at >= elements) return;
  const float lg = log2_decay(a.log_decay, h);
  const int slot = REVERSE ? segs.out[seg] : segs.in[seg];
  f32x4 sum{};
  if (a.first && slot >= 0) sum = *reinterpret_cast<const f32x4*>(a.first + ((int64_t)slot * a.heads + h) * elements + at) * a.first_scale;
  const float whole = power(lg, segs.piece_rows);
  f32x4* const x = reinterpret_cast<f32x4*>(a.inner + ((int64_t)segs.place0[seg] * a.heads + h) * elements + at);
  const int64_t apart = (int64_t)a.heads * elements / 4;
  constexpr int kAhead = 8;  // states are loaded eight at a time: one after the other a sequence of 32 pieces took 20 us
  for (int n0 = 0; n0 < pieces; n0 += kAhead) {
    f32x4 own[kAhead];
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
      if (n0 + n < pieces - 1) own[n] = x[(REVERSE ? pieces - 1 - n0 - n : n0 + n) * apart];
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
      if (n0 + n < pieces) {
        const int i = REVERSE ? pieces - 1 - n0 - n : n0 + n;
        x[i * apart] = sum;
        if (n0 + n < pieces - 1) sum = sum * (i == pieces - 1 ? power(lg, len - i * segs.piece_rows) : whole) + own[n];
      }
  }
}

// Four neighbouring elements of a row from either half of the wave (registers 4 g .. 4 g + 3 of an output tile are elements 8 g + 4 hh ..): stored as 16 bytes, the lower half
// of the lanes takes those of an even g, the upper one those of the odd g behind it.
__device__ __forceinline__ void store_row(const Rows& to, int row, int byte, const f32x16& o, float by, int hh) {
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    union {
      bf16x4 h;
      unsigned u[2];
    } even, odd;
    even.h = pack4(o[4 * g] * by, o[4 * g + 1] * by, o[4 * g + 2] * by, o[4 * g + 3] * by);
    odd.h = pack4(o[4 * g + 4] * by, o[4 * g + 5] * by, o[4 * g + 6] * by, o[4 * g + 7] * by);
    const u32x2 x = __builtin_amdgcn_permlane32_swap(even.u[0], odd.u[0], false, false), y = __builtin_amdgcn_permlane32_swap(even.u[1], odd.u[1], false, false);
    to.store(row, byte + 16 * (g + hh), u32x4{x[0], y[0], x[1], y[1]});
  }
}

// The walk.  Forwards a workgroup takes all query heads of its key/value head, one after the other in each block; backwards all of them stand in the roles of k and v.
// The next step's rows are fetched while this one's products run; two workgroups share a compute unit (head_dim 128: 56 KB of LDS and at most 256 registers each).
template <int D, bool REVERSE, bool TRANSPOSED, int PARTS>
__global__ __launch_bounds__(2 * D, 2) void walk_kernel(const WalkArgs a, const LinearSegs segs) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  lds_bf16* const qs = (lds_bf16*)smem;
  lds_bf16* const ks = qs + kBlock * pitch(D);
  lds_bf16* const vs = ks + kBlock * pitch(D);
  lds_bf16* const ps = vs + kBlock * pitch(D);  // weighted scores, 64 x 64
  lds_f32* const near = (lds_f32*)(ps + kBlock * pitch(64));
  constexpr int kWaves = D / 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hh = lane >> 5, l32 = lane & 31;
  const int h = blockIdx.x % a.heads;
  const Piece p = find_piece(segs, blockIdx.x / a.heads);
  const float lg = log2_decay(a.log_decay, h);
  const int group = a.group, q_group = REVERSE ? 1 : group, kv_group = REVERSE ? group : 1;
  const int64_t q_stride = (int64_t)a.heads * q_group * D, kv_stride = (int64_t)a.heads * kv_group * D;
  const int blocks = (p.rows + kBlock - 1) / kBlock;

  struct Step {  // one block and one query head
    int g, rows, empty;
    int64_t row0;
  };
  auto step_of = [&](int n, int g) {
    const int b = REVERSE ? blocks - 1 - n : n, rows = min(kBlock, p.rows - b * kBlock);
    return Step{g, rows, REVERSE ? 0 : kBlock - rows, (int64_t)p.row + b * kBlock};
  };
  Tile<D> qt, kt, vt;
  auto fetch = [&](const Step& x) {
    if (!REVERSE || x.g == 0) qt.fetch(Rows(a.q + x.row0 * q_stride + (h * q_group + (REVERSE ? 0 : x.g)) * D, 2 * (int)q_stride, x.rows, 2 * D), x.empty);
    if (REVERSE || x.g == 0) {
      const int64_t at = x.row0 * kv_stride + (h * kv_group + (REVERSE ? x.g : 0)) * D;
      kt.fetch(Rows(a.k + at, 2 * (int)kv_stride, x.rows, 2 * D), x.empty);
      vt.fetch(Rows(a.v + at, 2 * (int)kv_stride, x.rows, 2 * D), x.empty);
    }
  };
  Step now = step_of(0, 0);
  fetch(now);

  const int col = 32 * wave + l32;
  State<D> s;
  const int from = REVERSE ? segs.out[p.seg] : segs.in[p.seg];
  if (p.pieces > 1) s.template load<TRANSPOSED>(a.inner + ((int64_t)(segs.place0[p.seg] + p.index) * a.heads + h) * D * D, col, hh, 1.f);
  else if (a.first && from >= 0) s.template load<TRANSPOSED>(a.first + ((int64_t)from * a.heads + h) * D * D, col, hh, a.first_scale);
  else s.clear();

  const StateWeights<REVERSE> weights(lg, hh);
  // Scores are taken in tiles of 32 x 32, 0: (0, 0), 1: the one off the diagonal, 2: (1, 1).  Their weights, as a lane needs them, lie in LDS: on the diagonal, and off it.
  for (int i = threadIdx.x; i < 2 * 16 * 64; i += 2 * D) {
    const int l = i >> 2 & 63, j = 8 * (i >> 8 & 3) + 4 * (l >> 5) + (i & 3), far = (REVERSE ? j - (l & 31) : (l & 31) - j) + 32 * (i >> 10);
    near[i] = far >= 0 ? power(lg, far) : 0.f;
  }
  const int off = wave == 1 ? 1024 : 0;  // (with two waves the first takes tiles 0 and 2)
  const int ti = REVERSE ? wave >> 1 : (wave + 1) >> 1, tj = REVERSE ? (wave + 1) >> 1 : wave >> 1;  // the wave's tile, if it has one

  wait_all_but<0>();  // (else the compiler has the loop wait for all loads wherever it uses the state)
  f32x16 o[2];
  for (int n = 0; n < blocks; ++n) {
    for (int g = 0; g < group; ++g) {
      const bool last = g == group - 1;
      __syncthreads();
      if (!REVERSE || g == 0) qt.store(qs);
      if (REVERSE || g == 0) {
        kt.store(ks);
        vt.store(vs);
      }
      __syncthreads();
      const Step x = now;
      if (!last || n + 1 < blocks) {
        now = step_of(last ? n + 1 : n, last ? 0 : g + 1);
        fetch(now);
      }
      // Scores, transposed (a lane: one row i, four columns j at a time), only tiles with j <= i (backwards j >= i).  Operands are read two stages ahead, here and below.
      constexpr int kSteps = D / 16, kAhead = 2;
      auto scores = [&](int off, int ti, int tj) {
        f32x16 c{};
        bf16x8 kf[kSteps], qf[kSteps];
        auto read = [&](int st) {
          kf[st] = row_operand<D>(ks, 32 * tj, st, lane);
          qf[st] = row_operand<D>(qs, 32 * ti, st, lane);
        };
#pragma unroll
        for (int st = 0; st < kAhead; ++st) read(st);
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
          if (st + kAhead < kSteps) read(st + kAhead);
          __builtin_amdgcn_sched_barrier(0);
          c = mfma32(kf[st], qf[st], c);
          __builtin_amdgcn_sched_barrier(0);
        }
        f32x4 w[4];
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) w[q4] = lds_load4f(near + off + q4 * 256 + lane * 4);
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *(__attribute__((address_space(3))) bf16x4*)(ps + (l32 * pitch(64) + 4 * hh) + (32 * ti * pitch(64) + 32 * tj + 8 * q4)) =
              pack4(c[4 * q4] * w[q4][0], c[4 * q4 + 1] * w[q4][1], c[4 * q4 + 2] * w[q4][2], c[4 * q4 + 3] * w[q4][3]);
      };
      if (wave < 3) scores(off, ti, tj);
      if (kWaves == 2 && wave == 0) scores(0, 1, 1);
      const bool from_state = !REVERSE || g == 0;
      if (from_state) {
        bf16x8 qf[kSteps][2];
        auto read = [&](int st) {
          qf[st][0] = row_operand<D>(qs, 0, st, lane);
          qf[st][1] = row_operand<D>(qs, 32, st, lane);
        };
        o[0] = o[1] = f32x16{};
#pragma unroll
        for (int st = 0; st < kAhead; ++st) read(st);
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
          if (st + kAhead < kSteps) read(st + kAhead);
          __builtin_amdgcn_sched_barrier(0);
          const bf16x8 sb = s.operand(st);
          o[0] = mfma32(sb, qf[st][0], o[0]);
          o[1] = mfma32(sb, qf[st][1], o[1]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (from_state) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int i = 32 * half + l32 - x.empty;
          const float by = power(lg, max(REVERSE ? x.rows - 1 - i : i + 1, 0));
#pragma unroll
          for (int e = 0; e < 16; ++e) o[half][e] *= by;
        }
      }
      __syncthreads();
      bf16x8 vop[4];
      {
        bf16x8 pf[4][2];
        auto read = [&](int st) {
          vop[st] = column_operand<D, false>(vs, 16 * st, 32 * wave, lane);
#pragma unroll
          for (int half = 0; half < 2; ++half)
            if (REVERSE ? st >= 2 * half : st < 2 * half + 2) pf[st][half] = row_operand<64>(ps, 32 * half, st, lane);
        };
        read(0);
#pragma unroll
        for (int st = 0; st < 4; ++st) {
          if (st < 3) read(st + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int half = 0; half < 2; ++half)
            if (REVERSE ? st >= 2 * half : st < 2 * half + 2) o[half] = mfma32(vop[st], pf[st][half], o[half]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (!REVERSE || last) {
        const Rows out(a.o + x.row0 * q_stride + (h * q_group + (REVERSE ? 0 : g)) * D, 2 * (int)q_stride, x.rows, 2 * D);
#pragma unroll
        for (int half = 0; half < 2; ++half) store_row(out, 32 * half + l32 - x.empty, 64 * wave, o[half], a.scale, hh);
      }
      if (REVERSE ? g == 0 : last) s.scale(power(lg, x.rows));
      if (REVERSE || last) {
#pragma unroll
        for (int st = 0; st < 4; ++st) s.template add<PARTS>(ks, 16 * st, vop[st], weights.lead[st], weights.base, lane);
      }
    }
  }
  const int to = REVERSE ? segs.in[p.seg] : segs.out[p.seg];
  if (a.last && to >= 0 && p.index == (REVERSE ? 0 : p.pieces - 1)) s.store(a.last + ((int64_t)to * a.heads + h) * D * D, col, hh, a.last_scale);
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
constexpr int kStepHeads = 4;  // query heads at a time

// A workgroup takes one row of the batch and one key/value head: a thread four columns of the state and every so many rows.  Bound by memory (the state, read and written).
template <int D>
__global__ __launch_bounds__(step_threads(D)) void step_kernel(const StepArgs a) {
  constexpr int kGroups = step_groups(D), kThreads = step_threads(D), kRows = D / kGroups;
  __shared__ float ks[D], qs[kStepHeads][D], sums[kStepHeads][kGroups][D];
  __shared__ int next_row;
  const int h = blockIdx.x % a.heads, first = blockIdx.x / a.heads, slot = a.slots[first];
  if (slot < 0 || slot >= a.num_states) return;
  const int group = threadIdx.x / (D / 4), col = threadIdx.x % (D / 4) * 4;
  const int64_t at = ((int64_t)slot * a.heads + h) * D * D;
  const float decay = power(log2_decay(a.log_decay, h), 1);
  const float* from = a.states_in + at;
  float* const to = a.states_out + at;
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
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)a.v[kv + col + e];
    for (int g0 = 0; g0 < a.group; g0 += kStepHeads) {
      const int heads = min(kStepHeads, a.group - g0);
      const int64_t q0 = (((int64_t)row * a.heads + h) * a.group + g0) * D;
      for (int i = threadIdx.x; i < heads * D; i += kThreads) qs[i / D][i % D] = (float)a.q[q0 + i];
      __syncthreads();
      float acc[kStepHeads][4] = {};
#pragma unroll 16
      for (int n = 0; n < kRows; ++n) {
        const int r = n * kGroups + group;
        f32x4 x = *reinterpret_cast<const f32x4*>((g0 == 0 ? from : to) + (int64_t)r * D + col);
        if (g0 == 0) {
          const float kr = ks[r];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = x[e] * decay + kr * v[e];
          *reinterpret_cast<f32x4*>(to + (int64_t)r * D + col) = x;
        }
#pragma unroll
        for (int g = 0; g < kStepHeads; ++g) {
          if (g < heads) {
            const float qr = qs[g][r];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[g][e] += qr * x[e];
          }
        }
      }
#pragma unroll
      for (int g = 0; g < kStepHeads; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[g][group][col + e] = acc[g][e];
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

// Rows of a piece: a walk's even share when two walks run on each compute unit (one at head_dim 256).
int piece_rows(const chunk_linear_desc* d) {
  int64_t rows = 0, longest = 0;
  for (int i = 0; i < d->num_segments; ++i) {
    rows += d->segments[i].len;
    longest = std::max<int64_t>(longest, d->segments[i].len);
  }
  const int64_t share = rows * d->num_kv_heads / (d->head_dim > 128 ? kCus : 2 * kCus);
  const int64_t blocks = std::max<int64_t>(1, (share + kBlock - 1) / kBlock);
  return (int)std::min<int64_t>(blocks, (longest + kBlock - 1) / kBlock) * kBlock;
}
int pieces_of(int len, int rows) { return (len - 1) / rows + 1; }
int64_t count_places(const chunk_linear_desc* d, int rows) {
  int64_t n = 0;
  for (int i = 0; i < d->num_segments; ++i)
    if (d->segments[i].len > rows) n += pieces_of(d->segments[i].len, rows);
  return n;
}
size_t states_bytes(const chunk_linear_desc* d, int64_t n) { return (size_t)n * d->num_kv_heads * d->head_dim * d->head_dim * sizeof(float); }

template <class F>
hipError_t by_dim(int d, F&& f) {
  using std::integral_constant;
  if (d == 64) return f(integral_constant<int, 64>{});
  if (d == 96) return f(integral_constant<int, 96>{});
  if (d == 128) return f(integral_constant<int, 128>{});
  return f(integral_constant<int, 256>{});
}

template <int D, bool REVERSE, int PARTS>
hipError_t launch_piece_states(const WalkArgs& a, const LinearSegs& segs, hipStream_t stream) {
  constexpr size_t smem = 2 * tile_bytes(D);
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(&piece_states_kernel<D, REVERSE, PARTS>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((piece_states_kernel<D, REVERSE, PARTS>), dim3((unsigned)(segs.num_pieces * a.heads)), dim3(2 * D), smem, stream, a, segs);
  hipLaunchKernelGGL((join_states_kernel<REVERSE>), dim3((D * D / 4 + 255) / 256, (unsigned)(segs.n * a.heads)), dim3(256), 0, stream, a, segs, D * D);
  return hipGetLastError();
}
template <int D, bool REVERSE, bool TRANSPOSED, int PARTS>
hipError_t launch_walk(const WalkArgs& a, const LinearSegs& segs, hipStream_t stream) {
  constexpr size_t smem = 3 * tile_bytes(D) + tile_bytes(kBlock) + 2 * 16 * 64 * sizeof(float);
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(&walk_kernel<D, REVERSE, TRANSPOSED, PARTS>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((walk_kernel<D, REVERSE, TRANSPOSED, PARTS>), dim3((unsigned)(segs.num_pieces * a.heads)), dim3(2 * D), smem, stream, a, segs);
  return hipGetLastError();
}

// Goes through the segments, as many at a time as travel with a launch.
template <class F>
hipError_t for_segments(const chunk_linear_desc* d, int rows, F&& f) {
  LinearSegs s;
  int64_t places = 0;
  for (int s0 = 0; s0 < d->num_segments; s0 += kLinearSegs) {
    s.n = std::min(kLinearSegs, d->num_segments - s0);
    s.piece_rows = rows;
    s.num_pieces = 0;
    bool cut = false;
    for (int i = 0; i < s.n; ++i) {
      const chunk_linear_seg& x = d->segments[s0 + i];
      s.start[i] = x.start;
      s.len[i] = x.len;
      s.in[i] = x.state_in;
      s.out[i] = x.state_out;
      s.piece0[i] = s.num_pieces;
      s.place0[i] = (int)places;
      const int pieces = pieces_of(x.len, rows);
      s.num_pieces += pieces;
      if (pieces > 1) places += pieces;
      cut |= pieces > 1;
    }
    const hipError_t e = f(s, cut);
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
  *fwd_bytes = states_bytes(d, count_places(d, piece_rows(d)));
  *bwd_bytes = 2 * *fwd_bytes;
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
  const int rows = piece_rows(d);
  const size_t need = states_bytes(d, count_places(d, rows));
  if (need > 0) {
    if (!workspace || ((uintptr_t)workspace & 255) != 0) return CHUNK_ATTN_INVALID_ARG;
    if (workspace_bytes < need) return CHUNK_ATTN_WORKSPACE_TOO_SMALL;
  }
  WalkArgs a{(const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (__bf16*)o, log_decay, states_in, states_out, (float*)workspace, d->num_kv_heads,
             d->num_q_heads / d->num_kv_heads, 1.f, 1.f, d->scale};
  const hipStream_t stream = (hipStream_t)hip_stream;
  const hipError_t e = for_segments(d, rows, [&](const LinearSegs& segs, bool cut) {
    return by_dim(d->head_dim, [&](auto dim) {
      constexpr int D = decltype(dim)::value;
      auto with_parts = [&](auto parts) {
        constexpr int kParts = decltype(parts)::value;
        const hipError_t e = cut ? launch_piece_states<D, false, kParts>(a, segs, stream) : hipSuccess;
        return e != hipSuccess ? e : launch_walk<D, false, false, kParts>(a, segs, stream);
      };
      return states_out ? with_parts(std::integral_constant<int, 3>{}) : with_parts(std::integral_constant<int, 2>{});
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
  const int rows = piece_rows(d);
  const size_t need = states_bytes(d, count_places(d, rows));
  if (need > 0) {
    if (!workspace || ((uintptr_t)workspace & 255) != 0) return CHUNK_ATTN_INVALID_ARG;
    if (workspace_bytes < 2 * need) return CHUNK_ATTN_WORKSPACE_TOO_SMALL;
  }
  const __bf16 *bq = (const __bf16*)q, *bk = (const __bf16*)k, *bv = (const __bf16*)v, *bo = (const __bf16*)d_o;
  float* const inner_s = (float*)workspace;
  float* const inner_r = need > 0 ? inner_s + need / sizeof(float) : nullptr;
  const int heads = d->num_kv_heads, group = d->num_q_heads / heads;
  const float inv = 1.f / d->scale;
  // The walks' states backwards are the gradients' over `scale`, which all results are multiplied with.
  const WalkArgs s_states{nullptr, bk, bv, nullptr, log_decay, states_in, nullptr, inner_s, heads, group, 1.f, 1.f, d->scale};
  const WalkArgs r_states{nullptr, bq, bo, nullptr, log_decay, d_states_out, nullptr, inner_r, heads, group, inv, d->scale, d->scale};
  WalkArgs to_q = s_states, to_k = r_states, to_v = r_states;
  to_q.q = bo; to_q.k = bv; to_q.v = bk; to_q.o = (__bf16*)dq;
  to_k.q = bv; to_k.k = bo; to_k.v = bq; to_k.o = (__bf16*)dk;
  to_v.q = bk; to_v.k = bq; to_v.v = bo; to_v.o = (__bf16*)dv;
  to_v.last = d_states_in;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const hipError_t e = for_segments(d, rows, [&](const LinearSegs& segs, bool cut) {
    return by_dim(d->head_dim, [&](auto dim) {
      constexpr int D = decltype(dim)::value;
      hipError_t e = hipSuccess;
      if (cut) {
        if ((e = launch_piece_states<D, false, 2>(s_states, segs, stream)) != hipSuccess) return e;
        if ((e = d_states_in ? launch_piece_states<D, true, 3>(r_states, segs, stream) : launch_piece_states<D, true, 2>(r_states, segs, stream)) != hipSuccess) return e;
      }
      if ((e = launch_walk<D, false, true, 2>(to_q, segs, stream)) != hipSuccess) return e;
      if ((e = launch_walk<D, true, true, 2>(to_k, segs, stream)) != hipSuccess) return e;
      return d_states_in ? launch_walk<D, true, false, 3>(to_v, segs, stream) : launch_walk<D, true, false, 2>(to_v, segs, stream);
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
      (((uintptr_t)log_decay | (uintptr_t)slots) & 3) != 0 || (int64_t)batch * num_kv_heads > INT32_MAX)
    return CHUNK_ATTN_INVALID_ARG;
  const StepArgs a{(const __bf16*)q, (const __bf16*)k, (const __bf16*)v, log_decay, states_in, states_out, slots, (__bf16*)o, batch, num_states, num_kv_heads,
                   num_q_heads / num_kv_heads, scale};
  const hipError_t e = by_dim(head_dim, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    hipLaunchKernelGGL(step_kernel<D>, dim3((unsigned)(batch * num_kv_heads)), dim3(step_threads(D)), 0, (hipStream_t)hip_stream, a);
    return hipGetLastError();
  });
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, "linear attention step");
}
