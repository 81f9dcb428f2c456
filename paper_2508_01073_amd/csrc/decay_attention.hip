// Linear attention with a decay for each head on gfx950.
//
// Forward and all three gradients are one scan with different operands. With
// rows a_t, b_t of `di` values and c_t of `dout` values, over the tokens in
// ascending order (or descending for a reverse scan, u counting the tokens
// already passed),
//
//   out_u = oscale * (sum_{w <= u} gamma^{u-w} (a_u . b_w) c_w * sscale + gamma^{u+e} S^T a_u)
//   S_end = sscale * sum_u gamma^{L-e-u} b_u c_u^T + gamma^L S
//
//            a   b   c   S (di x dout)       e  oscale sscale
//   out      q   k   v   state               1  scale  1
//   dq       do  v   k   state transposed    1  scale  1
//   dk       v   do  q   dstate_out transp.  0  1      scale      reverse
//   dv       k   q   do  dstate_out          0  1      scale      reverse
//
// e: a forward scan decays the state before it adds a token, a reverse scan
// adds the token's term to the gradient of S_t and decays it on the way to
// S_{t-1}. The final S of `out` is state_out and that of `dv` is dstate.

#include "model.hpp"

namespace rdf2v {
namespace {

struct ScanOperand {
  const void *data;
  int64_t row, token, head;  // strides in elements
  int32_t share;             // query heads that read one of its heads
};

struct ScanArgs {
  ScanOperand a, b, c;
  const float *log_decay;
  const int32_t *len;
  const float *s0;  // S, or null for zeros
  float *s1;        // where S_end goes, or null
  void *out;        // [rows][length][heads][dout]
  int32_t *status;
  int64_t rows, length;
  int32_t heads, di, dout;
  float oscale, sscale;
  bool transposed;  // s0 and seg_state are stored [dout][di]
  bool reverse;
  // set by launch_scan
  float pscale;              // oscale * sscale
  int64_t segments, segment; // segments of a row, and their tokens (whole chunks)
  // [rows][heads][segments][dk][dv] states that the segments begin with (a state scan: their own), or null
  float *seg_state;
  bool wide, wide_out;       // 16-byte reads (short rows: of four values), stores of four values
  bool whole_out;            // out is bfloat16 in rows of whole 16 bytes
  bool out_f32;              // out is float32 whatever the element type: to be summed over heads
};

// Scans that run side by side.
struct ScanRoles {
  ScanArgs role[3];
  int32_t count;
};

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float head_log_decay(const float *log_decay, int h, int32_t *status, bool report) {
  const float g = log_decay[h];
  const bool ok = g <= 0.0f;
  if (!ok && report && status != nullptr) atomicOr(status, RDF2V_STATUS_BAD_VALUE);
  return ok ? fmaxf(g, -1e30f) : 0.0f;  // finite, so that 0 tokens of it are 0
}

__device__ __forceinline__ int64_t row_length(const int32_t *len, int64_t row, int64_t length, int32_t *status,
                                              bool report) {
  if (len == nullptr) return length;
  const int64_t n = len[row];
  if ((n < 0 || n > length) && report && status != nullptr) atomicOr(status, RDF2V_STATUS_BAD_LENGTH);
  return n < 0 ? 0 : n > length ? length : n;
}

template <class T>
__device__ __forceinline__ const T *operand_row(const ScanOperand &x, int64_t row, int h) {
  return static_cast<const T *>(x.data) + row * x.row + (h / x.share) * x.head;
}

constexpr int kChunk = 64;      // tokens of a chunk
constexpr int kThreads = 256;   // of the kernels below that are not scans
constexpr int kTile = 16;       // rows and columns of a matrix instruction

// Eight values of a row or column are what one lane feeds to a matrix
// instruction. Lane l serves row (of the first factor) or column (of the second)
// l % 16, and with g = l / 16 its values are any eight of a block of 32
// contraction indices, the same for both factors. A result holds rows 4 g + r of
// column l % 16: two results are an operand of the next product as they stand,
// if its other factor is read in their order.
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

template <class T>
struct Vec;
template <>
struct Vec<bf16> {
  typedef bf16x4 four;
  typedef bf16x8 eight;
  typedef bf16x8 load;  // 16 bytes
  // Operands of the matrix products that are computed values: the weights of a chunk's pairs, and a float32
  // state that tokens are multiplied with, are fed as two bfloat16 pieces, 16 bits, each off by at most 2^-16
  // of itself. The outputs' error is then that of their own rounding, 1.66e-3 in the 2-norm for random inputs
  // (one piece for the states: 2.05e-3, and far more where a state's large values cancel). Of four rows of
  // 4,096 x 16 heads of 128, forward and backward, the states take 438, 458 and 485 us with one, two and three
  // pieces; three for weights and states 576. What is added to a state keeps 24 bits, as three pieces, where
  // the state is an output in float32, and 16 where only bfloat16 outputs are made of it.
  static constexpr int kPieces = 2, kOperand = 2, kStatePieces = 3;
};
template <>
struct Vec<float> {
  typedef f32x4 four;
  typedef f32x8 eight;
  typedef f32x4 load;
  static constexpr int kPieces = 1, kOperand = 1, kStatePieces = 1;
};

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x8 a, f32x8 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// The same where the last four values of each lane are zeros.
__device__ __forceinline__ f32x4 mma_low(bf16x8 a, bf16x8 b, f32x4 c) { return mma(a, b, c); }
__device__ __forceinline__ f32x4 mma_low(f32x8 a, f32x8 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ bf16x8 join(bf16x4 a, bf16x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
__device__ __forceinline__ f32x8 join(f32x4 a, f32x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// The next piece of x: x rounded to the element type, and what is left in x.
template <class F>
__device__ __forceinline__ auto take_piece(F &x, bf16) {
  constexpr int kN = sizeof(F) / 4;
  typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef unsigned words __attribute__((ext_vector_type(kN / 2)));
  typedef bf16 piece __attribute__((ext_vector_type(kN)));
  words p;
#pragma unroll
  for (int j = 0; j < kN; j += 2) {
    p[j / 2] = __builtin_bit_cast(unsigned, bf16x2{bf16(x[j]), bf16(x[j + 1])});
    x[j] -= __uint_as_float(p[j / 2] << 16);
    x[j + 1] -= __uint_as_float(p[j / 2] & 0xffff0000u);
  }
  return __builtin_bit_cast(piece, p);
}
template <class F>
__device__ __forceinline__ F take_piece(F &x, float) {
  return x;
}

// Values that are no numbers have to stay where the sum over w <= u has them: a weight of 0 does not take them
// out of a matrix product. So columns with any are products without them, and NaN from the first of them on.
template <class E>
__device__ __forceinline__ bool any_odd(const E &x) {  // an exponent of ones, to which a one carries
  constexpr bool kHalf = sizeof(x[0]) == 2;
  constexpr unsigned kExponent = kHalf ? 0x7f807f80u : 0x7f800000u, kOne = kHalf ? 0x00800080u : 0x00800000u,
                     kCarry = kHalf ? 0x80008000u : 0x80000000u;
  typedef unsigned words __attribute__((ext_vector_type(sizeof(E) / 4)));
  const words w = __builtin_bit_cast(words, x);
  unsigned any = 0;
#pragma unroll
  for (unsigned i = 0; i < sizeof(E) / 4; ++i) any |= (w[i] & kExponent) + kOne;
  return (any & kCarry) != 0;
}
// Takes them out of x, whose value j is that of place(j); returns the least place that had one, or `first`.
template <class E, class Place>
__device__ __forceinline__ int take_odd(E &x, int first, Place place) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (__builtin_isfinite(to_f32(x[j]))) continue;
    first = min(first, place(j));
    x[j] = 0.0f;
  }
  return first;
}
// The least place of column l % 16 over the lane groups.
__device__ __forceinline__ int least_odd(int first) {
  first = min(first, __shfl_xor(first, 16, kWave));
  return min(first, __shfl_xor(first, 32, kWave));
}
// Result o holds columns 4 g + r of token u; `first` is that of column l % 16. NaN where u is at or behind its
// column's first.
__device__ __forceinline__ void spread_odd(f32x4 &o, int first, int u, int g) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (u >= __shfl(first, 4 * g + r, kWave)) o[r] = __builtin_nanf("");
}

// A tile of rows of W values in LDS. In bfloat16 the groups of four values of a
// row are permuted by the row: the 16-byte reads of 16 rows at one place, and
// the transposing reads of four neighbouring groups of eight rows, then meet
// every bank once. Pairs of groups stay together for the 16-byte accesses.
// Float32 rows are padded by 16 bytes.
template <class T, int W>
struct Tile;
template <int W>
struct Tile<bf16, W> {
  static constexpr int kSize = kChunk * W;
  static __device__ __forceinline__ int swap(int row) {
    const int low = W == 128 ? row % 4 * 4 : W == 64 ? row / 2 % 2 * 4 : 0;
    return low | row / 8 % 2 * (W / 8) | row / 4 % 2 * 2;
  }
  static __device__ __forceinline__ int at(int row, int group) { return row * W + (group ^ swap(row)) * 4; }
};
template <int W>
struct Tile<float, W> {
  static constexpr int kSize = kChunk * (W + 4);
  static __device__ __forceinline__ int at(int row, int group) { return row * (W + 4) + group * 4; }
};

// Operands of the chunks' products: lane l holds values 32 kk + 8 g + j of row
// (or column) l % 16.
//
// Values of row `row`, indices of block kk.
template <int W>
__device__ __forceinline__ bf16x8 row_values(const bf16 *tile, int row, int kk, int g) {
  return *reinterpret_cast<const bf16x8 *>(tile + Tile<bf16, W>::at(row, kk * 8 + 2 * g));
}
template <int W>
__device__ __forceinline__ f32x8 row_values(const float *tile, int row, int kk, int g) {
  const float *p = tile + Tile<float, W>::at(row, kk * 8 + 2 * g);
  return join(*reinterpret_cast<const f32x4 *>(p), *reinterpret_cast<const f32x4 *>(p + 4));
}
// Values of 16 columns, rows of block kk: columns group0 * 4 + step * 4 * (l16 / 4)
// + l16 % 4. In bfloat16 the transposing LDS read gives lane l of 16 the column l
// of the four groups of four rows that the lanes 4 row + (0 .. 3) address.
template <int W>
__device__ __forceinline__ bf16x8 column_values(const bf16 *tile, int group0, int step, int kk, int lane) {
  typedef __attribute__((address_space(3))) i16x4 lds4;
  const int row = kk * 32 + 8 * (lane / 16) + lane % 16 / 4, group = group0 + step * (lane % 4);
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(tile + Tile<bf16, W>::at(row, group)));
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(tile + Tile<bf16, W>::at(row + 4, group)));
  return join(__builtin_bit_cast(bf16x4, lo), __builtin_bit_cast(bf16x4, hi));
}
template <int W>
__device__ __forceinline__ f32x8 column_values(const float *tile, int group0, int step, int kk, int lane) {
  const int group = group0 + step * (lane % 16 / 4);
  const float *p = tile + Tile<float, W>::at(kk * 32 + 8 * (lane / 16), group) + lane % 4;
  f32x8 x;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = p[j * (W + 4)];
  return x;
}
// Row r of tile i of a state, in lane group g: such that the accumulators of
// tiles 2 kk and 2 kk + 1 are the operand of block kk.
__device__ __forceinline__ int state_row(int i, int g, int r) { return i / 2 * 32 + 8 * g + i % 2 * 4 + r; }

// A chunk's rows of one operand on their way from memory to LDS: 64 rows of W
// values, zeros beyond the operand's size and beyond the chunk's `n` tokens.
// `low` points to the chunk's token of the lowest number, `token` is the
// distance to the next one (64 of them stay below 2^31 bytes).
template <class T, int W, int THREADS>
struct Loader {
  typedef typename Vec<T>::load load;
  static constexpr int kPer = 16 / sizeof(T), kCols = W / kPer;
  // Whole bfloat16 rows go to LDS past the registers, 1 KB a wave and instruction: lane l's 16 bytes land
  // at 16 l, so each lane reads what the permuted tile has there. Float32 rows, which are padded, wait in
  // registers.
  static constexpr bool kDirect = sizeof(T) == 2;
  static constexpr int kRows = THREADS / kCols < kChunk ? THREADS / kCols : kChunk;
  static constexpr int kLoads = kChunk / kRows;
  load r[kDirect ? 1 : kLoads];

  __device__ __forceinline__ void fetch(unsigned thread, T *tile, const T *low, int token, bool reverse) {
    if constexpr (kDirect) {
      typedef __attribute__((address_space(3))) void lds;
      typedef const __attribute__((address_space(1))) void global;
      constexpr int kAtOnce = 512 / W, kSteps = kChunk / kAtOnce;  // rows of an instruction, instructions
      const int wave = __builtin_amdgcn_readfirstlane(thread / kWave), lane = thread % kWave;
#pragma unroll
      for (int i = 0; i < (kSteps + THREADS / kWave - 1) / (THREADS / kWave); ++i) {
        const int step = i * (THREADS / kWave) + wave;
        if (step >= kSteps) break;
        const int row = step * kAtOnce + lane / kCols;
        const int col = (lane % kCols ^ Tile<T, W>::swap(row) / 2) * kPer;
        const T *from = low + unsigned(__mul24(reverse ? kChunk - 1 - row : row, token) + col);
        __builtin_amdgcn_global_load_lds((global *)from, (lds *)(tile + step * 512), 16, 0, 0);
      }
    } else {
      const int u = thread / kCols, col = thread % kCols * kPer;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = min(u + i * kRows, kChunk - 1);
        r[i] = *reinterpret_cast<const load *>(low + unsigned(__mul24(reverse ? kChunk - 1 - row : row, token) + col));
      }
    }
  }
  __device__ __forceinline__ void store(unsigned thread, T *tile) const {
    if constexpr (!kDirect) {
      const int u = thread / kCols, col = thread % kCols * kPer;
      if (THREADS / kCols > kChunk && u >= kRows) return;
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        *reinterpret_cast<load *>(tile + Tile<T, W>::at(u + i * kRows, col / 4)) = r[i];
    }
  }
  // A chunk that is not whole, or narrower than the tile.
  static __device__ __forceinline__ void copy_part(unsigned thread, T *tile, const T *low, int token, bool reverse,
                                                   int n, int size) {
    for (int at = thread; at < kChunk * kCols; at += THREADS) {
      const int row = at / kCols, col = at % kCols * kPer;
      load x{};
      if (row < n && col < size)
        x = *reinterpret_cast<const load *>(low + unsigned(__mul24(reverse ? n - 1 - row : row, token) + col));
      *reinterpret_cast<load *>(tile + Tile<T, W>::at(row, col / 4)) = x;
    }
  }
  // Value by value, for rows that 16-byte reads do not fit.
  static __device__ __forceinline__ void copy(unsigned thread, T *tile, const T *chunk, int64_t token, int n,
                                              int size) {
    for (int at = thread; at < kChunk * W; at += THREADS) {
      const int u = at / W, col = at % W;
      tile[Tile<T, W>::at(u, col / 4) + col % 4] = u < n && col < size ? chunk[u * token + col] : T(0.0f);
    }
  }
};

// Role and item of a workgroup: the roles of an item, which read the same
// operands, run on one XCD (workgroups are dealt to the 8 in turn) and soon
// after one another.
constexpr int kXcds = 8;
__device__ __forceinline__ int role_of(int64_t block, int count, int64_t &item) {
  const int per = kXcds * count;
  item = block / per * kXcds + block % kXcds;
  return int(block % per) / kXcds;
}

// Four values of an output row, of which `col` is the first column.
template <class T>
__device__ __forceinline__ void store_four(const ScanArgs &p, int64_t at, int col, f32x4 x) {
  typedef typename Vec<T>::four four;
  if (p.out_f32) {
    float *to = static_cast<float *>(p.out) + at;
    if (p.wide_out) {
      if (col < p.dout) *reinterpret_cast<f32x4 *>(to) = x;
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (col + r < p.dout) to[r] = x[r];
    }
  } else {
    T *to = static_cast<T *>(p.out) + at;
    if (p.wide_out) {
      four y;
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = from_f32<T>(x[r]);
      if (col < p.dout) *reinterpret_cast<four *>(to) = y;
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (col + r < p.dout) to[r] = from_f32<T>(x[r]);
    }
  }
}

// One workgroup scans the chunks of one segment of a row for one head and NB
// columns of c and S.
//
// A chunk's part of the sum is the matrix product of the weights
// P[t][s] = gamma^{t-s} (a_t . b_s), s <= t, with c; the earlier chunks' part is
// gamma^{t+e} S^T a_t; then S becomes gamma^n S + sum_s gamma^{n-e-s} b_s c_s^T.
// Every wave owns some columns of S, which stay in its registers as the
// accumulators of the update and, in the order above, are the operands of the
// earlier chunks' part; the weights are computed once, a wave a tile of 16
// tokens, and shared through LDS. The next chunk is fetched while this one is
// computed.
//
// OUT: outputs are wanted; otherwise only S of the segment (from zeros).
//
// One row of 20,011 tokens, 8 heads of 128 in bfloat16, in 63 segments: 55 us
// with outputs (197 MB beyond L2, 3.6 TB/s), 30 us for the states alone (116 MB,
// 3.8) and 16 us to join them (67 MB, 4.2). Four rows of 4,096, 16 heads: 83 us
// for the outputs and 240 for the three gradients. Vector instructions issue in
// 58 to 63 % of the busy cycles of all of these scans, matrix instructions are
// busy for 22 to 26 %, and waves wait for 43 to 48 % of their time: the issue,
// and the waits at a chunk's barriers, bound them.
//
// A tile of 16 columns to a wave keeps all of that in 128 registers up to heads
// of 128, so that 16 waves share a CU; two tiles to a wave spilled, and the
// waits for the spills made it more than twice as slow.
constexpr int scan_waves(int nb) { return nb > 64 ? 8 : 4; }

template <class T, int DI, int NB, bool OUT>
__global__ __launch_bounds__(scan_waves(NB) * kWave, sizeof(T) == 2 ? 4 : 2) void scan_kernel(ScanRoles roles,
                                                                                             int64_t items,
                                                                                             int64_t first) {
  constexpr int kWaves = scan_waves(NB), kThreads = kWaves * kWave;
  constexpr int kWavesN = NB / kTile;                      // waves side by side over the columns
  constexpr int kWavesT = kWaves / kWavesN;                // and over the chunk's tokens
  constexpr int kTilesN = 1, kTilesT = 4 / kWavesT, kTilesI = DI / kTile, kK = DI / 32;
  constexpr int kPieces = Vec<T>::kPieces, kOperand = Vec<T>::kOperand, kStatePieces = Vec<T>::kStatePieces;
  // A scan for the state alone has LDS for two chunks: the next one is on its way while this one is used, and
  // a chunk has one barrier.
  constexpr int kBuffers = !OUT && Loader<T, DI, kThreads>::kDirect ? 2 : 1;
  __shared__ __attribute__((aligned(16))) T as[OUT ? Tile<T, DI>::kSize : 1], b_tiles[kBuffers][Tile<T, DI>::kSize],
      c_tiles[kBuffers][Tile<T, NB>::kSize];
  __shared__ __attribute__((aligned(16))) T ps[OUT ? kPieces : 1][OUT ? Tile<T, kChunk>::kSize : 1];
  // A chunk's outputs, put together to whole rows: a wave's 32 bytes of a row each would make four times the
  // requests. They are stored when the next chunk is in LDS, behind the same barrier.
  constexpr bool kStage = OUT && sizeof(T) == 2;
  __shared__ __attribute__((aligned(16))) T os[kStage ? Tile<T, NB>::kSize : 1];
  typedef typename Vec<T>::four four;
  typedef typename Vec<T>::eight eight;

  int64_t item;
  const ScanArgs &p = roles.role[role_of(first + blockIdx.x, roles.count, item)];
  if (item >= items) return;
  const int64_t seg = item % p.segments, rh = item / p.segments, row = rh / p.heads;
  const int h = int(rh % p.heads);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = lane_id(), l16 = lane % 16, g = lane / 16;
  const int wn = wave % kWavesN, wt = wave / kWavesN;
  const int nw = wn * kTilesN * kTile;                     // first column of the wave
  const bool report = seg == 0 && threadIdx.x == 0;
  const float head_log2_gamma =
      head_log_decay(p.log_decay, h, p.status, report && row == 0) * kLog2e;
  // Decays over 1 .. 7 tokens and over a tile of them, the same in all lanes: of neighbouring tokens' decays
  // one is computed and the others are its products (two rows of 8,192 x 16 heads of 64 with gradients 6 %
  // faster, 12 of 2,048 x 16 of 128 2 %).
  float by_tokens[7], by_tile;
  auto uniform = [](float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); };
#pragma unroll
  for (int j = 0; j < 7; ++j) by_tokens[j] = uniform(__builtin_amdgcn_exp2f(float(j + 1) * head_log2_gamma));
  by_tile = uniform(__builtin_amdgcn_exp2f(float(kTile) * head_log2_gamma));
  const int64_t len = row_length(p.len, row, p.length, p.status, report && h == 0);
  const int e = p.reverse ? 0 : 1;
  const T *a = operand_row<T>(p.a, row, h), *b = operand_row<T>(p.b, row, h), *c = operand_row<T>(p.c, row, h);
  const int64_t u_begin = seg * p.segment, u_end = min(p.length, u_begin + p.segment);
  const int64_t u_valid = min(u_end, len);
  const int dt = p.reverse ? -1 : 1;
  // a state that is written needs all three pieces of its addends; one that only outputs are made of, two
  const bool exact_state = !OUT || (p.s1 != nullptr && p.seg_state == nullptr);

  f32x4 s[kTilesN][kTilesI];
  const int64_t size = int64_t(p.di) * p.dout;
  {
    const float *s0 = !OUT                     ? nullptr
                      : p.seg_state != nullptr ? p.seg_state + (rh * p.segments + seg) * size
                      : p.s0 != nullptr        ? p.s0 + rh * size
                                               : nullptr;
    const int per_k = p.transposed ? 1 : p.dout, per_col = p.transposed ? p.di : 1;
#pragma unroll
    for (int n = 0; n < kTilesN; ++n)
#pragma unroll
      for (int i = 0; i < kTilesI; ++i) {
        s[n][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (s0 == nullptr) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int col = nw + n * kTile + l16, k = state_row(i, g, r);
          if (k < p.di && col < p.dout) s[n][i][r] = s0[unsigned(k * per_k + col * per_col)];
        }
      }
  }

  Loader<T, DI, kThreads> la, lb;
  Loader<T, NB, kThreads> lc;
  // Chunks that fill the tiles are fetched ahead.
  const bool fills = p.wide && p.di == DI && p.dout == NB;
  auto whole = [&](int64_t u0) { return fills && u0 + kChunk <= u_valid; };
  int buffer = 0;
  auto fetch = [&](unsigned thread, int64_t u0, int to) {
    const int64_t low = p.reverse ? len - u0 - kChunk : u0;
    if (OUT) la.fetch(thread, as, a + low * p.a.token, int(p.a.token), p.reverse);
    lb.fetch(thread, b_tiles[to], b + low * p.b.token, int(p.b.token), p.reverse);
    lc.fetch(thread, c_tiles[to], c + low * p.c.token, int(p.c.token), p.reverse);
  };
  const bool stage = kStage && p.whole_out;
  auto flush = [&](unsigned thread, int64_t u0) {  // the staged outputs of the chunk at u0
    constexpr int kCols = NB / 8;
    typedef bf16x8 vec;
    const int n = int(min(int64_t(kChunk), u_valid - u0));
    const int64_t t0 = p.reverse ? len - 1 - u0 : u0;
    T *out = static_cast<T *>(p.out) + ((row * p.length + t0) * p.heads + h) * int64_t(p.dout);
#pragma unroll
    for (int i = 0; i < kChunk * kCols / kThreads; ++i) {
      const int at = i * kThreads + thread, u = at / kCols, col = at % kCols * 8;
      if (u < n && col < p.dout)
        *reinterpret_cast<vec *>(out + dt * u * (p.heads * p.dout) + col) =
            *reinterpret_cast<const vec *>(os + Tile<T, NB>::at(u, col / 4));
    }
  };
  if (whole(u_begin)) fetch(threadIdx.x, u_begin, 0);
  __builtin_amdgcn_s_waitcnt(0x0f70);  // all loads: the loop then waits for its own chunks only

  for (int64_t u0 = u_begin; u0 < u_valid; u0 += kChunk) {
    // The decays and places of a chunk's tokens are the same in every chunk; kept for all of them they
    // would take the registers that the products need, so they are computed again.
    float log2_gamma = head_log2_gamma;
    unsigned thread = threadIdx.x;
    asm volatile("" : "+v"(log2_gamma), "+v"(thread));
    const int lane = thread % kWave, l16 = lane % 16, g = lane / 16;
    const int n_valid = int(min(int64_t(kChunk), u_valid - u0));
    const int64_t t0 = p.reverse ? len - 1 - u0 : u0;
    const bool last = u0 + kChunk >= u_valid;
    T *bs = b_tiles[buffer], *cs = c_tiles[buffer];
    buffer = (buffer + 1) % kBuffers;
    if (whole(u0)) {
      if (OUT) la.store(thread, as);
      lb.store(thread, bs);
      lc.store(thread, cs);
      if (la.kDirect) __builtin_amdgcn_s_waitcnt(0x0f70);  // this wave's part of the chunk is in LDS
    } else if (p.wide) {
      const int64_t low = p.reverse ? t0 - (n_valid - 1) : t0;
      if (OUT) la.copy_part(thread, as, a + low * p.a.token, int(p.a.token), p.reverse, n_valid, p.di);
      lb.copy_part(thread, bs, b + low * p.b.token, int(p.b.token), p.reverse, n_valid, p.di);
      lc.copy_part(thread, cs, c + low * p.c.token, int(p.c.token), p.reverse, n_valid, p.dout);
    } else {
      if (OUT) la.copy(thread, as, a + t0 * p.a.token, dt * p.a.token, n_valid, p.di);
      lb.copy(thread, bs, b + t0 * p.b.token, dt * p.b.token, n_valid, p.di);
      lc.copy(thread, cs, c + t0 * p.c.token, dt * p.c.token, n_valid, p.dout);
    }
    __syncthreads();
    if constexpr (kStage)
      if (stage && u0 > u_begin) flush(thread, u0 - kChunk);
    if (!OUT && whole(u0 + kChunk)) fetch(thread, u0 + kChunk, buffer);
    if (OUT) {
      // the weights of tokens 16 w .. 16 w + 15, and of half of the tokens before them where two waves share
      const int w4 = wave % 4, t = w4 * kTile + l16;
      eight av[kK];
#pragma unroll
      for (int kk = 0; kk < kK; ++kk) av[kk] = row_values<DI>(as, t, kk, g);
#pragma unroll
      for (int j = 0; j < 16 / kWaves; ++j) {
        const int i = wave / 4 * (16 / kWaves) + j;
        // blocks of 32 that the products below read
        if (kWavesT == 1 && i > (w4 | 1)) continue;
        f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
        if (i <= w4) {
#pragma unroll
          for (int kk = 0; kk < kK; ++kk) w = mma(row_values<DI>(bs, i * kTile + l16, kk, g), av[kk], w);
          const int d3 = t - (i * kTile + 4 * g + 3);  // of r = 3; positive off the diagonal
          if (i < w4) {
            const float decay = p.pscale * __builtin_amdgcn_exp2f(float(d3) * log2_gamma);
            w *= f32x4{decay * by_tokens[2], decay * by_tokens[1], decay * by_tokens[0], decay};
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int d = d3 + 3 - r;
              const float y = w[r] * (p.pscale * __builtin_amdgcn_exp2f(float(d) * log2_gamma));
              w[r] = d >= 0 ? y : 0.0f;
            }
          }
        }
#pragma unroll
        for (int x = 0; x < kPieces; ++x)
          *reinterpret_cast<four *>(ps[x] + Tile<T, kChunk>::at(t, i * 4 + g)) = take_piece(w, T());
      }
    }

    eight cv[kTilesN][2];
#pragma unroll
    for (int n = 0; n < kTilesN; ++n)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) cv[n][kk] = column_values<NB>(cs, (nw + n * kTile) / 4, 1, kk, lane);

    f32x4 o[kTilesT][kTilesN];
    if (OUT) {
#pragma unroll
      for (int t = 0; t < kTilesT; ++t)
#pragma unroll
        for (int n = 0; n < kTilesN; ++n) o[t][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kk = 0; kk < kK; ++kk) {
        eight sv[kTilesN][kOperand];
#pragma unroll
        for (int n = 0; n < kTilesN; ++n) {
          f32x8 x = join(s[n][2 * kk], s[n][2 * kk + 1]);
#pragma unroll
          for (int i = 0; i < kOperand; ++i) sv[n][i] = take_piece(x, T());
        }
        eight av[kTilesT];
#pragma unroll
        for (int t = 0; t < kTilesT; ++t) av[t] = row_values<DI>(as, (wt * kTilesT + t) * kTile + l16, kk, g);
        // one piece for all tiles, then the next: no product waits for the one before it
#pragma unroll
        for (int i = 0; i < kOperand; ++i)
#pragma unroll
          for (int t = 0; t < kTilesT; ++t)
#pragma unroll
            for (int n = 0; n < kTilesN; ++n) o[t][n] = mma(sv[n][i], av[t], o[t][n]);
      }
      float d = p.oscale * __builtin_amdgcn_exp2f(float(wt * kTilesT * kTile + l16 + e) * log2_gamma);
#pragma unroll
      for (int t = 0; t < kTilesT; ++t) {
#pragma unroll
        for (int n = 0; n < kTilesN; ++n) o[t][n] *= d;
        d *= by_tile;
      }
    }

    if (!last || exact_state) {
      const float d = __builtin_amdgcn_exp2f(float(n_valid) * log2_gamma);
      float near[8];
      near[7] = __builtin_amdgcn_exp2f(float(24 - 8 * g) * log2_gamma);
#pragma unroll
      for (int j = 0; j < 7; ++j) near[j] = near[7] * by_tokens[6 - j];
#pragma unroll
      for (int n = 0; n < kTilesN; ++n)
#pragma unroll
        for (int i = 0; i < kTilesI; ++i) s[n][i] *= d;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        if (kk * 32 >= n_valid) continue;
        eight wv[kTilesN][kStatePieces];
        f32x8 x[kTilesN];
        float w[8];  // gamma^{n-e-u}, u = 32 kk + 8 g + j; tokens u >= n have no c
        if (n_valid == kChunk) {
          const float far = p.sscale * __builtin_amdgcn_exp2f(float(33 - e - 32 * kk) * log2_gamma);
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = near[j] * far;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            w[j] = p.sscale * __builtin_amdgcn_exp2f(float(max(n_valid - e - 32 * kk - 8 * g - j, 0)) * log2_gamma);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int n = 0; n < kTilesN; ++n) x[n][j] = to_f32(cv[n][kk][j]) * w[j];
#pragma unroll
        for (int n = 0; n < kTilesN; ++n)
#pragma unroll
          for (int i = 0; i < kStatePieces; ++i)
            if (i < 2 || exact_state) wv[n][i] = take_piece(x[n], T());
        constexpr int kGroup = kTilesI < 4 ? kTilesI : 4;
#pragma unroll
        for (int i0 = 0; i0 < kTilesI; i0 += kGroup) {
          eight bv[kGroup];
#pragma unroll
          for (int i = 0; i < kGroup; ++i) bv[i] = column_values<DI>(bs, (i0 + i) / 2 * 8 + (i0 + i) % 2, 2, kk, lane);
#pragma unroll
          for (int x = 0; x < kStatePieces; ++x) {
            if (x >= 2 && !exact_state) continue;
#pragma unroll
            for (int i = 0; i < kGroup; ++i)
#pragma unroll
              for (int n = 0; n < kTilesN; ++n) s[n][i0 + i] = mma(bv[i], wv[n][x], s[n][i0 + i]);
          }
        }
      }
    }
    if (kBuffers == 2) continue;
    __syncthreads();  // the weights are there, and a, b and c are read
    if (OUT && whole(u0 + kChunk)) fetch(thread, u0 + kChunk, 0);

    if (OUT) {
      // a column of c that has NaN or infinities has made its column of S one, where S was computed
      bool odd = !last || exact_state ? !__builtin_isfinite(s[0][0][0]) : any_odd(cv[0][0]) || any_odd(cv[0][1]);
      if (__builtin_expect(__ballot(odd) != 0, 0)) {
#pragma unroll
        for (int n = 0; n < kTilesN; ++n) {
          int first = kChunk;
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) first = take_odd(cv[n][kk], first, [&](int j) { return 32 * kk + 8 * g + j; });
          first = least_odd(first);
#pragma unroll
          for (int t = 0; t < kTilesT; ++t) spread_odd(o[t][n], first, (wt * kTilesT + t) * kTile + l16, g);
        }
      }
      const int64_t out_at = ((row * p.length + t0) * p.heads + h) * int64_t(p.dout);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
          for (int t = 0; t < kTilesT; ++t) {
            const int tt = wt * kTilesT + t;
            if (kWavesT == 1 && kk * 2 > tt) continue;  // with more waves over the tokens: zeros
            const eight pv = row_values<kChunk>(ps[i], tt * kTile + l16, kk, g);
#pragma unroll
            for (int n = 0; n < kTilesN; ++n) o[t][n] = mma(cv[n][kk], pv, o[t][n]);
          }
#pragma unroll
      for (int t = 0; t < kTilesT; ++t) {
        const int u = (wt * kTilesT + t) * kTile + l16;
        if (kStage && stage) {
#pragma unroll
          for (int n = 0; n < kTilesN; ++n)
            *reinterpret_cast<four *>(os + Tile<T, NB>::at(u, (nw + n * kTile) / 4 + g)) =
                four{from_f32<T>(o[t][n][0]), from_f32<T>(o[t][n][1]), from_f32<T>(o[t][n][2]),
                     from_f32<T>(o[t][n][3])};
          continue;
        }
        if (u >= n_valid) continue;
        const int64_t at = out_at + dt * u * (p.heads * p.dout);  // 64 tokens of 65,535 heads stay below 2^31
#pragma unroll
        for (int n = 0; n < kTilesN; ++n) {
          const int col = nw + n * kTile + 4 * g;
          store_four<T>(p, at + col, col, o[t][n]);
        }
      }
    }
  }
  if constexpr (kStage)
    if (stage && u_begin < u_valid) {
      __syncthreads();
      flush(threadIdx.x, u_begin + (u_valid - 1 - u_begin) / kChunk * kChunk);
    }

  if (OUT && !p.out_f32) {  // tokens beyond the row's length (of a sum over heads, the sum has them)
    const int64_t t_begin = max(u_begin, len);
    const int64_t out_at = ((row * p.length + t_begin) * p.heads + h) * int64_t(p.dout);
    const int cols = (p.dout + 3) / 4;
    for (int64_t i = threadIdx.x; i < (u_end - t_begin) * cols; i += kThreads) {
      const int col = int(i % cols) * 4;
      store_four<T>(p, out_at + i / cols * p.heads * p.dout + col, col, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
    }
  }
  float *s1 = OUT ? (p.seg_state == nullptr ? p.s1 : nullptr) : p.seg_state;
  if (s1 == nullptr) return;
  s1 += OUT ? rh * size : (rh * p.segments + seg) * size;
#pragma unroll
  for (int n = 0; n < kTilesN; ++n)
#pragma unroll
    for (int i = 0; i < kTilesI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int col = nw + n * kTile + l16, k = state_row(i, g, r);
        if (wt == 0 && k < p.di && col < p.dout) s1[unsigned(k * p.dout + col)] = s[n][i][r];
      }
}

// Short rows: one wave to a row and head, in registers alone.
//
// The results of the weights' products are, in the order of the contractions
// above, operands of the products with c as they stand, so the wave needs no
// LDS and no barrier, and many waves share a CU; a workgroup to a row leaves
// most of its waves idle at its barriers. 4,000 rows of up to 17 tokens (half
// of them there), 4 heads of 32 in bfloat16: 20 us, 2.1 TB/s, bound by the
// latency of a wave's few dependent loads; 101 us with workgroups. 1,024 rows of
// up to 33 in float32, 6 heads on 3 of 48 and 80: 39 us, and 80 for the three
// gradients; vector instructions issue in 27 and 31 % of the busy cycles, matrix
// instructions are busy for 16 and 23 %, and waves wait for half of their time.
//
// TT: most tiles of 16 tokens.
constexpr int kShortWaves = 4;  // of a workgroup, each for itself

template <class T>
__device__ __forceinline__ typename Vec<T>::eight short_row(const T *token, int kk, int g, int di, bool quads) {
  typedef typename Vec<T>::four four;
  typedef T any_four __attribute__((ext_vector_type(4), aligned(2)));
  four x[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = kk * 32 + i * 16 + 4 * g;
    if (kk * 32 + i * 16 + 16 <= di) {
      x[i] = *reinterpret_cast<const any_four *>(token + col);
    } else if (quads) {
      const four y = *reinterpret_cast<const any_four *>(token + (col < di ? col : 0));
      x[i] = col < di ? y : four{};
    } else {
      x[i] = four{};
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (col + r < di) x[i][r] = token[col + r];
    }
  }
  return join(x[0], x[1]);
}

// The values of a column at the byte offsets of eight rows: of tokens that are
// there, whatever the chunk's length, so what is not a token's has to meet a
// weight of 0.
template <class T>
__device__ __forceinline__ typename Vec<T>::eight short_column(const T *base, const unsigned (&at)[8], unsigned col) {
  typename Vec<T>::eight x;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    x[j] = *reinterpret_cast<const T *>(reinterpret_cast<const char *>(base) + (at[j] + col));
  return x;
}

// Columns of a short row whose c has NaN or infinities: the outputs before the first of them, which the matrix
// products have made none, one by one.
template <class T, class TokenOf>
__device__ __forceinline__ void short_odd(const ScanArgs &p, const T *a, const T *b, const T *c, const float *s0,
                                          int64_t out_at, int64_t out_step, int len, float log2_gamma,
                                          TokenOf token_of) {
  int lane = lane_id();
  asm volatile("" : "+v"(lane));  // nothing of this is kept for it
  const int per_k = p.transposed ? 1 : p.dout, per_col = p.transposed ? p.di : 1, e = p.reverse ? 0 : 1;
#pragma unroll 1
  for (int n0 = 0; n0 < p.dout; n0 += kWave) {
    const bool there = n0 + lane < p.dout;
    const int col = there ? n0 + lane : 0;
    int first = len;
#pragma unroll 1
    for (int u = len - 1; u >= 0; --u)
      if (!__builtin_isfinite(to_f32(c[token_of(u) * p.c.token + col]))) first = u;
    const bool mends = there && first < len;
#pragma unroll 1
    for (int u = 0; __ballot(mends && u < first) != 0; ++u) {
      const T *au = a + token_of(u) * p.a.token;
      float o = 0.0f;
#pragma unroll 1
      for (int w = 0; w <= u; ++w) {
        const T *bw = b + token_of(w) * p.b.token;
        float x = 0.0f;
        for (int i = lane; i < p.di; i += kWave) x += to_f32(au[i]) * to_f32(bw[i]);
#pragma unroll
        for (int off = kWave / 2; off > 0; off >>= 1) x += __shfl_xor(x, off, kWave);
        x *= p.pscale * __builtin_amdgcn_exp2f(float(u - w) * log2_gamma);
        o += x * to_f32(c[token_of(w) * p.c.token + col]);
      }
      if (s0 != nullptr) {
        float x = 0.0f;
#pragma unroll 1
        for (int k = 0; k < p.di; ++k) x += to_f32(au[k]) * s0[unsigned(k * per_k + col * per_col)];
        o += x * p.oscale * __builtin_amdgcn_exp2f(float(u + e) * log2_gamma);
      }
      if (!mends || u >= first) continue;
      const int64_t at = out_at + token_of(u) * out_step + col;
      if (p.out_f32)
        static_cast<float *>(p.out)[at] = o;
      else
        static_cast<T *>(p.out)[at] = from_f32<T>(o);
    }
  }
}

template <class T, int DI, int TT>
__global__ __launch_bounds__(kShortWaves * kWave, TT <= 2 ? 6 : 4) void short_scan_kernel(ScanRoles roles,
                                                                                          int64_t items,
                                                                                          int64_t first) {
  constexpr int kK = DI / 32, kBlocks = (TT + 1) / 2, kPieces = Vec<T>::kPieces, kOperand = Vec<T>::kOperand,
                kStatePieces = Vec<T>::kStatePieces;
  typedef typename Vec<T>::eight eight;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t item = (first + blockIdx.x) * kShortWaves + wave;
  if (item >= items) return;
  const ScanArgs &p = roles.role[item % roles.count];
  const int64_t rh = item / roles.count, row = rh / p.heads;
  const int h = int(rh % p.heads);
  const int lane = lane_id(), l16 = lane % 16, g = lane / 16;
  const bool report = lane == 0;
  const float log2_gamma = head_log_decay(p.log_decay, h, p.status, report && row == 0) * kLog2e;
  const int len = int(row_length(p.len, row, p.length, p.status, report && h == 0));
  const int tiles = (len + kTile - 1) / kTile, blocks = (len + 31) / 32;
  const int e = p.reverse ? 0 : 1;
  const T *a = operand_row<T>(p.a, row, h), *b = operand_row<T>(p.b, row, h), *c = operand_row<T>(p.c, row, h);
  // the token that is u-th in the scan's order, or one that is there
  auto token_of = [&](int u) { return p.reverse ? max(len - 1 - u, 0) : min(u, len - 1); };
  const int64_t state_at = rh * int64_t(p.di) * p.dout;
  const float *s0 = p.s0 == nullptr ? nullptr : p.s0 + state_at;

  if (len > 0) {
    // a_t . b_s of the pairs of tiles: every row is read once, and of all tiles together
    f32x4 x[TT][TT];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int st = 0; st < TT; ++st) x[t][st] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int kk = 0; kk < kK; ++kk) {
      if (kk * 32 >= p.di) break;
      eight av[TT], bv[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        if (t >= tiles) break;
        const int64_t u = token_of(t * kTile + l16);
        av[t] = short_row(a + u * p.a.token, kk, g, p.di, p.wide);
        bv[t] = short_row(b + u * p.b.token, kk, g, p.di, p.wide);
      }
      const bool low = kk * 32 + kTile >= p.di;
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        if (t >= tiles) break;
#pragma unroll
        for (int st = 0; st <= t; ++st)
          x[t][st] = low ? mma_low(bv[st], av[t], x[t][st]) : mma(bv[st], av[t], x[t][st]);
      }
    }
    // weights of the pairs (t, s) as operands: tile t, blocks of 32 of s
    eight w[TT][kBlocks][kPieces];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      if (t >= tiles) break;
#pragma unroll
      for (int s32 = 0; s32 <= t / 2; ++s32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int st = 2 * s32 + i;
          if (st > t) continue;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = (t - st) * kTile + l16 - 4 * g - r;
            const float y = x[t][st][r] * p.pscale * __builtin_amdgcn_exp2f(float(d) * log2_gamma);
            x[t][st][r] = d >= 0 ? y : 0.0f;
          }
        }
        f32x8 both = join(x[t][2 * s32], 2 * s32 + 1 <= t ? x[t][2 * s32 + 1 < TT ? 2 * s32 + 1 : 0] : f32x4{});
#pragma unroll
        for (int i = 0; i < kPieces; ++i) w[t][s32][i] = take_piece(both, T());
      }
    }

    // places of the rows of c that a lane reads columns of
    unsigned c_at[kBlocks][8];
#pragma unroll
    for (int kk = 0; kk < kBlocks; ++kk)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        c_at[kk][j] = unsigned(token_of(kk * 32 + 16 * (j / 4) + 4 * g + j % 4)) * unsigned(p.c.token) *
                      unsigned(sizeof(T));

    const int per_k = p.transposed ? 1 : p.dout, per_col = p.transposed ? p.di : 1;
    const int64_t out_step = int64_t(p.heads) * p.dout, out_at = (row * p.length * p.heads + h) * p.dout;
    const float whole = __builtin_amdgcn_exp2f(float(len) * log2_gamma);
    bool odd = false;
    for (int n0 = 0; n0 < p.dout; n0 += kTile) {
      const int col = min(n0 + l16, p.dout - 1);  // columns beyond the last are not stored
      eight cv[kBlocks];
#pragma unroll
      for (int kk = 0; kk < kBlocks; ++kk) {
        if (kk >= blocks) break;
        cv[kk] = short_column(c, c_at[kk], unsigned(col) * unsigned(sizeof(T)));
      }
      f32x4 o[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) o[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (s0 != nullptr) {
        int g = lane / 16, l16 = lane % 16;
        asm volatile("" : "+v"(g), "+v"(l16));
#pragma unroll
        for (int kk = 0; kk < kK; ++kk) {
          if (kk * 32 >= p.di) break;
          f32x8 x;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int k = kk * 32 + 16 * (j / 4) + 4 * g + j % 4;
            x[j] = k < p.di ? s0[unsigned(k * per_k + col * per_col)] : 0.0f;
          }
          eight sv[kOperand];
#pragma unroll
          for (int i = 0; i < kOperand; ++i) sv[i] = take_piece(x, T());
#pragma unroll
          for (int t = 0; t < TT; ++t) {
            if (t >= tiles) break;
            const T *at = a + token_of(t * kTile + l16) * p.a.token;
            const eight av = short_row(at, kk, g, p.di, p.wide);
#pragma unroll
            for (int i = 0; i < kOperand; ++i) o[t] = mma(sv[i], av, o[t]);
          }
        }
#pragma unroll
        for (int t = 0; t < TT; ++t)
          o[t] *= p.oscale * __builtin_amdgcn_exp2f(float(t * kTile + l16 + e) * log2_gamma);
      }
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        if (t >= tiles) break;
#pragma unroll
        for (int kk = 0; kk <= t / 2; ++kk)
#pragma unroll
          for (int i = 0; i < kPieces; ++i)  // of the last block an even tile has the lower half
            o[t] = 2 * kk == t ? mma_low(cv[kk], w[t][kk][i], o[t]) : mma(cv[kk], w[t][kk][i], o[t]);
        const int u = t * kTile + l16;
#pragma unroll
        for (int r = 0; r < 4; ++r) odd |= !__builtin_isfinite(o[t][r]);
        if (u < len) store_four<T>(p, out_at + token_of(u) * out_step + n0 + 4 * g, n0 + 4 * g, o[t]);
      }
    }
    if (__builtin_expect(__ballot(odd) != 0, 0))
      short_odd<T>(p, a, b, c, s0, out_at, out_step, len, log2_gamma, token_of);
    // S at the row's end, a tile at a time; what it needs is made here, not kept
    for (int n0 = 0; p.s1 != nullptr && n0 < p.dout; n0 += kTile) {
      const int col = min(n0 + l16, p.dout - 1);  // columns beyond the last are not stored
      int g = lane / 16;
      asm volatile("" : "+v"(g));
      unsigned b_at[kBlocks][8];
#pragma unroll
      for (int kk = 0; kk < kBlocks; ++kk)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          b_at[kk][j] = unsigned(token_of(kk * 32 + 16 * (j / 4) + 4 * g + j % 4)) * unsigned(p.b.token) *
                        unsigned(sizeof(T));
      eight wv[kBlocks][kStatePieces];
#pragma unroll
      for (int kk = 0; kk < kBlocks; ++kk) {
        if (kk >= blocks) break;
        const eight cv = short_column(c, c_at[kk], unsigned(col) * unsigned(sizeof(T)));
        f32x8 x;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int u = kk * 32 + 16 * (j / 4) + 4 * g + j % 4;
          const float y = to_f32(cv[j]) * p.sscale * __builtin_amdgcn_exp2f(float(len - e - u) * log2_gamma);
          x[j] = u < len ? y : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < kStatePieces; ++i) wv[kk][i] = take_piece(x, T());
      }
      for (int i0 = 0; i0 < p.di; i0 += kTile) {
        const unsigned k_of = min(i0 + l16, p.di - 1);  // rows beyond the last are not stored
        f32x4 s;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int k = min(i0 + 4 * g + r, p.di - 1);
          s[r] = s0 != nullptr ? s0[unsigned(k * per_k + col * per_col)] * whole : 0.0f;
        }
#pragma unroll
        for (int kk = 0; kk < kBlocks; ++kk) {
          if (kk >= blocks) break;
          const eight bv = short_column(b, b_at[kk], k_of * unsigned(sizeof(T)));
#pragma unroll
          for (int i = 0; i < kStatePieces; ++i) s = mma(bv, wv[kk][i], s);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int k = i0 + 4 * g + r;
          if (k < p.di && n0 + l16 < p.dout) p.s1[state_at + k * p.dout + n0 + l16] = s[r];
        }
      }
    }
  } else if (p.s1 != nullptr) {  // a row without tokens leaves its state as it is
    for (int i = lane; i < p.di * p.dout; i += kWave)
      p.s1[state_at + i] = s0 == nullptr ? 0.0f : s0[p.transposed ? i % p.dout * p.di + i / p.dout : i];
  }
  if (p.out_f32) return;
  // tokens beyond the row's length (of a sum over heads, the sum has them)
  const int cols = (p.dout + 3) / 4;
  for (int i = lane; i < (int(p.length) - len) * cols; i += kWave) {
    const int col = i % cols * 4;
    store_four<T>(p, ((row * p.length + len + i / cols) * p.heads + h) * p.dout + col, col,
                  f32x4{0.0f, 0.0f, 0.0f, 0.0f});
  }
}

// The states that the segments of a row begin with, in place of the segments'
// own, and the row's last state.
__global__ __launch_bounds__(kThreads) void join_kernel(ScanRoles roles, int64_t first) {
  const int64_t block = first + blockIdx.x;
  const ScanArgs &p = roles.role[block % roles.count];
  const int64_t size = int64_t(p.di) * p.dout, parts = (size + kThreads - 1) / kThreads;
  const int64_t rh = block / roles.count / parts, at = block / roles.count % parts * kThreads + threadIdx.x;
  if (at >= size) return;
  const float log2_gamma = head_log_decay(p.log_decay, int(rh % p.heads), nullptr, false) * kLog2e;
  const int64_t len = row_length(p.len, rh / p.heads, p.length, nullptr, false);
  float cur = 0.0f;
  if (p.s0 != nullptr) cur = p.s0[rh * size + at];
  float *x = p.seg_state + rh * p.segments * size + at;
  constexpr int kAhead = 8;
  for (int64_t seg = 0; seg < p.segments; seg += kAhead) {
    float own[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) own[i] = seg + i < p.segments ? x[(seg + i) * size] : 0.0f;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (seg + i >= p.segments) break;
      x[(seg + i) * size] = cur;
      const int64_t n = max(int64_t(0), min(p.segment, len - (seg + i) * p.segment));
      cur = fmaf(cur, __builtin_amdgcn_exp2f(float(n) * log2_gamma), own[i]);
    }
  }
  if (p.s1 != nullptr) p.s1[rh * size + at] = cur;
}

int padded(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }

// Scans of one size side by side.
template <class T, bool OUT>
rdf2v_status launch_chunks(const ScanRoles &roles, hipStream_t stream) {
  const ScanArgs &p = roles.role[0];
  const int64_t items = p.rows * p.heads * p.segments;
  const int64_t blocks = (items + kXcds - 1) / kXcds * kXcds * roles.count;
  return for_each_launch(blocks, 8 * kWave, 1, [&](int64_t first, int64_t count) {
    const int di = padded(p.di), nb = padded(p.dout);
    const dim3 grid{unsigned(count)}, threads{unsigned(scan_waves(nb) * kWave)};
#define RDF2V_SCAN(DI, NB) \
  if (di == DI && nb == NB) scan_kernel<T, DI, NB, OUT><<<grid, threads, 0, stream>>>(roles, items, first);
    RDF2V_SCAN(32, 32) RDF2V_SCAN(32, 64) RDF2V_SCAN(32, 128)
    RDF2V_SCAN(64, 32) RDF2V_SCAN(64, 64) RDF2V_SCAN(64, 128)
    RDF2V_SCAN(128, 32) RDF2V_SCAN(128, 64) RDF2V_SCAN(128, 128)
#undef RDF2V_SCAN
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

template <class T>
rdf2v_status launch_short(const ScanRoles &roles, hipStream_t stream) {
  const int64_t items = roles.role[0].rows * roles.role[0].heads * roles.count;
  int di = 0;
  for (int i = 0; i < roles.count; ++i) di = roles.role[i].di > di ? roles.role[i].di : di;
  const int64_t blocks = (items + kShortWaves - 1) / kShortWaves;
  return for_each_launch(blocks, kShortWaves * kWave, 1, [&](int64_t first, int64_t count) {
    const dim3 grid{unsigned(count)}, threads{kShortWaves * kWave};
    const int64_t length = roles.role[0].length;
    const int tiles = length <= kTile ? 1 : int((length + kTile - 1) / kTile);
#define RDF2V_SHORT(DI, TT) \
  if (padded(di) == DI && tiles == TT) short_scan_kernel<T, DI, TT><<<grid, threads, 0, stream>>>(roles, items, first);
    RDF2V_SHORT(32, 1) RDF2V_SHORT(64, 1) RDF2V_SHORT(128, 1)
    RDF2V_SHORT(32, 2) RDF2V_SHORT(64, 2) RDF2V_SHORT(128, 2)
    RDF2V_SHORT(32, 3) RDF2V_SHORT(64, 3) RDF2V_SHORT(128, 3)
#undef RDF2V_SHORT
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

// Segments of a row: one, unless there are too few rows and heads to fill the
// chip with a workgroup each. Then a row is cut into segments of whole chunks,
// the states of the segments are computed first and joined, and all segments
// run at once: b and c are read twice, and a state is written and read for
// each segment. At least kLeastChunks chunks to a segment keep that traffic
// below what the segment itself reads.
//
// kFill: two workgroups of a scan share a CU, so 512 are one round of them.
// One row of 20,011 x 8 heads of 128, forward, takes 113, 116, 110 and 107 us
// with 256, 384, 512 and 768. The segments are as many as the state scans (two
// of them backwards) need to fill a round: with the 512 counted over the three
// scans of the gradients, four rows of 4,096 x 16 heads of 128, forward and
// backward, take 523 us, not 473, and two of 8,192 x 16 heads of 64 take 241,
// not 211. But rows whose three scans fill a round by themselves are not cut:
// 12 rows of 2,048 x 16 heads of 128 take 639 us whole and 775 in two.
constexpr int64_t kFill = 512;
constexpr int64_t kLeastChunks = 4;

int64_t segment_count(int64_t rows_heads, int scans, int state_scans, int64_t length) {
  const int64_t chunks = (length + kChunk - 1) / kChunk, states = rows_heads * state_scans;
  if (rows_heads == 0 || rows_heads * scans >= kFill || chunks < 2 * kLeastChunks) return 1;
  const int64_t want = (kFill + states - 1) / states, most = chunks / kLeastChunks;
  const int64_t count = want < most ? want : most, per = (chunks + count - 1) / count;
  return (chunks + per - 1) / per;
}

template <class T>
void finish(ScanArgs &p, bool short_rows, int64_t segments) {
  p.pscale = p.oscale * p.sscale;
  const int64_t chunks = (p.length + kChunk - 1) / kChunk;
  p.segments = segments;
  p.segment = (chunks + segments - 1) / segments * kChunk;
  auto fits = [](const ScanOperand &x, int d) {
    if (x.token < 0 || x.token >= int64_t(1) << 23) return false;
    const uintptr_t all = reinterpret_cast<uintptr_t>(x.data) |
                          uintptr_t(x.row | x.token | x.head | int64_t(d)) * sizeof(T);
    return (all & 15) == 0;
  };
  p.wide = short_rows ? p.di % 4 == 0 : (p.a.data == nullptr || fits(p.a, p.di)) && fits(p.b, p.di) && fits(p.c, p.dout);
  p.whole_out = !p.out_f32 && sizeof(T) == 2 && p.dout % 8 == 0 && (reinterpret_cast<uintptr_t>(p.out) & 15) == 0;
  p.wide_out = p.dout % 4 == 0 && (reinterpret_cast<uintptr_t>(p.out) & (p.out_f32 || sizeof(T) == 4 ? 15 : 7)) == 0;
}

// Whether a wave to a row and head is the faster way. us with a wave / with a workgroup and chunks, forward and
// the three gradients, 8 heads; many rows are 256 MB of q, k, v and out:
//                      tokens  sizes 32             64                    128
//   bfloat16           16      57/366  200/1055     61/282   214/830      64/250    234/731
//                      33      69/181   227/539     76/153   244/463      75/136    246/396
//                      48      57/127   207/377     84/112   238/346      89/101    242/287
//   with states        16      284/538  587/1351    679/535  1079/1263    1371/666  2060/1669
//                      33      236/294  563/720     440/304  911/703      919/367   1683/896
//                      48      197/209  448/509     436/223  714/507      827/268   1322/636
//   float32            16      45/315   132/940     47/321   139/946      48/406    146/1213
//                      33      59/176   180/546     57/188   173/563      56/227    175/665
//                      48      52/128   150/396     56/136   151/406      51/167    162/485
//   with states        16      208/451  340/1139    410/493  591/1231     780/759   1166/1979
//                      33      175/266  365/650     277/328  582/722      539/460   1169/1049
//                      48      160/193  286/468     278/236  450/518      489/331   874/754
// With states a wave does in turn what a workgroup does side by side, so few rows are faster with workgroups:
//   rows of 8 heads            64               128              256               512
//   bfloat16, 33 tokens, 32    18/14   25/24    18/15   29/32    25/24   51/52     35/40    80/93
//   float32, 33 tokens, 32     19/14   28/28    21/22   35/49    30/38   61/87     47/68    97/162
//   float32, 16 tokens, 64     34/19   48/47    48/35   64/86    60/63   92/157    91/116   167/300
//   float32, 48 tokens, 64     60/23   80/55    73/42   104/98   96/77   200/182   189/175  349/395
// (states: float32 in and out). A wave's 32-bit places take tokens less than
// 2^23 values apart, in ascending order.
template <class T>
bool use_short(const ScanArgs *scans, int count) {
  constexpr int kStates = sizeof(T) == 4 ? 64 : 32;
  for (int i = 0; i < count; ++i) {
    const ScanArgs &p = scans[i];
    if (p.length > 3 * kTile) return false;
    if (p.s0 != nullptr || p.s1 != nullptr) {
      const int size = p.di > p.dout ? p.di : p.dout;
      if (size > kStates || p.rows * p.heads < (size > 32 ? 2048 : 1024)) return false;
    }
    for (const ScanOperand *x : {&p.a, &p.b, &p.c})
      if (x->token < 0 || x->token >= int64_t(1) << 23) return false;
  }
  return true;
}

// `count` scans; states[state_of[i]] is the scan that gives scan i its states
// where rows are cut into segments (its own s0 and s1 are then not used).
template <class T>
rdf2v_status launch_scans(ScanArgs *scans, int count, ScanArgs *states, int num_states, const int *state_of,
                          float *seg_state, bool together, hipStream_t stream) {
  const bool short_rows = use_short<T>(scans, count);
  const int64_t segments = segment_count(scans[0].rows * scans[0].heads, count, num_states, scans[0].length);
  if (segments > 1) {
    ScanRoles roles{};
    for (int i = 0; i < num_states; ++i) {
      finish<T>(states[i], false, segments);
      states[i].seg_state = seg_state + i * states[i].rows * states[i].heads * segments * states[i].di * states[i].dout;
      roles.role[roles.count++] = states[i];
    }
    rdf2v_status st = launch_chunks<T, false>(roles, stream);
    if (st != RDF2V_OK) return st;
    const ScanArgs &p = states[0];
    const int64_t parts = (int64_t(p.di) * p.dout + kThreads - 1) / kThreads;
    st = for_each_launch(p.rows * p.heads * parts * num_states, kThreads, 1, [&](int64_t first, int64_t blocks) {
      join_kernel<<<dim3(unsigned(blocks)), dim3(kThreads), 0, stream>>>(roles, first);
      RDF2V_LAUNCH_CHECK();
      return RDF2V_OK;
    });
    if (st != RDF2V_OK) return st;
    for (int i = 0; i < count; ++i) {
      scans[i].seg_state = states[state_of[i]].seg_state;
      scans[i].s1 = nullptr;
    }
    together = true;
  }
  bool done[3] = {};
  for (int i = 0; i < count; ++i) {
    if (done[i]) continue;
    ScanRoles roles{};
    for (int j = i; j < count; ++j) {
      const bool same = short_rows || (padded(scans[j].di) == padded(scans[i].di) &&
                                      padded(scans[j].dout) == padded(scans[i].dout));
      if (done[j] || !same || (j > i && !together)) continue;
      finish<T>(scans[j], short_rows, segments);
      roles.role[roles.count++] = scans[j];
      done[j] = true;
    }
    const rdf2v_status st = short_rows ? launch_short<T>(roles, stream) : launch_chunks<T, true>(roles, stream);
    if (st != RDF2V_OK) return st;
  }
  return RDF2V_OK;
}

size_t segment_state_bytes(const rdf2v_attention &a, bool backward) {
  const int64_t segments = segment_count(a.rows * a.heads, backward ? 3 : 1, backward ? 2 : 1, a.length);
  if (segments == 1) return 0;
  return align_up(size_t(a.rows) * a.heads * segments * a.dk * a.dv * sizeof(float) * (backward ? 2 : 1), 256);
}

// The gradients of `share` query heads' keys and values summed in head order,
// and zeros for the tokens beyond a row's length, whose parts are not there. A
// wave takes a token, VEC values a lane: HBM-bound. 1,024 rows of up to 33
// tokens (half of them there), 6 heads on 3 of 48 and 80 in float32: 16 us,
// where a launch for each gradient over the padding too takes 37.
struct ShareArgs {
  const float *part[2];
  void *out[2];
  int32_t d[2];
  const int32_t *len;
  int64_t rows, length;
  int32_t kv_heads, share;
};

template <class T, int VEC>
__global__ __launch_bounds__(kThreads) void share_sum_kernel(ShareArgs p, int64_t first) {
  typedef float in __attribute__((ext_vector_type(VEC), aligned(4)));
  typedef T to __attribute__((ext_vector_type(VEC), aligned(sizeof(T))));
  constexpr int kWaves = kThreads / kWave;
  const int64_t token = (first + blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (token >= p.rows * p.length) return;
  const bool there = token % p.length < row_length(p.len, token / p.length, p.length, nullptr, false);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int per = p.d[i] / VEC;
    const float *part = p.part[i] + token * p.kv_heads * p.share * p.d[i];
    T *out = static_cast<T *>(p.out[i]) + token * p.kv_heads * p.d[i];
    for (int at = lane_id(); at < p.kv_heads * per; at += kWave) {
      const float *x = part + (unsigned(at) / unsigned(per) * p.share * per + unsigned(at) % unsigned(per)) * VEC;
      in sum{};
      if (there)
        for (int j = 0; j < p.share; ++j) sum += *reinterpret_cast<const in *>(x + j * p.d[i]);
      to y;
#pragma unroll
      for (int r = 0; r < VEC; ++r) y[r] = from_f32<T>(sum[r]);
      *reinterpret_cast<to *>(out + at * VEC) = y;
    }
  }
}

template <class T>
rdf2v_status launch_share_sum(const ShareArgs &p, hipStream_t stream) {
  constexpr int kWaves = kThreads / kWave;
  return for_each_launch((p.rows * p.length + kWaves - 1) / kWaves, kThreads, 1, [&](int64_t first, int64_t count) {
    const dim3 grid{unsigned(count)}, threads{kThreads};
    if (p.d[0] % 4 == 0 && p.d[1] % 4 == 0)
      share_sum_kernel<T, 4><<<grid, threads, 0, stream>>>(p, first);
    else
      share_sum_kernel<T, 1><<<grid, threads, 0, stream>>>(p, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

ScanOperand operand(const rdf2v_heads_view &v, int share) {
  return {v.data, v.row_stride, v.token_stride, v.head_stride, share};
}

ScanArgs scan_args(const rdf2v_attention &a, int32_t *status) {
  ScanArgs p{};
  p.log_decay = a.log_decay;
  p.len = a.len;
  p.rows = a.rows;
  p.length = a.length;
  p.heads = a.heads;
  p.oscale = p.sscale = 1.0f;
  p.status = status;
  return p;
}

template <class T>
rdf2v_status forward(const rdf2v_attention &a, const rdf2v_heads_view &q, const rdf2v_heads_view &k,
                     const rdf2v_heads_view &v, const float *state, void *out, float *state_out, void *workspace,
                     int32_t *status, hipStream_t stream) {
  const int share = a.heads / a.kv_heads, state_of[1] = {0};
  ScanArgs p = scan_args(a, status);
  p.a = operand(q, 1);
  p.b = operand(k, share);
  p.c = operand(v, share);
  p.di = a.dk;
  p.dout = a.dv;
  p.s0 = state;
  p.s1 = state_out;
  p.out = out;
  p.oscale = a.scale;
  ScanArgs own = p;
  own.a = ScanOperand{};
  return launch_scans<T>(&p, 1, &own, 1, state_of, static_cast<float *>(workspace), true, stream);
}

template <class T>
rdf2v_status backward(const rdf2v_attention &a, const rdf2v_heads_view &q, const rdf2v_heads_view &k,
                      const rdf2v_heads_view &v, const rdf2v_heads_view &dout, const float *state,
                      const float *dstate_out, void *dq, void *dk, void *dv, float *dstate, void *workspace,
                      int32_t *status, hipStream_t stream) {
  const int share = a.heads / a.kv_heads, state_of[3] = {0, 1, 1};
  const int64_t tokens = a.rows * a.length;
  float *seg = static_cast<float *>(workspace);
  float *part_k = seg + segment_state_bytes(a, true) / sizeof(float), *part_v = part_k + tokens * a.heads * a.dk;

  ScanArgs scans[3], states[2];
  ScanArgs &s = states[0], &r = states[1];  // S of the forward pass, and its gradient
  s = r = scan_args(a, status);
  s.di = r.di = a.dk;
  s.dout = r.dout = a.dv;
  s.b = operand(k, share);
  s.c = operand(v, share);
  s.s0 = state;
  r.b = operand(q, 1);
  r.c = operand(dout, 1);
  r.reverse = true;
  r.sscale = a.scale;
  r.s0 = dstate_out;
  r.s1 = dstate;

  ScanArgs &pq = scans[0], &pk = scans[1], &pv = scans[2];
  pq = scan_args(a, status);
  pq.a = operand(dout, 1);
  pq.b = operand(v, share);
  pq.c = operand(k, share);
  pq.di = a.dv;
  pq.dout = a.dk;
  pq.s0 = state;
  pq.transposed = true;
  pq.out = dq;
  pq.oscale = a.scale;
  pk = scan_args(a, status);
  pk.a = operand(v, share);
  pk.b = operand(dout, 1);
  pk.c = operand(q, 1);
  pk.di = a.dv;
  pk.dout = a.dk;
  pk.s0 = dstate_out;
  pk.transposed = true;
  pk.reverse = true;
  pk.sscale = a.scale;
  pk.out = share > 1 ? part_k : dk;
  pk.out_f32 = share > 1;
  pv = r;
  pv.a = operand(k, share);
  pv.out = share > 1 ? part_v : dv;
  pv.out_f32 = share > 1;

  // dv's scan writes dstate while dk's reads dstate_out: one after the other where they are one array
  const bool together = dstate == nullptr || dstate != dstate_out;
  rdf2v_status st = launch_scans<T>(scans, 3, states, 2, state_of, seg, together, stream);
  if (st != RDF2V_OK || share == 1) return st;
  return launch_share_sum<T>({{part_k, part_v}, {dk, dv}, {a.dk, a.dv}, a.len, a.rows, a.length, a.kv_heads, share},
                             stream);
}

struct StepArgs {
  ScanOperand q, k, v;
  const float *log_decay, *state;
  const int32_t *parents;
  void *out;
  float *state_out;
  int32_t *status;
  int64_t num_states, rows;
  int32_t heads, dk, dv;
  float scale;
};

// One workgroup to a row and head. HBM-bound: a state is read and written once,
// 2 operations a byte, VEC values a lane and kAhead loads of a lane in flight
// (a state of 128 x 128 is 16 loads of 16 bytes a thread). 512 rows of 8 heads
// of 128 x 128 that take over the states of their parents: 82 us, 5.4 TB/s.
template <class T, int VEC>
__global__ __launch_bounds__(kThreads) void step_kernel(StepArgs p, int64_t first) {
  typedef float vec __attribute__((ext_vector_type(VEC)));
  constexpr int kAhead = 16;
  __shared__ float ks[RDF2V_MAX_HEAD_SIZE], qs[RDF2V_MAX_HEAD_SIZE];
  __shared__ vec part[kThreads];
  const int64_t block = first + blockIdx.x, row = block / p.heads;
  const int h = int(block % p.heads);
  const bool report = threadIdx.x == 0;
  int64_t from = row;
  if (p.parents != nullptr) {
    from = p.parents[row];
    if (from < 0 || from >= p.num_states) {
      from = -1;
      if (report && h == 0 && p.status != nullptr) atomicOr(p.status, RDF2V_STATUS_ID_OUT_OF_RANGE);
    }
  }
  const int cols = p.dv / VEC, rows = kThreads / cols;  // lanes over a row of the state, rows side by side
  const int col = threadIdx.x % cols, r0 = threadIdx.x / cols;
  const bool active = r0 < rows;
  const int64_t size = int64_t(p.dk) * p.dv;
  const vec *s0 = reinterpret_cast<const vec *>(p.state + (from < 0 ? 0 : from * p.heads + h) * size);
  vec *s1 = reinterpret_cast<vec *>(p.state_out + (row * p.heads + h) * size);
  const int last = from < 0 || !active ? 0 : p.dk;      // rows of the state that are read
  vec s[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int r = r0 + i * rows;
    s[i] = vec(0.0f);
    if (r < last) s[i] = __builtin_nontemporal_load(s0 + r * cols + col);
  }
  const float gamma = expf(head_log_decay(p.log_decay, h, p.status, report && row == 0));
  if (int(threadIdx.x) < p.dk) {
    ks[threadIdx.x] = to_f32(operand_row<T>(p.k, row, h)[threadIdx.x]);
    qs[threadIdx.x] = to_f32(operand_row<T>(p.q, row, h)[threadIdx.x]);
  }
  const T *v = operand_row<T>(p.v, row, h) + col * VEC;
  vec vn;
#pragma unroll
  for (int j = 0; j < VEC; ++j) vn[j] = to_f32(v[j]);
  __syncthreads();
  vec o = vec(0.0f);
  if (active)
    for (int base = r0; base < p.dk; base += kAhead * rows) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int r = base + i * rows;
        if (base != r0) s[i] = r < last ? s0[r * cols + col] : vec(0.0f);
        if (r >= p.dk) continue;
        const vec x = s[i] * gamma + vn * ks[r];
        __builtin_nontemporal_store(x, s1 + r * cols + col);
        o += x * qs[r];
      }
    }
  part[threadIdx.x] = o;
  __syncthreads();
  T *out = static_cast<T *>(p.out) + (row * p.heads + h) * p.dv;
  for (int n = threadIdx.x; n < p.dv; n += kThreads) {
    float sum = 0.0f;
    for (int r = 0; r < rows; ++r) sum += part[r * cols + n / VEC][n % VEC];
    out[n] = from_f32<T>(sum * p.scale);
  }
}

template <class T>
rdf2v_status launch_step(const StepArgs &p, hipStream_t stream) {
  const bool wide = p.dv % 4 == 0 &&
                    ((reinterpret_cast<uintptr_t>(p.state) | reinterpret_cast<uintptr_t>(p.state_out)) & 15) == 0;
  return for_each_launch(p.rows * p.heads, kThreads, 1, [&](int64_t first, int64_t count) {
    if (wide)
      step_kernel<T, 4><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
    else
      step_kernel<T, 1><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

}  // namespace

size_t decay_attention_workspace_bytes(const rdf2v_attention &a, bool backward) {
  const size_t seg = segment_state_bytes(a, backward);
  if (!backward || a.heads == a.kv_heads) return seg;
  return seg + align_up(size_t(a.rows) * a.length * a.heads * (a.dk + a.dv) * sizeof(float), 256);
}

rdf2v_status launch_decay_attention(const rdf2v_attention &a, const rdf2v_heads_view &q, const rdf2v_heads_view &k,
                                    const rdf2v_heads_view &v, const float *state, void *out, float *state_out,
                                    void *workspace, int32_t *status_dev, hipStream_t stream) {
  return a.dtype == RDF2V_BF16 ? forward<bf16>(a, q, k, v, state, out, state_out, workspace, status_dev, stream)
                               : forward<float>(a, q, k, v, state, out, state_out, workspace, status_dev, stream);
}

rdf2v_status launch_decay_attention_backward(const rdf2v_attention &a, const rdf2v_heads_view &q,
                                             const rdf2v_heads_view &k, const rdf2v_heads_view &v,
                                             const rdf2v_heads_view &dout, const float *state,
                                             const float *dstate_out, void *dq, void *dk, void *dv, float *dstate,
                                             void *workspace, int32_t *status_dev, hipStream_t stream) {
  return a.dtype == RDF2V_BF16 ? backward<bf16>(a, q, k, v, dout, state, dstate_out, dq, dk, dv, dstate, workspace,
                                                status_dev, stream)
                               : backward<float>(a, q, k, v, dout, state, dstate_out, dq, dk, dv, dstate, workspace,
                                                 status_dev, stream);
}

rdf2v_status launch_decay_attention_step(const rdf2v_attention &a, const rdf2v_heads_view &q,
                                         const rdf2v_heads_view &k, const rdf2v_heads_view &v, const float *state,
                                         int64_t num_states, const int32_t *parents, void *out, float *state_out,
                                         int32_t *status_dev, hipStream_t stream) {
  const int share = a.heads / a.kv_heads;
  const StepArgs p{operand(q, 1), operand(k, share), operand(v, share), a.log_decay, state, parents, out, state_out,
                   status_dev, num_states, a.rows, a.heads, a.dk, a.dv, a.scale};
  return a.dtype == RDF2V_BF16 ? launch_step<bf16>(p, stream) : launch_step<float>(p, stream);
}

}  // namespace rdf2v
