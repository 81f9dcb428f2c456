// Selective scan over rows of tokens on gfx950, its gradients and its step.
//
//   h_t[n] = exp(delta_t a[n]) h_{t-1}[n] + delta_t x_t b_t[n],   y_t = sum_n c_t[n] h_t[n] + skip x_t
//
// for every channel by itself: per token, channel and state one exponential and three multiply-adds, so with 16
// states vector instructions bound it, memory comes next. An exponential takes the time of two other instructions.
//
// A wave takes 64 channels (a lane each) of a row, or of a segment of it, 16 tokens at a time, and nothing but the
// gradients' rates is shared with other waves: no barrier, no value made twice. It takes the channels' states in
// turn, each through the chunk's 16 tokens, whose values stay in registers meanwhile: the number of states is a
// loop's, not a register file's. b and c of the chunk lie in LDS and are read by all lanes at once.
//
// Rows too few to fill the chip are cut into segments: every segment's state from zeros (scan_states_kernel), the
// states' way through the segments (scan_join_kernel), then all segments at once. That costs the exponentials
// twice.
//
// Gradients go backwards through the chunks: a chunk's states are made again from the one before it, which
// scan_states_kernel has left in memory, and stay in registers for the way back. The sums over states (for x and
// dt) are a lane's own; the sums over channels (for b and c) are taken for sixteen values at once, see sixteen_sums.
//
// Kernels' times here and below are means under the profiler, up to an eighth longer than among other calls; times of
// calls are without it.

#include "vectors.hpp"

#include "layer.hpp"
#include "logits.hpp"

namespace rdf2v {
namespace {

constexpr int kTokens = 16;  // of a chunk
constexpr int kBackTokens = 8;  // of a chunk in the gradients: what is held of each sets how many waves there are
constexpr int kGang = 4;        // waves of a workgroup in the gradients, which have the rates in common
constexpr int kThreads = 256;  // of a workgroup where waves need not be alone

struct Scan {
  rdf2v_tokens_view x, dt, gate, dout;
  rdf2v_heads_view b, c;
  const float *a, *dt_bias, *skip, *state, *dstate_out;
  const int32_t *len, *parents;
  int32_t *status;
  void *out, *dx, *ddt, *dgate, *db, *dc;
  float *state_out, *dstate;
  // workspace; [..][channels] each
  float *carry;   // [rows][segments][states]: a segment's state from zeros, then the state it begins with
  float *back;    // the same of the gradients: of the state before a segment, then of the one it ends with
  float *steps;   // [rows][segments]: sum of delta
  float *starts;  // [rows][chunks][states]: the state before a chunk, from zeros at the segment's begin
  float *until;   // [rows][chunks]: sum of delta from the segment's begin to the chunk
  float *partial; // [parts]: gradients of a, dt_bias and skip
  float *bc;      // [blocks of a group][rows][chunks][groups][states][2][tokens]: parts of the gradients of b and c
  int64_t rows, length, num_states;
  int64_t segments, segment, chunks;  // segments of a row, tokens of a segment, chunks of a row
  int64_t blocks, parts;              // waves side by side in a group's channels, and along rows and segments
  int32_t channels, groups, states, per_group;
  uint32_t by_states;                 // 2^16 / states, rounded up: i / states = i by_states / 2^16 for i < 1024
};

// The part of the work that a workgroup has.
struct Place {
  int64_t row, begin, end, stop;  // tokens of the segment, and where those that count end
  int64_t seg, block;             // block of the group's channels
  int32_t group, c0, count;       // its first channel, its channels
};

__device__ __forceinline__ Place place_of(const Scan &p, int64_t column, int64_t row_and_seg, bool report) {
  Place w;
  w.block = column % p.blocks;
  w.group = int32_t(column / p.blocks);
  w.row = row_and_seg / p.segments;
  w.seg = row_and_seg % p.segments;
  w.c0 = __builtin_amdgcn_readfirstlane(w.group * p.per_group + int32_t(w.block) * kWave);
  w.count = min(int32_t(kWave), p.per_group - int32_t(w.block) * kWave);
  // the same in all lanes, and the compiler is to know
  const int64_t length = __builtin_amdgcn_readfirstlane(
      int32_t(row_length(p.len, w.row, p.length, report && column == 0 && w.seg == 0, p.status)));
  w.begin = w.seg * p.segment;
  w.end = min(w.begin + p.segment, p.length);
  w.stop = max(w.begin, min(w.end, length));
  return w;
}

// delta, from dt + dt_bias: log(1 + e^v) = max(v, 0) + log(1 + e), e = e^-|v|. The logarithm as 2 artanh(s / 2),
// s = e / (1 + e / 2), whose series in s^2 / 4, 1 / 9 at most, keeps the relative precision of small steps: the first
// term that is left out is 2^-25.
__device__ __forceinline__ float log1p_series(float e) {
  const float s = e * __builtin_amdgcn_rcpf(fmaf(e, 0.5f, 1.0f)), q = s * s;
  float r = 1.0f / (13.0f * 4096.0f);
  r = fmaf(r, q, 1.0f / (11.0f * 1024.0f));
  r = fmaf(r, q, 1.0f / (9.0f * 256.0f));
  r = fmaf(r, q, 1.0f / (7.0f * 64.0f));
  r = fmaf(r, q, 1.0f / (5.0f * 16.0f));
  r = fmaf(r, q, 1.0f / (3.0f * 4.0f));
  return fmaf(r * q, s, s);
}
__device__ __forceinline__ float softplus(float v) {
  const float log1 = log1p_series(exp_negative(-fabsf(v)));
  return v <= 0.0f ? log1 : v + log1;  // and what is no number stays that
}
// The same with its slope, 1 / (1 + e^-v).
__device__ __forceinline__ float softplus(float v, float &slope) {
  const float e = exp_negative(-fabsf(v)), log1 = log1p_series(e), d = __builtin_amdgcn_rcpf(1.0f + e);
  slope = v < 0.0f ? e * d : d;
  return v <= 0.0f ? log1 : v + log1;
}

// A rate as the kernels take it. Not below -2^95, which forgets all in a step of 2^-88: the lowest finite values would
// be -inf over ln 2, and a step of 0, as the tokens have that fill a chunk, times that no number.
__device__ __forceinline__ float checked_rate(float a, int32_t *status) {
  if (a <= 0.0f && a > -kInf) return fmaxf(a, -0x1p95f);
  if (status != nullptr) atomicOr(status, RDF2V_STATUS_BAD_VALUE);
  return 0.0f;
}

// Element `offset` of an array: 32 bits of a lane's own beside an address that all lanes have in common.
template <class T>
__device__ __forceinline__ T &lane_of(T *common, uint32_t offset) {
  typedef std::conditional_t<std::is_const_v<T>, const char, char> Byte;
  return *reinterpret_cast<T *>(reinterpret_cast<Byte *>(common) + offset * uint32_t(sizeof(T)));
}

// put(i, load(i)) for i = 0 .. count - 1, eight loads in flight at a time.
template <class Load, class Put>
__device__ __forceinline__ void in_batches(int count, Load load, Put put) {
  constexpr int kBatch = 8;
  for (int first = 0; first < count; first += kBatch) {
    decltype(load(0)) x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) x[k] = load(min(first + k, count - 1));
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (first + k < count) put(first + k, x[k]);
  }
}

// The rates over ln 2, [states][64], and zeros for channels that are not there.
__device__ __forceinline__ void load_rates(const Scan &p, const Place &w, float *rates, bool report) {
  const float *from = p.a + int64_t(w.c0) * p.states;
  in_batches(
      p.states, [&](int k) { return from[min(k * kWave + lane_id(), w.count * p.states - 1)]; },
      [&](int k, float a) {
        const int i = k * kWave + lane_id(), channel = i / p.states, n = i - channel * p.states;
        rates[n * kWave + channel] =
            channel < w.count ? checked_rate(a, report ? p.status : nullptr) * kLog2e : 0.0f;
      });
}

// States [channels][states] of memory from or to [states][64]; null: zeros.
__device__ __forceinline__ void load_states(const Scan &p, const Place &w, const float *from, float *to) {
  if (from == nullptr) {
    for (int n = 0; n < p.states; ++n) to[n * kWave + lane_id()] = 0.0f;
    return;
  }
  from += (w.row * p.channels + w.c0) * p.states;
  in_batches(
      p.states, [&](int k) { return from[min(k * kWave + lane_id(), w.count * p.states - 1)]; },
      [&](int k, float h) {
        const int i = k * kWave + lane_id(), channel = i / p.states, n = i - channel * p.states;
        to[n * kWave + channel] = channel < w.count ? h : 0.0f;
      });
}
__device__ __forceinline__ void store_states(const Scan &p, const Place &w, const float *from, float *to) {
  for (int i = lane_id(); i < w.count * p.states; i += kWave)
    to[(w.row * p.channels + w.c0) * p.states + i] = from[i % p.states * kWave + i / p.states];
}
// The same of the workspace, [states][channels].
__device__ __forceinline__ void load_carry(const Scan &p, const Place &w, const float *from, uint32_t near, float *to) {
  in_batches(
      p.states, [&](int n) { return lane_of(from + int64_t(n) * p.channels + w.c0, near); },
      [&](int n, float h) { to[n * kWave + lane_id()] = lane_id() < w.count ? h : 0.0f; });
}

// A chunk's work is written for N = 4, 8, .. K tokens, the fewest that hold those that count: rows of a few tokens
// leave most of a chunk out, and no token has a branch of its own.
template <int K, class Chunk>
__device__ __forceinline__ void with_tokens(int count, Chunk chunk) {
  if constexpr (K > 4) {
    if (count <= K - 4) {
      with_tokens<K - 4>(count, chunk);
      return;
    }
  }
  chunk(std::integral_constant<int, K>{});
}

// What the lanes of a wave hand to one another through LDS is there after this: a wave's accesses are made in order.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Whether token t of N is known to count, or does. Lanes without a channel go along with the block's first channel's
// values and write nothing.
template <int N>
__device__ __forceinline__ bool counts(int t, int count) {
  return t < N - 3 || t < count;
}

// The lane's channel (`near` the block's first) of a chunk's first `count` tokens; what follows is the last of them
// again. Addresses are made
// one after the other: all at once they would not fit the scalar registers.
template <class T, int N>
__device__ __forceinline__ void load_tokens(const rdf2v_tokens_view &view, const Place &w, uint32_t near, int64_t t0,
                                            int count, T (&x)[N]) {
  const T *base = static_cast<const T *>(view.data);
  int64_t at = w.row * view.row_stride + t0 * view.token_stride + w.c0;
#pragma unroll
  for (int t = 0; t < N; ++t) {
    x[t] = lane_of(base + at, near);
    at += counts<N>(t + 1, count) ? view.token_stride : 0;
    asm volatile("" : "+s"(at));
  }
}

// The same of an output, from token `first` of all rows on.
template <class T, int N>
__device__ __forceinline__ void store_tokens(void *out, int64_t first, int64_t channels, const Place &w, uint32_t near,
                                             int count, const float (&x)[N]) {
  T *base = static_cast<T *>(out);
  int64_t at = first * channels + w.c0;
#pragma unroll
  for (int t = 0; t < N; ++t) {
    if (counts<N>(t, count)) lane_of(base + at, near) = from_f32<T>(x[t]);
    at += channels;
    asm volatile("" : "+s"(at));
  }
}

// b or c of a chunk of K tokens to [states][K] in LDS; zeros for tokens that do not count.
template <class T, int NMAX, int K>
__device__ __forceinline__ void load_heads(const Scan &p, const rdf2v_heads_view &view, const Place &w, int lane,
                                           int64_t t0, int count, float *lds) {
  const T *at = static_cast<const T *>(view.data) + w.row * view.row_stride + t0 * view.token_stride +
                w.group * view.head_stride;
  constexpr int kEach = K * NMAX / kWave;
  T x[kEach];
  asm volatile("" : "+v"(lane));  // offsets are made anew for each chunk: kept, they would cost the registers of four
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = lane + k * kWave, token = i * p.by_states >> 16, n = i - token * p.states;
    x[k] = T(0.0f);
    if (token < count) x[k] = at[token * view.token_stride + n];
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = lane + k * kWave, token = i * p.by_states >> 16, n = i - token * p.states;
    if (token < K) lds[n * K + token] = to_f32(x[k]);
  }
}

// A state's values of a chunk's tokens, the same in every lane.
template <int K, int N>
__device__ __forceinline__ void read_head(const float *lds, int n, float (&x)[N]) {
  typedef float Four __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const Four v = reinterpret_cast<const Four *>(lds + n * K)[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * i + j] = v[j];
  }
}

// delta and delta x of a chunk's tokens; 0 beyond the last that counts: nothing decays and nothing is added.
template <class T, int N>
__device__ __forceinline__ void make_steps(const T (&x)[N], const T (&dt)[N], float bias, int count, float (&delta)[N],
                                           float (&u)[N]) {
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const float d = softplus(to_f32(dt[t]) + bias);
    delta[t] = counts<N>(t, count) ? d : 0.0f;
    u[t] = counts<N>(t, count) ? d * to_f32(x[t]) : 0.0f;
  }
}

__device__ __forceinline__ float silu(float x) { return x * sigmoid(x); }

// The gradients of y of a chunk's tokens.
template <class T, int N>
__device__ __forceinline__ void make_gradients(const T (&dout)[N], const T (&gate)[N], bool gated, int count,
                                               float (&g)[N]) {
#pragma unroll
  for (int t = 0; t < N; ++t) g[t] = counts<N>(t, count) ? to_f32(dout[t]) : 0.0f;
  if (!gated) return;
#pragma unroll
  for (int t = 0; t < N; ++t) g[t] = counts<N>(t, count) ? g[t] * silu(to_f32(gate[t])) : 0.0f;
}

template <class T>
__device__ __forceinline__ void store_zeros(void *out, int64_t from, int64_t to, int64_t row, int64_t length,
                                            int64_t width, int64_t at, int count) {
  T *p = static_cast<T *>(out) + row * length * width + at;
  for (int64_t t = from; t < to; ++t)
    for (int i = lane_id(); i < count; i += kWave) p[t * width + i] = from_f32<T>(0.0f);
}

// What a wave keeps for its channels.
struct Lane {
  int lane, channel;
  uint32_t near;  // what the channel is beyond the block's first
  bool there, gated, skips;  // skips: 0 in the place of a skip that is not there would make no number of infinity
  float bias, skip;
  __device__ __forceinline__ Lane(const Scan &p, const Place &w)
      : lane(lane_id()), channel(w.c0 + (lane < w.count ? lane : 0)), near(lane < w.count ? lane : 0),
        there(lane < w.count), gated(p.gate.data != nullptr), skips(p.skip != nullptr),
        bias(p.dt_bias != nullptr ? p.dt_bias[channel] : 0.0f), skip(p.skip != nullptr ? p.skip[channel] : 0.0f) {}
};

// The outputs of a segment. A wave's barriers cost nothing: it is alone in its workgroup. Bound by the issue of vector
// instructions: 9 for a token's state, its share of the token's own (the step's logarithm, conversions, the gate)
// among them. 20,011 tokens of 2,048 channels by 16 states: 208 us, 94 % of the issue with exponentials as two
// instructions each; 4,000 ragged rows of 17 tokens by 256 channels: 78 us, 81 %, 14 instructions for a token's state.
template <class T, int NMAX>
__global__ __launch_bounds__(kWave, NMAX <= 16 ? 4 : 1) void scan_out_kernel(Scan p, int64_t first) {
  __shared__ float rates[NMAX * kWave], held[NMAX * kWave], b[NMAX * kTokens], c[NMAX * kTokens];
  const int64_t columns = p.blocks * p.groups, column = (first + blockIdx.x) % columns,
                part = (first + blockIdx.x) / columns;
  Place w = place_of(p, column, 0, false);
  const Lane me(p, w);
  load_rates(p, w, rates, part == 0);
  for (int64_t item = part; item < p.rows * p.segments; item += p.parts) {
    w = place_of(p, column, item, me.lane == 0);
    __syncthreads();
    if (p.segments == 1) {
      load_states(p, w, p.state, held);
    } else {
      load_carry(p, w, p.carry + item * p.states * p.channels, me.near, held);
    }
    for (int64_t t0 = w.begin; t0 < w.stop; t0 += kTokens) {
      const int count = int(min(int64_t(kTokens), w.stop - t0));
      with_tokens<kTokens>(count, [&](auto tokens) {
        constexpr int N = tokens();
        T x[N], dt[N], gate[N];
        load_tokens(p.x, w, me.near, t0, count, x);
        load_tokens(p.dt, w, me.near, t0, count, dt);
        if (me.gated) load_tokens(p.gate, w, me.near, t0, count, gate);
        __syncthreads();
        load_heads<T, NMAX, kTokens>(p, p.b, w, me.lane, t0, count, b);
        load_heads<T, NMAX, kTokens>(p, p.c, w, me.lane, t0, count, c);
        float delta[N], u[N], y[N];
        make_steps(x, dt, me.bias, count, delta, u);
#pragma unroll
        for (int t = 0; t < N; ++t) y[t] = me.skips ? me.skip * to_f32(x[t]) : 0.0f;
        __syncthreads();
        for (int n = 0; n < p.states; ++n) {
          const float rate = rates[n * kWave + me.lane];
          float h = held[n * kWave + me.lane], bn[N], cn[N];
          read_head<kTokens>(b, n, bn);
          read_head<kTokens>(c, n, cn);
#pragma unroll
          for (int t = 0; t < N; ++t) {
            h = fmaf(exp2_fast(delta[t] * rate), h, u[t] * bn[t]);
            y[t] = fmaf(h, cn[t], y[t]);
          }
          held[n * kWave + me.lane] = h;
        }
        if (me.gated)
#pragma unroll
          for (int t = 0; t < N; ++t) y[t] *= silu(to_f32(gate[t]));
        if (me.there) store_tokens<T>(p.out, w.row * p.length + t0, p.channels, w, me.near, count, y);
      });
    }
    store_zeros<T>(p.out, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
    if (p.segments > 1 || p.state_out == nullptr) continue;
    __syncthreads();
    store_states(p, w, held, p.state_out);
  }
}

// The states that a segment ends with, from zeros; BACK, for the gradients: the states before its chunks (from the
// row's own state where there is one segment), and the gradient that its outputs give the state before it,
// sum_t (product of the decays up to t) c_t g_t, which needs no second way through the tokens. 20,011 tokens of 2,048
// channels by 16 states: 154 us, 88 % of the issue; 4 rows of 4,096 tokens, BACK: 284 us, 66 %. Reading a chunk's
// inputs while the one before is worked on takes the registers of a wave (164 us for 157; BACK 261 for 280, a hundredth
// of a training case).
template <class T, int NMAX, bool BACK, bool CUT>
__global__ __launch_bounds__(kWave) void scan_states_kernel(Scan p, int64_t first) {
  constexpr bool kBoth = BACK && CUT;
  constexpr int K = BACK ? kBackTokens : kTokens;
  __shared__ float rates[NMAX * kWave], held[NMAX * kWave], b[NMAX * K];
  __shared__ float grad[kBoth ? NMAX * kWave : 1], c[kBoth ? NMAX * K : 1];
  const int64_t columns = p.blocks * p.groups, column = (first + blockIdx.x) % columns,
                part = (first + blockIdx.x) / columns;
  Place w = place_of(p, column, 0, false);
  const Lane me(p, w);
  const int lane = me.lane;
  load_rates(p, w, rates, false);
  for (int64_t item = part; item < p.rows * p.segments; item += p.parts) {
    w = place_of(p, column, item, false);
    __syncthreads();
    load_states(p, w, CUT ? nullptr : p.state, held);
    if (kBoth)
      for (int n = 0; n < p.states; ++n) grad[n * kWave + lane] = 0.0f;
    float sum = 0.0f;  // of delta
    // without segments the state after the last chunk is not needed
    const int64_t stop = CUT ? w.stop : w.stop - K;
    for (int64_t t0 = w.begin; t0 < stop; t0 += K) {
      const int count = int(min(int64_t(K), w.stop - t0));
      const int64_t chunk = w.row * p.chunks + t0 / K;
      with_tokens<K>(count, [&](auto tokens) {
        constexpr int N = tokens();
        T x[N], dt[N];
        float delta[N], u[N], g[N];
        load_tokens(p.x, w, me.near, t0, count, x);
        load_tokens(p.dt, w, me.near, t0, count, dt);
        __syncthreads();
        load_heads<T, NMAX, K>(p, p.b, w, lane, t0, count, b);
        if constexpr (kBoth) {
          T o[N], gate[N];
          load_tokens(p.dout, w, me.near, t0, count, o);
          if (me.gated) load_tokens(p.gate, w, me.near, t0, count, gate);
          load_heads<T, NMAX, K>(p, p.c, w, lane, t0, count, c);
          make_gradients(o, gate, me.gated, count, g);
        }
        make_steps(x, dt, me.bias, count, delta, u);
        __syncthreads();
        if (kBoth && me.there) lane_of(p.until + chunk * p.channels + w.c0, me.near) = sum;
        const float before = sum;
        if constexpr (CUT)
#pragma unroll
          for (int t = 0; t < N; ++t) sum += delta[t];
        for (int n = 0; n < p.states; ++n) {
          const float rate = rates[n * kWave + lane];
          float h = held[n * kWave + lane], bn[N];
          if (kBoth && me.there) lane_of(p.starts + (chunk * p.states + n) * p.channels + w.c0, me.near) = h;
          read_head<K>(b, n, bn);
          if constexpr (kBoth) {
            float cn[N], most = exp2_fast(before * rate), r = grad[n * kWave + lane];
            read_head<K>(c, n, cn);
#pragma unroll
            for (int t = 0; t < N; ++t) {
              const float e = exp2_fast(delta[t] * rate);
              h = fmaf(e, h, u[t] * bn[t]);
              most *= e;
              r = fmaf(most, g[t] * cn[t], r);
            }
            grad[n * kWave + lane] = r;
          } else {
#pragma unroll
            for (int t = 0; t < N; ++t) h = fmaf(exp2_fast(delta[t] * rate), h, u[t] * bn[t]);
          }
          held[n * kWave + lane] = h;
          if (BACK && !CUT && me.there)
            lane_of(p.starts + ((chunk + 1) * p.states + n) * p.channels + w.c0, me.near) = h;
        }
      });
    }
    if (!CUT || !me.there) continue;
    lane_of(p.steps + item * p.channels + w.c0, me.near) = sum;
    for (int n = 0; n < p.states; ++n) {
      const int64_t at = (item * p.states + n) * p.channels + w.c0;
      lane_of(p.carry + at, me.near) = held[n * kWave + lane];
      if (kBoth) lane_of(p.back + at, me.near) = grad[n * kWave + lane];
    }
  }
}

// A row's states from segment to segment, a thread to a channel's state; BACK: also their gradients, backwards. Each
// segment's values are read ahead of the chain that needs them.
template <bool BACK>
__global__ __launch_bounds__(kThreads) void scan_join_kernel(Scan p, int64_t first) {
  constexpr int kAhead = 16;
  const int64_t item = (first + blockIdx.x) * kThreads + threadIdx.x;
  if (item >= p.rows * p.states * p.channels) return;
  const int64_t channel = item % p.channels, n = item / p.channels % p.states, row = item / p.channels / p.states;
  const float rate = checked_rate(p.a[channel * p.states + n], nullptr) * kLog2e;
  const int64_t held = (row * p.channels + channel) * p.states + n;
  const float *steps = p.steps + row * p.segments * p.channels + channel;
  const int64_t stride = int64_t(p.states) * p.channels, at = row * p.segments * stride + n * p.channels + channel;
  // From x on through the segments s, s + by, ..: `values` holds what each adds, and then what each begins with.
  const auto chain = [&](float x, float *values, int64_t s, int64_t by) {
    for (int64_t left = p.segments; left > 0; left -= kAhead) {
      const int count = int(min(left, int64_t(kAhead)));
      float mine[kAhead], decay[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int64_t from = s + by * min(k, count - 1);
        mine[k] = values[from * stride];
        decay[k] = steps[from * p.channels];
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (k >= count) break;
        values[(s + by * k) * stride] = x;
        x = fmaf(exp2_fast(decay[k] * rate), x, mine[k]);
      }
      s += by * kAhead;
    }
    return x;
  };
  const float h = chain(p.state != nullptr ? p.state[held] : 0.0f, p.carry + at, 0, 1);
  if (BACK)
    chain(p.dstate_out != nullptr ? p.dstate_out[held] : 0.0f, p.back + at, p.segments - 1, -1);
  else if (p.state_out != nullptr)
    p.state_out[held] = h;
}

// Sums over a wave's lanes of sixteen values at once: value lane / 4's in each lane. Every step adds two lanes of
// each value and leaves half as many values in a lane, so that 35 instructions do: two values meet in a swap of the
// wave's halves, then of rows, then (a lane's bit chooses what it keeps) of halves and quarters of rows, and quarters
// are added up. Matrix products with unit columns take 3 instructions a value less, but the f32 ones keep the vector
// instructions waiting, 8 for each product, and spread what is no number over all of the columns.
__device__ __forceinline__ float sixteen_sums(const float (&v)[16]) {
  const int lane = lane_id();
  float w[8], x[4], y[2];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 8]), false, false);
    w[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(w[i]), __float_as_uint(w[i + 4]), false, false);
    x[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
#define RDF2V_DPP(VALUE, CTRL) \
  __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(VALUE), CTRL, 0xf, 0xf, false))
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float keep = lane & 8 ? x[i + 2] : x[i], give = lane & 8 ? x[i] : x[i + 2];
    y[i] = keep + RDF2V_DPP(give, 0x128);  // row_ror:8
  }
  const float keep = lane & 4 ? y[1] : y[0], give = lane & 4 ? y[0] : y[1];
  float z = keep + RDF2V_DPP(give, 0x141);  // row_half_mirror
  z += RDF2V_DPP(z, 0xb1);                  // quad_perm:[1,0,3,2]
  z += RDF2V_DPP(z, 0x4e);                  // quad_perm:[2,3,0,1]
#undef RDF2V_DPP
  return z;
}

// Calls each(constant) for N - 1, N - 2, .. 0.
template <int N, class Each>
__device__ __forceinline__ void backwards(Each each) {
  if constexpr (N > 0) {
    each(std::integral_constant<int, N - 1>{});
    backwards<N - 1>(each);
  }
}

// Gradients of a segment, chunk after chunk from its end; a wave takes several segments of its channels in turn
// and holds the parameters' gradients meanwhile. 25 instructions for a token's state, 4 of them the sums over channels.
// 4 rows of 4,096 tokens by 2,048 channels of 16 states: 541 us, 73 % of the issue, the rest waits of the two waves
// that a SIMD's registers hold. Three, with segments for them, took 570 us for 589, but the states 352 for 279.
template <class T, int NMAX>
__global__ __launch_bounds__(kGang *kWave, NMAX <= 32 ? 2 : 1) void scan_backward_kernel(Scan p, int64_t first) {
  constexpr int K = kBackTokens, kStarts = 4;
  // what a segment begins with; of more states it would cost every other wave (64: 3,855 us for 2,529)
  constexpr bool kHeld = NMAX <= 16;
  __shared__ float rates[NMAX * kWave], all_grads[kGang][NMAX * kWave], all_da[kGang][NMAX * kWave];
  __shared__ float all_held[kGang][kHeld ? NMAX * kWave : 1], all_b[kGang][NMAX * K], all_c[kGang][NMAX * K];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  float *grads = all_grads[wave], *da = all_da[wave], *held = all_held[wave], *b = all_b[wave], *c = all_c[wave];
  const int64_t columns = p.blocks * p.groups, column = (first + blockIdx.x) % columns,
                part = (first + blockIdx.x) / columns * kGang + wave;
  const bool cut = p.segments > 1;
  Place w = place_of(p, column, 0, false);
  const Lane me(p, w);
  const int lane = me.lane;
  const bool whole = w.count == kWave;
  if (wave == 0) load_rates(p, w, rates, part == 0);
  __syncthreads();
  if (part >= p.parts) return;
  for (int n = 0; n < p.states; ++n) da[n * kWave + lane] = 0.0f;
  float ddt_bias = 0.0f, dskip = 0.0f;
  for (int64_t item = part; item < p.rows * p.segments; item += p.parts) {
    w = place_of(p, column, item, lane == 0);
    wave_sync();
    if (!cut) {
      load_states(p, w, p.dstate_out, grads);
    } else {
      load_carry(p, w, p.back + item * p.states * p.channels, me.near, grads);
      if (kHeld) load_carry(p, w, p.carry + item * p.states * p.channels, me.near, held);
    }
    const float *carry = p.carry + item * p.states * p.channels + w.c0;
    const int64_t last = w.begin + (w.stop - w.begin - 1) / K * K;  // chunk
    for (int64_t t0 = last; t0 >= w.begin && w.begin < w.stop; t0 -= K) {
      const int count = int(min(int64_t(K), w.stop - t0));
      const int64_t chunk = w.row * p.chunks + t0 / K, token = w.row * p.length + t0;
      // the states before the chunk: the row's, or its own and what the segment begins with
      const bool own = cut || t0 > w.begin;
      const float *starts = own ? p.starts + chunk * p.states * p.channels + w.c0
                            : p.state != nullptr ? p.state + (w.row * p.channels + w.c0) * p.states
                                                 : nullptr;
      const int64_t stride = own ? p.channels : 1;
      const uint32_t near = own ? me.near : me.near * uint32_t(p.states);
      const float until = cut ? lane_of(p.until + chunk * p.channels + w.c0, me.near) : 0.0f;
      float *sums = p.bc + (((w.block * p.rows * p.chunks + chunk) * p.groups + w.group) * p.states) * (2 * K);
      with_tokens<K>(count, [&](auto tokens) {
        constexpr int N = tokens();
        // four states' at a time, read while the four before are worked on
        const auto load_starts = [&](int n0, float (&from)[kStarts], float (&begin)[kStarts]) {
#pragma unroll
          for (int k = 0; k < kStarts; ++k) {
            const int n = min(n0 + k, p.states - 1);
            from[k] = starts != nullptr ? lane_of(starts + n * stride, near) : 0.0f;
            begin[k] = !kHeld && cut ? lane_of(carry + int64_t(n) * p.channels, me.near) : 0.0f;
          }
        };
        float from[kStarts], begin[kStarts];
        load_starts(0, from, begin);
        float xs[N], delta[N], slope[N], u[N], g[N], y[N], dgate[N], du[N] = {}, dd[N] = {};
        wave_sync();
        {
          T x[N], dt[N], gate[N], o[N];
          load_tokens(p.x, w, me.near, t0, count, x);
          load_tokens(p.dt, w, me.near, t0, count, dt);
          if (me.gated) load_tokens(p.gate, w, me.near, t0, count, gate);
          load_tokens(p.dout, w, me.near, t0, count, o);
          load_heads<T, NMAX, K>(p, p.b, w, lane, t0, count, b);
          load_heads<T, NMAX, K>(p, p.c, w, lane, t0, count, c);
#pragma unroll
          for (int t = 0; t < N; ++t) {
            const bool on = counts<N>(t, count);
            const float d = softplus(to_f32(dt[t]) + me.bias, slope[t]);
            xs[t] = to_f32(x[t]);
            delta[t] = on ? d : 0.0f;
            u[t] = on ? d * xs[t] : 0.0f;
            g[t] = on ? to_f32(o[t]) : 0.0f;
            dgate[t] = 0.0f;
          }
          if (me.gated)
#pragma unroll
            for (int t = 0; t < N; ++t) {
              const float z = to_f32(gate[t]), s = sigmoid(z);
              dgate[t] = g[t] * silu_slope(z, s);
              g[t] = counts<N>(t, count) ? g[t] * (z * s) : 0.0f;
            }
#pragma unroll
          for (int t = 0; t < N; ++t) {
            dskip = counts<N>(t, count) ? fmaf(g[t], xs[t], dskip) : dskip;
            y[t] = me.skips ? me.skip * xs[t] : 0.0f;
          }
        }
        wave_sync();
        const auto work = [&](int n, float start, float first) {
          const float rate = rates[n * kWave + lane];
          if (kHeld && cut) first = held[n * kWave + lane];
          const float h0 = cut ? fmaf(exp2_fast(until * rate), first, start) : start;
          float bn[N], cn[N], e[N], h[N];
          read_head<K>(b, n, bn);
          read_head<K>(c, n, cn);
#pragma unroll
          for (int t = 0; t < N; ++t) {
            e[t] = exp2_fast(delta[t] * rate);
            h[t] = fmaf(e[t], t > 0 ? h[t > 0 ? t - 1 : 0] : h0, u[t] * bn[t]);
            y[t] = fmaf(h[t], cn[t], y[t]);
          }
          float r = grads[n * kWave + lane], rates_sum = 0.0f, each[2 * K] = {};
          backwards<N>([&](auto token) {
            constexpr int t = token();
            r = fmaf(g[t], cn[t], r);
            each[t] = r * u[t];
            each[K + t] = g[t] * h[t];
            du[t] = fmaf(r, bn[t], du[t]);
            r *= e[t];
            const float q = r * (t > 0 ? h[t > 0 ? t - 1 : 0] : h0);
            dd[t] = fmaf(q, rate, dd[t]);
            // of the tokens that count: what the row leaves behind, infinite or no number, is no part of the sum
            rates_sum = counts<N>(t, count) ? fmaf(q, delta[t], rates_sum) : rates_sum;
          });
          grads[n * kWave + lane] = r;
          da[n * kWave + lane] += rates_sum;
          if (!whole) {
            asm volatile("");  // a branch, not selects for all
#pragma unroll
            for (int i = 0; i < 2 * K; ++i) each[i] = me.there ? each[i] : 0.0f;
          }
          const float total = sixteen_sums(each);
          if (lane % 4 == 0) lane_of(sums + n * 2 * K, uint32_t(lane) / 4) = total;
        };
        for (int n0 = 0; n0 < p.states; n0 += kStarts) {
          float ahead[kStarts], begin_ahead[kStarts];
          load_starts(n0 + kStarts, ahead, begin_ahead);
#pragma unroll
          for (int k = 0; k < kStarts; ++k)
            if (n0 + k < p.states) work(n0 + k, from[k], begin[k]);
#pragma unroll
          for (int k = 0; k < kStarts; ++k) from[k] = ahead[k], begin[k] = begin_ahead[k];
        }
#pragma unroll
        for (int t = 0; t < N; ++t) {
          dd[t] = fmaf(dd[t], kLn2, xs[t] * du[t]) * slope[t];
          du[t] = fmaf(delta[t], du[t], me.skips ? me.skip * g[t] : 0.0f);
          y[t] *= dgate[t];
          if (counts<N>(t, count)) ddt_bias += dd[t];
        }
        if (!me.there) return;
        store_tokens<T>(p.dx, token, p.channels, w, me.near, count, du);
        store_tokens<T>(p.ddt, token, p.channels, w, me.near, count, dd);
        if (me.gated) store_tokens<T>(p.dgate, token, p.channels, w, me.near, count, y);
      });
    }
    store_zeros<T>(p.dx, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
    store_zeros<T>(p.ddt, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
    if (me.gated) store_zeros<T>(p.dgate, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
    if (w.seg == 0 && p.dstate != nullptr) {
      wave_sync();
      store_states(p, w, grads, p.dstate);
    }
  }
  float *partial = p.partial + part * p.channels * (p.states + 2);
  wave_sync();
  for (int i = lane; i < w.count * p.states; i += kWave)
    partial[int64_t(w.c0) * p.states + i] = da[i % p.states * kWave + i / p.states];
  if (!me.there) return;
  partial[int64_t(p.channels) * p.states + me.channel] = ddt_bias;
  partial[int64_t(p.channels) * (p.states + 1) + me.channel] = dskip;
}

// Gradients of b and c: the sums over a group's blocks of channels, in order, from [states][2][tokens of a chunk] to
// [tokens][states]. A thread to a value of the output.
template <class T>
__global__ __launch_bounds__(kThreads) void scan_bc_kernel(Scan p, int64_t first) {
  constexpr int K = kBackTokens;
  const int64_t item = (first + blockIdx.x) * kThreads + threadIdx.x;
  if (item >= p.rows * p.length * p.groups * p.states) return;
  const int64_t n = item % p.states, head = item / p.states, group = head % p.groups, token = head / p.groups;
  const int64_t row = token / p.length, t = token % p.length;
  float db = 0.0f, dc = 0.0f;
  if (t < row_length(p.len, row, p.length, false, nullptr)) {
    const int64_t all = p.rows * p.chunks * p.groups * p.states * (2 * K);
    const float *from =
        p.bc + (((row * p.chunks + t / K) * p.groups + group) * p.states + n) * (2 * K) + t % K;
    for (int64_t k = 0; k < p.blocks; ++k) {
      db += from[k * all];
      dc += from[k * all + K];
    }
  }
  static_cast<T *>(p.db)[item] = from_f32<T>(db);
  static_cast<T *>(p.dc)[item] = from_f32<T>(dc);
}

// One token more. `lanes` threads, a power of two, take a channel's states, four neighbouring ones at a time (WHOLE:
// the last of them has four, too); a workgroup takes a tile of channels of kStepRows rows, whose loads are all in
// flight at once, and the rates once for them. HBM-bound: states are read and written. 512 rows of 2,048 channels by 16
// states: 32 us, 143 MB; by 17 states 74 us, and 147 with a thread to each state.
constexpr int kStepRows = 4;
template <class T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void scan_step_kernel(Scan p, int lanes, int64_t tiles, int64_t first) {
  constexpr int V = 4;
  const int64_t block = first + blockIdx.x, row0 = block / tiles * kStepRows;
  const int lane = threadIdx.x % lanes;
  const int64_t at = block % tiles * (kThreads / lanes) + threadIdx.x / lanes;
  const bool there = at < p.channels;
  const int64_t channel = there ? at : p.channels - 1, group = channel / p.per_group;
  const int rows = int(min(int64_t(kStepRows), p.rows - row0));
  const float bias = p.dt_bias != nullptr ? p.dt_bias[channel] : 0.0f;
  const float skip = p.skip != nullptr ? p.skip[channel] : 0.0f;
  int64_t from[kStepRows];
  float x[kStepRows], d[kStepRows], z[kStepRows], y[kStepRows] = {};
#pragma unroll
  for (int r = 0; r < kStepRows; ++r) {
    const int64_t row = row0 + min(r, rows - 1);
    from[r] = p.parents != nullptr ? p.parents[row] : row;
    x[r] = to_f32(static_cast<const T *>(p.x.data)[row * p.x.row_stride + channel]);
    d[r] = to_f32(static_cast<const T *>(p.dt.data)[row * p.dt.row_stride + channel]);
    z[r] = p.gate.data != nullptr
               ? to_f32(static_cast<const T *>(p.gate.data)[row * p.gate.row_stride + channel])
               : 0.0f;
  }
  for (int n = lane * V; n < p.states; n += lanes * V) {
    float rate[V], h[kStepRows][V], b[kStepRows][V], c[kStepRows][V];
    const int count = WHOLE ? V : min(V, p.states - n);
    load_values<float, V>(p.a + channel * p.states + n, count, rate);
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
      const int64_t row = row0 + min(r, rows - 1);
      const bool known = from[r] >= 0 && from[r] < p.num_states;
      load_values<float, V>(p.state + ((known ? from[r] : 0) * p.channels + channel) * p.states + n,
                            p.num_states > 0 ? count : 0, h[r]);
      load_values<T, V>(static_cast<const T *>(p.b.data) + row * p.b.row_stride + group * p.b.head_stride + n, count,
                        b[r]);
      load_values<T, V>(static_cast<const T *>(p.c.data) + row * p.c.row_stride + group * p.c.head_stride + n, count,
                        c[r]);
#pragma unroll
      for (int i = 0; i < V; ++i) h[r][i] = known ? h[r][i] : 0.0f;
    }
    if (n == lane * V)
#pragma unroll
      for (int r = 0; r < kStepRows; ++r) d[r] = softplus(d[r] + bias);
#pragma unroll
    for (int i = 0; i < V; ++i) rate[i] = checked_rate(rate[i], row0 == 0 ? p.status : nullptr) * kLog2e;
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
      const float u = d[r] * x[r];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!WHOLE && i >= count) break;  // 0 times an infinite u would be no number
        h[r][i] = fmaf(exp2_fast(d[r] * rate[i]), h[r][i], u * b[r][i]);
        y[r] = fmaf(h[r][i], c[r][i], y[r]);
      }
      if (there && r < rows)
        store_values<float, V>(p.state_out + ((row0 + r) * p.channels + channel) * p.states + n, count, h[r]);
    }
  }
#pragma unroll
  for (int r = 0; r < kStepRows; ++r) {
    for (int m = lanes / 2; m > 0; m /= 2) y[r] += __shfl_xor(y[r], m, kWave);
    if (r >= rows || lane != 0 || !there) continue;
    if (channel == 0 && p.status != nullptr && (from[r] < 0 || from[r] >= p.num_states))
      atomicOr(p.status, RDF2V_STATUS_ID_OUT_OF_RANGE);
    if (p.skip != nullptr) y[r] = fmaf(skip, x[r], y[r]);
    if (p.gate.data != nullptr) y[r] *= silu(z[r]);
    static_cast<T *>(p.out)[(row0 + r) * p.channels + channel] = from_f32<T>(y[r]);
  }
}

Scan base(const rdf2v_scan &a, const ScanInputs &in, int32_t *status) {
  Scan p{};
  p.x = in.x;
  p.dt = in.dt;
  p.gate = in.gate;
  p.b = in.b;
  p.c = in.c;
  p.a = a.a;
  p.dt_bias = a.dt_bias;
  p.skip = a.skip;
  p.len = a.len;
  p.status = status;
  p.rows = a.rows;
  p.length = a.length;
  p.channels = a.channels;
  p.groups = a.groups;
  p.states = a.states;
  p.per_group = a.channels / a.groups;
  p.blocks = (p.per_group + kWave - 1) / kWave;
  p.by_states = (65536u + uint32_t(a.states) - 1) / uint32_t(a.states);
  return p;
}

// Waves along rows and segments, of at most `most` in all.
int64_t parts_of(const Scan &p, int64_t most) {
  return std::max<int64_t>(1, std::min(p.rows * p.segments, most / (p.blocks * p.groups)));
}

// Sets how many tokens a segment has, and how many segments, `segments` or fewer, that makes.
void cut_rows(Scan &p, int64_t segments, int64_t chunk) {
  p.segment = (p.length + segments - 1) / segments;
  p.segment = std::max(chunk, (p.segment + chunk - 1) / chunk * chunk);
  p.segments = std::max<int64_t>(1, (p.length + p.segment - 1) / p.segment);
}

constexpr int64_t kSimds = 1024;
constexpr int64_t kShortest = 32;  // tokens of a segment at least

// Forward rows are cut where a wave to a row's column of channels is less than one to a SIMD, as it takes a second look
// at all tokens: into as many segments as there are waves that the registers let the chip have at once, four to a SIMD.
void plan_forward(Scan &p) {
  const int64_t whole = std::max<int64_t>(1, p.rows * p.blocks * p.groups);
  const int64_t segments = whole < kSimds ? std::min(4 * kSimds / whole, p.length / kShortest) : 1;
  cut_rows(p, std::max<int64_t>(1, segments), kTokens);
  p.parts = parts_of(p, 8 * kSimds);
}

// The gradients look at all tokens twice anyway, and their waves, two to a SIMD, take segments in turn. Where whole
// rows are fewer: of the numbers of segments that fill 1, 2, .. turns the one that gives the busiest wave the fewest
// tokens, with 8 for what a segment costs by itself; a wave alone on its SIMD takes three quarters of the time, and
// rows that are cut an eighth more. Rows of 256 tokens by 1,024 channels, 16 states, bf16: calls with 64 of them take 521 us
// whole and 464 cut, 80 651 and 584, 110 695 and 720. With more rows cutting costs (130 rows of 126 tokens: 471 and 516).
void plan_backward(Scan &p) {
  const int64_t most = 2 * kSimds, columns = p.blocks * p.groups, rows = std::max<int64_t>(1, p.rows);
  const auto cost = [&](int64_t segments) {
    cut_rows(p, segments, kBackTokens);
    p.parts = parts_of(p, most);
    const int64_t turns = (rows * p.segments + p.parts - 1) / p.parts;
    return turns * (p.segment + 8) * (p.parts * columns <= kSimds ? 3 : 4) * (p.segments > 1 ? 9 : 8);
  };
  int64_t best = 1, least = cost(1);
  for (int64_t turns = 1; turns <= 8 && rows * columns < most; ++turns) {
    const int64_t segments = std::min(turns * std::max<int64_t>(1, most / columns) / rows, p.length / kShortest);
    if (segments < 2) continue;
    const int64_t of = cost(segments);
    if (of < least) best = segments, least = of;
  }
  cost(best);
}

// Segments of a row, chunks, the waves along rows and segments, and where the workspace's arrays lie; its bytes.
size_t plan(Scan &p, bool backward, void *workspace) {
  backward ? plan_backward(p) : plan_forward(p);
  p.chunks = (p.length + kBackTokens - 1) / kBackTokens;
  size_t bytes = 0;
  const auto take = [&](float *&at, int64_t count) {
    at = workspace != nullptr ? reinterpret_cast<float *>(static_cast<char *>(workspace) + bytes) : nullptr;
    bytes += align_up(size_t(count) * sizeof(float), 256);
  };
  const bool cut = p.segments > 1;
  if (cut) {
    take(p.carry, p.rows * p.segments * p.states * p.channels);
    take(p.steps, p.rows * p.segments * p.channels);
  }
  if (!backward) return bytes;
  if (cut) {
    take(p.back, p.rows * p.segments * p.states * p.channels);
    take(p.until, p.rows * p.chunks * p.channels);
  }
  if (p.chunks > 1) take(p.starts, p.rows * p.chunks * p.states * p.channels);
  if (p.rows > 0) take(p.partial, p.parts * p.channels * (p.states + 2));
  take(p.bc, p.blocks * p.rows * p.chunks * p.groups * p.states * 2 * kBackTokens);
  return bytes;
}

// Calls launch with a value of the element type and a constant for the most states. Shared memory sets how many waves
// there are: 16 states leave four to a SIMD (two in the gradients, by their registers), 32 two, 64 one. 4 rows of 4,096
// tokens by 1,024 channels of 24 states: a call takes 240 us by the kernels for 32, 402 by those for 64.
template <class Launch>
rdf2v_status with_types(int dtype, int states, Launch launch) {
  const auto sized = [&](auto t) {
    if (states <= 16) return launch(t, std::integral_constant<int, 16>{});
    if (states <= 32) return launch(t, std::integral_constant<int, 32>{});
    return launch(t, std::integral_constant<int, 64>{});
  };
  return dtype == RDF2V_BF16 ? sized(bf16{}) : sized(float{});
}

// Calls launch for the waves of a call.
template <class Launch>
rdf2v_status for_waves(const Scan &p, Launch launch) {
  return for_each_launch(p.parts * p.blocks * p.groups, kWave, 1, [&](int64_t first, int64_t count) {
    launch(first, dim3(unsigned(count)));
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

template <bool BACK, bool CUT>
rdf2v_status launch_states(Scan p, int dtype, hipStream_t stream) {
  p.parts = parts_of(p, 8192);
  return with_types(dtype, p.states, [&](auto t, auto most) {
    return for_waves(p, [&](int64_t first, dim3 grid) {
      scan_states_kernel<decltype(t), most(), BACK, CUT><<<grid, dim3(kWave), 0, stream>>>(p, first);
    });
  });
}

template <bool BACK>
rdf2v_status launch_join(const Scan &p, hipStream_t stream) {
  const int64_t blocks = (p.rows * p.states * p.channels + kThreads - 1) / kThreads;
  return for_each_launch(blocks, kThreads, 1, [&](int64_t first, int64_t count) {
    scan_join_kernel<BACK><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

}  // namespace

size_t selective_scan_workspace_bytes(const rdf2v_scan &a, bool backward) {
  Scan p = base(a, {}, nullptr);
  return plan(p, backward, nullptr);
}

rdf2v_status launch_selective_scan(const rdf2v_scan &a, const ScanInputs &in, const float *state, void *out,
                                   float *state_out, void *workspace, int32_t *status_dev, hipStream_t stream) {
  Scan p = base(a, in, status_dev);
  p.state = state;
  p.out = out;
  p.state_out = state_out;
  plan(p, false, workspace);
  if (p.segments > 1) {
    rdf2v_status st = launch_states<false, true>(p, a.dtype, stream);
    if (st == RDF2V_OK) st = launch_join<false>(p, stream);
    if (st != RDF2V_OK) return st;
  }
  return with_types(a.dtype, p.states, [&](auto t, auto most) {
    return for_waves(p, [&](int64_t first, dim3 grid) {
      scan_out_kernel<decltype(t), most()><<<grid, dim3(kWave), 0, stream>>>(p, first);
    });
  });
}

rdf2v_status launch_selective_scan_backward(const rdf2v_scan &a, const ScanInputs &in, const rdf2v_tokens_view &dout,
                                            const float *state, const float *dstate_out,
                                            const rdf2v_scan_gradients &grads, void *workspace, int32_t *status_dev,
                                            hipStream_t stream) {
  Scan p = base(a, in, status_dev);
  p.dout = dout;
  p.state = state;
  p.dstate_out = dstate_out;
  p.dx = grads.dx;
  p.ddt = grads.ddt;
  p.dgate = grads.dgate;
  p.db = grads.db;
  p.dc = grads.dc;
  p.dstate = grads.dstate;
  plan(p, true, workspace);
  rdf2v_status st = RDF2V_OK;
  if (p.rows > 0) {
    if (p.segments > 1) {
      st = launch_states<true, true>(p, a.dtype, stream);
      if (st == RDF2V_OK) st = launch_join<true>(p, stream);
    } else if (p.chunks > 1) {
      st = launch_states<true, false>(p, a.dtype, stream);
    }
    if (st != RDF2V_OK) return st;
    st = with_types(a.dtype, p.states, [&](auto t, auto most) {
      const int64_t gangs = (p.parts + kGang - 1) / kGang * p.blocks * p.groups;
      return for_each_launch(gangs, kGang * kWave, 1, [&](int64_t first, int64_t count) {
        scan_backward_kernel<decltype(t), most()><<<dim3(unsigned(count)), dim3(kGang * kWave), 0, stream>>>(p, first);
        RDF2V_LAUNCH_CHECK();
        return RDF2V_OK;
      });
    });
    if (st != RDF2V_OK) return st;
    if (p.length > 0) {
      const int64_t blocks = (p.rows * p.length * p.groups * p.states + kThreads - 1) / kThreads;
      st = for_each_launch(blocks, kThreads, 1, [&](int64_t first, int64_t count) {
        if (a.dtype == RDF2V_BF16)
          scan_bc_kernel<bf16><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
        else
          scan_bc_kernel<float><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
        RDF2V_LAUNCH_CHECK();
        return RDF2V_OK;
      });
      if (st != RDF2V_OK) return st;
    }
  }
  return launch_part_sums({p.partial, p.rows > 0 ? p.parts : 0,
                           {int64_t(p.channels) * p.states, p.channels, p.channels},
                           {grads.da, grads.ddt_bias, grads.dskip}}, stream);
}

rdf2v_status launch_selective_scan_step(const rdf2v_scan &a, const ScanInputs &in, const float *state,
                                        int64_t num_states, const int32_t *parents, void *out, float *state_out,
                                        int32_t *status_dev, hipStream_t stream) {
  Scan p = base(a, in, status_dev);
  p.state = state;
  p.num_states = num_states;
  p.parents = parents;
  p.out = out;
  p.state_out = state_out;
  const bool whole = p.states % 4 == 0;
  int lanes = 1;
  while (lanes < kWave && lanes * 4 < p.states) lanes *= 2;
  const int64_t per = kThreads / lanes, tiles = (p.channels + per - 1) / per;
  return for_each_launch((p.rows + kStepRows - 1) / kStepRows * tiles, kThreads, 1, [&](int64_t first, int64_t count) {
    const dim3 grid(static_cast<unsigned>(count)), block(kThreads);
    if (a.dtype == RDF2V_BF16 && whole)
      scan_step_kernel<bf16, true><<<grid, block, 0, stream>>>(p, lanes, tiles, first);
    else if (a.dtype == RDF2V_BF16)
      scan_step_kernel<bf16, false><<<grid, block, 0, stream>>>(p, lanes, tiles, first);
    else if (whole)
      scan_step_kernel<float, true><<<grid, block, 0, stream>>>(p, lanes, tiles, first);
    else
      scan_step_kernel<float, false><<<grid, block, 0, stream>>>(p, lanes, tiles, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

}  // namespace rdf2v
