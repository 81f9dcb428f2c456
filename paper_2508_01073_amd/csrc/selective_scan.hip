// Selective scan over rows of tokens on gfx950, its gradients and its step.
//
//   h_t[n] = exp(delta_t a[n]) h_{t-1}[n] + delta_t x_t b_t[n],   y_t = sum_n c_t[n] h_t[n] + skip x_t
//
// for every channel by itself: per token, channel and state one exponential and three multiply-adds, so with 16
// states vector instructions bound it, the exponentials (a quarter of the rate) half of them; memory comes next.
//
// A wave takes 64 channels (a lane each) of a row, or of a segment of it, 16 tokens at a time, and nothing is
// shared with other waves: no barrier, no value made twice. It takes the channels' states in turn, each through
// the chunk's 16 tokens, whose values stay in registers meanwhile: the number of states is a loop's, not a
// register file's. b and c of the chunk lie in LDS and are read by all lanes at once.
//
// Rows too few to fill the chip are cut into segments: every segment's state from zeros (scan_states_kernel), the
// states' way through the segments (scan_join_kernel), then all segments at once. That costs the exponentials
// twice.
//
// Gradients go backwards through the chunks: a chunk's states are made again from the one before it, which
// scan_states_kernel has left in memory, and stay in registers for the way back. The sums over states (for x and
// dt) are a lane's own; the sums over channels (for b and c) are taken by matrix instructions, see ChannelSums.

#include "vectors.hpp"

#include "layer.hpp"
#include "logits.hpp"

namespace rdf2v {
namespace {

constexpr int kTokens = 16;  // of a chunk
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
  float *bc;      // [blocks of a group][rows][length][groups][2 states]: parts of the gradients of b and c
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
  w.c0 = w.group * p.per_group + int32_t(w.block) * kWave;
  w.count = min(int32_t(kWave), p.per_group - int32_t(w.block) * kWave);
  // the same in all lanes, and the compiler is to know
  const int64_t length = __builtin_amdgcn_readfirstlane(
      int32_t(row_length(p.len, w.row, p.length, report && column == 0 && w.seg == 0, p.status)));
  w.begin = w.seg * p.segment;
  w.end = min(w.begin + p.segment, p.length);
  w.stop = max(w.begin, min(w.end, length));
  return w;
}

// delta, from dt + dt_bias: log(1 + e^v) = max(v, 0) + log(1 + e), e = e^-|v|. The logarithm as
// 2 artanh(e / (2 + e)), whose series in squares of at most 1 / 9 keeps the relative precision of small steps.
__device__ __forceinline__ float softplus(float v) {
  const float e = exp_negative(-fabsf(v)), s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
  float r = 1.0f / 15.0f;
  r = fmaf(r, q, 1.0f / 13.0f);
  r = fmaf(r, q, 1.0f / 11.0f);
  r = fmaf(r, q, 1.0f / 9.0f);
  r = fmaf(r, q, 1.0f / 7.0f);
  r = fmaf(r, q, 1.0f / 5.0f);
  r = fmaf(r, q, 1.0f / 3.0f);
  const float log1 = 2.0f * fmaf(r * q, s, s);
  return v > 0.0f ? v + log1 : log1;
}

__device__ __forceinline__ float checked_rate(float a, int32_t *status) {
  if (a <= 0.0f && a > -kInf) return a;
  if (status != nullptr) atomicOr(status, RDF2V_STATUS_BAD_VALUE);
  return 0.0f;
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
      p.states, [&](int k) { return from[min(k * kWave + int(threadIdx.x), w.count * p.states - 1)]; },
      [&](int k, float a) {
        const int i = k * kWave + threadIdx.x, channel = i / p.states, n = i - channel * p.states;
        rates[n * kWave + channel] =
            channel < w.count ? checked_rate(a, report ? p.status : nullptr) * kLog2e : 0.0f;
      });
}

// States [channels][states] of memory from or to [states][64]; null: zeros.
__device__ __forceinline__ void load_states(const Scan &p, const Place &w, const float *from, float *to) {
  if (from == nullptr) {
    for (int n = 0; n < p.states; ++n) to[n * kWave + threadIdx.x] = 0.0f;
    return;
  }
  from += (w.row * p.channels + w.c0) * p.states;
  in_batches(
      p.states, [&](int k) { return from[min(k * kWave + int(threadIdx.x), w.count * p.states - 1)]; },
      [&](int k, float h) {
        const int i = k * kWave + threadIdx.x, channel = i / p.states, n = i - channel * p.states;
        to[n * kWave + channel] = channel < w.count ? h : 0.0f;
      });
}
__device__ __forceinline__ void store_states(const Scan &p, const Place &w, const float *from, float *to) {
  for (int i = threadIdx.x; i < w.count * p.states; i += kWave)
    to[(w.row * p.channels + w.c0) * p.states + i] = from[i % p.states * kWave + i / p.states];
}
// The same of the workspace, [states][channels].
__device__ __forceinline__ void load_carry(const Scan &p, const Place &w, const float *from, int channel, float *to) {
  in_batches(
      p.states, [&](int n) { return from[int64_t(n) * p.channels + channel]; },
      [&](int n, float h) { to[n * kWave + threadIdx.x] = int(threadIdx.x) < w.count ? h : 0.0f; });
}

// A chunk's work is written for N = 4, 8, 12 or 16 tokens, the fewest that hold those that count: rows of a few
// tokens leave most of a chunk out, and no token has a branch of its own.
template <class Chunk>
__device__ __forceinline__ void with_tokens(int count, Chunk chunk) {
  if (count > 12)
    chunk(std::integral_constant<int, 16>{});
  else if (count > 8)
    chunk(std::integral_constant<int, 12>{});
  else if (count > 4)
    chunk(std::integral_constant<int, 8>{});
  else
    chunk(std::integral_constant<int, 4>{});
}

// The lane's channel of a token: 32 bits of offset beside an address that all lanes have in common.
template <class T>
__device__ __forceinline__ T *lane_of(T *token, int channel) {
  typedef std::conditional_t<std::is_const_v<T>, const char, char> Byte;
  return reinterpret_cast<T *>(reinterpret_cast<Byte *>(token) + uint32_t(channel) * uint32_t(sizeof(T)));
}

// The lane's channel of a chunk's first `count` tokens; what follows is the last of them again. Addresses are made
// one after the other: all at once they would not fit the scalar registers.
template <class T, int N>
__device__ __forceinline__ void load_tokens(const rdf2v_tokens_view &view, const Place &w, int channel, int64_t t0,
                                            int count, T (&x)[N]) {
  const T *base = static_cast<const T *>(view.data);
  int64_t at = w.row * view.row_stride + t0 * view.token_stride;
#pragma unroll
  for (int t = 0; t < N; ++t) {
    x[t] = *lane_of(base + at, channel);
    at += t + 1 < N - 3 || t + 1 < count ? view.token_stride : 0;
    asm volatile("" : "+s"(at));
  }
}

// The same of an output, from token `first` of all rows on.
template <class T, int N>
__device__ __forceinline__ void store_tokens(void *out, int64_t first, int64_t channels, int channel, int count,
                                             const float (&x)[N]) {
  T *base = static_cast<T *>(out);
  int64_t at = first * channels;
#pragma unroll
  for (int t = 0; t < N; ++t) {
    if (t < N - 3 || t < count) *lane_of(base + at, channel) = from_f32<T>(x[t]);
    at += channels;
    asm volatile("" : "+s"(at));
  }
}

// b or c of a chunk to [states][16] in LDS; zeros for tokens that do not count.
template <class T, int NMAX>
__device__ __forceinline__ void load_heads(const Scan &p, const rdf2v_heads_view &view, const Place &w, int64_t t0,
                                           int count, float *lds) {
  const T *at = static_cast<const T *>(view.data) + w.row * view.row_stride + t0 * view.token_stride +
                w.group * view.head_stride;
  constexpr int kEach = kTokens * NMAX / kWave;
  T x[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = threadIdx.x + k * kWave, token = i * p.by_states >> 16, n = i - token * p.states;
    x[k] = T(0.0f);
    if (token < count) x[k] = at[token * view.token_stride + n];
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = threadIdx.x + k * kWave, token = i * p.by_states >> 16, n = i - token * p.states;
    if (token < kTokens) lds[n * kTokens + token] = to_f32(x[k]);
  }
}

// A state's values of a chunk's tokens, the same in every lane.
template <int N>
__device__ __forceinline__ void read_head(const float *lds, int n, float (&x)[N]) {
  typedef float Four __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const Four v = reinterpret_cast<const Four *>(lds + n * kTokens)[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * i + j] = v[j];
  }
}

// delta and delta x of a chunk's tokens; 0 beyond the last that counts: nothing decays and nothing is added.
template <class T, int N>
__device__ __forceinline__ void make_steps(const T (&x)[N], const T (&dt)[N], float bias, int count, bool there,
                                           float (&delta)[N], float (&u)[N]) {
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const bool on = there && t < count;
    const float d = softplus(to_f32(dt[t]) + bias);
    delta[t] = on ? d : 0.0f;
    u[t] = on ? d * to_f32(x[t]) : 0.0f;
  }
}

__device__ __forceinline__ float silu(float x) { return x * sigmoid(x); }

// The gradients of y of a chunk's tokens.
template <class T, int N>
__device__ __forceinline__ void make_gradients(const T (&dout)[N], const T (&gate)[N], bool gated, int count,
                                               bool there, float (&g)[N]) {
#pragma unroll
  for (int t = 0; t < N; ++t) g[t] = there && t < count ? to_f32(dout[t]) : 0.0f;
  if (!gated) return;
#pragma unroll
  for (int t = 0; t < N; ++t) g[t] = there && t < count ? g[t] * silu(to_f32(gate[t])) : 0.0f;
}

template <class T>
__device__ __forceinline__ void store_zeros(void *out, int64_t from, int64_t to, int64_t row, int64_t length,
                                            int64_t width, int64_t at, int count) {
  T *p = static_cast<T *>(out) + row * length * width + at;
  for (int64_t t = from; t < to; ++t)
    for (int i = threadIdx.x; i < count; i += kWave) p[t * width + i] = from_f32<T>(0.0f);
}

// What a wave keeps for its channels.
struct Lane {
  int lane, channel;
  bool there, gated;
  float bias, skip;
  __device__ __forceinline__ Lane(const Scan &p, const Place &w)
      : lane(threadIdx.x), channel(w.c0 + (int(threadIdx.x) < w.count ? threadIdx.x : 0)),
        there(int(threadIdx.x) < w.count), gated(p.gate.data != nullptr),
        bias(p.dt_bias != nullptr ? p.dt_bias[channel] : 0.0f), skip(p.skip != nullptr ? p.skip[channel] : 0.0f) {}
};

// The outputs of a segment. A wave's barriers cost nothing: it is alone in its workgroup.
template <class T, int NMAX>
__global__ __launch_bounds__(kWave) void scan_out_kernel(Scan p, int64_t first) {
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
      load_carry(p, w, p.carry + item * p.states * p.channels, me.channel, held);
    }
    for (int64_t t0 = w.begin; t0 < w.stop; t0 += kTokens) {
      const int count = int(min(int64_t(kTokens), w.stop - t0));
      with_tokens(count, [&](auto tokens) {
        constexpr int N = tokens();
        T x[N], dt[N], gate[N];
        load_tokens(p.x, w, me.channel, t0, count, x);
        load_tokens(p.dt, w, me.channel, t0, count, dt);
        if (me.gated) load_tokens(p.gate, w, me.channel, t0, count, gate);
        __syncthreads();
        load_heads<T, NMAX>(p, p.b, w, t0, count, b);
        load_heads<T, NMAX>(p, p.c, w, t0, count, c);
        float delta[N], u[N], y[N];
        make_steps(x, dt, me.bias, count, me.there, delta, u);
#pragma unroll
        for (int t = 0; t < N; ++t) y[t] = me.skip * to_f32(x[t]);
        __syncthreads();
        for (int n = 0; n < p.states; ++n) {
          const float rate = rates[n * kWave + me.lane];
          float h = held[n * kWave + me.lane], bn[N], cn[N];
          read_head(b, n, bn);
          read_head(c, n, cn);
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
        if (me.there) store_tokens<T>(p.out, w.row * p.length + t0, p.channels, me.channel, count, y);
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
// sum_t (product of the decays up to t) c_t g_t, which needs no second way through the tokens.
template <class T, int NMAX, bool BACK, bool CUT>
__global__ __launch_bounds__(kWave) void scan_states_kernel(Scan p, int64_t first) {
  constexpr bool kBoth = BACK && CUT;
  __shared__ float rates[NMAX * kWave], held[NMAX * kWave], b[NMAX * kTokens];
  __shared__ float decay[kBoth ? NMAX * kWave : 1], grad[kBoth ? NMAX * kWave : 1], c[kBoth ? NMAX * kTokens : 1];
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
      for (int n = 0; n < p.states; ++n) {
        decay[n * kWave + lane] = 1.0f;
        grad[n * kWave + lane] = 0.0f;
      }
    float sum = 0.0f;  // of delta
    // without segments the state after the last chunk is not needed
    const int64_t stop = CUT ? w.stop : w.stop - kTokens;
    for (int64_t t0 = w.begin; t0 < stop; t0 += kTokens) {
      const int count = int(min(int64_t(kTokens), w.stop - t0));
      const int64_t chunk = w.row * p.chunks + t0 / kTokens;
      with_tokens(count, [&](auto tokens) {
        constexpr int N = tokens();
        T x[N], dt[N];
        float delta[N], u[N], g[N];
        load_tokens(p.x, w, me.channel, t0, count, x);
        load_tokens(p.dt, w, me.channel, t0, count, dt);
        __syncthreads();
        load_heads<T, NMAX>(p, p.b, w, t0, count, b);
        if constexpr (kBoth) {
          T o[N], gate[N];
          load_tokens(p.dout, w, me.channel, t0, count, o);
          if (me.gated) load_tokens(p.gate, w, me.channel, t0, count, gate);
          load_heads<T, NMAX>(p, p.c, w, t0, count, c);
          make_gradients(o, gate, me.gated, count, me.there, g);
        }
        make_steps(x, dt, me.bias, count, me.there, delta, u);
        __syncthreads();
        if (kBoth && me.there) p.until[chunk * p.channels + me.channel] = sum;
        if constexpr (CUT)
#pragma unroll
          for (int t = 0; t < N; ++t) sum += delta[t];
        for (int n = 0; n < p.states; ++n) {
          const float rate = rates[n * kWave + lane];
          float h = held[n * kWave + lane], bn[N];
          if (kBoth && me.there) p.starts[(chunk * p.states + n) * p.channels + me.channel] = h;
          read_head(b, n, bn);
          if constexpr (kBoth) {
            float cn[N], most = decay[n * kWave + lane], r = grad[n * kWave + lane];
            read_head(c, n, cn);
#pragma unroll
            for (int t = 0; t < N; ++t) {
              const float e = exp2_fast(delta[t] * rate);
              h = fmaf(e, h, u[t] * bn[t]);
              most *= e;
              r = fmaf(most, g[t] * cn[t], r);
            }
            decay[n * kWave + lane] = most;
            grad[n * kWave + lane] = r;
          } else {
#pragma unroll
            for (int t = 0; t < N; ++t) h = fmaf(exp2_fast(delta[t] * rate), h, u[t] * bn[t]);
          }
          held[n * kWave + lane] = h;
          if (BACK && !CUT && me.there) p.starts[((chunk + 1) * p.states + n) * p.channels + me.channel] = h;
        }
      });
    }
    if (!CUT || !me.there) continue;
    p.steps[item * p.channels + me.channel] = sum;
    for (int n = 0; n < p.states; ++n) {
      p.carry[(item * p.states + n) * p.channels + me.channel] = held[n * kWave + lane];
      if (kBoth) p.back[(item * p.states + n) * p.channels + me.channel] = grad[n * kWave + lane];
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

typedef float Four __attribute__((ext_vector_type(4)));

// Sums over a wave's channels of a value for each of 16 tokens, by matrix products with a unit column: with A the
// value of lane 16 k + i at (i, k) and B ones in column t, a product adds the sums over k to column t of its
// accumulator. Sixteen products of 32 cycles beside the vector instructions take the place of sixteen sums over
// 64 lanes, at most 2 instructions a value instead of 7.
struct ChannelSums {
  Four sum = {0.0f, 0.0f, 0.0f, 0.0f};
  // `unit`: 1 in the lanes of column t, from unit_column
  __device__ __forceinline__ void add(float value, float unit) {
    sum = __builtin_amdgcn_mfma_f32_16x16x4f32(value, unit, sum, 0, 0, 0);
  }
  // of the lane's column
  __device__ __forceinline__ float part() const { return (sum[0] + sum[1]) + (sum[2] + sum[3]); }
};

// The columns' totals of two sums: lane t has token t's of the first, lane 32 + t of the second.
__device__ __forceinline__ float two_totals(const ChannelSums &one, const ChannelSums &two) {
  const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(one.part()), __float_as_uint(two.part()), false,
                                                       false);
  const uint32_t x = __float_as_uint(__uint_as_float(halves[0]) + __uint_as_float(halves[1]));
  const auto rows = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return __uint_as_float(rows[0]) + __uint_as_float(rows[1]);
}

// `first`, 1 in lanes 0, 16, 32 and 48 and 0 in the others, moved up by T lanes in its rows of 16.
template <int T>
__device__ __forceinline__ float unit_column(float first) {
  if constexpr (T == 0)
    return first;
  else
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(first), 0x110 + T, 0xf, 0xf, true));
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
// and holds the parameters' gradients meanwhile. Inputs are read twice, before the states' loop and after it:
// what is made of them would not fit the registers beside it.
template <class T, int NMAX>
__global__ __launch_bounds__(kWave, NMAX <= 16 ? 2 : 1) void scan_backward_kernel(Scan p, int64_t first) {
  __shared__ float rates[NMAX * kWave], grads[NMAX * kWave], da[NMAX * kWave], held[NMAX * kWave];
  __shared__ float b[NMAX * kTokens], c[NMAX * kTokens], db[kTokens * NMAX], dc[kTokens * NMAX];
  const int64_t columns = p.blocks * p.groups, column = (first + blockIdx.x) % columns,
                part = (first + blockIdx.x) / columns;
  const bool cut = p.segments > 1, direct = p.blocks == 1;
  Place w = place_of(p, column, 0, false);
  const Lane me(p, w);
  const int lane = me.lane;
  load_rates(p, w, rates, part == 0);
  for (int n = 0; n < p.states; ++n) da[n * kWave + lane] = 0.0f;
  float ddt_bias = 0.0f, dskip = 0.0f;
  for (int64_t item = part; item < p.rows * p.segments; item += p.parts) {
    w = place_of(p, column, item, lane == 0);
    __syncthreads();
    if (!cut) {
      load_states(p, w, p.dstate_out, grads);
    } else {
      load_carry(p, w, p.back + item * p.states * p.channels, me.channel, grads);
    }
    const int64_t last = w.begin + (w.stop - w.begin - 1) / kTokens * kTokens;  // chunk
    for (int64_t t0 = last; t0 >= w.begin && w.begin < w.stop; t0 -= kTokens) {
      const int count = int(min(int64_t(kTokens), w.stop - t0));
      const int64_t chunk = w.row * p.chunks + t0 / kTokens, token = w.row * p.length + t0;
      // the states before the chunk: the row's, or its own and what the segment begins with
      const float *starts = p.starts + chunk * p.states * p.channels + me.channel;
      if (cut) {
        const float *carry = p.carry + item * p.states * p.channels + me.channel;
        const float until = p.until[chunk * p.channels + me.channel];
        in_batches(
            p.states,
            [&](int n) { return make_float2(starts[int64_t(n) * p.channels], carry[int64_t(n) * p.channels]); },
            [&](int n, float2 h) {
              held[n * kWave + lane] =
                  me.there ? fmaf(exp2_fast(until * rates[n * kWave + lane]), h.y, h.x) : 0.0f;
            });
      } else if (t0 > w.begin) {
        load_carry(p, w, starts - me.channel, me.channel, held);
      } else {
        load_states(p, w, p.state, held);
      }
      with_tokens(count, [&](auto tokens) {
        constexpr int N = tokens();
        float delta[N], u[N], g[N], y[N], du[N] = {}, dd[N] = {};
        __syncthreads();
        {
          T x[N], dt[N], gate[N], o[N];
          load_tokens(p.x, w, me.channel, t0, count, x);
          load_tokens(p.dt, w, me.channel, t0, count, dt);
          if (me.gated) load_tokens(p.gate, w, me.channel, t0, count, gate);
          load_tokens(p.dout, w, me.channel, t0, count, o);
          load_heads<T, NMAX>(p, p.b, w, t0, count, b);
          load_heads<T, NMAX>(p, p.c, w, t0, count, c);
          make_steps(x, dt, me.bias, count, me.there, delta, u);
          make_gradients(o, gate, me.gated, count, me.there, g);
#pragma unroll
          for (int t = 0; t < N; ++t) {
            const float xv = to_f32(x[t]);
            dskip = t < count ? fmaf(g[t], xv, dskip) : dskip;
            y[t] = me.skip * xv;
          }
        }
        __syncthreads();
        float first = lane % kTokens == 0 ? 1.0f : 0.0f;
        for (int n = 0; n < p.states; ++n) {
          asm volatile("" : "+v"(first));  // its columns are made anew: kept, they would cost 16 registers
          const float rate = rates[n * kWave + lane], h0 = held[n * kWave + lane], after = grads[n * kWave + lane];
          float bn[N], cn[N], e[N], h[N];
          read_head(b, n, bn);
          read_head(c, n, cn);
#pragma unroll
          for (int t = 0; t < N; ++t) {
            e[t] = exp2_fast(delta[t] * rate);
            h[t] = fmaf(e[t], t > 0 ? h[t > 0 ? t - 1 : 0] : h0, u[t] * bn[t]);
            y[t] = fmaf(h[t], cn[t], y[t]);
          }
          float r = after, rates_sum = 0.0f;
          ChannelSums sb, sc;
          backwards<N>([&](auto token) {
            constexpr int t = token();
            const float unit = unit_column<t>(first);
            r = fmaf(g[t], cn[t], r);
            sb.add(r * u[t], unit);
            sc.add(g[t] * h[t], unit);
            du[t] = fmaf(r, bn[t], du[t]);
            r *= e[t];
            const float q = r * (t > 0 ? h[t > 0 ? t - 1 : 0] : h0);
            dd[t] = fmaf(q, rate, dd[t]);
            rates_sum = fmaf(q, delta[t], rates_sum);
          });
          grads[n * kWave + lane] = r;
          da[n * kWave + lane] += rates_sum;
          float total = two_totals(sb, sc);
          if (__builtin_expect(__ballot(!(fabsf(total) < kInf)) != 0, 0)) {
            // What is no number has spread over the unit columns' zeros: the same sums token by token.
            r = after;
            backwards<N>([&](auto token) {
              constexpr int t = token();
              const float unit = unit_column<t>(first);
              r = fmaf(g[t], cn[t], r);
              ChannelSums ob, oc;
              ob.add(me.there ? r * u[t] : 0.0f, unit);
              oc.add(me.there ? g[t] * h[t] : 0.0f, unit);
              r *= e[t];
              const float one = two_totals(ob, oc);
              if (lane % kTokens == t) total = one;
            });
          }
          if (lane % 32 < kTokens) (lane < 32 ? db : dc)[lane % kTokens * p.states + n] = total;
        }
        T x[N], dt[N], gate[N], o[N];
        load_tokens(p.x, w, me.channel, t0, count, x);
        load_tokens(p.dt, w, me.channel, t0, count, dt);
        if (me.gated) {
          load_tokens(p.gate, w, me.channel, t0, count, gate);
          load_tokens(p.dout, w, me.channel, t0, count, o);
        }
#pragma unroll
        for (int t = 0; t < N; ++t) {
          dd[t] = fmaf(dd[t], kLn2, to_f32(x[t]) * du[t]) * sigmoid(to_f32(dt[t]) + me.bias);
          du[t] = fmaf(delta[t], du[t], me.skip * g[t]);
          if (t < count) ddt_bias += dd[t];
        }
        if (me.there) {
          store_tokens<T>(p.dx, token, p.channels, me.channel, count, du);
          store_tokens<T>(p.ddt, token, p.channels, me.channel, count, dd);
        }
        if (!me.gated) return;
#pragma unroll
        for (int t = 0; t < N; ++t) {
          const float z = to_f32(gate[t]);
          y[t] = to_f32(o[t]) * y[t] * silu_slope(z, sigmoid(z));
        }
        if (me.there) store_tokens<T>(p.dgate, token, p.channels, me.channel, count, y);
      });
      __syncthreads();
      for (int i = lane; i < count * p.states; i += kWave) {
        const int t = i * p.by_states >> 16, n = i - t * p.states;
        if (direct) {
          const int64_t to = ((token + t) * p.groups + w.group) * p.states + n;
          static_cast<T *>(p.db)[to] = from_f32<T>(db[i]);
          static_cast<T *>(p.dc)[to] = from_f32<T>(dc[i]);
        } else {
          float *to = p.bc + ((w.block * p.rows * p.length + token + t) * p.groups + w.group) * 2 * p.states + n;
          to[0] = db[i];
          to[p.states] = dc[i];
        }
      }
    }
    store_zeros<T>(p.dx, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
    store_zeros<T>(p.ddt, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
    if (me.gated) store_zeros<T>(p.dgate, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
    if (direct) {
      store_zeros<T>(p.db, w.stop, w.end, w.row, p.length, int64_t(p.groups) * p.states, w.group * p.states, p.states);
      store_zeros<T>(p.dc, w.stop, w.end, w.row, p.length, int64_t(p.groups) * p.states, w.group * p.states, p.states);
    }
    if (w.seg == 0 && p.dstate != nullptr) {
      __syncthreads();
      store_states(p, w, grads, p.dstate);
    }
  }
  float *partial = p.partial + part * p.channels * (p.states + 2);
  __syncthreads();
  for (int i = lane; i < w.count * p.states; i += kWave)
    partial[int64_t(w.c0) * p.states + i] = da[i % p.states * kWave + i / p.states];
  if (!me.there) return;
  partial[int64_t(p.channels) * p.states + me.channel] = ddt_bias;
  partial[int64_t(p.channels) * (p.states + 1) + me.channel] = dskip;
}

// Gradients of b and c: the sums over a group's workgroups, in order.
template <class T>
__global__ __launch_bounds__(kThreads) void scan_bc_kernel(Scan p, int64_t first) {
  const int64_t width = int64_t(p.groups) * 2 * p.states, all = p.rows * p.length * width;
  const int64_t item = (first + blockIdx.x) * kThreads + threadIdx.x;
  if (item >= all) return;
  const int64_t token = item / width, row = token / p.length, n = item % (2 * p.states);
  float sum = 0.0f;
  if (token % p.length < row_length(p.len, row, p.length, false, nullptr))
    for (int64_t k = 0; k < p.blocks; ++k) sum += p.bc[k * all + item];
  const int64_t head = item / (2 * p.states);
  if (n < p.states)
    static_cast<T *>(p.db)[head * p.states + n] = from_f32<T>(sum);
  else
    static_cast<T *>(p.dc)[head * p.states + n - p.states] = from_f32<T>(sum);
}

// One token more. `lanes` threads, a power of two, take a channel's states, V neighbouring ones at a time; a
// workgroup takes a tile of channels of kStepRows rows, whose loads are all in flight at once, and the rates once
// for them. HBM-bound: states are read and written.
constexpr int kStepRows = 4;
template <class T, int V>
__global__ __launch_bounds__(kThreads) void scan_step_kernel(Scan p, int lanes, int64_t tiles, int64_t first) {
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
    load_values<float, V>(p.a + channel * p.states + n, V, rate);
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
      const int64_t row = row0 + min(r, rows - 1);
      const bool known = from[r] >= 0 && from[r] < p.num_states;
      load_values<float, V>(p.state + ((known ? from[r] : 0) * p.channels + channel) * p.states + n,
                            p.num_states > 0 ? V : 0, h[r]);
      load_values<T, V>(static_cast<const T *>(p.b.data) + row * p.b.row_stride + group * p.b.head_stride + n, V, b[r]);
      load_values<T, V>(static_cast<const T *>(p.c.data) + row * p.c.row_stride + group * p.c.head_stride + n, V, c[r]);
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
        h[r][i] = fmaf(exp2_fast(d[r] * rate[i]), h[r][i], u * b[r][i]);
        y[r] = fmaf(h[r][i], c[r][i], y[r]);
      }
      if (there && r < rows)
        store_values<float, V>(p.state_out + ((row0 + r) * p.channels + channel) * p.states + n, V, h[r]);
    }
  }
#pragma unroll
  for (int r = 0; r < kStepRows; ++r) {
    for (int m = lanes / 2; m > 0; m /= 2) y[r] += __shfl_xor(y[r], m, kWave);
    if (r >= rows || lane != 0 || !there) continue;
    if (channel == 0 && p.status != nullptr && (from[r] < 0 || from[r] >= p.num_states))
      atomicOr(p.status, RDF2V_STATUS_ID_OUT_OF_RANGE);
    y[r] = fmaf(skip, x[r], y[r]);
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

// Segments of a row, chunks, the waves along rows and segments, and where the workspace's arrays lie; its bytes.
size_t plan(Scan &p, bool backward, void *workspace) {
  // Waves that fill the chip are 1,024 times two or three.
  constexpr int64_t kFew = 1024, kFill = 4096, kMost = 8192, kShortest = 2 * kTokens;
  const int64_t columns = p.blocks * p.groups, whole = std::max<int64_t>(1, p.rows * columns);
  int64_t segments = 1;
  if (whole < kFew) segments = std::max<int64_t>(1, std::min(kFill / whole, p.length / kShortest));
  p.segment = std::max<int64_t>(1, (p.length + segments - 1) / segments);
  p.segment = (p.segment + kTokens - 1) / kTokens * kTokens;
  p.segments = std::max<int64_t>(1, (p.length + p.segment - 1) / p.segment);
  p.chunks = (p.length + kTokens - 1) / kTokens;
  p.parts = std::max<int64_t>(1, std::min(p.rows * p.segments, (backward ? kMost / 2 : kMost) / columns));
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
  if (p.blocks > 1) take(p.bc, p.blocks * p.rows * p.length * p.groups * 2 * p.states);
  return bytes;
}

// Calls launch with a value of the element type and a constant for the most states.
template <class Launch>
rdf2v_status with_types(int dtype, int states, Launch launch) {
  const auto sized = [&](auto t) {
    return states <= 16 ? launch(t, std::integral_constant<int, 16>{}) : launch(t, std::integral_constant<int, 64>{});
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
rdf2v_status launch_states(const Scan &p, int dtype, hipStream_t stream) {
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
      return for_waves(p, [&](int64_t first, dim3 grid) {
        scan_backward_kernel<decltype(t), most()><<<grid, dim3(kWave), 0, stream>>>(p, first);
      });
    });
    if (st != RDF2V_OK) return st;
    if (p.blocks > 1 && p.length > 0) {
      const int64_t blocks = (p.rows * p.length * p.groups * 2 * p.states + kThreads - 1) / kThreads;
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
  // whole vectors of four states where there are no others
  const int each = p.states % 4 == 0 ? 4 : 1;
  int lanes = 1;
  while (lanes < kWave && lanes * each < p.states) lanes *= 2;
  const int64_t per = kThreads / lanes, tiles = (p.channels + per - 1) / per;
  return for_each_launch((p.rows + kStepRows - 1) / kStepRows * tiles, kThreads, 1, [&](int64_t first, int64_t count) {
    const dim3 grid(static_cast<unsigned>(count)), block(kThreads);
    if (a.dtype == RDF2V_BF16 && each == 4)
      scan_step_kernel<bf16, 4><<<grid, block, 0, stream>>>(p, lanes, tiles, first);
    else if (a.dtype == RDF2V_BF16)
      scan_step_kernel<bf16, 1><<<grid, block, 0, stream>>>(p, lanes, tiles, first);
    else if (each == 4)
      scan_step_kernel<float, 4><<<grid, block, 0, stream>>>(p, lanes, tiles, first);
    else
      scan_step_kernel<float, 1><<<grid, block, 0, stream>>>(p, lanes, tiles, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

}  // namespace rdf2v
