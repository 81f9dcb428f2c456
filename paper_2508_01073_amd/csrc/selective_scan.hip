// Selective scan over rows of tokens on gfx950, its gradients and its step.
//
//   h_t[n] = exp(delta_t a[n]) h_{t-1}[n] + delta_t x_t b_t[n],   y_t = sum_n c_t[n] h_t[n] + skip x_t
//
// for every channel by itself: per token, channel and state one exponential and three multiply-adds, so with 16
// states vector instructions bound it, the exponentials (a quarter of the rate) half of them; memory comes next.
//
// A workgroup takes 64 channels (a lane each) of a row, or of a segment of it, 16 tokens at a time. The channels'
// states are dealt to its four waves: what is made of a token once (delta and delta x) goes through LDS to all of
// them, and their parts of y come back the same way. A wave takes its states in turn, each through the chunk's 16
// tokens, whose values stay in registers meanwhile: the number of states is a loop's, not a register file's.
// b and c of the chunk lie in LDS and are read by all lanes at once.
//
// Rows too few to fill the chip are cut into segments: every segment's state from zeros (scan_states_kernel), the
// states' way through the segments (scan_join_kernel), then all segments at once. That costs the exponentials
// twice.
//
// Gradients go backwards through the chunks: a chunk's states are made again from the one before it, which
// scan_states_kernel has left in memory, and stay in registers for the way back. The sums over states (for x and
// dt) are a lane's own; the sums over channels (for b and c) are taken by matrix instructions, see channel_sums.

#include "vectors.hpp"

#include "layer.hpp"
#include "logits.hpp"

namespace rdf2v {
namespace {

constexpr int kTokens = 16;  // of a chunk
constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kOwn = kTokens / kWaves;  // tokens of a chunk that a wave prepares and finishes

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
  int64_t blocks, parts;              // workgroups side by side in a group's channels; gradients: along rows and segments
  int32_t channels, groups, states, per_group;
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
  const int64_t length = row_length(p.len, w.row, p.length, report && column == 0 && w.seg == 0, p.status);
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

// The rates over ln 2, [states][64], and zeros for channels that are not there.
__device__ __forceinline__ void load_rates(const Scan &p, const Place &w, float *rates, bool report) {
  for (int i = threadIdx.x; i < kWave * p.states; i += kThreads) {
    const int channel = i / p.states, n = i % p.states;
    rates[n * kWave + channel] =
        channel < w.count
            ? checked_rate(p.a[int64_t(w.c0) * p.states + i], report ? p.status : nullptr) * kLog2e
            : 0.0f;
  }
}

// States [channels][states] of memory from or to [states][64]; null: zeros.
__device__ __forceinline__ void load_states(const Scan &p, const Place &w, const float *from, float *to) {
  for (int i = threadIdx.x; i < kWave * p.states; i += kThreads) {
    const int channel = i / p.states, n = i % p.states;
    to[n * kWave + channel] = from != nullptr && channel < w.count
                                  ? from[(w.row * p.channels + w.c0) * p.states + i]
                                  : 0.0f;
  }
}
__device__ __forceinline__ void store_states(const Scan &p, const Place &w, const float *from, float *to) {
  for (int i = threadIdx.x; i < w.count * p.states; i += kThreads)
    to[(w.row * p.channels + w.c0) * p.states + i] = from[i % p.states * kWave + i / p.states];
}

// A wave's tokens of a chunk, the lane's channel: values in flight as they lie in memory.
template <class T>
struct Ahead {
  T v[kOwn];
  __device__ __forceinline__ void load(const rdf2v_tokens_view &view, const Place &w, int64_t t0, int wave, int lane) {
    const T *at = static_cast<const T *>(view.data) + w.row * view.row_stride + w.c0 + lane;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int64_t t = t0 + wave * kOwn + i;
      v[i] = T(0.0f);
      if (t < w.stop && lane < w.count) v[i] = at[t * view.token_stride];
    }
  }
};

// b or c of a chunk: a thread's values in flight, then [states][16] in LDS; zeros for tokens that do not count.
template <class T, int NMAX>
struct AheadHeads {
  static constexpr int kEach = kTokens * NMAX / kThreads;
  T v[kEach];
  __device__ __forceinline__ void load(const Scan &p, const rdf2v_heads_view &view, const Place &w, int64_t t0) {
    const T *at = static_cast<const T *>(view.data) + w.row * view.row_stride + w.group * view.head_stride;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int i = threadIdx.x + k * kThreads, token = i / p.states, n = i % p.states;
      v[k] = T(0.0f);
      if (token < kTokens && t0 + token < w.stop) v[k] = at[(t0 + token) * view.token_stride + n];
    }
  }
  __device__ __forceinline__ void put(const Scan &p, float *lds) const {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int i = threadIdx.x + k * kThreads, token = i / p.states, n = i % p.states;
      if (token < kTokens) lds[n * kTokens + token] = to_f32(v[k]);
    }
  }
};

// A lane's values of a chunk's tokens, [16][64] in LDS.
__device__ __forceinline__ void read_tokens(const float (*lds)[kWave], int lane, float (&x)[kTokens]) {
#pragma unroll
  for (int t = 0; t < kTokens; ++t) x[t] = lds[t][lane];
}
// A state's values of a chunk's tokens, the same in every lane.
__device__ __forceinline__ void read_head(const float *lds, int n, float (&x)[kTokens]) {
  typedef float Four __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < kTokens / 4; ++i) {
    const Four v = reinterpret_cast<const Four *>(lds + n * kTokens)[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * i + j] = v[j];
  }
}

template <class T>
__device__ __forceinline__ void store_zeros(void *out, int64_t from, int64_t to, int64_t row, int64_t length,
                                            int64_t width, int64_t at, int count) {
  T *p = static_cast<T *>(out) + row * length * width + at;
  for (int64_t t = from + threadIdx.x / kWave; t < to; t += kWaves)
    for (int i = threadIdx.x % kWave; i < count; i += kWave) p[t * width + i] = from_f32<T>(0.0f);
}

// The outputs of a segment.
template <class T, int NMAX>
__global__ __launch_bounds__(kThreads) void scan_out_kernel(Scan p, int64_t first) {
  __shared__ float rates[NMAX * kWave], held[NMAX * kWave], b[NMAX * kTokens], c[NMAX * kTokens];
  __shared__ float delta[kTokens][kWave], u[kTokens][kWave], sums[kWaves][kTokens][kWave];
  const int64_t item = first + blockIdx.x, columns = p.blocks * p.groups;
  const Place w = place_of(p, item % columns, item / columns, threadIdx.x == 0);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const bool there = lane < w.count;
  const int channel = w.c0 + (there ? lane : 0);
  load_rates(p, w, rates, w.row == 0 && w.seg == 0);
  if (p.segments == 1) {
    load_states(p, w, p.state, held);
  } else {
    const float *from = p.carry + (w.row * p.segments + w.seg) * p.states * p.channels + channel;
    for (int n = wave; n < p.states; n += kWaves) held[n * kWave + lane] = there ? from[int64_t(n) * p.channels] : 0.0f;
  }
  const float bias = p.dt_bias != nullptr ? p.dt_bias[channel] : 0.0f;
  const float skip = p.skip != nullptr ? p.skip[channel] : 0.0f;
  const bool gated = p.gate.data != nullptr;
  T *out = static_cast<T *>(p.out) + w.row * p.length * p.channels + w.c0 + lane;
  Ahead<T> x, dt, gate;
  AheadHeads<T, NMAX> bs, cs;
  const auto load = [&](int64_t t0) {
    x.load(p.x, w, t0, wave, lane);
    dt.load(p.dt, w, t0, wave, lane);
    if (gated) gate.load(p.gate, w, t0, wave, lane);
    bs.load(p, p.b, w, t0);
    cs.load(p, p.c, w, t0);
  };
  load(w.begin);
  for (int64_t t0 = w.begin; t0 < w.stop; t0 += kTokens) {
    float kept[kOwn], open[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int t = wave * kOwn + i;
      const bool on = there && t0 + t < w.stop;
      const float d = on ? softplus(to_f32(dt.v[i]) + bias) : 0.0f, xv = to_f32(x.v[i]);
      delta[t][lane] = d;
      u[t][lane] = on ? d * xv : 0.0f;
      kept[i] = skip * xv;
      const float z = gated ? to_f32(gate.v[i]) : 0.0f;
      open[i] = z * sigmoid(z);
    }
    bs.put(p, b);
    cs.put(p, c);
    __syncthreads();
    load(t0 + kTokens);
    const int count = int(min(int64_t(kTokens), w.stop - t0));
    float dl[kTokens], ul[kTokens], y[kTokens] = {};
    read_tokens(delta, lane, dl);
    read_tokens(u, lane, ul);
    for (int n = wave; n < p.states; n += kWaves) {
      const float rate = rates[n * kWave + lane];
      float h = held[n * kWave + lane], bn[kTokens], cn[kTokens];
      read_head(b, n, bn);
      read_head(c, n, cn);
#pragma unroll
      for (int t = 0; t < kTokens; ++t) {
        if (t % 4 == 0 && t >= count) break;
        h = fmaf(exp2_fast(dl[t] * rate), h, ul[t] * bn[t]);
        y[t] = fmaf(h, cn[t], y[t]);
      }
      held[n * kWave + lane] = h;
    }
#pragma unroll
    for (int t = 0; t < kTokens; ++t) sums[wave][t][lane] = y[t];
    __syncthreads();
    if (!there) continue;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int t = wave * kOwn + i;
      if (t >= count) break;
      float sum = kept[i];
#pragma unroll
      for (int v = 0; v < kWaves; ++v) sum += sums[v][t][lane];
      out[(t0 + t) * p.channels] = from_f32<T>(gated ? sum * open[i] : sum);
    }
  }
  store_zeros<T>(p.out, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
  if (p.segments > 1 || p.state_out == nullptr) return;
  __syncthreads();
  store_states(p, w, held, p.state_out);
}

// The states that a segment ends with, from zeros; BACK, for the gradients: the states before its chunks (from the
// row's own state where there is one segment), and the gradient that its outputs give the state before it,
// sum_t (product of the decays up to t) c_t g_t, which needs no second way through the tokens.
template <class T, int NMAX, bool BACK>
__global__ __launch_bounds__(kThreads) void scan_states_kernel(Scan p, int64_t first) {
  __shared__ float rates[NMAX * kWave], held[NMAX * kWave], b[NMAX * kTokens];
  __shared__ float decay[BACK ? NMAX * kWave : 1], grad[BACK ? NMAX * kWave : 1], c[BACK ? NMAX * kTokens : 1];
  __shared__ float delta[kTokens][kWave], u[kTokens][kWave], g[BACK ? kTokens : 1][kWave];
  const int64_t item = first + blockIdx.x, columns = p.blocks * p.groups;
  const Place w = place_of(p, item % columns, item / columns, false);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const bool there = lane < w.count, cut = p.segments > 1, gated = p.gate.data != nullptr;
  const int channel = w.c0 + (there ? lane : 0);
  load_rates(p, w, rates, false);
  load_states(p, w, cut ? nullptr : p.state, held);
  if (BACK && cut)
    for (int n = wave; n < p.states; n += kWaves) {
      decay[n * kWave + lane] = 1.0f;
      grad[n * kWave + lane] = 0.0f;
    }
  const float bias = p.dt_bias != nullptr ? p.dt_bias[channel] : 0.0f;
  Ahead<T> x, dt, gate, dout;
  AheadHeads<T, NMAX> bs, cs;
  const auto load = [&](int64_t t0) {
    x.load(p.x, w, t0, wave, lane);
    dt.load(p.dt, w, t0, wave, lane);
    bs.load(p, p.b, w, t0);
    if (!BACK || !cut) return;
    if (gated) gate.load(p.gate, w, t0, wave, lane);
    dout.load(p.dout, w, t0, wave, lane);
    cs.load(p, p.c, w, t0);
  };
  float sum = 0.0f;  // of delta
  // without segments the state after the last chunk is not needed
  const int64_t stop = cut ? w.stop : w.stop - kTokens;
  if (w.begin < stop) load(w.begin);
  for (int64_t t0 = w.begin; t0 < stop; t0 += kTokens) {
    __syncthreads();  // the chunk before has been read
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int t = wave * kOwn + i;
      const bool on = there && t0 + t < w.stop;
      const float d = on ? softplus(to_f32(dt.v[i]) + bias) : 0.0f;
      delta[t][lane] = d;
      u[t][lane] = on ? d * to_f32(x.v[i]) : 0.0f;
      if (BACK && cut) {
        const float z = gated ? to_f32(gate.v[i]) : 0.0f, o = to_f32(dout.v[i]);
        g[BACK ? t : 0][lane] = gated ? o * (z * sigmoid(z)) : o;
      }
    }
    bs.put(p, b);
    if (BACK && cut) cs.put(p, c);
    __syncthreads();
    load(t0 + kTokens);
    const int count = int(min(int64_t(kTokens), w.stop - t0));
    float dl[kTokens], ul[kTokens], gl[kTokens];
    read_tokens(delta, lane, dl);
    read_tokens(u, lane, ul);
    if (BACK && cut) read_tokens(g, lane, gl);
    if (BACK && cut && wave == 0 && there)
      p.until[(w.row * p.chunks + t0 / kTokens) * p.channels + channel] = sum;
#pragma unroll
    for (int t = 0; t < kTokens; ++t) sum += dl[t];
    for (int n = wave; n < p.states; n += kWaves) {
      const float rate = rates[n * kWave + lane];
      float h = held[n * kWave + lane], bn[kTokens], cn[kTokens];
      if (BACK && cut && there)
        p.starts[((w.row * p.chunks + t0 / kTokens) * p.states + n) * p.channels + channel] = h;
      read_head(b, n, bn);
      if (BACK && cut) {
        read_head(c, n, cn);
        float most = decay[n * kWave + lane], r = grad[n * kWave + lane];
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
          if (t % 4 == 0 && t >= count) break;
          const float e = exp2_fast(dl[t] * rate);
          h = fmaf(e, h, ul[t] * bn[t]);
          most *= e;
          r = fmaf(most, gl[t] * cn[t], r);
        }
        decay[n * kWave + lane] = most;
        grad[n * kWave + lane] = r;
      } else {
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
          if (t % 4 == 0 && t >= count) break;
          h = fmaf(exp2_fast(dl[t] * rate), h, ul[t] * bn[t]);
        }
      }
      held[n * kWave + lane] = h;
      if (BACK && !cut && there)
        p.starts[((w.row * p.chunks + t0 / kTokens + 1) * p.states + n) * p.channels + channel] = h;
    }
  }
  if (!cut || !there) return;
  const int64_t at = w.row * p.segments + w.seg;
  if (wave == 0) p.steps[at * p.channels + channel] = sum;
  for (int n = wave; n < p.states; n += kWaves) {
    p.carry[(at * p.states + n) * p.channels + channel] = held[n * kWave + lane];
    if (BACK) p.back[(at * p.states + n) * p.channels + channel] = grad[n * kWave + lane];
  }
}

// A row's states from segment to segment, a thread to a channel's state; BACK: also their gradients, backwards.
template <bool BACK>
__global__ __launch_bounds__(kThreads) void scan_join_kernel(Scan p, int64_t first) {
  const int64_t item = (first + blockIdx.x) * kThreads + threadIdx.x;
  if (item >= p.rows * p.states * p.channels) return;
  const int64_t channel = item % p.channels, n = item / p.channels % p.states, row = item / p.channels / p.states;
  const float rate = checked_rate(p.a[channel * p.states + n], nullptr) * kLog2e;
  const int64_t held = (row * p.channels + channel) * p.states + n;
  const float *steps = p.steps + row * p.segments * p.channels + channel;
  const int64_t stride = int64_t(p.states) * p.channels, at = row * p.segments * stride + n * p.channels + channel;
  float h = p.state != nullptr ? p.state[held] : 0.0f;
#pragma unroll 8
  for (int64_t s = 0; s < p.segments; ++s) {
    const float mine = p.carry[at + s * stride];
    p.carry[at + s * stride] = h;
    h = fmaf(exp2_fast(steps[s * p.channels] * rate), h, mine);
  }
  if (!BACK) {
    if (p.state_out != nullptr) p.state_out[held] = h;
    return;
  }
  float r = p.dstate_out != nullptr ? p.dstate_out[held] : 0.0f;
#pragma unroll 8
  for (int64_t s = p.segments - 1; s >= 0; --s) {
    const float mine = p.back[at + s * stride];
    p.back[at + s * stride] = r;
    r = fmaf(exp2_fast(steps[s * p.channels] * rate), r, mine);
  }
}

typedef float Four __attribute__((ext_vector_type(4)));

// Sums over a wave's channels of a value for each of 16 tokens, by matrix products with a unit column: with A the
// value of lane 16 k + i at (i, k) and B ones in column t, a product adds the sums over k to column t of its
// accumulator. Sixteen products of 32 cycles beside the vector instructions take the place of sixteen sums over
// 64 lanes, at most 2 instructions a value instead of 7.
struct ChannelSums {
  Four sum = {0.0f, 0.0f, 0.0f, 0.0f};
  __device__ __forceinline__ void add(float value, int t, int lane) {
    sum = __builtin_amdgcn_mfma_f32_16x16x4f32(value, lane % kTokens == t ? 1.0f : 0.0f, sum, 0, 0, 0);
  }
  // token lane % 16's, in every lane
  __device__ __forceinline__ float total() const {
    float x = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    x += __shfl_xor(x, 16, kWave);
    return x + __shfl_xor(x, 32, kWave);
  }
};

// Gradients of a segment, chunk after chunk from its end; a workgroup takes several segments of its channels in
// turn and holds the parameters' gradients meanwhile.
template <class T, int NMAX>
__global__ __launch_bounds__(kThreads, NMAX <= 16 ? 2 : 1) void scan_backward_kernel(Scan p, int64_t first) {
  __shared__ float rates[NMAX * kWave], grads[NMAX * kWave], da[NMAX * kWave];
  __shared__ float b[NMAX * kTokens], c[NMAX * kTokens], db[kTokens * NMAX], dc[kTokens * NMAX];
  __shared__ float delta[kTokens][kWave], u[kTokens][kWave], g[kTokens][kWave];
  __shared__ float ys[kWaves][kTokens][kWave], dus[kWaves][kTokens][kWave], dds[kWaves][kTokens][kWave];
  const int64_t columns = p.blocks * p.groups, column = (first + blockIdx.x) % columns,
                part = (first + blockIdx.x) / columns;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const bool gated = p.gate.data != nullptr, cut = p.segments > 1, direct = p.blocks == 1;
  Place w = place_of(p, column, 0, false);
  const bool there = lane < w.count;
  const int channel = w.c0 + (there ? lane : 0);
  const float bias = p.dt_bias != nullptr ? p.dt_bias[channel] : 0.0f;
  const float skip = p.skip != nullptr ? p.skip[channel] : 0.0f;
  load_rates(p, w, rates, part == 0);
  for (int i = threadIdx.x; i < NMAX * kWave; i += kThreads) da[i] = 0.0f;
  float ddt_bias = 0.0f, dskip = 0.0f;
  for (int64_t item = part; item < p.rows * p.segments; item += p.parts) {
    w = place_of(p, column, item, threadIdx.x == 0);
    const int64_t at = w.row * p.segments + w.seg, tokens = w.row * p.length * p.channels + w.c0 + lane;
    __syncthreads();
    if (!cut) {
      load_states(p, w, p.dstate_out, grads);
    } else {
      for (int n = wave; n < p.states; n += kWaves)
        grads[n * kWave + lane] = there ? p.back[(at * p.states + n) * p.channels + channel] : 0.0f;
    }
    Ahead<T> x, dt, gate, dout;
    AheadHeads<T, NMAX> bs, cs;
    const auto load = [&](int64_t t0) {
      x.load(p.x, w, t0, wave, lane);
      dt.load(p.dt, w, t0, wave, lane);
      if (gated) gate.load(p.gate, w, t0, wave, lane);
      dout.load(p.dout, w, t0, wave, lane);
      bs.load(p, p.b, w, t0);
      cs.load(p, p.c, w, t0);
    };
    const int64_t last = w.begin + (w.stop - w.begin - 1) / kTokens * kTokens;  // chunk
    if (w.begin < w.stop) load(last);
    for (int64_t t0 = last; t0 >= w.begin && w.begin < w.stop; t0 -= kTokens) {
      float xv[kOwn], dv[kOwn], raw[kOwn], z[kOwn], sig[kOwn], o[kOwn], gv[kOwn];
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const int t = wave * kOwn + i;
        const bool on = there && t0 + t < w.stop;
        xv[i] = to_f32(x.v[i]);
        raw[i] = to_f32(dt.v[i]) + bias;
        dv[i] = on ? softplus(raw[i]) : 0.0f;
        o[i] = to_f32(dout.v[i]);
        z[i] = gated ? to_f32(gate.v[i]) : 0.0f;
        sig[i] = gated ? sigmoid(z[i]) : 0.0f;
        gv[i] = gated ? o[i] * (z[i] * sig[i]) : o[i];
        delta[t][lane] = dv[i];
        u[t][lane] = on ? dv[i] * xv[i] : 0.0f;
        g[t][lane] = on ? gv[i] : 0.0f;
      }
      bs.put(p, b);
      cs.put(p, c);
      __syncthreads();
      if (t0 > w.begin) load(t0 - kTokens);
      const int count = int(min(int64_t(kTokens), w.stop - t0));
      float dl[kTokens], ul[kTokens], gl[kTokens], y[kTokens] = {}, du[kTokens] = {}, dd[kTokens] = {};
      read_tokens(delta, lane, dl);
      read_tokens(u, lane, ul);
      read_tokens(g, lane, gl);
      const int64_t chunk = w.row * p.chunks + t0 / kTokens;
      const float until = cut && there ? p.until[chunk * p.channels + channel] : 0.0f;
      for (int n = wave; n < p.states; n += kWaves) {
        const float rate = rates[n * kWave + lane];
        float h = 0.0f;
        if (there) {
          if (cut)
            h = fmaf(exp2_fast(until * rate), p.carry[(at * p.states + n) * p.channels + channel],
                     p.starts[(chunk * p.states + n) * p.channels + channel]);
          else if (t0 > w.begin)
            h = p.starts[(chunk * p.states + n) * p.channels + channel];
          else if (p.state != nullptr)
            h = p.state[(w.row * p.channels + channel) * p.states + n];
        }
        float bn[kTokens], cn[kTokens], e[kTokens], kept[kTokens];
        read_head(b, n, bn);
        read_head(c, n, cn);
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
          if (t % 4 == 0 && t >= count) break;
          e[t] = exp2_fast(dl[t] * rate);
          kept[t] = e[t] * h;
          h = fmaf(ul[t], bn[t], kept[t]);
          y[t] = fmaf(h, cn[t], y[t]);
        }
        const float after = grads[n * kWave + lane];
        float r = after, rates_sum = 0.0f;
        ChannelSums sb, sc;
#pragma unroll
        for (int t = kTokens - 1; t >= 0; --t) {
          if (t / 4 * 4 >= count) continue;
          r = fmaf(gl[t], cn[t], r);
          sb.add(r * ul[t], t, lane);
          sc.add(gl[t] * fmaf(ul[t], bn[t], kept[t]), t, lane);
          du[t] = fmaf(r, bn[t], du[t]);
          const float q = r * kept[t];
          dd[t] = fmaf(q, rate, dd[t]);
          rates_sum = fmaf(q, dl[t], rates_sum);
          r *= e[t];
        }
        grads[n * kWave + lane] = r;
        da[n * kWave + lane] += rates_sum;
        float tb = sb.total(), tc = sc.total();
        if (__builtin_expect(__ballot(!(fabsf(tb) < kInf) || !(fabsf(tc) < kInf)) != 0, 0)) {
          // What is no number has spread over the unit columns' zeros: the same sums token by token.
          r = after;
          for (int t = kTokens - 1; t >= 0; --t) {
            if (t >= count) continue;
            const float ct = c[n * kTokens + t], bt = b[n * kTokens + t], ut = u[t][lane], gt = g[t][lane];
            float et = 0.0f, kt = 0.0f;
#pragma unroll
            for (int k = 0; k < kTokens; ++k) {
              et = k == t ? e[k] : et;
              kt = k == t ? kept[k] : kt;
            }
            r = fmaf(gt, ct, r);
            ChannelSums ob, oc;
            ob.add(there ? r * ut : 0.0f, t, lane);
            oc.add(there ? gt * fmaf(ut, bt, kt) : 0.0f, t, lane);
            r *= et;
            const float one = ob.total(), two = oc.total();
            if (lane % kTokens == t) {
              tb = one;
              tc = two;
            }
          }
        }
        if (lane < kTokens) {
          db[lane * p.states + n] = tb;
          dc[lane * p.states + n] = tc;
        }
      }
#pragma unroll
      for (int t = 0; t < kTokens; ++t) {
        ys[wave][t][lane] = y[t];
        dus[wave][t][lane] = du[t];
        dds[wave][t][lane] = dd[t];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const int t = wave * kOwn + i;
        if (t >= count) break;
        if (!there) break;
        float sy = skip * xv[i], su = 0.0f, sd = 0.0f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
          sy += ys[v][t][lane];
          su += dus[v][t][lane];
          sd += dds[v][t][lane];
        }
        const float dstep = fmaf(sd, kLn2, xv[i] * su) * sigmoid(raw[i]);
        ddt_bias += dstep;
        dskip = fmaf(gv[i], xv[i], dskip);
        const int64_t to = tokens + (t0 + t) * p.channels;
        static_cast<T *>(p.dx)[to] = from_f32<T>(fmaf(dv[i], su, skip * gv[i]));
        static_cast<T *>(p.ddt)[to] = from_f32<T>(dstep);
        if (gated) static_cast<T *>(p.dgate)[to] = from_f32<T>(o[i] * sy * silu_slope(z[i], sig[i]));
      }
      for (int i = threadIdx.x; i < count * p.states; i += kThreads) {
        const int64_t token = w.row * p.length + t0 + i / p.states;
        const int n = i % p.states;
        if (direct) {
          const int64_t to = (token * p.groups + w.group) * p.states + n;
          static_cast<T *>(p.db)[to] = from_f32<T>(db[i]);
          static_cast<T *>(p.dc)[to] = from_f32<T>(dc[i]);
        } else {
          float *to = p.bc + ((w.block * p.rows * p.length + token) * p.groups + w.group) * 2 * p.states + n;
          to[0] = db[i];
          to[p.states] = dc[i];
        }
      }
    }
    store_zeros<T>(p.dx, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
    store_zeros<T>(p.ddt, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
    if (gated) store_zeros<T>(p.dgate, w.stop, w.end, w.row, p.length, p.channels, w.c0, w.count);
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
  for (int i = threadIdx.x; i < w.count * p.states; i += kThreads)
    partial[int64_t(w.c0) * p.states + i] = da[i % p.states * kWave + i / p.states];
  ys[wave][0][lane] = ddt_bias;
  ys[wave][1][lane] = dskip;
  __syncthreads();
  if (wave >= 2 || !there) return;
  float sum = 0.0f;
  for (int v = 0; v < kWaves; ++v) sum += ys[v][wave][lane];
  partial[int64_t(p.channels) * (p.states + wave) + channel] = sum;
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

// One token more: `lanes` threads, a power of two, to a row's channel, its states dealt to them.
template <class T>
__global__ __launch_bounds__(kThreads) void scan_step_kernel(Scan p, int lanes, int64_t first) {
  const int64_t item = ((first + blockIdx.x) * kThreads + threadIdx.x) / lanes;
  const int lane = threadIdx.x % lanes;
  if (item >= p.rows * p.channels) return;  // whole teams leave
  const int64_t channel = item % p.channels, row = item / p.channels, group = channel / p.per_group;
  const int64_t from = p.parents != nullptr ? p.parents[row] : row;
  const bool known = from >= 0 && from < p.num_states;
  if (!known && channel == 0 && lane == 0 && p.status != nullptr) atomicOr(p.status, RDF2V_STATUS_ID_OUT_OF_RANGE);
  const float x = to_f32(static_cast<const T *>(p.x.data)[row * p.x.row_stride + channel]);
  const float raw = to_f32(static_cast<const T *>(p.dt.data)[row * p.dt.row_stride + channel]);
  const float d = softplus(raw + (p.dt_bias != nullptr ? p.dt_bias[channel] : 0.0f)), u = d * x;
  const T *b = static_cast<const T *>(p.b.data) + row * p.b.row_stride + group * p.b.head_stride;
  const T *c = static_cast<const T *>(p.c.data) + row * p.c.row_stride + group * p.c.head_stride;
  float y = 0.0f;
  for (int n = lane; n < p.states; n += lanes) {
    const float rate = checked_rate(p.a[channel * p.states + n], row == 0 ? p.status : nullptr) * kLog2e;
    const float old = known ? p.state[(from * p.channels + channel) * p.states + n] : 0.0f;
    const float h = fmaf(exp2_fast(d * rate), old, u * to_f32(b[n]));
    p.state_out[item * p.states + n] = h;
    y = fmaf(h, to_f32(c[n]), y);
  }
  for (int m = lanes / 2; m > 0; m /= 2) y += __shfl_xor(y, m, kWave);
  if (lane != 0) return;
  y = fmaf(p.skip != nullptr ? p.skip[channel] : 0.0f, x, y);
  if (p.gate.data != nullptr) {
    const float z = to_f32(static_cast<const T *>(p.gate.data)[row * p.gate.row_stride + channel]);
    y *= z * sigmoid(z);
  }
  static_cast<T *>(p.out)[item] = from_f32<T>(y);
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
  return p;
}

// Segments of a row, chunks, the gradients' workgroups, and where the workspace's arrays lie; its bytes.
size_t plan(Scan &p, bool backward, void *workspace) {
  constexpr int64_t kFill = 512, kShortest = 4 * kTokens;
  const int64_t columns = p.blocks * p.groups, whole = std::max<int64_t>(1, p.rows * columns);
  int64_t segments = 1;
  if (whole < kFill) segments = std::max<int64_t>(1, std::min((2 * kFill) / whole, p.length / kShortest));
  p.segment = std::max<int64_t>(1, (p.length + segments - 1) / segments);
  p.segment = (p.segment + kTokens - 1) / kTokens * kTokens;
  p.segments = std::max<int64_t>(1, (p.length + p.segment - 1) / p.segment);
  p.chunks = (p.length + kTokens - 1) / kTokens;
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
  p.parts = std::max<int64_t>(1, std::min(p.rows * p.segments, 4096 / columns));
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

template <bool BACK>
rdf2v_status launch_states(const Scan &p, int dtype, hipStream_t stream) {
  return with_types(dtype, p.states, [&](auto t, auto most) {
    return for_each_launch(p.rows * p.segments * p.blocks * p.groups, kThreads, 1, [&](int64_t first, int64_t count) {
      scan_states_kernel<decltype(t), most(), BACK><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
      RDF2V_LAUNCH_CHECK();
      return RDF2V_OK;
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
    rdf2v_status st = launch_states<false>(p, a.dtype, stream);
    if (st == RDF2V_OK) st = launch_join<false>(p, stream);
    if (st != RDF2V_OK) return st;
  }
  return with_types(a.dtype, p.states, [&](auto t, auto most) {
    return for_each_launch(p.rows * p.segments * p.blocks * p.groups, kThreads, 1, [&](int64_t first, int64_t count) {
      scan_out_kernel<decltype(t), most()><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
      RDF2V_LAUNCH_CHECK();
      return RDF2V_OK;
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
    if (p.chunks > 1) st = launch_states<true>(p, a.dtype, stream);
    if (st == RDF2V_OK && p.segments > 1) st = launch_join<true>(p, stream);
    if (st != RDF2V_OK) return st;
    st = with_types(a.dtype, p.states, [&](auto t, auto most) {
      return for_each_launch(p.parts * p.blocks * p.groups, kThreads, 1, [&](int64_t first, int64_t count) {
        scan_backward_kernel<decltype(t), most()><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
        RDF2V_LAUNCH_CHECK();
        return RDF2V_OK;
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
  int lanes = 1;
  while (lanes < kWave && lanes < p.states) lanes *= 2;
  const int64_t blocks = (p.rows * p.channels + kThreads / lanes - 1) / (kThreads / lanes);
  return for_each_launch(blocks, kThreads, 1, [&](int64_t first, int64_t count) {
    if (a.dtype == RDF2V_BF16)
      scan_step_kernel<bf16><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, lanes, first);
    else
      scan_step_kernel<float><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, lanes, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

}  // namespace rdf2v
