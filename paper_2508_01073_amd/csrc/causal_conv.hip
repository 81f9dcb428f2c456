// Causal convolution of each channel by itself on gfx950, its gradients and its step.
//
// u_t = bias + sum_j w_j x_{t - width + 1 + j}: 2 width operations a value, so HBM bounds every form: the floor
// is x read once and the output written once; for the gradients x and dout read, dx written. A thread takes a
// few channels side by side and a tile of tokens, holding the width - 1 inputs before it in registers: all that
// is read twice are these, at the tiles' ends.
//
// Kernels' times here and below are means under the profiler, up to an eighth longer than among other calls; times of
// calls are without it.

#include "vectors.hpp"

#include "layer.hpp"

namespace rdf2v {
namespace {

constexpr int kThreads = 256;

struct Conv {
  const void *x, *dout, *state, *dstate_out;
  void *out, *state_out, *dstate;  // out: dx in the gradients
  const float *weight, *bias;
  const int32_t *len, *parents;
  float *partial;
  int32_t *status;
  int64_t row_stride, token_stride, dout_row_stride, dout_token_stride;
  int64_t rows, length, num_states;
  int64_t vectors, tiles, tile;  // vectors of channels in a token, tiles of tokens in a row
  int64_t blocks, parts;         // gradients: workgroups side by side in the channels, and along the tokens
  int32_t channels, lanes;       // gradients: threads side by side in the channels
};

// Channels of a vector in the gradients: what is held of each, 5 width + 8 values, sets how many waves there are.
template <class T>
constexpr int kBackwardVector = sizeof(T) == 2 ? 4 : 2;

// The taps of V neighbouring channels, which lie one behind the other: read four at a time (a step of 512 rows by 2,048
// channels: 7.8 us, one at a time 10.2).
template <int W, int V>
struct Taps {
  float w[W][V], bias[V];
  __device__ __forceinline__ void load(const Conv &a, int64_t c, int n) {
    constexpr int kWide = V < 4 ? V : 4;
#pragma unroll
    for (int i = 0; i < W * V; i += kWide) {
      float x[kWide];
      load_values<float, kWide>(a.weight + c * W + i, n * W - i, x);
#pragma unroll
      for (int k = 0; k < kWide; ++k) w[(i + k) % W][(i + k) / W] = x[k];
    }
    if (a.bias != nullptr) {
      load_values<float, V>(a.bias + c, n, bias);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) bias[i] = 0.0f;
    }
  }
  __device__ __forceinline__ bool finite() const {
    bool all = true;
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) all = all && fabsf(w[j][i]) < __builtin_inff();
    return all;
  }
};

// The input `at` tokens after a row's first: of the row, of the state before it, or zeros.
template <class T, int W, int V>
__device__ __forceinline__ void load_input(const Conv &a, int64_t row, int64_t at, int64_t c, int n, float (&x)[V]) {
  if (at >= 0) {
    load_values<T, V>(static_cast<const T *>(a.x) + row * a.row_stride + at * a.token_stride + c, n, x);
  } else if (a.state != nullptr && at >= -(W - 1)) {
    load_values<T, V>(static_cast<const T *>(a.state) + (row * (W - 1) + at + W - 1) * a.channels + c, n, x);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.0f;
  }
}

template <int W, int V>
__device__ __forceinline__ void shift(float (&x)[W][V]) {
#pragma unroll
  for (int j = 0; j + 1 < W; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) x[j][i] = x[j + 1][i];
}

template <int W, int V>
__device__ __forceinline__ float tap_sum(const Taps<W, V> &taps, const float (&x)[W][V], int i) {
  float u = taps.bias[i];
#pragma unroll
  for (int j = 0; j < W; ++j) u = fmaf(taps.w[j][i], x[j][i], u);
  return u;
}

// Whole rows: a thread to a vector of channels and a tile of tokens, four of which are read at once. 20,011 tokens of
// 2,048 channels in bf16: 37 us, 4.4 TB/s of what has to be read and written; vectors of eight channels need twice the
// registers and leave half as many waves (48 us for 58 when both were timed).
template <class T, int W, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_kernel(Conv a, int64_t first) {
  constexpr int V = 4, kAhead = 4;
  const int64_t item = (first + blockIdx.x) * kThreads + threadIdx.x;
  if (item >= a.rows * a.tiles * a.vectors) return;
  const int64_t vector = item % a.vectors, rest = item / a.vectors, tile = rest % a.tiles, row = rest / a.tiles;
  const int64_t c = vector * V;
  const int n = int(min(int64_t(V), a.channels - c));
  const int64_t length = row_length(a.len, row, a.length, vector == 0 && tile == 0, a.status);
  const int64_t begin = tile * a.tile, end = min(begin + a.tile, a.length), stop = min(end, length);
  T *out = static_cast<T *>(a.out) + row * a.length * a.channels + c;
  if (begin < stop) {
    Taps<W, V> taps;
    taps.load(a, c, n);
    float x[W][V];
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) load_input<T, W, V>(a, row, begin - (W - 1) + j, c, n, x[j + 1]);
    const T *from = static_cast<const T *>(a.x) + row * a.row_stride + begin * a.token_stride + c;
    T *to = out + begin * a.channels;
    for (int left = int(stop - begin); left > 0; left -= kAhead) {
      Values<T, V> next[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        next[k].load(from, n);
        if (k + 1 < left) from += a.token_stride;
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (k >= left) break;
        shift<W, V>(x);
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          x[W - 1][i] = next[k][i];
          const float u = tap_sum<W, V>(taps, x, i);
          y[i] = SILU ? u * sigmoid(u) : u;
        }
        store_values<T, V>(to, n, y);
        to += a.channels;
      }
    }
  }
  const float zeros[V] = {};
  for (int64_t t = max(begin, stop); t < end; ++t) store_values<T, V>(out + t * a.channels, n, zeros);
  if (tile != 0 || a.state_out == nullptr) return;
  for (int j = 0; j + 1 < W; ++j) {
    float y[V];
    load_input<T, W, V>(a, row, length - (W - 1) + j, c, n, y);
    store_values<T, V>(static_cast<T *>(a.state_out) + (row * (W - 1) + j) * a.channels + c, n, y);
  }
}

// Gradients. `lanes` threads side by side take vectors of channels, the workgroup's others (what is left of them has
// nothing to do) and the `parts` workgroups the tiles of tokens in turn; the parameters' gradients stay in registers
// until the end. dx_p is a sum over the `width` tokens from p on, so a tile goes width - 1 tokens beyond its end; the
// first tile begins with the state's inputs. 4,096 ragged rows of 17 tokens by 408 channels in float32: 74 us, 268 MB
// at 3.6 TB/s.
template <class T, int W, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_backward_kernel(Conv a, int64_t first) {
  constexpr int V = kBackwardVector<T>, kAhead = 4;
  __shared__ float scratch[kThreads][V];
  const int64_t block = first + blockIdx.x, part = block / a.blocks;
  const int subs = kThreads / a.lanes, sub = threadIdx.x / a.lanes, lane = threadIdx.x % a.lanes;
  const int64_t vector = block % a.blocks * a.lanes + lane, c = vector * V;
  const bool there = vector < a.vectors && sub < subs;
  const int n = there ? int(min(int64_t(V), a.channels - c)) : 0;
  float dw[W][V] = {}, db[V] = {};
  if (there) {
    Taps<W, V> taps;
    taps.load(a, c, n);
    for (int64_t item = part * subs + sub; item < a.rows * a.tiles; item += a.parts * subs) {
      const int64_t row = item / a.tiles, tile = item % a.tiles;
      const int64_t length = row_length(a.len, row, a.length, vector == 0 && tile == 0, a.status);
      const int64_t begin = tile * a.tile, end = min(begin + a.tile, a.length), stop = min(end, length);
      const bool states = tile == 0 && a.dstate != nullptr;  // the state's inputs are the tile's too
      T *dx = static_cast<T *>(a.out) + (row * a.length + begin) * a.channels + c;
      int zeros = int(end - begin);
      if (begin < stop || states) {
        float x[W][V], du[W][V] = {};  // inputs of the tokens up to t; gradients of u of the tokens up to t
#pragma unroll
        for (int j = 0; j + 1 < W; ++j) load_input<T, W, V>(a, row, begin - (W - 1) + j, c, n, x[j + 1]);
        const T *px = static_cast<const T *>(a.x) + row * a.row_stride + begin * a.token_stride + c;
        const T *pd = static_cast<const T *>(a.dout) + row * a.dout_row_stride + begin * a.dout_token_stride + c;
        // counted from `begin`: tokens of the row, of the tile, and those whose gradients reach an input of the tile
        const int64_t rest = length - begin;
        const int own = int(stop - begin), to = own + W - 1, real = int(min(rest, int64_t(to)));
        zeros -= own;
        const auto walk = [&](auto finite) {
          constexpr bool FINITE = finite();
          for (int t = 0; t < to; t += kAhead) {
            Values<T, V> nx[kAhead], nd[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
              nx[k].load(px, t + k < real ? n : 0);
              nd[k].load(pd, t + k < real ? n : 0);
              if (t + k + 1 < real) {
                px += a.token_stride;
                pd += a.dout_token_stride;
              }
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
              const int s = t + k, p = s - (W - 1);
              if (s >= to) break;
              shift<W, V>(x);
              shift<W, V>(du);
#pragma unroll
              for (int i = 0; i < V; ++i) {
                x[W - 1][i] = nx[k][i];
                float d = nd[k][i];
                if (SILU && s < real) {
                  const float u = tap_sum<W, V>(taps, x, i);
                  d *= silu_slope(u, sigmoid(u));
                }
                du[W - 1][i] = d;
                if (s < own) {
                  db[i] += d;
#pragma unroll
                  for (int j = 0; j < W; ++j) dw[j][i] = fmaf(d, x[j][i], dw[j][i]);
                }
              }
              if (p < 0 && !states) continue;
              float g[V] = {};
              const int64_t slot = p - (rest - (W - 1));  // of the state that the row leaves
              if (slot >= 0 && a.dstate_out != nullptr)
                load_values<T, V>(static_cast<const T *>(a.dstate_out) + (row * (W - 1) + slot) * a.channels + c, n, g);
#pragma unroll
              for (int j = 0; j < W; ++j)
                if (FINITE || (s >= j && s - j < real))  // what is not there is 0, and no number times infinity
#pragma unroll
                  for (int i = 0; i < V; ++i) g[i] = fmaf(taps.w[j][i], du[W - 1 - j][i], g[i]);
              if (p >= 0) {
                store_values<T, V>(dx, n, g);
                dx += a.channels;
              } else {
                store_values<T, V>(static_cast<T *>(a.dstate) + (row * (W - 1) + p + W - 1) * a.channels + c, n, g);
              }
            }
          }
        };
        // Taps that are all finite, as ever but by accident, need no look at where a tap's token lies: with one for
        // each tap 4,096 rows of 17 tokens by 408 channels take 84 us for 74.
        if (taps.finite())
          walk(std::true_type{});
        else
          walk(std::false_type{});
      }
      const float zero[V] = {};
      for (; zeros > 0; --zeros, dx += a.channels) store_values<T, V>(dx, n, zero);
    }
  }
  // the workgroup's threads of one vector, in order
  float *partial = a.partial + part * a.channels * (W + 1);
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) scratch[threadIdx.x][i] = j < W ? dw[j < W ? j : 0][i] : db[i];
    __syncthreads();
    if (sub != 0 || !there) continue;
    float sum[V] = {};
    for (int s = 0; s < subs; ++s)
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += scratch[s * a.lanes + lane][i];
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) partial[j < W ? (c + i) * W + j : int64_t(a.channels) * W + c + i] = sum[i];
  }
}

// One token more: a thread to a row's vector of channels. 512 rows of 2,048 channels in bf16, width 4: 7.5 us for
// 15 MB, most of it the latency of a parent's id and then its state.
template <class T, int W, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_step_kernel(Conv a, int64_t first) {
  constexpr int V = 16 / sizeof(T);
  const int64_t item = (first + blockIdx.x) * kThreads + threadIdx.x;
  if (item >= a.rows * a.vectors) return;
  const int64_t vector = item % a.vectors, row = item / a.vectors, c = vector * V;
  const int n = int(min(int64_t(V), a.channels - c));
  float x[W][V];
  load_values<T, V>(static_cast<const T *>(a.x) + row * a.row_stride + c, n, x[W - 1]);
  const int64_t from = a.parents != nullptr ? a.parents[row] : row;
  const bool known = from >= 0 && from < a.num_states;
  if (!known && vector == 0 && a.status != nullptr) atomicOr(a.status, RDF2V_STATUS_ID_OUT_OF_RANGE);
#pragma unroll
  for (int j = 0; j + 1 < W; ++j) {
    if (known)
      load_values<T, V>(static_cast<const T *>(a.state) + (from * (W - 1) + j) * a.channels + c, n, x[j]);
    else
#pragma unroll
      for (int i = 0; i < V; ++i) x[j][i] = 0.0f;
  }
  Taps<W, V> taps;
  taps.load(a, c, n);
  float y[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float u = tap_sum<W, V>(taps, x, i);
    y[i] = SILU ? u * sigmoid(u) : u;
  }
  store_values<T, V>(static_cast<T *>(a.out) + row * a.channels + c, n, y);
#pragma unroll
  for (int j = 0; j + 1 < W; ++j)
    store_values<T, V>(static_cast<T *>(a.state_out) + (row * (W - 1) + j) * a.channels + c, n, x[j + 1]);
}

// Calls launch with a constant for the width and whether there is an activation.
template <class Launch>
rdf2v_status with_width(int width, bool silu, Launch launch) {
#define RDF2V_WIDTH(W)                                                                             \
  case W:                                                                                          \
    return silu ? launch(std::integral_constant<int, W>{}, std::true_type{})                       \
                : launch(std::integral_constant<int, W>{}, std::false_type{});
  switch (width) {
    RDF2V_WIDTH(1)
    RDF2V_WIDTH(2)
    RDF2V_WIDTH(3)
    RDF2V_WIDTH(4)
    RDF2V_WIDTH(5)
    RDF2V_WIDTH(6)
    RDF2V_WIDTH(7)
    RDF2V_WIDTH(8)
    default:
      return RDF2V_ERR_INVALID_ARGUMENT;
  }
#undef RDF2V_WIDTH
}

Conv base(const rdf2v_conv &a, const rdf2v_tokens_view &x, int32_t *status) {
  Conv c{};
  c.x = x.data;
  c.row_stride = x.row_stride;
  c.token_stride = x.token_stride;
  c.weight = a.weight;
  c.bias = a.bias;
  c.len = a.len;
  c.rows = a.rows;
  c.length = a.length;
  c.channels = a.channels;
  c.status = status;
  return c;
}

// Tiles of at most `most` tokens, of one size but for the last; one also for rows without tokens.
void tile_rows(Conv &c, int64_t most) {
  c.tiles = c.length == 0 ? 1 : (c.length + most - 1) / most;
  c.tile = c.length == 0 ? 1 : (c.length + c.tiles - 1) / c.tiles;
  c.tiles = c.length == 0 ? 1 : (c.length + c.tile - 1) / c.tile;
}

// The gradients' workgroups. A tile reads width - 1 tokens more at either end, so tiles are long where there are
// enough of them (4,096 rows of 17 tokens by 408 channels in float32: a call takes 92 us, with 16 tokens to a tile 107;
// 64 rows of 64 tokens by 512 channels: 17 us with 16 tokens, 36 with 64).
void plan_backward(Conv &c, int32_t dtype) {
  const int64_t each = dtype == RDF2V_BF16 ? kBackwardVector<bf16> : kBackwardVector<float>;
  c.vectors = (int64_t(c.channels) + each - 1) / each;
  c.blocks = (c.vectors + kWave - 1) / kWave;
  c.lanes = int32_t((c.vectors + c.blocks - 1) / c.blocks);
  tile_rows(c, 64);
  if (c.rows * c.tiles * c.vectors < (int64_t(1) << 18)) tile_rows(c, 16);
  const int64_t subs = kThreads / c.lanes, most = (c.rows * c.tiles + subs - 1) / subs;
  c.parts = std::max<int64_t>(1, std::min(most, 2048 / c.blocks));
}

}  // namespace

size_t causal_conv_backward_workspace_bytes(const rdf2v_conv &a) {
  if (a.rows == 0) return 0;
  Conv c = base(a, {}, nullptr);
  plan_backward(c, a.dtype);
  return align_up(size_t(c.parts) * a.channels * (a.width + 1) * sizeof(float), 256);
}

rdf2v_status launch_causal_conv(const rdf2v_conv &a, const rdf2v_tokens_view &x, const void *state, void *out,
                                void *state_out, int32_t *status_dev, hipStream_t stream) {
  Conv c = base(a, x, status_dev);
  c.state = state;
  c.out = out;
  c.state_out = state_out;
  tile_rows(c, 16);
  const int per = 4;
  c.vectors = (int64_t(a.channels) + per - 1) / per;
  const int64_t blocks = (a.rows * c.tiles * c.vectors + kThreads - 1) / kThreads;
  return with_width(a.width, a.silu != 0, [&](auto width, auto silu) {
    return for_each_launch(blocks, kThreads, 1, [&](int64_t first, int64_t count) {
      if (a.dtype == RDF2V_BF16)
        conv_kernel<bf16, width(), silu()><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(c, first);
      else
        conv_kernel<float, width(), silu()><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(c, first);
      RDF2V_LAUNCH_CHECK();
      return RDF2V_OK;
    });
  });
}

rdf2v_status launch_causal_conv_backward(const rdf2v_conv &a, const rdf2v_tokens_view &x,
                                         const rdf2v_tokens_view &dout, const void *state, const void *dstate_out,
                                         void *dx, float *dweight, float *dbias, void *dstate, void *workspace,
                                         int32_t *status_dev, hipStream_t stream) {
  Conv c = base(a, x, status_dev);
  c.state = state;
  c.dout = dout.data;
  c.dout_row_stride = dout.row_stride;
  c.dout_token_stride = dout.token_stride;
  c.dstate_out = dstate_out;
  c.out = dx;
  c.dstate = a.width > 1 ? dstate : nullptr;
  c.partial = static_cast<float *>(workspace);
  plan_backward(c, a.dtype);
  if (a.rows > 0) {
    const rdf2v_status st = with_width(a.width, a.silu != 0, [&](auto width, auto silu) {
      return for_each_launch(c.blocks * c.parts, kThreads, 1, [&](int64_t first, int64_t count) {
        if (a.dtype == RDF2V_BF16)
          conv_backward_kernel<bf16, width(), silu()><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(c, first);
        else
          conv_backward_kernel<float, width(), silu()><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(c, first);
        RDF2V_LAUNCH_CHECK();
        return RDF2V_OK;
      });
    });
    if (st != RDF2V_OK) return st;
  }
  return launch_part_sums({c.partial, a.rows > 0 ? c.parts : 0, {int64_t(a.channels) * a.width, a.channels, 0},
                           {dweight, dbias, nullptr}}, stream);
}

rdf2v_status launch_causal_conv_step(const rdf2v_conv &a, const rdf2v_tokens_view &x, const void *state,
                                     int64_t num_states, const int32_t *parents, void *out, void *state_out,
                                     int32_t *status_dev, hipStream_t stream) {
  Conv c = base(a, x, status_dev);
  c.state = state;
  c.num_states = num_states;
  c.parents = parents;
  c.out = out;
  c.state_out = state_out;
  const int per = a.dtype == RDF2V_BF16 ? 8 : 4;
  c.vectors = (int64_t(a.channels) + per - 1) / per;
  const int64_t blocks = (a.rows * c.vectors + kThreads - 1) / kThreads;
  return with_width(a.width, a.silu != 0, [&](auto width, auto silu) {
    return for_each_launch(blocks, kThreads, 1, [&](int64_t first, int64_t count) {
      if (a.dtype == RDF2V_BF16)
        conv_step_kernel<bf16, width(), silu()><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(c, first);
      else
        conv_step_kernel<float, width(), silu()><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(c, first);
      RDF2V_LAUNCH_CHECK();
      return RDF2V_OK;
    });
  });
}

}  // namespace rdf2v
