// Residual connection, dropout and norm on gfx950, and their gradients.
//
// hidden = residual + scale * dropout(x), out = weight * (hidden - mean) / std + bias: HBM-bound, the floor is
// each array read or written once. A token's channels stay in the registers of a team of threads between the
// sums and what needs them; a team takes tokens in turn and holds the parameters, and in the gradients their
// sums, in registers too. The dropout mask is made from counters where it is needed and never stored: ten
// rounds for four channels, in the shadow of the loads.
//
// Gradients are computed from x and residual again, not from hidden as it was rounded: the parameters'
// gradients have 32 bits, and would have lost them.
//
// Kernels' times here and below are means under the profiler, up to an eighth longer than among other calls; times of
// calls are without it.

#include "vectors.hpp"

#include "layer.hpp"
#include "logits.hpp"

namespace rdf2v {
namespace {

constexpr int kThreads = 256;
constexpr int V = 4;  // channels of a vector: what a block of the generator serves

struct Norm {
  const void *x, *residual, *dout, *dhidden;
  void *out, *hidden;  // dx and dresidual in the gradients
  const float *weight, *bias, *scale, *stats_in;
  float *stats, *partial;
  const int32_t *len;
  const int64_t *seed_offset;
  int32_t *status;
  int64_t x_row, x_token, residual_row, residual_token, dout_row, dout_token, dhidden_row, dhidden_token;
  int64_t length, tokens, row_begin, workgroups;
  uint64_t seed;
  int32_t channels;
  uint32_t threshold;
  float keep, eps;  // keep: 1 without dropout
  bool center;
};

// Four words of Philox4x32-10 (Salmon, Moraes, Dror & Shaw, SC'11).
struct Words4 {
  uint32_t w[4];
};
__device__ __forceinline__ Words4 philox(uint32_t x0, uint32_t x1, uint64_t row, uint64_t key) {
  uint32_t x2 = uint32_t(row), x3 = uint32_t(row >> 32), k0 = uint32_t(key), k1 = uint32_t(key >> 32);
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const uint64_t a = uint64_t(x0) * 0xD2511F53u, b = uint64_t(x2) * 0xCD9E8D57u;
    x0 = uint32_t(b >> 32) ^ x1 ^ k0;
    x1 = uint32_t(b);
    x2 = uint32_t(a >> 32) ^ x3 ^ k1;
    x3 = uint32_t(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{x0, x1, x2, x3}};
}

// Sums over a team of TEAM threads, in each of them: over rows of 16 lanes with DPP rotations, over the rows of a
// wave with swaps, over a team's waves through LDS. Teams of more than a wave: one barrier, and `scratch`, a place
// for each wave, is not used in the call that follows.
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&x)[N], float (*scratch)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
#define RDF2V_ROTATE(BY) \
  x[i] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x[i]), 0x120 + BY, 0xf, 0xf, false));
    RDF2V_ROTATE(8)
    RDF2V_ROTATE(4)
    RDF2V_ROTATE(2)
    RDF2V_ROTATE(1)
#undef RDF2V_ROTATE
    if constexpr (TEAM > 16) {
      const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[i]), __float_as_uint(x[i]), false, false);
      x[i] = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    if constexpr (TEAM > 32) {
      const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[i]), __float_as_uint(x[i]), false, false);
      x[i] = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
  }
  if constexpr (TEAM > kWave) {
    if (lane_id() == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) scratch[threadIdx.x / kWave][i] = x[i];
    __syncthreads();
    const int first = threadIdx.x / TEAM * (TEAM / kWave);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = scratch[first][i];
      for (int w = 1; w < TEAM / kWave; ++w) x[i] += scratch[first + w][i];
    }
  }
}

// What of a token's channels a thread has: vectors lane, lane + TEAM, ...
template <int TEAM, int PER>
struct Own {
  int lane;
  int channels;
  __device__ __forceinline__ int at(int i) const { return (lane + i * TEAM) * V; }
  __device__ __forceinline__ int count(int i) const { return min(V, channels - at(i)); }  // 0 or less: nothing there
};

template <class T, int TEAM, int PER>
__device__ __forceinline__ void load_token(const T *p, const Own<TEAM, PER> &own, float (&x)[PER][V]) {
#pragma unroll
  for (int i = 0; i < PER; ++i) load_values<T, V>(p + own.at(i), own.count(i), x[i]);
}
template <class T, int TEAM, int PER>
__device__ __forceinline__ void store_token(T *p, const Own<TEAM, PER> &own, const float (&x)[PER][V]) {
#pragma unroll
  for (int i = 0; i < PER; ++i) store_values<T, V>(p + own.at(i), own.count(i), x[i]);
}

// The residual's scale: ones where there is none.
template <int TEAM, int PER>
__device__ __forceinline__ void load_scale(const Norm &a, const Own<TEAM, PER> &own, float (&scale)[PER][V]) {
  if (a.scale != nullptr) {
    load_token(a.scale, own, scale);
    return;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) scale[i][j] = 1.0f;
}

// x after dropout, where there is any, and what is kept, a bit for each value. What is dropped counts as 0, whatever
// it holds.
template <int TEAM, int PER>
__device__ __forceinline__ void dropout(const Norm &a, const Own<TEAM, PER> &own, int64_t row, int64_t token,
                                        uint64_t key, float (&x)[PER][V], uint32_t &kept) {
  kept = ~uint32_t(0);
  if (a.threshold == 0) return;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const Words4 r = philox(uint32_t(own.at(i) / V), uint32_t(token + 1), uint64_t(a.row_begin + row), key);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const bool keep = r.w[j] >= a.threshold;
      x[i][j] = keep ? x[i][j] * a.keep : 0.0f;
      if (!keep) kept &= ~(uint32_t(1) << (i * V + j));
    }
  }
}

// Row and token of one of all tokens.
__device__ __forceinline__ void locate(const Norm &a, int64_t id, int64_t &row, int64_t &token) {
  if (a.tokens <= 0xffffffffll) {  // a division of 32 bits is a fifth of one of 64
    row = uint32_t(id) / uint32_t(a.length);
    token = uint32_t(id) - uint32_t(row) * uint32_t(a.length);
  } else {
    row = id / a.length;
    token = id % a.length;
  }
}

constexpr int workgroup_of(int team) { return team < kThreads ? kThreads : team; }
// Waves of each of a compute unit's four SIMDs, as the registers for a thread's vectors let them have.
constexpr int waves_of(bool backward, int per) { return backward || per > 3 ? 4 : per > 2 ? 5 : 6; }

// 16,384 tokens of 4,096 channels, bf16 beside a float32 residual: 145 us, 805 MB at 5.6 TB/s; 69,632 tokens of 301
// channels, half of them padding, float32: 70 us, 250 MB.
template <class T, class R, int TEAM, int PER>
__global__ __launch_bounds__(workgroup_of(TEAM), waves_of(false, PER)) void norm_kernel(Norm a) {
  constexpr int kBlock = workgroup_of(TEAM), kTeams = kBlock / TEAM;
  __shared__ float scratch[2][kBlock / kWave][1];
  const Own<TEAM, PER> own{int(threadIdx.x) % TEAM, a.channels};
  const uint64_t key = a.seed + (a.seed_offset != nullptr ? uint64_t(*a.seed_offset) : 0);
  const float inverse = 1.0f / float(a.channels);
  float weight[PER][V], scale[PER][V], bias[PER][V] = {};
  load_token(a.weight, own, weight);
  if (a.bias != nullptr) load_token(a.bias, own, bias);
  load_scale(a, own, scale);
  int turn = 0;
  for (int64_t at = int64_t(blockIdx.x) * kTeams; at < a.tokens; at += a.workgroups * kTeams) {
    // a team without a token goes along: it has lanes in common with those that have one
    const bool mine = at + int(threadIdx.x) / TEAM < a.tokens;
    const int64_t id = mine ? at + int(threadIdx.x) / TEAM : a.tokens - 1;
    int64_t row, token;
    locate(a, id, row, token);
    const bool live = token < row_length(a.len, row, a.length, mine && token == 0 && own.lane == 0, a.status);
    float h[PER][V] = {};
    if (live) {
      load_token(static_cast<const T *>(a.x) + row * a.x_row + token * a.x_token, own, h);
      float from[PER][V] = {};
      if (a.residual != nullptr)
        load_token(static_cast<const R *>(a.residual) + row * a.residual_row + token * a.residual_token, own, from);
      uint32_t kept;
      dropout(a, own, row, token, key, h, kept);
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) h[i][j] = fmaf(h[i][j], scale[i][j], from[i][j]);
    }
    if (mine && a.hidden != nullptr) store_token(static_cast<R *>(a.hidden) + id * a.channels, own, h);
    float mean = 0.0f, sum[1] = {0.0f};
    if (a.center) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += h[i][j];
      team_sum<TEAM>(sum, scratch[turn]);
      turn ^= 1;
      mean = sum[0] * inverse;
      sum[0] = 0.0f;
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) h[i][j] = j < own.count(i) ? h[i][j] - mean : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] = fmaf(h[i][j], h[i][j], sum[0]);
    team_sum<TEAM>(sum, scratch[turn]);
    turn ^= 1;
    const float inv = live ? 1.0f / sqrtf(fmaf(sum[0], inverse, a.eps)) : 0.0f;
    if (!mine) continue;
    if (a.stats != nullptr && own.lane == 0) {
      a.stats[2 * id] = mean;
      a.stats[2 * id + 1] = inv;
    }
    if (live) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) h[i][j] = fmaf(h[i][j] * inv, weight[i][j], bias[i][j]);
    }
    store_token(static_cast<T *>(a.out) + id * a.channels, own, h);
  }
}

// The teams' sums of one parameter's gradient, in order, to the workgroup's part.
template <int TEAM, int PER>
__device__ __forceinline__ void store_part(float *part, const Own<TEAM, PER> &own, const float (&x)[PER][V],
                                           float (*scratch)[V]) {
  constexpr int kTeams = workgroup_of(TEAM) / TEAM;
  if constexpr (kTeams == 1) {
    store_token(part, own, x);
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) scratch[threadIdx.x][j] = x[i][j];
      __syncthreads();
      if (threadIdx.x >= TEAM) continue;
      float sum[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        sum[j] = x[i][j];
        for (int t = 1; t < kTeams; ++t) sum[j] += scratch[t * TEAM + threadIdx.x][j];
      }
      store_values<float, V>(part + own.at(i), own.count(i), sum);
    }
  }
}

// With n = (hidden - mean) / std and dn = dout * weight, a token's gradient is
//   dhidden + (dn - n mean(dn n) - mean(dn)) / std        (the last mean where the norm is centred)
// MORE: there is a scale, or gradients of the bias or the scale are wanted. The same tokens as above: 276 us, 1.2 GB at
// 4.4 TB/s, and 100 us, 341 MB: loads, sums and stores of a token follow one another, and 16 waves to a compute unit are
// what the parameters' sums leave registers for.
template <class T, class R, bool MORE, int TEAM, int PER>
__global__ __launch_bounds__(workgroup_of(TEAM), waves_of(true, PER)) void norm_backward_kernel(Norm a) {
  constexpr int kBlock = workgroup_of(TEAM), kTeams = kBlock / TEAM;
  __shared__ float scratch[2][kBlock / kWave][2];
  __shared__ float parts[kTeams > 1 ? kBlock : 1][V];
  const Own<TEAM, PER> own{int(threadIdx.x) % TEAM, a.channels};
  const uint64_t key = a.seed + (a.seed_offset != nullptr ? uint64_t(*a.seed_offset) : 0);
  const float inverse = 1.0f / float(a.channels);
  float weight[PER][V], scale[PER][V];
  load_token(a.weight, own, weight);
  load_scale(a, own, scale);
  float dweight[PER][V] = {}, dbias[PER][V] = {}, dscale[PER][V] = {};
  int turn = 0;
  for (int64_t at = int64_t(blockIdx.x) * kTeams; at < a.tokens; at += a.workgroups * kTeams) {
    const bool mine = at + int(threadIdx.x) / TEAM < a.tokens;
    const int64_t id = mine ? at + int(threadIdx.x) / TEAM : a.tokens - 1;
    int64_t row, token;
    locate(a, id, row, token);
    const bool live =
        token < row_length(a.len, row, a.length, mine && token == 0 && own.lane == 0, a.status) && mine;
    float x[PER][V] = {}, h[PER][V] = {}, d[PER][V] = {}, dh[PER][V] = {};
    uint32_t kept = 0;
    float inv = 0.0f, sums[2] = {0.0f, 0.0f};
    if (live) {
      load_token(static_cast<const T *>(a.x) + row * a.x_row + token * a.x_token, own, x);
      if (a.residual != nullptr)
        load_token(static_cast<const R *>(a.residual) + row * a.residual_row + token * a.residual_token, own, h);
      load_token(static_cast<const T *>(a.dout) + row * a.dout_row + token * a.dout_token, own, d);
      if (a.dhidden != nullptr)
        load_token(static_cast<const R *>(a.dhidden) + row * a.dhidden_row + token * a.dhidden_token, own, dh);
      const float mean = a.stats_in[2 * id];
      inv = a.stats_in[2 * id + 1];
      dropout(a, own, row, token, key, x, kept);
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float n = ((MORE ? x[i][j] * scale[i][j] : x[i][j]) + h[i][j] - mean) * inv;
          h[i][j] = n;
          dweight[i][j] = fmaf(d[i][j], n, dweight[i][j]);
          if (MORE) dbias[i][j] += d[i][j];
          d[i][j] *= weight[i][j];
          if (j < own.count(i)) sums[0] = fmaf(d[i][j], n, sums[0]);
          sums[1] += d[i][j];
        }
    }
    team_sum<TEAM>(sums, scratch[turn]);
    turn ^= 1;
    if (!mine) continue;
    if (live) {
      const float along = sums[0] * inverse, level = a.center ? sums[1] * inverse : 0.0f;
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float g = fmaf(d[i][j] - fmaf(h[i][j], along, level), inv, dh[i][j]);
          dh[i][j] = g;
          if (MORE) dscale[i][j] = fmaf(g, x[i][j], dscale[i][j]);
          d[i][j] = MORE ? g * scale[i][j] : g;
          d[i][j] = kept >> (i * V + j) & 1 ? d[i][j] * a.keep : 0.0f;
        }
    }
    store_token(static_cast<T *>(a.out) + id * a.channels, own, d);
    if (a.hidden != nullptr) store_token(static_cast<R *>(a.hidden) + id * a.channels, own, dh);
  }
  float *part = a.partial + int64_t(blockIdx.x) * a.channels * (MORE ? 3 : 1);
  store_part(part, own, dweight, parts);
  if constexpr (MORE) {
    store_part(part + a.channels, own, dbias, parts);
    store_part(part + 2 * a.channels, own, dscale, parts);
  }
}

// Calls launch with constants for the size of a team and the vectors of a thread: the smallest team that needs two
// at most, three in the forward call: the generator works for all lanes, with channels or without. In the gradients
// a third costs in waves what idle lanes do (69,632 tokens of 301 channels: teams of 32 with three vectors and of 64
// with two take 69 and 80 us forward, 99 us both backward).
template <bool BACKWARD, class Launch>
rdf2v_status with_team(int channels, Launch launch) {
#define RDF2V_TEAM(TEAM, PER) \
  if (channels <= TEAM * PER * V) return launch(std::integral_constant<int, TEAM>{}, std::integral_constant<int, PER>{});
  RDF2V_TEAM(16, 1)
  RDF2V_TEAM(16, 2)
  RDF2V_TEAM(32, 2)
  if constexpr (!BACKWARD) {
    RDF2V_TEAM(32, 3)
  }
  RDF2V_TEAM(64, 2)
  if constexpr (!BACKWARD) {
    RDF2V_TEAM(64, 3)
  }
  RDF2V_TEAM(128, 2)
  RDF2V_TEAM(256, 2)
  RDF2V_TEAM(512, 2)
  RDF2V_TEAM(1024, 2)
  RDF2V_TEAM(1024, 4)
#undef RDF2V_TEAM
  return RDF2V_ERR_INVALID_ARGUMENT;
}

template <class Launch>
rdf2v_status with_types(int dtype, int residual_dtype, Launch launch) {
  if (dtype == RDF2V_F32) return launch(float{}, float{});
  if (residual_dtype == RDF2V_F32) return launch(bf16{}, float{});
  return launch(bf16{}, bf16{});
}

template <class Launch>
rdf2v_status with_flag(bool flag, Launch launch) {
  return flag ? launch(std::true_type{}) : launch(std::false_type{});
}

// As many workgroups as the chip's 256 compute units hold at once, at most one for each workgroup's teams of tokens:
// they take tokens in turn, and a second round of some would leave units idle (16,384 tokens of 4,096 channels,
// gradients: 349 us with 1,024 workgroups where 768 fit).
template <bool BACKWARD>
int64_t workgroups_of(int64_t tokens, int channels) {
  int64_t count = 1;
  with_team<BACKWARD>(channels, [&](auto team, auto per) {
    const int64_t waves = 4 * waves_of(BACKWARD, per());
    const int64_t teams = workgroup_of(team()) / team();
    count = std::min((tokens + teams - 1) / teams, 256 * std::max<int64_t>(1, waves * kWave / workgroup_of(team())));
    return RDF2V_OK;
  });
  return std::max<int64_t>(1, count);
}

Norm base(const rdf2v_norm &a, const rdf2v_tokens_view &x, const rdf2v_tokens_view &residual, int32_t *status) {
  Norm n{};
  n.x = x.data;
  n.x_row = x.row_stride;
  n.x_token = x.token_stride;
  n.residual = residual.data;
  n.residual_row = residual.row_stride;
  n.residual_token = residual.token_stride;
  n.weight = a.weight;
  n.bias = a.bias;
  n.scale = a.scale;
  n.len = a.len;
  n.seed_offset = a.seed_offset;
  n.status = status;
  n.length = a.length;
  n.tokens = a.rows * a.length;
  n.row_begin = a.row_begin;
  n.seed = a.seed;
  n.channels = a.channels;
  n.threshold = uint32_t(std::nearbyint(a.drop * 0x1p32));
  n.keep = n.threshold != 0 ? float(1.0 / (1.0 - a.drop)) : 1.0f;
  n.center = a.center != 0;
  n.eps = a.eps;
  return n;
}

}  // namespace

size_t residual_norm_backward_workspace_bytes(const rdf2v_norm &a) {
  if (a.rows == 0 || a.length == 0) return 0;
  return align_up(size_t(workgroups_of<true>(a.rows * a.length, a.channels)) * a.channels * 3 * sizeof(float),
                  256);
}

rdf2v_status launch_residual_norm(const rdf2v_norm &a, const rdf2v_tokens_view &x, const rdf2v_tokens_view &residual,
                                  void *out, void *hidden, float *stats, int32_t *status_dev, hipStream_t stream) {
  Norm n = base(a, x, residual, status_dev);
  n.out = out;
  n.hidden = hidden;
  n.stats = stats;
  n.workgroups = workgroups_of<false>(n.tokens, a.channels);
  return with_types(a.dtype, a.residual_dtype, [&](auto t, auto r) {
    return with_team<false>(a.channels, [&](auto team, auto per) {
      norm_kernel<decltype(t), decltype(r), team(), per()>
          <<<dim3(unsigned(n.workgroups)), dim3(workgroup_of(team())), 0, stream>>>(n);
      RDF2V_LAUNCH_CHECK();
      return RDF2V_OK;
    });
  });
}

rdf2v_status launch_residual_norm_backward(const rdf2v_norm &a, const rdf2v_tokens_view &x,
                                           const rdf2v_tokens_view &residual, const float *stats,
                                           const rdf2v_tokens_view &dout, const rdf2v_tokens_view &dhidden, void *dx,
                                           void *dresidual, float *dweight, float *dbias, float *dscale,
                                           void *workspace, int32_t *status_dev, hipStream_t stream) {
  Norm n = base(a, x, residual, status_dev);
  n.stats_in = stats;
  n.dout = dout.data;
  n.dout_row = dout.row_stride;
  n.dout_token = dout.token_stride;
  n.dhidden = dhidden.data;
  n.dhidden_row = dhidden.row_stride;
  n.dhidden_token = dhidden.token_stride;
  n.out = dx;
  n.hidden = dresidual;
  n.partial = static_cast<float *>(workspace);
  n.workgroups = n.tokens > 0 ? workgroups_of<true>(n.tokens, a.channels) : 0;
  const bool more = a.scale != nullptr || dbias != nullptr || dscale != nullptr;
  if (n.tokens > 0) {
    const rdf2v_status st = with_types(a.dtype, a.residual_dtype, [&](auto t, auto r) {
      return with_flag(more, [&](auto has) {
        return with_team<true>(a.channels, [&](auto team, auto per) {
          norm_backward_kernel<decltype(t), decltype(r), has(), team(), per()>
              <<<dim3(unsigned(n.workgroups)), dim3(workgroup_of(team())), 0, stream>>>(n);
          RDF2V_LAUNCH_CHECK();
          return RDF2V_OK;
        });
      });
    });
    if (st != RDF2V_OK) return st;
  }
  const int64_t rest = more ? a.channels : 0;
  return launch_part_sums({n.partial, n.workgroups, {a.channels, rest, rest}, {dweight, dbias, dscale}}, stream);
}

}  // namespace rdf2v
