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
  bool transposed;  // s0 is stored [dout][di]
  bool reverse;
};

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

constexpr int kColumns = 64;  // columns of S per workgroup, one to a lane

// Token by token: lane n holds column n of S in registers.
template <class T, class O, int DI>
__global__ __launch_bounds__(kColumns) void scan_kernel(ScanArgs p, int64_t first) {
  __shared__ float as[DI], bs[DI];
  const int blocks_n = (p.dout + kColumns - 1) / kColumns;
  const int64_t block = first + blockIdx.x;
  const int nb = int(block % blocks_n);
  const int h = int(block / blocks_n % p.heads);
  const int64_t row = block / blocks_n / p.heads;
  const int lane = threadIdx.x, n = nb * kColumns + lane;
  const bool report = nb == 0 && lane == 0;
  const float g = head_log_decay(p.log_decay, h, p.status, report && row == 0);
  const float gamma = expf(g);
  const int64_t len = row_length(p.len, row, p.length, p.status, report && h == 0);
  const T *a = operand_row<T>(p.a, row, h), *b = operand_row<T>(p.b, row, h), *c = operand_row<T>(p.c, row, h);
  float s[DI];
#pragma unroll
  for (int i = 0; i < DI; ++i) {
    s[i] = 0.0f;
    if (p.s0 != nullptr && i < p.di && n < p.dout) {
      const float *s0 = p.s0 + (row * p.heads + h) * int64_t(p.di) * p.dout;
      s[i] = p.transposed ? s0[int64_t(n) * p.di + i] : s0[int64_t(i) * p.dout + n];
    }
  }
  O *out = static_cast<O *>(p.out) + (row * p.length * p.heads + h) * int64_t(p.dout);
  const int64_t step = int64_t(p.heads) * p.dout;
  for (int64_t u = 0; u < len; ++u) {
    const int64_t t = p.reverse ? len - 1 - u : u;
    __syncthreads();
    for (int i = lane; i < DI; i += kColumns) {
      as[i] = i < p.di ? to_f32(a[t * p.a.token + i]) : 0.0f;
      bs[i] = i < p.di ? to_f32(b[t * p.b.token + i]) * p.sscale : 0.0f;
    }
    __syncthreads();
    const float cv = n < p.dout ? to_f32(c[t * p.c.token + n]) : 0.0f;
    const float d = p.reverse && u == 0 ? 1.0f : gamma;
    float o = 0.0f;
#pragma unroll
    for (int i = 0; i < DI; ++i) {
      s[i] = fmaf(s[i], d, bs[i] * cv);
      o = fmaf(as[i], s[i], o);
    }
    if (n < p.dout) out[t * step + n] = from_f32<O>(o * p.oscale);
  }
  for (int64_t t = len; t < p.length; ++t)
    if (n < p.dout) out[t * step + n] = from_f32<O>(0.0f);
  if (p.s1 != nullptr && n < p.dout) {
    float *s1 = p.s1 + (row * p.heads + h) * int64_t(p.di) * p.dout;
    const float d = p.reverse && len > 0 ? gamma : 1.0f;
#pragma unroll
    for (int i = 0; i < DI; ++i)
      if (i < p.di) s1[int64_t(i) * p.dout + n] = s[i] * d;
  }
}

template <class T, class O>
rdf2v_status launch_scan(const ScanArgs &p, hipStream_t stream) {
  const int64_t blocks = p.rows * p.heads * ((p.dout + kColumns - 1) / kColumns);
  return for_each_launch(blocks, kColumns, 1, [&](int64_t first, int64_t count) {
    if (p.di <= 32)
      scan_kernel<T, O, 32><<<dim3(unsigned(count)), dim3(kColumns), 0, stream>>>(p, first);
    else if (p.di <= 64)
      scan_kernel<T, O, 64><<<dim3(unsigned(count)), dim3(kColumns), 0, stream>>>(p, first);
    else
      scan_kernel<T, O, 128><<<dim3(unsigned(count)), dim3(kColumns), 0, stream>>>(p, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

// Sums of the gradients of `share` query heads, in head order.
template <class T>
__global__ __launch_bounds__(256) void share_sum_kernel(const float *part, T *out, int64_t groups, int share, int d,
                                                        int64_t first) {
  const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x;
  if (i >= groups * d) return;
  const float *x = part + i / d * share * d + i % d;
  float sum = 0.0f;
  for (int j = 0; j < share; ++j) sum += x[int64_t(j) * d];
  out[i] = from_f32<T>(sum);
}

template <class T>
rdf2v_status launch_share_sum(const float *part, void *out, int64_t groups, int share, int d, hipStream_t stream) {
  return for_each_launch((groups * d + 255) / 256, 256, 1, [&](int64_t first, int64_t count) {
    share_sum_kernel<T>
        <<<dim3(unsigned(count)), dim3(256), 0, stream>>>(part, static_cast<T *>(out), groups, share, d, first);
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
                     const rdf2v_heads_view &v, const float *state, void *out, float *state_out, int32_t *status,
                     hipStream_t stream) {
  const int share = a.heads / a.kv_heads;
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
  return launch_scan<T, T>(p, stream);
}

template <class T>
rdf2v_status backward(const rdf2v_attention &a, const rdf2v_heads_view &q, const rdf2v_heads_view &k,
                      const rdf2v_heads_view &v, const rdf2v_heads_view &dout, const float *state,
                      const float *dstate_out, void *dq, void *dk, void *dv, float *dstate, void *workspace,
                      int32_t *status, hipStream_t stream) {
  const int share = a.heads / a.kv_heads;
  const int64_t tokens = a.rows * a.length;
  ScanArgs p = scan_args(a, status);
  p.a = operand(dout, 1);
  p.b = operand(v, share);
  p.c = operand(k, share);
  p.di = a.dv;
  p.dout = a.dk;
  p.s0 = state;
  p.transposed = true;
  p.out = dq;
  p.oscale = a.scale;
  rdf2v_status st = launch_scan<T, T>(p, stream);
  if (st != RDF2V_OK) return st;

  float *part = static_cast<float *>(workspace);
  p = scan_args(a, status);
  p.reverse = true;
  p.sscale = a.scale;
  p.a = operand(v, share);
  p.b = operand(dout, 1);
  p.c = operand(q, 1);
  p.di = a.dv;
  p.dout = a.dk;
  p.s0 = dstate_out;
  p.transposed = true;
  p.out = share > 1 ? part : dk;
  st = share > 1 ? launch_scan<T, float>(p, stream) : launch_scan<T, T>(p, stream);
  if (st == RDF2V_OK && share > 1) st = launch_share_sum<T>(part, dk, tokens * a.kv_heads, share, a.dk, stream);
  if (st != RDF2V_OK) return st;

  p.a = operand(k, share);
  p.b = operand(q, 1);
  p.c = operand(dout, 1);
  p.di = a.dk;
  p.dout = a.dv;
  p.transposed = false;
  p.out = share > 1 ? part : dv;
  p.s1 = dstate;
  st = share > 1 ? launch_scan<T, float>(p, stream) : launch_scan<T, T>(p, stream);
  if (st == RDF2V_OK && share > 1) st = launch_share_sum<T>(part, dv, tokens * a.kv_heads, share, a.dv, stream);
  return st;
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

template <class T>
__global__ __launch_bounds__(kColumns) void step_kernel(StepArgs p, int64_t first) {
  const int blocks_n = (p.dv + kColumns - 1) / kColumns;
  const int64_t block = first + blockIdx.x;
  const int nb = int(block % blocks_n);
  const int h = int(block / blocks_n % p.heads);
  const int64_t row = block / blocks_n / p.heads;
  const int n = nb * kColumns + threadIdx.x;
  const bool report = nb == 0 && threadIdx.x == 0;
  const float gamma = expf(head_log_decay(p.log_decay, h, p.status, report && row == 0));
  int64_t from = row;
  if (p.parents != nullptr) {
    from = p.parents[row];
    if (from < 0 || from >= p.num_states) {
      from = -1;
      if (report && h == 0 && p.status != nullptr) atomicOr(p.status, RDF2V_STATUS_ID_OUT_OF_RANGE);
    }
  }
  const T *q = operand_row<T>(p.q, row, h), *k = operand_row<T>(p.k, row, h), *v = operand_row<T>(p.v, row, h);
  if (n >= p.dv) return;
  const int64_t size = int64_t(p.dk) * p.dv;
  const float *s0 = p.state + (from * p.heads + h) * size + n;
  float *s1 = p.state_out + (row * p.heads + h) * size + n;
  const float vn = to_f32(v[n]);
  float o = 0.0f;
  for (int i = 0; i < p.dk; ++i) {
    const float s = fmaf(from < 0 ? 0.0f : s0[int64_t(i) * p.dv], gamma, to_f32(k[i]) * vn);
    s1[int64_t(i) * p.dv] = s;
    o = fmaf(to_f32(q[i]), s, o);
  }
  static_cast<T *>(p.out)[(row * p.heads + h) * p.dv + n] = from_f32<T>(o * p.scale);
}

}  // namespace

size_t decay_attention_workspace_bytes(const rdf2v_attention &a, bool backward) {
  if (!backward || a.heads == a.kv_heads) return 0;
  return align_up(size_t(a.rows) * a.length * a.heads * (a.dk > a.dv ? a.dk : a.dv) * sizeof(float), 256);
}

rdf2v_status launch_decay_attention(const rdf2v_attention &a, const rdf2v_heads_view &q, const rdf2v_heads_view &k,
                                    const rdf2v_heads_view &v, const float *state, void *out, float *state_out,
                                    void *, int32_t *status_dev, hipStream_t stream) {
  return a.dtype == RDF2V_BF16 ? forward<bf16>(a, q, k, v, state, out, state_out, status_dev, stream)
                               : forward<float>(a, q, k, v, state, out, state_out, status_dev, stream);
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
  const int64_t blocks = a.rows * a.heads * ((a.dv + kColumns - 1) / kColumns);
  return for_each_launch(blocks, kColumns, 1, [&](int64_t first, int64_t count) {
    if (a.dtype == RDF2V_BF16)
      step_kernel<bf16><<<dim3(unsigned(count)), dim3(kColumns), 0, stream>>>(p, first);
    else
      step_kernel<float><<<dim3(unsigned(count)), dim3(kColumns), 0, stream>>>(p, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

}  // namespace rdf2v
