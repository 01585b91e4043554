// Attention under the masks of packed, prefixed, padded and cached sequences, and its backward pass.
//
//   z_ij = scale q_i . k_j, capped: cap tanh(z / cap), minus slope_h |pos_i - j|;  p_i = softmax over first_i <= j < end_i;  o_i = sum p_ij v_j
//   dv_j = sum_i p_ij do_i;  dz = p (do_i . v_j - do_i . o_i) (1 - tanh^2);  dq_i = scale sum_j dz k_j;  dk_j = scale sum_i dz q_i
//
// A wavefront to a query (forward, dq) or to a key (dk, dv), its lanes over the head's columns, one pass with the running maximum and sum.

#include <math.h>

#include "hdet_ops.h"
#include "hdet_elem.h"

namespace {

constexpr int THREADS = 256;
constexpr int WAVES = THREADS / 64;

struct attend_args {
  const void *q, *k, *v, *o, *dout;
  void *out, *dq, *dk, *dv;
  int64_t q_s, q_z, k_s, k_z, v_s, v_z, o_s, o_z, do_s, do_z, out_s, out_z, dq_s, dq_z, dk_s, dk_z, dv_s, dv_z;
  float* lse;
  const float* lse_in;
  float* dot;                              // backward: [replica][head][row] sum_c do o
  const float* slopes;
  int64_t slopes_z;
  const int32_t *pos, *first, *end;
  int n, seqs, q_len, kv_len, heads, kv_heads, d, causal, window;
  float scale, cap, inv_cap;
};

struct key_range { int lo, hi; int64_t pos; };

// Keys that query i of sequence b attends: lo .. hi - 1
__device__ __forceinline__ key_range range_of(const attend_args& g, int r, int b, int i) {
  const int64_t row = (int64_t)b * g.q_len + i, at = (int64_t)r * g.seqs * g.q_len + row;
  const int64_t pos = g.pos ? g.pos[at] : (int64_t)i + g.kv_len - g.q_len;
  int64_t lo = 0, hi = g.kv_len;
  if (g.first && g.first[at] > lo) lo = g.first[at];
  if (g.window && pos - g.window + 1 > lo) lo = pos - g.window + 1;
  if (g.end && g.end[at] < hi) hi = g.end[at];
  if (g.causal && pos + 1 < hi) hi = pos + 1;
  if (hi <= lo) lo = hi = 0;
  return {(int)lo, (int)hi, pos};
}

// the score of a pair from q . k; `slope` receives the derivative of the cap
__device__ __forceinline__ float score(const attend_args& g, float qk, float slope, int64_t distance, float& bend) {
  float z = qk * g.scale;
  bend = 1.f;
  if (g.cap > 0.f) {
    const float t = tanhf(z * g.inv_cap);
    z = g.cap * t;
    bend = 1.f - t * t;
  }
  return __builtin_fmaf(-slope, (float)(distance < 0 ? -distance : distance), z);
}

template <typename T> struct lane_columns {            // columns lane and lane + 64 of a head
  float a, b;
  __device__ __forceinline__ lane_columns(const T* p, int lane, int d) : a(lane < d ? hdet_ld(p + lane) : 0.f), b(lane + 64 < d ? hdet_ld(p + lane + 64) : 0.f) {}
  __device__ __forceinline__ float dot(const lane_columns& o) const { return hdet_wave_sum(__builtin_fmaf(a, o.a, b * o.b)); }
};
template <typename T> __device__ __forceinline__ void store_columns(T* p, int lane, int d, float a, float b) {
  if (lane < d) hdet_st(p + lane, a);
  if (lane + 64 < d) hdet_st(p + lane + 64, b);
}

__device__ __forceinline__ int64_t wave_index() { return (((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * THREADS + threadIdx.x) >> 6; }

template <typename T> __global__ __launch_bounds__(THREADS) void attend_kernel(const attend_args g) {
  const int64_t w = wave_index(), rows = (int64_t)g.seqs * g.q_len;
  if (w >= rows * g.heads * g.n) return;
  const int lane = threadIdx.x & 63, h = (int)(w % g.heads), kh = h / (g.heads / g.kv_heads);
  const int64_t row = w / g.heads % rows;
  const int r = (int)(w / g.heads / rows), b = (int)(row / g.q_len);
  const key_range range = range_of(g, r, b, (int)(row % g.q_len));
  const lane_columns<T> q((const T*)g.q + r * g.q_z + row * g.q_s + (int64_t)h * g.d, lane, g.d);
  const T* k = (const T*)g.k + r * g.k_z + (int64_t)b * g.kv_len * g.k_s + (int64_t)kh * g.d;
  const T* v = (const T*)g.v + r * g.v_z + (int64_t)b * g.kv_len * g.v_s + (int64_t)kh * g.d;
  const float slope = g.slopes ? g.slopes[r * g.slopes_z + h] : 0.f;
  float m = -INFINITY, l = 0.f, oa = 0.f, ob = 0.f, bend;
  for (int j = range.lo; j < range.hi; ++j) {
    const float z = score(g, q.dot(lane_columns<T>(k + j * g.k_s, lane, g.d)), slope, range.pos - j, bend);
    const lane_columns<T> x(v + j * g.v_s, lane, g.d);
    const float top = fmaxf(m, z), ref = top == -INFINITY ? 0.f : top;
    const float keep = expf(m - ref), p = expf(z - ref);
    l = __builtin_fmaf(l, keep, p);
    oa = __builtin_fmaf(oa, keep, p * x.a);
    ob = __builtin_fmaf(ob, keep, p * x.b);
    m = top;
  }
  const float inv = range.hi > range.lo ? 1.f / l : 0.f;
  store_columns((T*)g.out + r * g.out_z + row * g.out_s + (int64_t)h * g.d, lane, g.d, oa * inv, ob * inv);
  if (g.lse && lane == 0) g.lse[((int64_t)r * g.heads + h) * rows + row] = range.hi > range.lo ? m + logf(l) : -INFINITY;
}

template <typename T> __global__ __launch_bounds__(THREADS) void attend_dq_kernel(const attend_args g) {
  const int64_t w = wave_index(), rows = (int64_t)g.seqs * g.q_len;
  if (w >= rows * g.heads * g.n) return;
  const int lane = threadIdx.x & 63, h = (int)(w % g.heads), kh = h / (g.heads / g.kv_heads);
  const int64_t row = w / g.heads % rows;
  const int r = (int)(w / g.heads / rows), b = (int)(row / g.q_len);
  const key_range range = range_of(g, r, b, (int)(row % g.q_len));
  const int64_t col = (int64_t)h * g.d, stat = ((int64_t)r * g.heads + h) * rows + row;
  T* const dq = (T*)g.dq + r * g.dq_z + row * g.dq_s + col;
  if (range.hi == range.lo) return store_columns(dq, lane, g.d, 0.f, 0.f);
  const lane_columns<T> q((const T*)g.q + r * g.q_z + row * g.q_s + col, lane, g.d), o((const T*)g.o + r * g.o_z + row * g.o_s + col, lane, g.d);
  const lane_columns<T> dout((const T*)g.dout + r * g.do_z + row * g.do_s + col, lane, g.d);
  const T* k = (const T*)g.k + r * g.k_z + (int64_t)b * g.kv_len * g.k_s + (int64_t)kh * g.d;
  const T* v = (const T*)g.v + r * g.v_z + (int64_t)b * g.kv_len * g.v_s + (int64_t)kh * g.d;
  const float slope = g.slopes ? g.slopes[r * g.slopes_z + h] : 0.f, lse = g.lse_in[stat], dot = dout.dot(o);
  float a = 0.f, c = 0.f, bend;
  for (int j = range.lo; j < range.hi; ++j) {
    const lane_columns<T> x(k + j * g.k_s, lane, g.d);
    const float p = expf(score(g, q.dot(x), slope, range.pos - j, bend) - lse);
    const float dz = p * (dout.dot(lane_columns<T>(v + j * g.v_s, lane, g.d)) - dot) * bend;
    a = __builtin_fmaf(dz, x.a, a);
    c = __builtin_fmaf(dz, x.b, c);
  }
  store_columns(dq, lane, g.d, a * g.scale, c * g.scale);
  if (lane == 0) g.dot[stat] = dot;
}

template <typename T> __global__ __launch_bounds__(THREADS) void attend_dkv_kernel(const attend_args g) {
  const int64_t w = wave_index(), keys = (int64_t)g.seqs * g.kv_len, rows = (int64_t)g.seqs * g.q_len;
  if (w >= keys * g.kv_heads * g.n) return;
  const int lane = threadIdx.x & 63, kh = (int)(w % g.kv_heads), group = g.heads / g.kv_heads;
  const int64_t key = w / g.kv_heads % keys;
  const int r = (int)(w / g.kv_heads / keys), b = (int)(key / g.kv_len), j = (int)(key % g.kv_len);
  const lane_columns<T> k((const T*)g.k + r * g.k_z + key * g.k_s + (int64_t)kh * g.d, lane, g.d), v((const T*)g.v + r * g.v_z + key * g.v_s + (int64_t)kh * g.d, lane, g.d);
  float ka = 0.f, kb = 0.f, va = 0.f, vb = 0.f, bend;
  for (int h = kh * group; h < (kh + 1) * group; ++h) {
    const float slope = g.slopes ? g.slopes[r * g.slopes_z + h] : 0.f;
    for (int i = 0; i < g.q_len; ++i) {
      const key_range range = range_of(g, r, b, i);
      if (j < range.lo || j >= range.hi) continue;
      const int64_t row = (int64_t)b * g.q_len + i, col = (int64_t)h * g.d, stat = ((int64_t)r * g.heads + h) * rows + row;
      const lane_columns<T> q((const T*)g.q + r * g.q_z + row * g.q_s + col, lane, g.d), dout((const T*)g.dout + r * g.do_z + row * g.do_s + col, lane, g.d);
      const float p = expf(score(g, q.dot(k), slope, range.pos - j, bend) - g.lse_in[stat]);
      const float dz = p * (dout.dot(v) - g.dot[stat]) * bend;
      ka = __builtin_fmaf(dz, q.a, ka);
      kb = __builtin_fmaf(dz, q.b, kb);
      va = __builtin_fmaf(p, dout.a, va);
      vb = __builtin_fmaf(p, dout.b, vb);
    }
  }
  store_columns((T*)g.dk + r * g.dk_z + key * g.dk_s + (int64_t)kh * g.d, lane, g.d, ka * g.scale, kb * g.scale);
  store_columns((T*)g.dv + r * g.dv_z + key * g.dv_s + (int64_t)kh * g.d, lane, g.d, va, vb);
}

template <typename A> attend_args common_args(const A& a) {
  attend_args g = {};
  g.q = a.q.dev; g.q_s = a.q.row_stride; g.q_z = a.q.replica_stride;
  g.k = a.k.dev; g.k_s = a.k.row_stride; g.k_z = a.k.replica_stride;
  g.v = a.v.dev; g.v_s = a.v.row_stride; g.v_z = a.v.replica_stride;
  g.slopes = a.slopes_dev; g.slopes_z = a.slopes_stride;
  g.pos = a.positions_dev; g.first = a.first_dev; g.end = a.end_dev;
  g.n = a.n_replicas; g.seqs = a.seqs; g.q_len = a.q_len; g.kv_len = a.kv_len; g.heads = a.heads; g.kv_heads = a.kv_heads; g.d = a.head_dim;
  g.causal = a.causal; g.window = a.window;
  g.scale = (float)a.scale; g.cap = (float)a.softcap; g.inv_cap = a.softcap > 0 ? (float)(1.0 / a.softcap) : 0.f;
  return g;
}
dim3 wave_grid(int64_t waves) {
  const int64_t blocks = (waves + WAVES - 1) / WAVES, x = blocks < (1 << 20) ? blocks : 1 << 20;
  return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

}  // namespace

size_t hdet_attend_bytes(int, int, int, int, int, int, int) { return 0; }
size_t hdet_attend_backward_bytes(int n, int seqs, int q_len, int, int heads, int, int) { return (size_t)n * seqs * q_len * heads * sizeof(float); }

hipError_t hdet_launch_attend(const hdet_attention_args& a, hipStream_t s) {
  attend_args g = common_args(a);
  g.out = a.out.dev; g.out_s = a.out.row_stride; g.out_z = a.out.replica_stride;
  g.lse = a.lse_dev;
  const int64_t waves = (int64_t)a.seqs * a.q_len * a.heads * a.n_replicas;
  if (waves == 0) return hipSuccess;
  if (a.dtype == HDET_TYPE_BF16) hipLaunchKernelGGL(attend_kernel<uint16_t>, wave_grid(waves), dim3(THREADS), 0, s, g);
  else hipLaunchKernelGGL(attend_kernel<float>, wave_grid(waves), dim3(THREADS), 0, s, g);
  return hipGetLastError();
}

hipError_t hdet_launch_attend_backward(const hdet_attention_grad_args& a, hipStream_t s) {
  attend_args g = common_args(a);
  g.o = a.out.dev; g.o_s = a.out.row_stride; g.o_z = a.out.replica_stride;
  g.dout = a.dout.dev; g.do_s = a.dout.row_stride; g.do_z = a.dout.replica_stride;
  g.dq = a.dq.dev; g.dq_s = a.dq.row_stride; g.dq_z = a.dq.replica_stride;
  g.dk = a.dk.dev; g.dk_s = a.dk.row_stride; g.dk_z = a.dk.replica_stride;
  g.dv = a.dv.dev; g.dv_s = a.dv.row_stride; g.dv_z = a.dv.replica_stride;
  g.lse_in = a.lse_dev;
  g.dot = (float*)a.workspace_dev;
  const int64_t q_waves = (int64_t)a.seqs * a.q_len * a.heads * a.n_replicas, k_waves = (int64_t)a.seqs * a.kv_len * a.kv_heads * a.n_replicas;
  auto go = [&](auto e) {
    typedef decltype(e) T;
    if (q_waves) hipLaunchKernelGGL(attend_dq_kernel<T>, wave_grid(q_waves), dim3(THREADS), 0, s, g);
    if (k_waves) hipLaunchKernelGGL(attend_dkv_kernel<T>, wave_grid(k_waves), dim3(THREADS), 0, s, g);
  };
  if (a.dtype == HDET_TYPE_BF16) go(uint16_t());
  else go(float());
  return hipGetLastError();
}
