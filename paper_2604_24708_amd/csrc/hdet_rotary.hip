// Norm of every head of the queries and keys with the rotation by position, and the backward pass.
//
//   xh = x rstd, rstd = 1 / sqrt(mean x^2 + eps);  u = xh g;  y = R(pos) u:  pairs (u_1, u_2) -> m (u_1 cos a - u_2 sin a, u_1 sin a + u_2 cos a), a = pos f_t
//   w = R(pos)^T dy;  dx = rstd (w g - xh mean(w g xh));  dg = sum w xh
//
// Bound by memory: heads are read once and written once.  A head is held by a team of T lanes, 8 pairs of columns each, so that a rotation
// never leaves a lane and the norm's sums are log2 T exchanges.  A block first forms the cosines and sines of its rows, once for all heads of
// a row, in LDS, then walks over the heads.

#include <algorithm>
#include <type_traits>

#include "hdet_ops.h"
#include "hdet_elem.h"

namespace {

constexpr int THREADS = 256;
constexpr int MAX_ROWS = 16;               // rows of a block's table at a time
constexpr int MAX_TABLE = 1024;            // pairs of the table: 8 KiB

// How a head's columns lie in the lanes' pairs: 8 neighbours and the 8 that they turn with (halves), 16 neighbours (pairs), or single elements of
// heads that are no whole pieces of 8 columns at 16-byte boundaries
enum { kHalves = 0, kPairs = 1, kLoose = 2 };

struct side {                              // the queries or the keys
  const void *x, *dy;
  void* y;                                 // forward: the output; backward: the gradient
  int64_t x_s, x_z, dy_s, dy_z, y_s, y_z;
  const float* gain;
  int64_t gain_z;
  int heads;
  int sums;                                // backward: the gain's gradient is wanted
};
struct rotary_args {
  side s[2];
  const int32_t* pos;
  const double* freq;
  float* partial;                          // [replica][block][2][d]
  int64_t rows;
  int d, half, period, table_rows;         // half: number of pairs that turn
  int paired;                              // kLoose: which columns are a pair
  double eps;
  float magnitude, inv_d;
};

// Cosine and sine of a in 64 bits' angle: the quarter turns are taken off in 64 bits (pi / 2 in two parts), what is left, at most pi / 4, goes
// through the Taylor polynomials of degree 10 and 9: off by less than 2^-29, and by fp32's roundings.
__device__ __forceinline__ float2 cos_sin(double a) {
  const double q = rint(a * 0.63661977236758134308);
  double r = __builtin_fma(-q, 1.5707963267948965580, a);
  r = __builtin_fma(-q, 6.1232339957367660359e-17, r);
  const float x = (float)r, x2 = x * x;
  const float s = __builtin_fmaf(x * x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -0.16666667f), x);
  const float c = __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f),
                                                                            4.1666668e-2f), -0.5f), 1.f);
  const int k = (int)(q - 4.0 * floor(q * 0.25));
  const float cc = k & 1 ? s : c, ss = k & 1 ? c : s;
  return make_float2(k == 1 || k == 2 ? -cc : cc, k >= 2 ? -ss : ss);
}

// Sum over the T lanes of a team, the same in each
template <int T> __device__ __forceinline__ float team_sum(float v) {
  if (T > 1) v += hdet_dpp<0xB1>(v);
  if (T > 2) v += hdet_dpp<0x4E>(v);
  if (T > 4) v += hdet_dpp<0x141>(v);
  if (T > 8) v += hdet_dpp<0x140>(v);
  return v;
}
template <int T> __device__ __forceinline__ double team_sum64(double v) {
  for (int o = 1; o < T; o <<= 1) v += __shfl_xor(v, o);
  return v;
}

struct pairs { float a[8], b[8]; };

// Column of the first and second of a lane's pairs, d and beyond: none
template <int MODE, int T> __device__ __forceinline__ void columns(const rotary_args& g, int l, int i, int& ca, int& cb, int& t) {
  if (MODE == kLoose) {
    t = l + T * i;
    if (t < g.half) {
      ca = g.paired ? 2 * t : t;
      cb = g.paired ? 2 * t + 1 : t + g.half;
    } else {
      ca = 2 * t;
      cb = 2 * t + 1;
    }
  } else {
    t = 8 * l + i;
    if (MODE == kHalves && 8 * l < g.half) {
      ca = t;
      cb = t + g.half;
    } else if (MODE == kHalves) {
      ca = 16 * l + i;
      cb = ca + 8;
    } else {
      ca = 2 * t;
      cb = 2 * t + 1;
    }
  }
}

// A lane's pairs of a head at p; zeros in columns that there are not
template <typename E, int MODE, int T> __device__ __forceinline__ pairs load_pairs(const rotary_args& g, const E* p, int l) {
  pairs v;
  if (MODE == kLoose) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int ca, cb, t;
      columns<MODE, T>(g, l, i, ca, cb, t);
      v.a[i] = ca < g.d ? hdet_ld(p + ca) : 0.f;
      v.b[i] = cb < g.d ? hdet_ld(p + cb) : 0.f;
    }
    return v;
  }
  int ca, cb, t;
  columns<MODE, T>(g, l, 0, ca, cb, t);
  if (MODE == kPairs) cb = ca + 8;
  hdet_f8 x = {}, y = {};
  if (ca < g.d) x = hdet_ld8(p + ca);
  if (cb < g.d) y = hdet_ld8(p + cb);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v.a[i] = MODE == kHalves ? x.v[i] : i < 4 ? x.v[2 * (i & 3)] : y.v[2 * (i & 3)];
    v.b[i] = MODE == kHalves ? y.v[i] : i < 4 ? x.v[2 * (i & 3) + 1] : y.v[2 * (i & 3) + 1];
  }
  return v;
}
template <typename E, int MODE, int T> __device__ __forceinline__ void store_pairs(const rotary_args& g, E* p, int l, const pairs& v) {
  if (MODE == kLoose) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int ca, cb, t;
      columns<MODE, T>(g, l, i, ca, cb, t);
      if (ca < g.d) hdet_st(p + ca, v.a[i]);
      if (cb < g.d) hdet_st(p + cb, v.b[i]);
    }
    return;
  }
  int ca, cb, t;
  columns<MODE, T>(g, l, 0, ca, cb, t);
  if (MODE == kPairs) cb = ca + 8;
  hdet_f8 x, y;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x.v[i] = MODE == kHalves ? v.a[i] : i & 1 ? v.b[i >> 1] : v.a[i >> 1];
    y.v[i] = MODE == kHalves ? v.b[i] : i & 1 ? v.b[4 + (i >> 1)] : v.a[4 + (i >> 1)];
  }
  if (ca < g.d) hdet_st8(p + ca, x);
  if (cb < g.d) hdet_st8(p + cb, y);
}

// 1 / sqrt(mean x^2 + eps): fp32 sums, in 64 bits where the squares leave fp32's range
template <int T> __device__ __forceinline__ float rstd_of(const rotary_args& g, const pairs& v) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = __builtin_fmaf(v.a[i], v.a[i], __builtin_fmaf(v.b[i], v.b[i], s));
  s = team_sum<T>(s);
  const float m = __builtin_fmaf(s, g.inv_d, (float)g.eps);
  if (m > 1e-30f && m < 1e30f) {
    const float r = __builtin_amdgcn_rsqf(m);
    return r * __builtin_fmaf(-0.5f * m * r, r, 1.5f);
  }
  double w = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) w += (double)v.a[i] * v.a[i] + (double)v.b[i] * v.b[i];
  return (float)(1.0 / sqrt(team_sum64<T>(w) / g.d + g.eps));
}

__device__ __forceinline__ double position(const rotary_args& g, int r, int64_t row) {
  return g.pos ? (double)g.pos[(int64_t)r * g.rows + row] : (double)(g.period ? row % g.period : row);
}

// One block: rows `table_rows` at a time, all heads of them.  BACK: the gradients, and the gains' partial sums.
template <typename E, int MODE, int T, bool BACK> __global__ __launch_bounds__(THREADS) void rotary_kernel(const rotary_args g) {
  __shared__ float2 table[MAX_TABLE];
  __shared__ float sums[BACK ? THREADS * 16 : 1];
  const int tid = threadIdx.x, l = tid % T, r = blockIdx.y;
  const int64_t chunks = (g.rows + g.table_rows - 1) / g.table_rows;
  pairs acc[2] = {};
  pairs gain[2];
#pragma unroll
  for (int z = 0; z < 2; ++z)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int ca, cb, t;
      columns<MODE, T>(g, l, i, ca, cb, t);
      const float* q = g.s[z].gain ? g.s[z].gain + r * g.s[z].gain_z : nullptr;
      gain[z].a[i] = q && ca < g.d ? q[ca] : 0.f;
      gain[z].b[i] = q && cb < g.d ? q[cb] : 0.f;
    }
  for (int64_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
    const int64_t row0 = chunk * g.table_rows;
    const int have = (int)(g.rows - row0 < g.table_rows ? g.rows - row0 : g.table_rows);
    __syncthreads();                       // the last rows' table has been read
    for (int i = tid; i < have * g.half; i += THREADS) {
      const int row = i / g.half;
      float2 cs = cos_sin(position(g, r, row0 + row) * g.freq[i - row * g.half]);
      table[i] = make_float2(cs.x * g.magnitude, (BACK ? -cs.y : cs.y) * g.magnitude);
    }
    __syncthreads();
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const side& s = g.s[z];
      const int items = have * s.heads * T;
      for (int i = tid; i < items; i += THREADS) {
        const int team = i / T, row = team / s.heads, head = team - row * s.heads;
        const int64_t at = row0 + row;
        pairs x = {}, dy;
        float rstd = 1.f;
        if (!BACK || s.gain) x = load_pairs<E, MODE, T>(g, (const E*)s.x + r * s.x_z + at * s.x_s + (int64_t)head * g.d, l);
        if (BACK) dy = load_pairs<E, MODE, T>(g, (const E*)s.dy + r * s.dy_z + at * s.dy_s + (int64_t)head * g.d, l);
        if (s.gain) rstd = rstd_of<T>(g, x);
        pairs& v = BACK ? dy : x;
        if (!BACK && s.gain) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v.a[e] = v.a[e] * rstd * gain[z].a[e];
            v.b[e] = v.b[e] * rstd * gain[z].b[e];
          }
        }
        const float2* cs = table + row * g.half;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int t = MODE == kLoose ? l + T * e : 8 * l + e;
          if (t < g.half) {
            const float2 c = cs[t];
            const float a = v.a[e], b = v.b[e];
            v.a[e] = __builtin_fmaf(a, c.x, -b * c.y);
            v.b[e] = __builtin_fmaf(a, c.y, b * c.x);
          }
        }
        if (BACK && s.gain) {
          float dot = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x.a[e] *= rstd;
            x.b[e] *= rstd;
            if (s.sums) {
              acc[z].a[e] = __builtin_fmaf(v.a[e], x.a[e], acc[z].a[e]);
              acc[z].b[e] = __builtin_fmaf(v.b[e], x.b[e], acc[z].b[e]);
            }
            v.a[e] *= gain[z].a[e];
            v.b[e] *= gain[z].b[e];
            dot = __builtin_fmaf(v.a[e], x.a[e], __builtin_fmaf(v.b[e], x.b[e], dot));
          }
          dot = team_sum<T>(dot) * g.inv_d;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v.a[e] = rstd * __builtin_fmaf(-x.a[e], dot, v.a[e]);
            v.b[e] = rstd * __builtin_fmaf(-x.b[e], dot, v.b[e]);
          }
        }
        store_pairs<E, MODE, T>(g, (E*)s.y + r * s.y_z + at * s.y_s + (int64_t)head * g.d, l, v);
      }
    }
  }
  if (!BACK) return;
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    if (!g.s[z].sums) continue;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sums[(tid / T) * (16 * T) + (2 * e) * T + l] = acc[z].a[e];
      sums[(tid / T) * (16 * T) + (2 * e + 1) * T + l] = acc[z].b[e];
    }
    __syncthreads();
    for (int j = tid; j < 16 * T; j += THREADS) {
      float v = 0.f;
      for (int team = 0; team < THREADS / T; ++team) v += sums[team * (16 * T) + j];
      int ca, cb, t;
      columns<MODE, T>(g, j % T, j / T / 2, ca, cb, t);
      const int c = j / T & 1 ? cb : ca;
      if (c < g.d) g.partial[(((int64_t)r * gridDim.x + blockIdx.x) * 2 + z) * g.d + c] = v;
    }
  }
}

// The gains' gradients from the blocks' sums: 16 rows of threads walk over the blocks, then their sums in order
__global__ __launch_bounds__(1024) void rotary_gain_kernel(const float* partial, int parts, int d, float* q, int64_t q_z, float* k, int64_t k_z) {
  __shared__ float part[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6, r = blockIdx.y, z = blockIdx.z;
  float* out = z ? k : q;
  if (!out) return;
  float v = 0.f;
  if (c < d)
    for (int p = w; p < parts; p += 16) v += partial[(((int64_t)r * parts + p) * 2 + z) * d + c];
  part[w][threadIdx.x & 63] = v;
  __syncthreads();
  if (w == 0 && c < d) {
    for (int i = 1; i < 16; ++i) v += part[i][threadIdx.x];
    out[r * (z ? k_z : q_z) + c] = v;
  }
}

int team_of(int d) { return d <= 32 ? 2 : d <= 64 ? 4 : d <= 128 ? 8 : 16; }

// Rows of a block's table: at least as many as give every thread a head, within the table
int table_rows_of(int64_t rows, int n, int d, int half, int heads) {
  int most = half ? MAX_TABLE / half : MAX_ROWS;
  if (most > MAX_ROWS) most = MAX_ROWS;
  int want = THREADS / team_of(d) / heads;
  if (want < 1) want = 1;
  // large calls: more rows a table, for fewer waits; small ones: a row a block, for more blocks
  while (want < most && rows * n / (2 * want) >= 8 * (int64_t)hdet_compute_units()) want *= 2;
  return want < most ? want : most;
}
// Blocks a replica of the backward pass: few partial sums
int grad_blocks(int64_t rows, int n, int table_rows) {
  const int64_t chunks = (rows + table_rows - 1) / table_rows;
  int64_t want = 8 * (int64_t)hdet_compute_units() / n;
  if (want < 1) want = 1;
  return (int)(chunks < want ? chunks : want);
}

// whole pieces of 8 columns at 16-byte boundaries
bool whole(const hdet_rows& m, int size) {
  const int64_t mask = 16 / size - 1;
  return !m.dev || (((uintptr_t)m.dev & 15) == 0 && ((m.row_stride | m.replica_stride) & mask) == 0);
}

template <bool BACK> hipError_t launch(const rotary_args& g, int dtype, int mode, int n, int blocks, hipStream_t s) {
  const dim3 grid(blocks, n);
  auto go = [&](auto e, auto m, auto t) { hipLaunchKernelGGL((rotary_kernel<decltype(e), m, t, BACK>), grid, dim3(THREADS), 0, s, g); };
  auto with_mode = [&](auto e, auto t) {
    if (mode == kHalves) go(e, std::integral_constant<int, kHalves>(), t);
    else if (mode == kPairs) go(e, std::integral_constant<int, kPairs>(), t);
    else go(e, std::integral_constant<int, kLoose>(), t);
  };
  auto with_team = [&](auto e) {
    switch (team_of(g.d)) {
      case 2: return with_mode(e, std::integral_constant<int, 2>());
      case 4: return with_mode(e, std::integral_constant<int, 4>());
      case 8: return with_mode(e, std::integral_constant<int, 8>());
      default: return with_mode(e, std::integral_constant<int, 16>());
    }
  };
  if (dtype == HDET_TYPE_BF16) with_team(uint16_t());
  else with_team(float());
  return hipGetLastError();
}

template <typename A> rotary_args common_args(const A& a, bool keys) {
  rotary_args g = {};
  g.s[0].heads = a.q_heads;
  g.s[1].heads = keys ? a.k_heads : 0;
  g.s[0].gain = a.q_gain_dev; g.s[0].gain_z = a.q_gain_stride;
  g.s[1].gain = keys ? a.k_gain_dev : nullptr; g.s[1].gain_z = a.k_gain_stride;
  g.pos = a.positions_dev; g.freq = a.freq_dev;
  g.rows = a.rows; g.d = a.head_dim; g.half = a.rotated / 2; g.period = a.period;
  g.paired = a.layout == HDET_ROTARY_PAIRS;
  g.eps = a.eps; g.magnitude = (float)a.magnitude; g.inv_d = 1.f / (float)a.head_dim;
  g.table_rows = table_rows_of(a.rows, a.n_replicas, g.d, g.half, g.s[0].heads + g.s[1].heads);
  return g;
}
int mode_of(const rotary_args& g, bool aligned) {
  if (!aligned || g.d % 8) return kLoose;
  if (g.paired) return kPairs;
  return g.half % 8 == 0 ? kHalves : kLoose;
}

}  // namespace

hipError_t hdet_launch_rotary(const hdet_rotary_args& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const bool keys = a.k.dev != nullptr;
  rotary_args g = common_args(a, keys);
  const int size = a.dtype == HDET_TYPE_BF16 ? 2 : 4;
  g.s[0].x = a.q.dev; g.s[0].x_s = a.q.row_stride; g.s[0].x_z = a.q.replica_stride;
  g.s[0].y = a.q_out.dev; g.s[0].y_s = a.q_out.row_stride; g.s[0].y_z = a.q_out.replica_stride;
  g.s[1].x = a.k.dev; g.s[1].x_s = a.k.row_stride; g.s[1].x_z = a.k.replica_stride;
  g.s[1].y = a.k_out.dev; g.s[1].y_s = a.k_out.row_stride; g.s[1].y_z = a.k_out.replica_stride;
  const bool aligned = whole(a.q, size) && whole(a.q_out, size) && (!keys || (whole(a.k, size) && whole(a.k_out, size)));
  const int64_t chunks = (a.rows + g.table_rows - 1) / g.table_rows;
  return launch<false>(g, a.dtype, mode_of(g, aligned), a.n_replicas, (int)chunks, s);
}

size_t hdet_rotary_backward_bytes(int n_replicas, int64_t rows, int head_dim, int q_heads, int k_heads) {
  if (rows == 0) return 0;
  // the most blocks that any number of turning pairs gives
  int64_t blocks = grad_blocks(rows, n_replicas, 1);
  return (size_t)n_replicas * blocks * 2 * head_dim * sizeof(float);
}

hipError_t hdet_launch_rotary_backward(const hdet_rotary_grad_args& a, hipStream_t s) {
  const bool keys = a.dk_out.dev != nullptr;
  rotary_args g = common_args(a, keys);
  const int size = a.dtype == HDET_TYPE_BF16 ? 2 : 4;
  g.s[0].x = a.q.dev; g.s[0].x_s = a.q.row_stride; g.s[0].x_z = a.q.replica_stride;
  g.s[0].dy = a.dq_out.dev; g.s[0].dy_s = a.dq_out.row_stride; g.s[0].dy_z = a.dq_out.replica_stride;
  g.s[0].y = a.dq.dev; g.s[0].y_s = a.dq.row_stride; g.s[0].y_z = a.dq.replica_stride;
  g.s[1].x = a.k.dev; g.s[1].x_s = a.k.row_stride; g.s[1].x_z = a.k.replica_stride;
  g.s[1].dy = a.dk_out.dev; g.s[1].dy_s = a.dk_out.row_stride; g.s[1].dy_z = a.dk_out.replica_stride;
  g.s[1].y = a.dk.dev; g.s[1].y_s = a.dk.row_stride; g.s[1].y_z = a.dk.replica_stride;
  g.s[0].sums = a.dq_gain_dev != nullptr;
  g.s[1].sums = a.dk_gain_dev != nullptr;
  g.partial = (float*)a.workspace_dev;
  int blocks = 0;
  if (a.rows > 0) {
    const bool aligned = whole(a.dq_out, size) && whole(a.dq, size) && (!a.q_gain_dev || whole(a.q, size)) &&
                         (!keys || (whole(a.dk_out, size) && whole(a.dk, size) && (!a.k_gain_dev || whole(a.k, size))));
    blocks = grad_blocks(a.rows, a.n_replicas, g.table_rows);
    const hipError_t e = launch<true>(g, a.dtype, mode_of(g, aligned), a.n_replicas, blocks, s);
    if (e != hipSuccess) return e;
  }
  if (!a.dq_gain_dev && !a.dk_gain_dev) return hipSuccess;
  hipLaunchKernelGGL(rotary_gain_kernel, dim3((a.head_dim + 63) / 64, a.n_replicas, 2), dim3(1024), 0, s, g.partial, blocks, a.head_dim, a.dq_gain_dev, a.dq_gain_stride,
                     a.dk_gain_dev, a.dk_gain_stride);
  return hipGetLastError();
}
