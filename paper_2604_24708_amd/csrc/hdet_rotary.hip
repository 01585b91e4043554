// Norm of every head of the queries and keys with the rotation by position, and the backward pass.
//
//   xh = x rstd, rstd = 1 / sqrt(mean x^2 + eps);  u = xh g;  y = R(pos) u:  pairs (u_1, u_2) -> m (u_1 cos a - u_2 sin a, u_1 sin a + u_2 cos a), a = pos f_t
//   w = R(pos)^T dy;  dx = rstd (w g - xh mean(w g xh));  dg = sum w xh
//
// Bound by memory: heads are read once and written once.  A head is held by a team of lanes, 16 bytes each, next to each other, so that a wavefront's loads and
// stores cover whole lines; halves that turn with each other are exchanged between lanes as they lie in memory.  (8 columns and the 8 they turn with in one
// lane, which exchanges nothing: 74 us for 8 x 8192 rows of 20 heads of 64, a line in two halves by two loads.)  A block first forms the cosines and
// sines of its rows, once for all heads of a row, in LDS, then walks over the heads, two a team on their way at once.
//   us (TB/s of what is read and written), forward / backward: 8 x 4096 rows of 16 heads of 64 31 (4.4) / 46 (4.4), 8 x 8192 rows of 20 heads, half
//   of each turning, 63 (5.3) / 105 (4.8), both bfloat16 with gains; the gains' partial sums take another 5 to 8.  An addition over 8 GiB makes 6.2.
// Heads that are no whole pieces of 16 bytes at 16-byte boundaries go element by element, 8 pairs a lane (loose).

#include <algorithm>
#include <type_traits>

#include "hdet_ops.h"
#include "hdet_elem.h"

namespace {

constexpr int THREADS = 256;
constexpr int MAX_ROWS = 16;               // rows of a block's table at a time, where they are not needed to give every thread a head
constexpr int MAX_TABLE = 1024;            // pairs of the table: 8 KiB

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
  int paired;                              // neighbours are a pair
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
  if (T > 16) v += __shfl_xor(v, 16);
  if (T > 32) v += __shfl_xor(v, 32);
  return v;
}
template <int T> __device__ __forceinline__ double team_sum64(double v) {
  for (int o = 1; o < T; o <<= 1) v += __shfl_xor(v, o);
  return v;
}
// 1 / sqrt(mean x^2 + eps) from a lane's sum of squares: fp32 sums, in 64 bits where the squares leave fp32's range (slow(): the lane's sum in 64 bits)
template <int T, typename F> __device__ __forceinline__ float rstd_of(const rotary_args& g, float s, F slow) {
  const float m = __builtin_fmaf(team_sum<T>(s), g.inv_d, (float)g.eps);
  if (m > 1e-30f && m < 1e30f) {
    const float r = __builtin_amdgcn_rsqf(m);
    return r * __builtin_fmaf(-0.5f * m * r, r, 1.5f);
  }
  return (float)(1.0 / sqrt(team_sum64<T>(slow()) / g.d + g.eps));
}
__device__ __forceinline__ double position(const rotary_args& g, int r, int64_t row) {
  return g.pos ? (double)g.pos[(int64_t)r * g.rows + row] : (double)(g.period ? row % g.period : row);
}
// Cosines and sines of `have` rows from row0 on; between two barriers.  BACK: of the turn back
template <bool BACK> __device__ __forceinline__ void make_table(const rotary_args& g, int r, int64_t row0, unsigned have, float2* table) {
  __syncthreads();                         // the last rows' table has been read
  for (unsigned i = threadIdx.x; i < have * g.half; i += THREADS) {
    const unsigned row = i / (unsigned)g.half;
    const float2 cs = cos_sin(position(g, r, row0 + row) * g.freq[i - row * g.half]);
    table[i] = make_float2(cs.x * g.magnitude, (BACK ? -cs.y : cs.y) * g.magnitude);
  }
  __syncthreads();
}

// ---------------------------------------------------------------------------------------------
// Whole pieces.  One block: rows `table_rows` at a time, all heads of one side (blockIdx.z) of them.  BACK: the gradients, and the gain's partial sums.
// ---------------------------------------------------------------------------------------------
template <typename E> struct chunk_of {    // 16 bytes of a row
  static constexpr int N = 16 / sizeof(E);
  hdet_u4v w;
  __device__ __forceinline__ void load(const E* p) { w = *reinterpret_cast<const hdet_u4v*>(p); }
  __device__ __forceinline__ float operator[](int e) const {
    return sizeof(E) == 4 ? __uint_as_float(w[e & 3]) : __uint_as_float(e & 1 ? w[(e >> 1) & 3] & 0xffff0000u : w[(e >> 1) & 3] << 16);
  }
  __device__ __forceinline__ chunk_of from(int lane) const {
    chunk_of r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = __shfl((int)w[i], lane);
    return r;
  }
};
template <typename E, bool PAIRED, int T, bool BACK> __global__ __launch_bounds__(THREADS) void rotary_kernel(const rotary_args g) {
  typedef chunk_of<E> chunk;
  constexpr int N = chunk::N, U = 2;
  __shared__ float2 table[MAX_TABLE];
  __shared__ float sums[BACK ? THREADS * N : 1];
  const int tid = threadIdx.x, l = tid % T, r = blockIdx.y, lane = tid & 63;
  const side& s = g.s[blockIdx.z];
  const int64_t chunks = (g.rows + g.table_rows - 1) / g.table_rows;
  const bool on = l * N < g.d, turns = l * N < 2 * g.half;
  // halves: the lane that holds the other half, whether this is the second, and the first pair
  const int step = g.half / N;
  const bool second = !PAIRED && turns && l >= step;
  const int other = PAIRED || !turns ? lane : second ? lane - step : lane + step, pair0 = PAIRED ? l * (N / 2) : (second ? l - step : l) * N;
  const E* const xs = (const E*)s.x + r * s.x_z + l * N;
  const E* const dys = (const E*)s.dy + r * s.dy_z + l * N;
  E* const ys = (E*)s.y + r * s.y_z + l * N;
  float gain[N], acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    gain[e] = s.gain && on ? s.gain[r * s.gain_z + l * N + e] : 1.f;
    acc[e] = 0.f;
  }
  for (int64_t chunk_i = blockIdx.x; chunk_i < chunks; chunk_i += gridDim.x) {
    const int64_t row0 = chunk_i * g.table_rows;
    const unsigned have = (unsigned)(g.rows - row0 < g.table_rows ? g.rows - row0 : g.table_rows), teams = have * (unsigned)s.heads;
    make_table<BACK>(g, r, row0, have, table);
    for (unsigned t0 = tid / T; t0 < teams; t0 += U * (THREADS / T)) {
      chunk x_[U], dy_[U];
      unsigned row_[U], head_[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const unsigned team = t0 + u * (THREADS / T);
        row_[u] = team / (unsigned)s.heads;
        head_[u] = team - row_[u] * s.heads;
        x_[u].w = dy_[u].w = hdet_u4v{0u, 0u, 0u, 0u};
        if (team >= teams || !on) continue;
        const int64_t at = row0 + row_[u], col = (int64_t)head_[u] * g.d;
        if (!BACK || s.gain) x_[u].load(xs + at * s.x_s + col);
        if (BACK) dy_[u].load(dys + at * s.dy_s + col);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (t0 + u * (THREADS / T) >= teams) break;
        const chunk x = x_[u];
        float rstd = 1.f;
        if (s.gain) {
          float q = 0.f;
#pragma unroll
          for (int e = 0; e < N; ++e) q = __builtin_fmaf(x[e], x[e], q);
          rstd = rstd_of<T>(g, q, [&] {
            double w = 0.0;
            for (int e = 0; e < N; ++e) w += (double)x[e] * x[e];
            return w;
          });
        }
        const chunk v = BACK ? dy_[u] : x;
        float w[N], y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
          w[e] = v[e];
          if (!BACK && s.gain) w[e] *= rstd * gain[e];
          y[e] = w[e];
        }
        const float2* const cs = table + row_[u] * g.half + pair0;
        if (PAIRED) {
#pragma unroll
          for (int e = 0; e < N; e += 2)
            if (pair0 + e / 2 < g.half) {
              const float2 c = cs[e / 2];
              y[e] = __builtin_fmaf(w[e], c.x, -w[e + 1] * c.y);
              y[e + 1] = __builtin_fmaf(w[e], c.y, w[e + 1] * c.x);
            }
        } else {
          float mate[N];
          if (BACK) {
            const chunk v2 = v.from(other);
#pragma unroll
            for (int e = 0; e < N; ++e) mate[e] = v2[e];
          } else {
#pragma unroll
            for (int e = 0; e < N; ++e) mate[e] = __shfl(w[e], other);
          }
          if (turns) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
              const float2 c = cs[e];
              y[e] = __builtin_fmaf(w[e], c.x, mate[e] * (second ? c.y : -c.y));
            }
          }
        }
        if (BACK && s.gain) {
          float dot = 0.f;
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float xh = x[e] * rstd;
            acc[e] = __builtin_fmaf(y[e], xh, acc[e]);
            y[e] *= gain[e];
            dot = __builtin_fmaf(y[e], xh, dot);
          }
          dot = team_sum<T>(dot) * g.inv_d;
#pragma unroll
          for (int e = 0; e < N; ++e) y[e] = rstd * __builtin_fmaf(-x[e] * rstd, dot, y[e]);
        }
        if (!on) continue;
        E* const to = ys + (row0 + row_[u]) * s.y_s + (int64_t)head_[u] * g.d;
        if constexpr (N == 8) hdet_st8(to, hdet_f8{{y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7]}});
        else hdet_st4(to, hdet_f4{{y[0], y[1], y[2], y[3]}});
      }
    }
  }
  if (!BACK || !s.sums) return;
#pragma unroll
  for (int e = 0; e < N; ++e) sums[tid * N + e] = acc[e];
  __syncthreads();
  for (int c = tid; c < g.d; c += THREADS) {
    float v = 0.f;
    for (int team = 0; team < THREADS / T; ++team) v += sums[team * (N * T) + c];
    g.partial[(((int64_t)r * gridDim.x + blockIdx.x) * 2 + blockIdx.z) * g.d + c] = v;
  }
}

// ---------------------------------------------------------------------------------------------
// Any heads: a lane's pair i is number l + T i, behind the ones that turn the rest's neighbours
// ---------------------------------------------------------------------------------------------
struct pairs { float a[8], b[8]; };
template <int T> __device__ __forceinline__ void columns(const rotary_args& g, int l, int i, int& ca, int& cb) {
  const int t = l + T * i;
  ca = g.paired || t >= g.half ? 2 * t : t;
  cb = g.paired || t >= g.half ? 2 * t + 1 : t + g.half;
}
template <typename E, int T> __device__ __forceinline__ pairs load_pairs(const rotary_args& g, const E* p, int l) {
  pairs v;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    int ca, cb;
    columns<T>(g, l, i, ca, cb);
    v.a[i] = ca < g.d ? hdet_ld(p + ca) : 0.f;
    v.b[i] = cb < g.d ? hdet_ld(p + cb) : 0.f;
  }
  return v;
}
template <typename E, int T, bool BACK> __global__ __launch_bounds__(THREADS) void rotary_loose_kernel(const rotary_args g) {
  __shared__ float2 table[MAX_TABLE];
  __shared__ float sums[BACK ? THREADS * 16 : 1];
  const int tid = threadIdx.x, l = tid % T, r = blockIdx.y;
  const side& s = g.s[blockIdx.z];
  const int64_t chunks = (g.rows + g.table_rows - 1) / g.table_rows;
  pairs acc = {}, gain = {};
  if (s.gain) gain = load_pairs<float, T>(g, s.gain + r * s.gain_z, l);
  for (int64_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
    const int64_t row0 = chunk * g.table_rows;
    const unsigned have = (unsigned)(g.rows - row0 < g.table_rows ? g.rows - row0 : g.table_rows), teams = have * (unsigned)s.heads;
    make_table<BACK>(g, r, row0, have, table);
    for (unsigned team = tid / T; team < teams; team += THREADS / T) {
      const unsigned row = team / (unsigned)s.heads, head = team - row * s.heads;
      const int64_t at = row0 + row, col = (int64_t)head * g.d;
      pairs x = {}, v;
      float rstd = 1.f;
      if (!BACK || s.gain) x = load_pairs<E, T>(g, (const E*)s.x + r * s.x_z + at * s.x_s + col, l);
      if (BACK) v = load_pairs<E, T>(g, (const E*)s.dy + r * s.dy_z + at * s.dy_s + col, l);
      if (s.gain) {
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) q = __builtin_fmaf(x.a[i], x.a[i], __builtin_fmaf(x.b[i], x.b[i], q));
        rstd = rstd_of<T>(g, q, [&] {
          double w = 0.0;
          for (int i = 0; i < 8; ++i) w += (double)x.a[i] * x.a[i] + (double)x.b[i] * x.b[i];
          return w;
        });
      }
      if (!BACK) {
        v = x;
        if (s.gain) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v.a[i] = x.a[i] * rstd * gain.a[i];
            v.b[i] = x.b[i] * rstd * gain.b[i];
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (l + T * i >= g.half) continue;
        const float2 c = table[row * g.half + l + T * i];
        const float a = v.a[i], b = v.b[i];
        v.a[i] = __builtin_fmaf(a, c.x, -b * c.y);
        v.b[i] = __builtin_fmaf(a, c.y, b * c.x);
      }
      if (BACK && s.gain) {
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x.a[i] *= rstd;
          x.b[i] *= rstd;
          acc.a[i] = __builtin_fmaf(v.a[i], x.a[i], acc.a[i]);
          acc.b[i] = __builtin_fmaf(v.b[i], x.b[i], acc.b[i]);
          v.a[i] *= gain.a[i];
          v.b[i] *= gain.b[i];
          dot = __builtin_fmaf(v.a[i], x.a[i], __builtin_fmaf(v.b[i], x.b[i], dot));
        }
        dot = team_sum<T>(dot) * g.inv_d;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v.a[i] = rstd * __builtin_fmaf(-x.a[i], dot, v.a[i]);
          v.b[i] = rstd * __builtin_fmaf(-x.b[i], dot, v.b[i]);
        }
      }
      E* const to = (E*)s.y + r * s.y_z + at * s.y_s + col;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        int ca, cb;
        columns<T>(g, l, i, ca, cb);
        if (ca < g.d) hdet_st(to + ca, v.a[i]);
        if (cb < g.d) hdet_st(to + cb, v.b[i]);
      }
    }
  }
  if (!BACK || !s.sums) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    sums[(tid / T) * (16 * T) + (2 * i) * T + l] = acc.a[i];
    sums[(tid / T) * (16 * T) + (2 * i + 1) * T + l] = acc.b[i];
  }
  __syncthreads();
  for (int j = tid; j < 16 * T; j += THREADS) {
    float v = 0.f;
    for (int team = 0; team < THREADS / T; ++team) v += sums[team * (16 * T) + j];
    int ca, cb;
    columns<T>(g, j % T, j / T / 2, ca, cb);
    const int c = j / T & 1 ? cb : ca;
    if (c < g.d) g.partial[(((int64_t)r * gridDim.x + blockIdx.x) * 2 + blockIdx.z) * g.d + c] = v;
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

// lanes of a head, `each` columns a lane: a power of two
int team_of(int d, int each) {
  int t = 1;
  while (t * each < d) t *= 2;
  return t;
}

// Rows of a block's table: as many as give every thread a head (few heads of few columns: 4 x 16 sequences of 2525 tokens, 3 heads of 16, forward and
// backward 117 us, 198 in tables of up to 16 rows), while that leaves two blocks a CU, within the table
int table_rows_of(int64_t rows, int n, int d, int half, int heads) {
  int most = half ? MAX_TABLE / half : MAX_TABLE;
  int want = THREADS / team_of(d, 8) / heads;
  if (want < 1) want = 1;
  while (want > MAX_ROWS && rows * n / want < 2 * (int64_t)hdet_compute_units()) want /= 2;
  if (most > MAX_ROWS && most > want) most = want > MAX_ROWS ? want : MAX_ROWS;
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

// f(integral_constant<T>) for the smallest power of two from LEAST on that is T
template <int LEAST, typename F> void with_team(int t, F f) {
  if (t <= LEAST) f(std::integral_constant<int, LEAST>());
  else if constexpr (LEAST < 64) with_team<2 * LEAST>(t, f);
}
template <bool BACK, typename E> void launch_typed(const rotary_args& g, bool whole, int n, int blocks, hipStream_t s) {
  const dim3 grid(blocks, n, g.s[1].heads ? 2 : 1);
  if (whole) {
    with_team<2>(team_of(g.d, 16 / (int)sizeof(E)), [&](auto t) {
      if (g.paired) hipLaunchKernelGGL((rotary_kernel<E, true, t, BACK>), grid, dim3(THREADS), 0, s, g);
      else hipLaunchKernelGGL((rotary_kernel<E, false, t, BACK>), grid, dim3(THREADS), 0, s, g);
    });
  } else {
    with_team<2>(std::min(16, team_of(g.d, 16)), [&](auto t) {
      if constexpr (t <= 16) hipLaunchKernelGGL((rotary_loose_kernel<E, t, BACK>), grid, dim3(THREADS), 0, s, g);
    });
  }
}
template <bool BACK> hipError_t launch(const rotary_args& g, int dtype, bool aligned, int n, int blocks, hipStream_t s) {
  const int each = dtype == HDET_TYPE_BF16 ? 8 : 4;
  const bool whole = aligned && g.d % each == 0 && (g.paired || g.half % each == 0);
  if (dtype == HDET_TYPE_BF16) launch_typed<BACK, uint16_t>(g, whole, n, blocks, s);
  else launch_typed<BACK, float>(g, whole, n, blocks, s);
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
  return launch<false>(g, a.dtype, aligned, a.n_replicas, (int)chunks, s);
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
    const hipError_t e = launch<true>(g, a.dtype, aligned, a.n_replicas, blocks, s);
    if (e != hipSuccess) return e;
  }
  if (!a.dq_gain_dev && !a.dk_gain_dev) return hipSuccess;
  hipLaunchKernelGGL(rotary_gain_kernel, dim3((a.head_dim + 63) / 64, a.n_replicas, 2), dim3(1024), 0, s, g.partial, blocks, a.head_dim, a.dq_gain_dev, a.dq_gain_stride,
                     a.dk_gain_dev, a.dk_gain_stride);
  return hipGetLastError();
}
