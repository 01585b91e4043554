// Root-mean-square norm of a residual sum with an output in 8 bits, its backward pass, rows to 8 bits and back, and sums over rows.
//
//   u = x + r,  rstd = 1 / sqrt(mean u^2 + eps),  y = u rstd g;  codes q = rint(y / s), s the power of two that takes max|y| to 127 or less
//   dx = rstd (dy g - xh mean(dy g xh)) + dtotal,  xh = h rstd;  dg = sum_rows dy xh
//
// All of it is bound by memory: a row is read once, stays in registers between its sums and its results, and nothing but the results is
// written.  L threads hold a row (8 .. 64: several rows to a wavefront or block, reductions by exchanges inside the wavefront; 256 and
// 1024: a block to a row, one pass through LDS), each in C pieces of 8 elements.

#include <type_traits>

#include "hdet_ops.h"
#include "hdet_elem.h"

namespace {

// How a launch's rows lie: anywhere; in whole pieces of 8 elements at 16-byte boundaries; the same, and so much of it that what is written
// would push what is still to be read out of the memory-side cache (256 MB): past the caches then.  us, through / past:  backward 8 x 8192
// rows of 1024 119 / 101, 8 x 4096 of 512 26.5 / 29;  forward 84 / 78 and 22 / 26
enum { kLoose = 0, kWhole = 1, kStream = 2 };

// Eight neighbouring elements of a row of `width`, as they lie in memory; zeros behind the row's end.  Where rows are not whole pieces one
// lies at any element, which the memory takes as it takes aligned ones but for the lines it crosses; the last piece of a row is loaded from
// 8 elements before the end and moved into place, so that no lane waits for another's single elements (an odd row of 1001: 14.5 us of a
// launch that takes 9 so).
typedef hdet_u4v hdet_u4v_any __attribute__((aligned(2)));
typedef hdet_f4v hdet_f4v_any __attribute__((aligned(4)));
template <typename T> struct piece;
template <> struct piece<uint16_t> {
  hdet_u4v w;
  __device__ __forceinline__ void zero() { w = hdet_u4v{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ float operator[](int e) const { return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16); }
  template <int WHOLE> __device__ __forceinline__ void load(const uint16_t* p, int col, int width) {
    if (WHOLE == kStream) {
      w = __builtin_nontemporal_load(reinterpret_cast<const hdet_u4v*>(p + col));
    } else if (WHOLE) {
      w = *reinterpret_cast<const hdet_u4v*>(p + col);
    } else if (width >= 8) {
      const int back = col + 8 > width ? col + 8 - width : 0;
      const hdet_u4v u = *reinterpret_cast<const hdet_u4v_any*>(p + col - back);
      const int d = back >> 1;
      unsigned x[5];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = d == 0 ? u[i] : d == 1 ? (i < 3 ? u[i + 1 & 3] : 0u) : d == 2 ? (i < 2 ? u[i + 2 & 3] : 0u) : (i < 1 ? u[3] : 0u);
      x[4] = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = back & 1 ? x[i] >> 16 | x[i + 1] << 16 : x[i];
    } else {
      zero();
      for (int e = 0; e < width; ++e) w[e >> 1] |= (unsigned)p[e] << (16 * (e & 1));
    }
  }
};
template <> struct piece<float> {
  hdet_f4v a, b;
  __device__ __forceinline__ void zero() { a = b = hdet_f4v{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ float operator[](int e) const { return e < 4 ? a[e & 3] : b[e & 3]; }
  template <int WHOLE> __device__ __forceinline__ void load(const float* p, int col, int width) {
    if (WHOLE == kStream) {
      a = __builtin_nontemporal_load(reinterpret_cast<const hdet_f4v*>(p + col));
      b = __builtin_nontemporal_load(reinterpret_cast<const hdet_f4v*>(p + col + 4));
    } else if (WHOLE) {
      a = *reinterpret_cast<const hdet_f4v*>(p + col);
      b = *reinterpret_cast<const hdet_f4v*>(p + col + 4);
    } else if (width >= 8) {
      const int back = col + 8 > width ? col + 8 - width : 0;
      const float* q = p + col - back;
      const hdet_f4v u = *reinterpret_cast<const hdet_f4v_any*>(q), v = *reinterpret_cast<const hdet_f4v_any*>(q + 4);
      float x[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
#pragma unroll
      for (int h = 4; h > 0; h >>= 1)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = back & h ? (e + h < 8 ? x[e + h < 8 ? e + h : 7] : 0.f) : x[e];
      a = hdet_f4v{x[0], x[1], x[2], x[3]};
      b = hdet_f4v{x[4], x[5], x[6], x[7]};
    } else {
      zero();
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < width) (e < 4 ? a : b)[e & 3] = p[e];
    }
  }
};
template <int WHOLE>
__device__ __forceinline__ void store_piece(uint16_t* p, const float (&v)[8], int left) {
  if (WHOLE || left >= 8) {
    hdet_u4v u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = hdet_bf16_pack(v[2 * i], v[2 * i + 1]);
    if (WHOLE == kStream) __builtin_nontemporal_store(u, reinterpret_cast<hdet_u4v*>(p));
    else if (WHOLE) *reinterpret_cast<hdet_u4v*>(p) = u;
    else *reinterpret_cast<hdet_u4v_any*>(p) = u;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) hdet_st(p + e, v[e]);
  }
}
template <int WHOLE>
__device__ __forceinline__ void store_piece(float* p, const float (&v)[8], int left) {
  if (WHOLE || left >= 8) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const hdet_f4v u = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
      if (WHOLE == kStream) __builtin_nontemporal_store(u, reinterpret_cast<hdet_f4v*>(p + 4 * h));
      else if (WHOLE) *reinterpret_cast<hdet_f4v*>(p + 4 * h) = u;
      else *reinterpret_cast<hdet_f4v_any*>(p + 4 * h) = u;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = v[e];
  }
}

// Reduction over the L threads of a row, the same value in each, in a fixed order.  L > 64 (a block to a row): through `buf`.
template <int L, typename V, typename F>
__device__ __forceinline__ V over_row(V x, V* buf, F op) {
#pragma unroll
  for (int o = 1; o < (L < 64 ? L : 64); o <<= 1) x = op(x, __shfl_xor(x, o));
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
    __syncthreads();
    x = buf[0];
#pragma unroll
    for (int w = 1; w < L / 64; ++w) x = op(x, buf[w]);
    __syncthreads();
  }
  return x;
}
template <int L, typename V> __device__ __forceinline__ V row_sum_of(V x, V* buf) { return over_row<L>(x, buf, [](V a, V b) { return a + b; }); }
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }

// Scale of a row from the bits of its largest absolute value.  With top = m 2^(E - 126), m in [1/2, 1): 127 2^e >= top from e = E - 133 on,
// or one more where m > 127 / 128.  Absolute values compare as their bits do, NaN above infinity above all numbers: either gives the
// exponent 255.
struct row_scale { float scale, inverse; };
__device__ __forceinline__ row_scale scale_of(unsigned top) {
  const int E = (int)(top >> 23);
  if (E == 255) return {__uint_as_float(0x7fc00000u), 0.f};
  int e = E - 133 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  if (e < -126) e = -126;
  return {__uint_as_float((unsigned)(e + 127) << 23), __uint_as_float((unsigned)(127 - e) << 23)};
}
// rint(x inverse) as the low bits of that + 1.5 2^52, halves to even; |x inverse| is 127 at most, up to what rounding the row's largest
// value to fp32 took off
__device__ __forceinline__ unsigned code_of(double x, double inverse) {
  return (unsigned)__builtin_bit_cast(unsigned long long, __builtin_fma(x, inverse, 6755399441055744.0));
}

struct norm_kernel_args {
  const void *x, *resid;
  void *total, *y;
  int8_t* codes;
  float *scale, *rstd;
  const float* gain;
  int64_t x_s, x_z, r_s, r_z, t_s, t_z, y_s, y_z, c_s, c_z, gain_z, rows;
  int width;
  double eps, inv_width;
};

}  // namespace

// The sum of squares, the norm and what is rounded to codes are held in 64 bits, which costs a tenth of the time (8 x 8192 rows of 1024,
// bf16, sum and codes: 80 us in 32 bits, 88 so) and puts a code where the formula has it: in 32 bits y is off by up to 3e-7 of itself, and
// about one row in 800 (normally distributed, 1000 columns) has a code one off.  Bound by memory: that size 87 us = 5.4 TB/s, 8 x 4096 rows
// of 512 25.5 us; one row of 512 3.6 us, a launch and its chain of load, two reductions and store.
// NORM: as above; otherwise y = x (rows to 8 bits).  Grid: (ceil(rows / rows a block), replicas).
// (The row is in registers from its two loads to its two or three stores; what is left between the loads and the stores are the two
// reductions.)
template <typename T, int WHOLE, int L, int C, bool NORM>
__global__ __launch_bounds__(L < 256 ? 256 : L) void hdet_norm_kernel(const norm_kernel_args a) {
  constexpr int THREADS = L < 256 ? 256 : L, RPB = THREADS / L;
  __shared__ unsigned buf[16];
  __shared__ double sums[16];
  const int j = threadIdx.x % L, z = blockIdx.y;
  const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / L;
  const bool here = row < a.rows;
  double u[C][8];
  const T* x = (const T*)a.x + z * a.x_z + row * a.x_s;
  const T* r = (const T*)a.resid + z * a.r_z + row * a.r_s;
  piece<T> p[C], q[C];      // the two summands
  piece<float> gain[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * L + j) * 8;
    p[c].zero();
    q[c].zero();
    if (NORM) gain[c].zero();
    if (here && col < a.width) {
      p[c].template load<WHOLE>(x, col, a.width);
      if (NORM && a.resid) q[c].template load<WHOLE>(r, col, a.width);
      if (NORM) gain[c].template load<kLoose>(a.gain + z * a.gain_z, col, a.width);
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e)      // (bfloat16 summands: the sum is exact in 32 bits unless one is 2^16 times the other)
      u[c][e] = !NORM ? (double)p[c][e] : sizeof(T) == 2 ? (double)(p[c][e] + q[c][e]) : (double)p[c][e] + (double)q[c][e];
  if constexpr (NORM) {
    double ss = 0.0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = __builtin_fma(u[c][e], u[c][e], ss);
    const double rstd = 1.0 / sqrt(row_sum_of<L>(ss, sums) * a.inv_width + a.eps);
    if (a.rstd && here && j == 0) a.rstd[z * a.rows + row] = (float)rstd;
    T* const total = (T*)a.total + z * a.t_z + row * a.t_s;
    T* const y = (T*)a.y + z * a.y_z + row * a.y_s;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * L + j) * 8;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (float)u[c][e];
      if (a.total && here && col < a.width) store_piece<WHOLE>(total + col, v, a.width - col);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[c][e] *= rstd * (double)gain[c][e];
        v[e] = (float)u[c][e];
      }
      if (a.y && here && col < a.width) store_piece<WHOLE>(y + col, v, a.width - col);
    }
  }
  if (!a.codes) return;
  unsigned top = 0u;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = larger(top, __float_as_uint((float)u[c][e]) & 0x7fffffffu);
  const row_scale sc = scale_of(over_row<L>(top, buf, larger));
  if (here && j == 0) a.scale[z * a.rows + row] = sc.scale;
  int8_t* const to = a.codes + z * a.c_z + row * a.c_s;
  const int padded = (a.width + 15) & ~15;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * L + j) * 8;
    if (here && col < padded) {                     // columns behind the last are 0 in u (a row of registers is a multiple of 16 long)
      unsigned w[2] = {0u, 0u};
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e >> 2] |= (code_of(u[c][e], sc.inverse) & 255u) << (8 * (e & 3));
      *reinterpret_cast<hdet_u2v*>(to + col) = sc.inverse == 0.f ? hdet_u2v{0u, 0u} : hdet_u2v{w[0], w[1]};      // rows that are not finite: codes 0
    }
  }
}

namespace {
struct norm_grad_kernel_args {
  const void *h, *dy, *dt;
  void* dx;
  const float *rstd, *gain;
  float* part;             // [replica][blocks][width], or the gradient itself where one block takes all rows; null: none wanted
  int64_t h_s, h_z, dy_s, dy_z, dt_s, dt_z, dx_s, dx_z, gain_z, part_z, rows;
  int width;
  float inv_width;
};
}  // namespace

// Grid: (blocks, replicas); a block takes every gridDim.x-th group of rows and adds up its columns' dy xh on the way (the gain's gradient
// is then `blocks` rows instead of all of them for a second launch).  A row stays in registers as it lies in memory, the gain is in LDS;
// other wavefronts cover a row's loads.  Bound by memory: 8 x 8192 rows of 1024, bf16, 96 us = 5.6 TB/s, 8 x 4096 of 512 24.  Not faster,
// us, of 115 to 119 through the caches: consecutive rows a block 128, four times the blocks 142, registers for 5, 6 or 8 wavefronts a SIMD
// 207, 292, 413 (spills); the next row's loads under a row 115, but 16.8 for 12.9 at 3 x 777 rows of 1001 in fp32.
template <typename T, int WHOLE, int L, int C>
__global__ __launch_bounds__(L < 256 ? 256 : L) void hdet_norm_grad_kernel(const norm_grad_kernel_args a) {
  constexpr int THREADS = L < 256 ? 256 : L, RPB = THREADS / L, COLS = L * 8 * C;
  constexpr bool kGainInLds = COLS <= 8192;
  __shared__ float buf[16];
  __shared__ __attribute__((aligned(16))) float s_gain[kGainInLds ? COLS : 1];
  __shared__ float sums[RPB > 1 ? RPB * COLS : 1];
  const int j = threadIdx.x % L, sub = threadIdx.x / L, z = blockIdx.y;
  const float* const gain = a.gain + z * a.gain_z;
  float acc[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[c][e] = 0.f;
  const T *const h = (const T*)a.h + z * a.h_z, *const dy = (const T*)a.dy + z * a.dy_z, *const dt = (const T*)a.dt + z * a.dt_z;
  auto gain_of = [&](int c, float (&g)[8]) {
    const int col = (c * L + j) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = kGainInLds ? s_gain[col + e] : col + e < a.width ? gain[col + e] : 0.f;
  };
  struct row_data { piece<T> h[C], dy[C], dt[C]; float rstd; };
  auto fetch = [&](row_data& d, int64_t row) {
    const bool here = row < a.rows;
    d.rstd = here ? a.rstd[z * a.rows + row] : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * L + j) * 8;
      d.h[c].zero();
      d.dy[c].zero();
      d.dt[c].zero();
      if (here && col < a.width) {
        d.h[c].template load<WHOLE>(h + row * a.h_s, col, a.width);
        d.dy[c].template load<WHOLE>(dy + row * a.dy_s, col, a.width);
        if (a.dt) d.dt[c].template load<WHOLE>(dt + row * a.dt_s, col, a.width);
      }
    }
  };
  auto finish = [&](const row_data& d, int64_t row) {
    float dot = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float g[8];
      gain_of(c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xh = d.h[c][e] * d.rstd, y = d.dy[c][e];
        acc[c][e] = __builtin_fmaf(y, xh, acc[c][e]);
        dot = __builtin_fmaf(y * g[e], xh, dot);
      }
    }
    const float mean = row_sum_of<L>(dot, buf) * a.inv_width;
    T* const dx = (T*)a.dx + z * a.dx_z + row * a.dx_s;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * L + j) * 8;
      float g[8], o[8];
      gain_of(c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = __builtin_fmaf(d.rstd, __builtin_fmaf(-(d.h[c][e] * d.rstd), mean, d.dy[c][e] * g[e]), d.dt[c][e]);
      if (row < a.rows && col < a.width) store_piece<WHOLE>(dx + col, o, a.width - col);
    }
  };
  const int64_t step = (int64_t)gridDim.x * RPB;
  row_data d;
  int64_t base = (int64_t)blockIdx.x * RPB;
  fetch(d, base + sub);         // in flight while the gain comes into LDS
  if (kGainInLds) {
    for (int c = threadIdx.x; c < COLS; c += THREADS) s_gain[c] = c < a.width ? gain[c] : 0.f;
    __syncthreads();
  }
  while (base < a.rows) {
    finish(d, base + sub);
    base += step;
    fetch(d, base + sub);
  }
  if (!a.part) return;
  float* const out = a.part + z * a.part_z + (int64_t)blockIdx.x * a.width;
  if constexpr (RPB > 1) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[sub * COLS + (c * L + j) * 8 + e] = acc[c][e];
    __syncthreads();
    for (int col = threadIdx.x; col < a.width; col += THREADS) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < RPB; ++w) s += sums[w * COLS + col];
      out[col] = s;
    }
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int col = (c * L + j) * 8 + e;
        if (col < a.width) out[col] = acc[c][e];
      }
  }
}

// out[z][col] = sum over p of part[z][p][col], ascending in 16 phases that are added in their order.  Block = 64 columns x 16 phases; grid
// (ceil(width / 64), replicas).
__global__ __launch_bounds__(1024) void hdet_partial_sum_kernel(const float* part, int parts, int width, int64_t pitch, float* out, int64_t out_z) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, col = blockIdx.x * 64 + lane, ph = threadIdx.x >> 6, z = blockIdx.y;
  float x = 0.f;
  if (col < width) {
    const float* p = part + (int64_t)z * parts * pitch + col;
#pragma unroll 4
    for (int i = ph; i < parts; i += 16) x += p[i * pitch];
  }
  s[ph][lane] = x;
  __syncthreads();
  if (ph != 0 || col >= width) return;
  x = s[0][lane];
#pragma unroll
  for (int w = 1; w < 16; ++w) x += s[w][lane];
  out[z * out_z + col] = x;
}

// Sums over `each` rows of a bfloat16 matrix.  Block = 64 pieces of 8 columns x 4 phases of rows, eight rows' loads in flight; grid (column
// blocks, row blocks, replicas).
// (8 x 8192 rows of 4096, more than the memory-side cache holds: 122 us, past the caches 93 = 5.8 TB/s.)
template <int WHOLE>
__global__ __launch_bounds__(256) void hdet_row_sum_kernel(const uint16_t* x, int64_t x_s, int64_t x_z, int64_t rows, int each, int width, float* part, int64_t part_z) {
  __shared__ float s[4][512 + 8];
  const int cg = threadIdx.x & 63, ph = threadIdx.x >> 6, z = blockIdx.z, col = blockIdx.x * 512 + cg * 8;
  const int64_t r0 = (int64_t)blockIdx.y * each, r1 = r0 + each < rows ? r0 + each : rows;
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  if (col < width) {
    const uint16_t* p = x + z * x_z;
#pragma unroll 8
    for (int64_t r = r0 + ph; r < r1; r += 4) {
      piece<uint16_t> v;
      v.load<WHOLE>(p + r * x_s, col, width);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s[ph][cg * 8 + e] = acc[e];
  __syncthreads();
  for (int c = threadIdx.x; c < 512; c += 256)
    if (blockIdx.x * 512 + c < width)
      part[z * part_z + (int64_t)blockIdx.y * width + blockIdx.x * 512 + c] = (s[0][c] + s[1][c]) + (s[2][c] + s[3][c]);
}

// Rows of codes to values: a thread takes 8 columns.  Bound by memory: 8 x 8192 rows of 1024 to bf16 31 us = 6.5 TB/s of what it reads and
// writes (part of it in the caches).  Grid: hdet_long_grid(rows * pieces).
template <typename T, int WHOLE>
__global__ __launch_bounds__(256) void hdet_restore_kernel(const int8_t* q, int64_t q_s, int64_t q_z, const float* scale, T* v, int64_t v_s, int64_t v_z,
                                                           int64_t rows, int width, int pieces) {
  const int64_t t = hdet_long_thread(), row = t / pieces;
  const int z = blockIdx.y, col = (int)(t - row * pieces) * 8;
  if (row >= rows) return;
  const hdet_u2v w = *reinterpret_cast<const hdet_u2v*>(q + z * q_z + row * q_s + col);
  const float s = scale[z * rows + row];
  float o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = (float)(int8_t)((w[e >> 2] >> (8 * (e & 3))) & 255u) * s;
  store_piece<WHOLE>(v + z * v_z + row * v_s + col, o, width - col);
}

// Rows of a bfloat16 matrix in rows of `pitch`, `copies` times, zeros for rows with a negative label: a thread takes 8 columns.  Grid:
// hdet_long_grid(rows * pieces).
template <int WHOLE>
__global__ __launch_bounds__(256) void hdet_pad_rows_kernel(const uint16_t* x, int64_t x_s, int64_t x_z, int64_t rows, int width, const int32_t* labels, uint16_t* out,
                                                            int64_t pitch, int copies) {
  const int64_t pieces = pitch >> 3, t = hdet_long_thread(), row = t / pieces, all = rows * pieces;
  const int col = (int)(t - row * pieces) * 8;
  if (row >= rows) return;
  piece<uint16_t> v;
  v.zero();
  if (col < width && !(labels && labels[blockIdx.y * rows + row] < 0)) v.load<WHOLE>(x + blockIdx.y * x_z + row * x_s, col, width);
  hdet_u4v* const to = reinterpret_cast<hdet_u4v*>(out) + blockIdx.y * copies * all + t;
  for (int c = 0; c < copies; ++c) to[c * all] = v.w;
}

namespace {

// Whether rows are whole 16-byte pieces of `size`-byte elements (8 of them) at 16-byte boundaries, or the matrix is absent
bool pieces_of_8(const hdet_rows& m, int size, int width) {
  if (!m.dev) return true;
  return (reinterpret_cast<uintptr_t>(m.dev) & 15) == 0 && ((m.row_stride | m.replica_stride) * size & 15) == 0 && (width & 7) == 0;
}

int mode_of(bool whole, int64_t bytes) { return !whole ? kLoose : bytes > (int64_t)256 << 20 ? kStream : kWhole; }

// f(T, mode, L, C) for the smallest row of registers that holds `width`
template <typename T, typename F>
void with_shape(int width, int mode, F f) {
#define HDET_SHAPE(L, C)                                                                              \
  if (width <= 8 * L * C) {                                                                           \
    if (mode == kStream) return f(T(), std::integral_constant<int, kStream>(), std::integral_constant<int, L>(), std::integral_constant<int, C>());   \
    if (mode == kWhole) return f(T(), std::integral_constant<int, kWhole>(), std::integral_constant<int, L>(), std::integral_constant<int, C>());     \
    return f(T(), std::integral_constant<int, kLoose>(), std::integral_constant<int, L>(), std::integral_constant<int, C>());                         \
  }
  HDET_SHAPE(8, 1)
  HDET_SHAPE(16, 1)
  HDET_SHAPE(32, 1)
  HDET_SHAPE(64, 1)
  HDET_SHAPE(64, 2)
  HDET_SHAPE(64, 4)
  HDET_SHAPE(256, 2)
  HDET_SHAPE(256, 4)
  HDET_SHAPE(1024, 2)
  HDET_SHAPE(1024, 4)
#undef HDET_SHAPE
}
int rows_per_block(int width) {
  int n = 1;
  with_shape<float>(width, kWhole, [&](auto, auto, auto l, auto) { n = l < 256 ? 256 / l : 1; });
  return n;
}
// blocks a replica of the backward pass: about eight a compute unit over all replicas, so that the gain's partial sums stay few
int grad_blocks(int n_replicas, int64_t rows, int width) {
  const int64_t most = (rows + rows_per_block(width) - 1) / rows_per_block(width);
  int64_t want = 8 * (int64_t)hdet_compute_units() / n_replicas;
  if (want < 1) want = 1;
  return (int)(most < want ? most : want);
}

template <typename T>
hipError_t launch_norm_typed(const norm_kernel_args& k, int n, int mode, bool norm, hipStream_t s) {
  with_shape<T>(k.width, mode, [&](auto t, auto v, auto l, auto c) {
    constexpr int THREADS = l < 256 ? 256 : l;
    const dim3 grid((unsigned)((k.rows + THREADS / l - 1) / (THREADS / l)), n);
    if (norm) hipLaunchKernelGGL((hdet_norm_kernel<decltype(t), v, l, c, true>), grid, dim3(THREADS), 0, s, k);
    else hipLaunchKernelGGL((hdet_norm_kernel<decltype(t), v, l, c, false>), grid, dim3(THREADS), 0, s, k);
  });
  return hipGetLastError();
}

}  // namespace

hipError_t hdet_launch_norm(const hdet_norm_args& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const int size = a.dtype == HDET_TYPE_BF16 ? 2 : 4;
  const bool vec = pieces_of_8(a.x, size, a.width) && pieces_of_8(a.resid, size, a.width) && pieces_of_8(a.total, size, a.width) && pieces_of_8(a.y, size, a.width);
  const int64_t each = (1 + (a.resid.dev != nullptr) + (a.total.dev != nullptr) + (a.y.dev != nullptr)) * size + (a.codes.dev != nullptr);
  const int mode = mode_of(vec, each * a.n_replicas * a.rows * a.width);
  norm_kernel_args k = {a.x.dev, a.resid.dev, a.total.dev, a.y.dev, (int8_t*)a.codes.dev, a.scale_dev, a.rstd_dev, a.gain_dev,
                        a.x.row_stride, a.x.replica_stride, a.resid.row_stride, a.resid.replica_stride, a.total.row_stride, a.total.replica_stride,
                        a.y.row_stride, a.y.replica_stride, a.codes.row_stride, a.codes.replica_stride, a.gain_stride, a.rows, a.width, a.eps, 1.0 / (double)a.width};
  return a.dtype == HDET_TYPE_BF16 ? launch_norm_typed<uint16_t>(k, a.n_replicas, mode, true, s) : launch_norm_typed<float>(k, a.n_replicas, mode, true, s);
}

hipError_t hdet_launch_quantise(const hdet_codes_args& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const int size = a.dtype == HDET_TYPE_BF16 ? 2 : 4, mode = mode_of(pieces_of_8(a.values, size, a.width), (int64_t)(size + 1) * a.n_replicas * a.rows * a.width);
  norm_kernel_args k = {};
  k.x = a.values.dev; k.x_s = a.values.row_stride; k.x_z = a.values.replica_stride;
  k.codes = (int8_t*)a.codes.dev; k.c_s = a.codes.row_stride; k.c_z = a.codes.replica_stride;
  k.scale = a.scale_dev; k.rows = a.rows; k.width = a.width;
  return a.dtype == HDET_TYPE_BF16 ? launch_norm_typed<uint16_t>(k, a.n_replicas, mode, false, s) : launch_norm_typed<float>(k, a.n_replicas, mode, false, s);
}

hipError_t hdet_launch_restore(const hdet_codes_args& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const int pieces = (a.width + 7) / 8;
  const bool bf = a.dtype == HDET_TYPE_BF16, vec = pieces_of_8(a.values, bf ? 2 : 4, a.width);
  const dim3 grid = hdet_long_grid(a.rows * pieces, a.n_replicas);
  auto go = [&](auto kernel, auto* v) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const int8_t*)a.codes.dev, a.codes.row_stride, a.codes.replica_stride, a.scale_dev, v,
                       a.values.row_stride, a.values.replica_stride, a.rows, a.width, pieces);
  };
  if (bf && vec) go(&hdet_restore_kernel<uint16_t, kWhole>, (uint16_t*)a.values.dev);
  else if (bf) go(&hdet_restore_kernel<uint16_t, kLoose>, (uint16_t*)a.values.dev);
  else if (vec) go(&hdet_restore_kernel<float, kWhole>, (float*)a.values.dev);
  else go(&hdet_restore_kernel<float, kLoose>, (float*)a.values.dev);
  return hipGetLastError();
}

hipError_t hdet_launch_pad_rows(const hdet_rows& x, int n_replicas, int64_t rows, int width, const int32_t* labels, uint16_t* out, int64_t pitch, int copies, hipStream_t s) {
  const dim3 grid = hdet_long_grid(rows * (pitch >> 3), n_replicas);
  const uint16_t* from = (const uint16_t*)x.dev;
  if (pieces_of_8(x, 2, width)) hipLaunchKernelGGL(hdet_pad_rows_kernel<kWhole>, grid, dim3(256), 0, s, from, x.row_stride, x.replica_stride, rows, width, labels, out, pitch, copies);
  else hipLaunchKernelGGL(hdet_pad_rows_kernel<kLoose>, grid, dim3(256), 0, s, from, x.row_stride, x.replica_stride, rows, width, labels, out, pitch, copies);
  return hipGetLastError();
}

size_t hdet_norm_backward_bytes(int n_replicas, int64_t rows, int width) {
  if (rows == 0) return 0;
  return (size_t)n_replicas * grad_blocks(n_replicas, rows, width) * width * sizeof(float);
}

hipError_t hdet_launch_partial_sum(const float* partial, int n_replicas, int parts, int width, int64_t pitch, float* out, int64_t out_stride, hipStream_t s) {
  hipLaunchKernelGGL(hdet_partial_sum_kernel, dim3((width + 63) / 64, n_replicas), dim3(1024), 0, s, partial, parts, width, pitch, out, out_stride);
  return hipGetLastError();
}

hipError_t hdet_launch_norm_backward(const hdet_norm_grad_args& a, hipStream_t s) {
  // no rows: the sum over none of them
  if (a.rows == 0) return a.dgain_dev ? hdet_launch_partial_sum(nullptr, a.n_replicas, 0, a.width, 0, a.dgain_dev, a.dgain_stride, s) : hipSuccess;
  const int size = a.dtype == HDET_TYPE_BF16 ? 2 : 4;
  const bool vec = pieces_of_8(a.total, size, a.width) && pieces_of_8(a.dy, size, a.width) && pieces_of_8(a.dtotal, size, a.width) && pieces_of_8(a.dx, size, a.width);
  const int blocks = grad_blocks(a.n_replicas, a.rows, a.width);
  const bool direct = blocks == 1;
  const norm_grad_kernel_args k = {a.total.dev, a.dy.dev, a.dtotal.dev, a.dx.dev, a.rstd_dev, a.gain_dev, !a.dgain_dev ? nullptr : direct ? a.dgain_dev : (float*)a.workspace_dev,
                                   a.total.row_stride, a.total.replica_stride, a.dy.row_stride, a.dy.replica_stride, a.dtotal.row_stride, a.dtotal.replica_stride,
                                   a.dx.row_stride, a.dx.replica_stride, a.gain_stride, direct ? a.dgain_stride : (int64_t)blocks * a.width, a.rows, a.width, 1.f / (float)a.width};
  auto go = [&](auto t, auto v, auto l, auto c) {
    hipLaunchKernelGGL((hdet_norm_grad_kernel<decltype(t), v, l, c>), dim3(blocks, a.n_replicas), dim3(l < 256 ? 256 : l), 0, s, k);
  };
  const int mode = mode_of(vec, (int64_t)(3 + (a.dtotal.dev != nullptr)) * size * a.n_replicas * a.rows * a.width);
  if (a.dtype == HDET_TYPE_BF16) with_shape<uint16_t>(a.width, mode, go);
  else with_shape<float>(a.width, mode, go);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || direct || !a.dgain_dev) return e;
  return hdet_launch_partial_sum((const float*)a.workspace_dev, a.n_replicas, blocks, a.width, a.width, a.dgain_dev, a.dgain_stride, s);
}

// Rows of a block of hdet_row_sum_kernel: 128, fewer until there are four blocks a compute unit (3 x 515 rows of 1501: 128 16 us, 64 10)
static int rows_each(int n_replicas, int64_t rows, int width) {
  int each = 128;
  while (each > 16 && (rows + each - 1) / each * ((width + 511) / 512) * n_replicas < 4 * hdet_compute_units()) each >>= 1;
  return each;
}
static int row_sum_parts(int n_replicas, int64_t rows, int width) {
  const int each = rows_each(n_replicas, rows, width);
  return (int)((rows + each - 1) / each);
}

size_t hdet_row_sum_bytes(int n_replicas, int64_t rows, int width) {
  const int parts = row_sum_parts(n_replicas, rows, width);
  return parts > 1 ? (size_t)n_replicas * parts * width * sizeof(float) : 0;
}

hipError_t hdet_launch_row_sum(const hdet_rows& x, int n_replicas, int64_t rows, int width, float* out, int64_t out_stride, void* scratch, hipStream_t s) {
  const int parts = row_sum_parts(n_replicas, rows, width), each = rows_each(n_replicas, rows, width);
  if (parts == 0) return hdet_launch_partial_sum(nullptr, n_replicas, 0, width, 0, out, out_stride, s);
  float* const to = parts == 1 ? out : (float*)scratch;
  const int64_t to_z = parts == 1 ? out_stride : (int64_t)parts * width;
  const int mode = mode_of(pieces_of_8(x, 2, width), (int64_t)2 * n_replicas * rows * width);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((width + 511) / 512, parts, n_replicas), dim3(256), 0, s, (const uint16_t*)x.dev, x.row_stride, x.replica_stride, rows, each, width, to, to_z);
  };
  if (mode == kStream) go(&hdet_row_sum_kernel<kStream>);
  else if (mode == kWhole) go(&hdet_row_sum_kernel<kWhole>);
  else go(&hdet_row_sum_kernel<kLoose>);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  return hdet_launch_partial_sum((const float*)scratch, n_replicas, parts, width, width, out, out_stride, s);
}
