// Root-mean-square norm of a residual sum with an output in 8 bits, its backward pass, rows to 8 bits and back, and sums over rows.
//
//   u = x + r,  rstd = 1 / sqrt(mean u^2 + eps),  y = u rstd g;  codes q = rint(y / s) with s the power of two that takes max|y| to 127 or less
//   dx = rstd (dy g - xh mean(dy g xh)) + dtotal,  xh = h rstd;  dg = sum_rows dy xh
//
// All of it is bound by memory: a row is read once, stays in registers between its sums and its results, and nothing but the results is
// written.  L threads hold a row (8 .. 64: several rows to a wavefront or block, reductions by exchanges inside the wavefront; 256 and
// 1024: a block to a row, one pass through LDS), each in C pieces of VEC elements: VEC = 8 where rows are whole 16-byte pieces at
// 16-byte boundaries, else single elements.

#include <type_traits>

#include "hdet_ops.h"
#include "hdet_elem.h"

namespace {

template <int VEC> struct piece_of { float v[VEC]; };
template <int VEC, typename T>
__device__ __forceinline__ piece_of<VEC> load_piece(const T* p) {
  piece_of<VEC> r;
  if constexpr (VEC == 8) {
    const hdet_f8 x = hdet_ld8(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = x.v[e];
  } else {
    r.v[0] = hdet_ld(p);
  }
  return r;
}
template <int VEC, typename T>
__device__ __forceinline__ void store_piece(T* p, const float (&v)[VEC]) {
  if constexpr (VEC == 8) {
    hdet_f8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = v[e];
    hdet_st8(p, x);
  } else {
    hdet_st(p, v[0]);
  }
}

// Reduction over the L threads of a row, the same value in each, in a fixed order.  L > 64 (a block to a row): through `buf`.
template <int L, typename F>
__device__ __forceinline__ unsigned over_row(unsigned x, unsigned* buf, F op) {
#pragma unroll
  for (int o = 1; o < (L < 64 ? L : 64); o <<= 1) x = op(x, (unsigned)__shfl_xor((int)x, o));
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
__device__ __forceinline__ unsigned add_floats(unsigned a, unsigned b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }
template <int L> __device__ __forceinline__ float row_sum_of(float x, unsigned* buf) { return __uint_as_float(over_row<L>(__float_as_uint(x), buf, add_floats)); }

// Scale of a row from the bits of its largest absolute value.  With top = m 2^(E - 126), m in [1/2, 1): 127 2^e >= top from e = E - 133 on, or one more
// where m > 127 / 128.  Absolute values compare as their bits do, NaN above infinity above all numbers: either gives the exponent 255.
struct row_scale { float scale, inverse; };
__device__ __forceinline__ row_scale scale_of(unsigned top) {
  const int E = (int)(top >> 23);
  if (E == 255) return {__uint_as_float(0x7fc00000u), 0.f};
  int e = E - 133 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  if (e < -126) e = -126;
  return {__uint_as_float((unsigned)(e + 127) << 23), __uint_as_float((unsigned)(127 - e) << 23)};
}
// |x| <= 127; rows that are not finite have the inverse 0 and get codes 0
__device__ __forceinline__ int code_of(float x, float inverse) { return inverse == 0.f ? 0 : (int)rintf(x * inverse); }

struct norm_kernel_args {
  const void *x, *resid;
  void *total, *y;
  int8_t* codes;
  float *scale, *rstd;
  const float* gain;
  int64_t x_s, x_z, r_s, r_z, t_s, t_z, y_s, y_z, c_s, c_z, gain_z, rows;
  int width;
  float eps, inv_width;
};

}  // namespace

// NORM: as above; otherwise y = x (rows to 8 bits).  Grid: (ceil(rows / rows a block), replicas).
// (The row is in registers from its two loads to its two or three stores; what is left between the loads and the stores are the two reductions.)
template <typename T, int VEC, int L, int C, bool NORM>
__global__ __launch_bounds__(L < 256 ? 256 : L) void hdet_norm_kernel(const norm_kernel_args a) {
  constexpr int THREADS = L < 256 ? 256 : L, RPB = THREADS / L;
  __shared__ unsigned buf[16];
  const int j = threadIdx.x % L, z = blockIdx.y;
  const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / L;
  const bool here = row < a.rows;
  float u[C][VEC];
  const T* x = (const T*)a.x + z * a.x_z + row * a.x_s;
  const T* r = (const T*)a.resid + z * a.r_z + row * a.r_s;
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * L + j) * VEC;
    if (here && col < a.width) {
      piece_of<VEC> p = load_piece<VEC>(x + col);
      if (NORM && a.resid) {
        const piece_of<VEC> q = load_piece<VEC>(r + col);
#pragma unroll
        for (int e = 0; e < VEC; ++e) p.v[e] += q.v[e];
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) u[c][e] = p.v[e];
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) u[c][e] = 0.f;
    }
  }
  if constexpr (NORM) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < VEC; ++e) ss = __builtin_fmaf(u[c][e], u[c][e], ss);
    ss = row_sum_of<L>(ss, buf);
    const float rstd = 1.f / sqrtf(__builtin_fmaf(ss, a.inv_width, a.eps));
    if (a.rstd && here && j == 0) a.rstd[z * a.rows + row] = rstd;
    T* const total = (T*)a.total + z * a.t_z + row * a.t_s;
    T* const y = (T*)a.y + z * a.y_z + row * a.y_s;
    const float* g = a.gain + z * a.gain_z;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * L + j) * VEC;
      if (here && col < a.width) {
        if (a.total) store_piece<VEC>(total + col, u[c]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[c][e] = u[c][e] * rstd * g[col + e];
        if (a.y) store_piece<VEC>(y + col, u[c]);
      }
    }
  }
  if (!a.codes) return;
  unsigned top = 0u;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < VEC; ++e) top = larger(top, __float_as_uint(u[c][e]) & 0x7fffffffu);
  const row_scale sc = scale_of(over_row<L>(top, buf, larger));
  if (here && j == 0) a.scale[z * a.rows + row] = sc.scale;
  int8_t* const q = a.codes + z * a.c_z + row * a.c_s;
  const int padded = (a.width + 15) & ~15;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * L + j) * VEC;
    if (here && col < padded) {                     // columns behind the last are 0 in u (a row of registers is a multiple of 16 long)
      if constexpr (VEC == 8) {
        unsigned w[2] = {0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2] |= ((unsigned)code_of(u[c][e], sc.inverse) & 255u) << (8 * (e & 3));
        *reinterpret_cast<hdet_u2v*>(q + col) = hdet_u2v{w[0], w[1]};
      } else {
        q[col] = (int8_t)code_of(u[c][0], sc.inverse);
      }
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

// Grid: (blocks, replicas); a block takes every gridDim.x-th group of rows and adds up its columns' dy xh on the way (the gain's gradient is then
// `blocks` rows instead of all of them for a second launch).
template <typename T, int VEC, int L, int C>
__global__ __launch_bounds__(L < 256 ? 256 : L) void hdet_norm_grad_kernel(const norm_grad_kernel_args a) {
  constexpr int THREADS = L < 256 ? 256 : L, RPB = THREADS / L, COLS = L * VEC * C;
  __shared__ unsigned buf[16];
  __shared__ float sums[RPB > 1 ? RPB * COLS : 1];
  const int j = threadIdx.x % L, sub = threadIdx.x / L, z = blockIdx.y;
  float g[C][VEC], acc[C][VEC];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const int col = (c * L + j) * VEC + e;
      g[c][e] = col < a.width ? a.gain[z * a.gain_z + col] : 0.f;
      acc[c][e] = 0.f;
    }
  for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += (int64_t)gridDim.x * RPB) {
    const int64_t row = base + sub;
    const bool here = row < a.rows;
    const T* h = (const T*)a.h + z * a.h_z + row * a.h_s;
    const T* dy = (const T*)a.dy + z * a.dy_z + row * a.dy_s;
    const T* dt = (const T*)a.dt + z * a.dt_z + row * a.dt_s;
    const float rstd = here ? a.rstd[z * a.rows + row] : 0.f;
    float xh[C][VEC], dn[C][VEC], add[C][VEC], dot = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * L + j) * VEC;
      const bool ok = here && col < a.width;
      piece_of<VEC> p, q, t;
#pragma unroll
      for (int e = 0; e < VEC; ++e) p.v[e] = q.v[e] = t.v[e] = 0.f;
      if (ok) {
        p = load_piece<VEC>(h + col);
        q = load_piece<VEC>(dy + col);
        if (a.dt) t = load_piece<VEC>(dt + col);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        xh[c][e] = p.v[e] * rstd;
        dn[c][e] = q.v[e];
        add[c][e] = t.v[e];
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        acc[c][e] = __builtin_fmaf(dn[c][e], xh[c][e], acc[c][e]);
        dn[c][e] *= g[c][e];
        dot = __builtin_fmaf(dn[c][e], xh[c][e], dot);
      }
    const float mean = row_sum_of<L>(dot, buf) * a.inv_width;
    T* const dx = (T*)a.dx + z * a.dx_z + row * a.dx_s;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * L + j) * VEC;
      if (here && col < a.width) {
        float o[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = __builtin_fmaf(rstd, __builtin_fmaf(-xh[c][e], mean, dn[c][e]), add[c][e]);
        store_piece<VEC>(dx + col, o);
      }
    }
  }
  if (!a.part) return;
  float* const out = a.part + z * a.part_z + (int64_t)blockIdx.x * a.width;
  if constexpr (RPB > 1) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sums[sub * COLS + (c * L + j) * VEC + e] = acc[c][e];
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
      for (int e = 0; e < VEC; ++e) {
        const int col = (c * L + j) * VEC + e;
        if (col < a.width) out[col] = acc[c][e];
      }
  }
}

// out[z][col] = sum over p of part[z][p][col], ascending in four phases.  Block = 64 columns x 4 phases; grid (ceil(width / 64), replicas).
__global__ __launch_bounds__(256) void hdet_partial_sum_kernel(const float* part, int parts, int width, int64_t pitch, float* out, int64_t out_z) {
  __shared__ float s[4][64];
  const int col = blockIdx.x * 64 + (threadIdx.x & 63), ph = threadIdx.x >> 6, z = blockIdx.y;
  float x = 0.f;
  if (col < width) {
    const float* p = part + (int64_t)z * parts * pitch + col;
#pragma unroll 4
    for (int i = ph; i < parts; i += 4) x += p[i * pitch];
  }
  s[ph][threadIdx.x & 63] = x;
  __syncthreads();
  if (ph == 0 && col < width) out[z * out_z + col] = (s[0][threadIdx.x] + s[1][threadIdx.x]) + (s[2][threadIdx.x] + s[3][threadIdx.x]);
}

// Sums over up to kSumRows rows of a bfloat16 matrix.  Block = 32 groups of VEC columns x 8 phases of rows; grid (column blocks, row blocks, replicas).
namespace { constexpr int kSumRows = 128; }
template <int VEC>
__global__ __launch_bounds__(256) void hdet_row_sum_kernel(const uint16_t* x, int64_t x_s, int64_t x_z, int64_t rows, int width, float* part, int64_t part_z) {
  constexpr int COLS = 32 * VEC;
  __shared__ float s[8][COLS + 1];
  const int cg = threadIdx.x & 31, ph = threadIdx.x >> 5, z = blockIdx.z, col = blockIdx.x * COLS + cg * VEC;
  const int64_t r0 = (int64_t)blockIdx.y * kSumRows, r1 = r0 + kSumRows < rows ? r0 + kSumRows : rows;
  float acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  if (col < width) {
    const uint16_t* p = x + z * x_z + col;
#pragma unroll 4
    for (int64_t r = r0 + ph; r < r1; r += 8) {
      const piece_of<VEC> v = load_piece<VEC>(p + r * x_s);
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += v.v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[ph][cg * VEC + e] = acc[e];
  __syncthreads();
  for (int c = threadIdx.x; c < COLS; c += 256) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += s[w][c];
    if (blockIdx.x * COLS + c < width) part[z * part_z + (int64_t)blockIdx.y * width + blockIdx.x * COLS + c] = v;
  }
}

// Rows of codes to values: a thread takes 8 columns.  Grid: (ceil(rows * pieces / 256), replicas).
template <typename T, int VEC>
__global__ __launch_bounds__(256) void hdet_restore_kernel(const int8_t* q, int64_t q_s, int64_t q_z, const float* scale, T* v, int64_t v_s, int64_t v_z,
                                                           int64_t rows, int width, int pieces) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, row = t / pieces;
  const int z = blockIdx.y, col = (int)(t - row * pieces) * 8;
  if (row >= rows) return;
  const hdet_u2v w = *reinterpret_cast<const hdet_u2v*>(q + z * q_z + row * q_s + col);
  const float s = scale[z * rows + row];
  float o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = (float)(int8_t)((w[e >> 2] >> (8 * (e & 3))) & 255u) * s;
  T* const p = v + z * v_z + row * v_s + col;
  if constexpr (VEC == 8) {
    store_piece<8>(p, o);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (col + e < width) hdet_st(p + e, o[e]);
  }
}

namespace {

// Whether rows are whole 16-byte pieces of `size`-byte elements (8 of them) at 16-byte boundaries, or the matrix is absent
bool pieces_of_8(const hdet_rows& m, int size, int width) {
  if (!m.dev) return true;
  return (reinterpret_cast<uintptr_t>(m.dev) & 15) == 0 && ((m.row_stride | m.replica_stride) * size & 15) == 0 && (width & 7) == 0;
}

// f(T, VEC, L, C) for the smallest row of registers that holds `width`
template <typename T, typename F>
void with_shape(int width, bool vec, F f) {
#define HDET_SHAPE(VEC, L, C)                                                                         \
  if (width <= VEC * L * C) return f(T(), std::integral_constant<int, VEC>(), std::integral_constant<int, L>(), std::integral_constant<int, C>())
  if (vec) {
    HDET_SHAPE(8, 8, 1);
    HDET_SHAPE(8, 16, 1);
    HDET_SHAPE(8, 32, 1);
    HDET_SHAPE(8, 64, 1);
    HDET_SHAPE(8, 64, 2);
    HDET_SHAPE(8, 64, 4);
    HDET_SHAPE(8, 256, 2);
    HDET_SHAPE(8, 256, 4);
    HDET_SHAPE(8, 1024, 2);
    HDET_SHAPE(8, 1024, 4);
  } else {
    HDET_SHAPE(1, 64, 8);
    HDET_SHAPE(1, 64, 32);
    HDET_SHAPE(1, 256, 32);
    HDET_SHAPE(1, 1024, 32);
  }
#undef HDET_SHAPE
}
int rows_per_block(int width, bool vec) {
  int n = 1;
  with_shape<float>(width, vec, [&](auto, auto, auto l, auto) { n = l < 256 ? 256 / l : 1; });
  return n;
}
// blocks a replica of the backward pass: about eight a compute unit over all replicas, so that the gain's partial sums stay few
int grad_blocks(int n_replicas, int64_t rows, int width, bool vec) {
  const int64_t most = (rows + rows_per_block(width, vec) - 1) / rows_per_block(width, vec);
  int64_t want = 8 * (int64_t)hdet_compute_units() / n_replicas;
  if (want < 1) want = 1;
  return (int)(most < want ? most : want);
}

template <typename T>
hipError_t launch_norm_typed(const norm_kernel_args& k, int n, bool vec, bool norm, hipStream_t s) {
  with_shape<T>(k.width, vec, [&](auto t, auto v, auto l, auto c) {
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
  norm_kernel_args k = {a.x.dev, a.resid.dev, a.total.dev, a.y.dev, (int8_t*)a.codes.dev, a.scale_dev, a.rstd_dev, a.gain_dev,
                        a.x.row_stride, a.x.replica_stride, a.resid.row_stride, a.resid.replica_stride, a.total.row_stride, a.total.replica_stride,
                        a.y.row_stride, a.y.replica_stride, a.codes.row_stride, a.codes.replica_stride, a.gain_stride, a.rows, a.width, (float)a.eps, 1.f / (float)a.width};
  return a.dtype == HDET_TYPE_BF16 ? launch_norm_typed<uint16_t>(k, a.n_replicas, vec, true, s) : launch_norm_typed<float>(k, a.n_replicas, vec, true, s);
}

hipError_t hdet_launch_quantise(const hdet_codes_args& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const bool vec = pieces_of_8(a.values, a.dtype == HDET_TYPE_BF16 ? 2 : 4, a.width);
  norm_kernel_args k = {};
  k.x = a.values.dev; k.x_s = a.values.row_stride; k.x_z = a.values.replica_stride;
  k.codes = (int8_t*)a.codes.dev; k.c_s = a.codes.row_stride; k.c_z = a.codes.replica_stride;
  k.scale = a.scale_dev; k.rows = a.rows; k.width = a.width;
  return a.dtype == HDET_TYPE_BF16 ? launch_norm_typed<uint16_t>(k, a.n_replicas, vec, false, s) : launch_norm_typed<float>(k, a.n_replicas, vec, false, s);
}

hipError_t hdet_launch_restore(const hdet_codes_args& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const int pieces = (a.width + 7) / 8;
  const bool bf = a.dtype == HDET_TYPE_BF16, vec = pieces_of_8(a.values, bf ? 2 : 4, a.width);
  const dim3 grid((unsigned)((a.rows * pieces + 255) / 256), a.n_replicas);
  auto go = [&](auto kernel, auto* v) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const int8_t*)a.codes.dev, a.codes.row_stride, a.codes.replica_stride, a.scale_dev, v,
                       a.values.row_stride, a.values.replica_stride, a.rows, a.width, pieces);
  };
  if (bf && vec) go(&hdet_restore_kernel<uint16_t, 8>, (uint16_t*)a.values.dev);
  else if (bf) go(&hdet_restore_kernel<uint16_t, 1>, (uint16_t*)a.values.dev);
  else if (vec) go(&hdet_restore_kernel<float, 8>, (float*)a.values.dev);
  else go(&hdet_restore_kernel<float, 1>, (float*)a.values.dev);
  return hipGetLastError();
}

size_t hdet_norm_backward_bytes(int n_replicas, int64_t rows, int width) {
  if (rows == 0) return 0;
  const int a = grad_blocks(n_replicas, rows, width, true), b = grad_blocks(n_replicas, rows, width, false);
  return (size_t)n_replicas * (a > b ? a : b) * width * sizeof(float);
}

hipError_t hdet_launch_partial_sum(const float* partial, int n_replicas, int parts, int width, int64_t pitch, float* out, int64_t out_stride, hipStream_t s) {
  hipLaunchKernelGGL(hdet_partial_sum_kernel, dim3((width + 63) / 64, n_replicas), dim3(256), 0, s, partial, parts, width, pitch, out, out_stride);
  return hipGetLastError();
}

hipError_t hdet_launch_norm_backward(const hdet_norm_grad_args& a, hipStream_t s) {
  // no rows: the sum over none of them
  if (a.rows == 0) return a.dgain_dev ? hdet_launch_partial_sum(nullptr, a.n_replicas, 0, a.width, 0, a.dgain_dev, a.dgain_stride, s) : hipSuccess;
  const int size = a.dtype == HDET_TYPE_BF16 ? 2 : 4;
  const bool vec = pieces_of_8(a.total, size, a.width) && pieces_of_8(a.dy, size, a.width) && pieces_of_8(a.dtotal, size, a.width) && pieces_of_8(a.dx, size, a.width);
  const int blocks = grad_blocks(a.n_replicas, a.rows, a.width, vec);
  const bool direct = blocks == 1;
  const norm_grad_kernel_args k = {a.total.dev, a.dy.dev, a.dtotal.dev, a.dx.dev, a.rstd_dev, a.gain_dev, !a.dgain_dev ? nullptr : direct ? a.dgain_dev : (float*)a.workspace_dev,
                                   a.total.row_stride, a.total.replica_stride, a.dy.row_stride, a.dy.replica_stride, a.dtotal.row_stride, a.dtotal.replica_stride,
                                   a.dx.row_stride, a.dx.replica_stride, a.gain_stride, direct ? a.dgain_stride : (int64_t)blocks * a.width, a.rows, a.width, 1.f / (float)a.width};
  auto go = [&](auto t, auto v, auto l, auto c) {
    hipLaunchKernelGGL((hdet_norm_grad_kernel<decltype(t), v, l, c>), dim3(blocks, a.n_replicas), dim3(l < 256 ? 256 : l), 0, s, k);
  };
  if (a.dtype == HDET_TYPE_BF16) with_shape<uint16_t>(a.width, vec, go);
  else with_shape<float>(a.width, vec, go);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || direct || !a.dgain_dev) return e;
  return hdet_launch_partial_sum((const float*)a.workspace_dev, a.n_replicas, blocks, a.width, a.width, a.dgain_dev, a.dgain_stride, s);
}

size_t hdet_row_sum_bytes(int n_replicas, int64_t rows, int width) { return (size_t)n_replicas * ((rows + kSumRows - 1) / kSumRows) * width * sizeof(float); }

hipError_t hdet_launch_row_sum(const hdet_rows& x, int n_replicas, int64_t rows, int width, float* out, int64_t out_stride, void* scratch, hipStream_t s) {
  const int parts = (int)((rows + kSumRows - 1) / kSumRows);
  if (parts == 0) return hdet_launch_partial_sum(nullptr, n_replicas, 0, width, 0, out, out_stride, s);
  float* const to = parts == 1 ? out : (float*)scratch;
  const int64_t to_z = parts == 1 ? out_stride : (int64_t)parts * width;
  if (pieces_of_8(x, 2, width))
    hipLaunchKernelGGL(hdet_row_sum_kernel<8>, dim3((width + 255) / 256, parts, n_replicas), dim3(256), 0, s, (const uint16_t*)x.dev, x.row_stride, x.replica_stride, rows, width, to, to_z);
  else
    hipLaunchKernelGGL(hdet_row_sum_kernel<1>, dim3((width + 31) / 32, parts, n_replicas), dim3(256), 0, s, (const uint16_t*)x.dev, x.row_stride, x.replica_stride, rows, width, to, to_z);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  return hdet_launch_partial_sum((const float*)scratch, n_replicas, parts, width, width, out, out_stride, s);
}
