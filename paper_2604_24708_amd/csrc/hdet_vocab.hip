// Output layer with its softmax cross-entropy in pieces of the vocabulary, N replicas:
//
//   z = h W^T + b,  loss = log sum exp z - z_label,  dz = (softmax(z) - onehot) / c,  dh = dz W,  dW = dz^T h,  db = sum_rows dz
//
// No more than `piece` classes of z and dz exist at a time.  A first round over the pieces forms each row's reference and sum of exponentials, a second
// forms z again, dz from it, and with dz the piece's share of dh (added up in fp32) and its rows of dW and db.  With one piece z is formed once.
//
// Exponentials are exp2(z log2(e) - r) with r the whole number next to max log2(e): pieces refer to each other by exact powers of two.
// dz leaves as bfloat16 -- what the matrix cores multiply -- for dh and a bfloat16 dW, whose own rounding is as coarse.  An fp32 dW takes dz in three bfloat16 parts,
// 24 bits: they stand below each other as rows, beside three copies of h, and make one product of three times the rows.

#include <type_traits>

#include "hdet_ops.h"
#include "hdet_elem.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;
constexpr int kRowChunk = 128;      // rows of a block's column sums

// Memory of a call, in the order it is carved.  What a member names: [replica][...].
struct vocab_layout {
  int piece;                // classes at a time
  int pieces;
  int planes;               // bfloat16 parts of dz
  int64_t pitch;            // columns of z and dz as they lie in memory
  size_t count, ref, a, sum, zy, z, dz, h3, acc, part, total;
};
size_t up(size_t x) { return (x + 255) & ~(size_t)255; }

vocab_layout layout_of(int n, int64_t rows, int width, int classes, int dw_dtype, int piece) {
  vocab_layout l;
  l.planes = dw_dtype == HDET_TYPE_F32 ? 3 : 1;
  const size_t all = (size_t)n * rows;
  if (piece <= 0) {
    // z and dz of a piece in a few hundred megabytes, at least 1024 classes
    const size_t a_class = all * (4 + 2 * l.planes);
    size_t p = a_class ? ((size_t)512 << 20) / a_class : (size_t)classes;
    p = p / 256 * 256;
    piece = p < 1024 ? 1024 : p > (size_t)classes ? classes : (int)p;
  }
  if (piece > classes) piece = classes;
  l.piece = piece;
  l.pieces = (classes + piece - 1) / piece;
  l.pitch = (piece + 7) & ~7;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += up(bytes); return here; };
  l.count = take((size_t)n * 4);
  l.ref = take(all * 4);
  l.a = take(all * 4);
  l.sum = take(all * 8);
  l.zy = take(all * 4);
  l.z = take(all * l.pitch * 4);
  l.dz = take(all * l.pitch * 2 * l.planes);
  l.h3 = take(l.planes == 3 ? all * 3 * width * 2 : 0);
  l.acc = take(l.pieces > 1 ? all * width * 4 : 0);
  l.part = take((size_t)n * ((rows + kRowChunk - 1) / kRowChunk) * l.pitch * 4);
  l.total = at;
  return l;
}

}  // namespace

// 1 / rows that count, and the losses of a replica without rows.  One block a replica.
__global__ __launch_bounds__(256) void hdet_vocab_count_kernel(const int32_t* labels, int64_t rows, int classes, float* inv, float* mean) {
  __shared__ int part[4];
  const int z = blockIdx.x;
  int n = 0;
  for (int64_t i = threadIdx.x; i < rows; i += 256) n += (unsigned)labels[z * rows + i] < (unsigned)classes ? 1 : 0;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = part[0] + part[1] + part[2] + part[3];
    inv[z] = 1.f / (float)(n > 1 ? n : 1);
    if (rows == 0) mean[z] = 0.f;
  }
}

// Reference and sum of a row over the classes so far, and its label's logit.  Block = one row of a piece; grid (rows, replicas).
__global__ __launch_bounds__(256) void hdet_vocab_stat_kernel(const float* z, int64_t pitch, int64_t rows, int cols, int v0, const int32_t* labels, float* ref,
                                                              double* sum, float* zy) {
  __shared__ float part[4];
  const int64_t row = blockIdx.x, at = (int64_t)blockIdx.y * rows + row;
  const float* p = z + at * pitch;
  float mx = -INFINITY;
  for (int c = threadIdx.x; c < cols; c += 256) mx = fmaxf(mx, p[c]);
  mx = hdet_wave_max(mx);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mx;
  __syncthreads();
  mx = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  __syncthreads();
  const float r = rintf(mx * kLog2e), rl = r == -INFINITY ? 0.f : r;
  float s = 0.f;
  for (int c = threadIdx.x; c < cols; c += 256) s += __builtin_amdgcn_exp2f(__builtin_fmaf(p[c], kLog2e, -rl));
  s = hdet_wave_sum(s);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = (part[0] + part[1]) + (part[2] + part[3]);
    const int y = labels[at] - v0;
    if ((unsigned)y < (unsigned)cols) zy[at] = p[y];
    if (v0 == 0) {
      ref[at] = r;
      sum[at] = (double)s;
    } else {
      const float r0 = ref[at], top = fmaxf(r0, r);
      // a side without classes has the sum 0 (or NaN) and no reference
      const double a = r0 == -INFINITY ? sum[at] : sum[at] * (double)__builtin_amdgcn_exp2f(r0 - top);
      const double b = r == -INFINITY ? (double)s : (double)(s * __builtin_amdgcn_exp2f(r - top));
      ref[at] = top;
      sum[at] = a + b;
    }
  }
}

// A row's loss and the factor of its exponentials in dz
__global__ __launch_bounds__(256) void hdet_vocab_rows_kernel(const float* ref, const double* sum, const float* zy, const int32_t* labels, const float* inv, int64_t rows,
                                                              int classes, float* a, float* row_loss) {
  const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int z = blockIdx.y;
  if (row >= rows) return;
  const int64_t at = z * rows + row;
  const bool counts = (unsigned)labels[at] < (unsigned)classes;
  a[at] = counts ? (float)((double)inv[z] / sum[at]) : 0.f;
  row_loss[at] = counts ? (float)(((double)ref[at] + log2(sum[at]) - (double)zy[at] * 1.4426950408889634) * kLn2) : 0.f;
}

__global__ __launch_bounds__(256) void hdet_vocab_mean_kernel(const float* row_loss, const float* inv, int64_t rows, float* mean) {
  __shared__ double part[4];
  const int z = blockIdx.x;
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < rows; i += 256) s += (double)row_loss[z * rows + i];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) mean[z] = (float)((part[0] + part[1] + part[2] + part[3]) * (double)inv[z]);
}

// dz of a piece from z, in PLANES bfloat16 parts, and its sums over 128 rows.  Thread = a column; grid (ceil(pitch / 256), row chunks, replicas).
template <int PLANES>
__global__ __launch_bounds__(256) void hdet_vocab_grad_kernel(const float* z, int64_t pitch, int64_t rows, int cols, int v0, int classes, const int32_t* labels, const float* ref,
                                                              const float* a, const float* inv, uint16_t* dz, float* part) {
  const int c = blockIdx.x * 256 + threadIdx.x, zr = blockIdx.z;
  if (c >= pitch) return;
  const int64_t r0 = (int64_t)blockIdx.y * kRowChunk, r1 = r0 + kRowChunk < rows ? r0 + kRowChunk : rows;
  const float invc = inv[zr];
  float sum = 0.f;
  for (int64_t r = r0; r < r1; ++r) {
    const int64_t at = zr * rows + r;
    const int y = labels[at] - v0;
    float v = 0.f;
    if (c < cols && a[at] != 0.f) v = __builtin_amdgcn_exp2f(__builtin_fmaf(z[at * pitch + c], kLog2e, -ref[at])) * a[at];
    if (c < cols && c == y) v -= invc;
    sum += v;
    uint16_t* p = dz + ((int64_t)zr * PLANES * rows + r) * pitch + c;
#pragma unroll
    for (int q = 0; q < PLANES; ++q) {
      const unsigned b = hdet_bf16_bits(v);
      p[q * rows * pitch] = (uint16_t)b;
      v -= __uint_as_float(b << 16);
    }
  }
  if (part) part[((int64_t)zr * gridDim.y + blockIdx.y) * pitch + c] = sum;
}

// three copies of h below each other: [replica][3][rows][width]
__global__ __launch_bounds__(256) void hdet_vocab_copy_kernel(const uint16_t* h, int64_t h_s, int64_t h_z, int64_t rows, int width, uint16_t* out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = rows * width;
  if (i >= all) return;
  const uint16_t v = h[blockIdx.y * h_z + i / width * h_s + i % width];
  uint16_t* p = out + blockIdx.y * 3 * all + i;
  p[0] = v; p[all] = v; p[2 * all] = v;
}

// zeros in a matrix of `size`-byte elements (2 or 4)
__global__ __launch_bounds__(256) void hdet_zero_rows_kernel(void* m, int64_t row_s, int64_t rep_s, int64_t rows, int width, int size) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * width) return;
  const int64_t at = blockIdx.y * rep_s + i / width * row_s + i % width;
  if (size == 2) ((uint16_t*)m)[at] = 0;
  else ((float*)m)[at] = 0.f;
}

hipError_t hdet_launch_zero_rows(const hdet_rows& m, int n_replicas, int64_t rows, int width, int dtype, hipStream_t s) {
  hipLaunchKernelGGL(hdet_zero_rows_kernel, dim3((unsigned)((rows * width + 255) / 256), n_replicas), dim3(256), 0, s, m.dev, m.row_stride, m.replica_stride, rows, width,
                     dtype == HDET_TYPE_BF16 ? 2 : 4);
  return hipGetLastError();
}

size_t hdet_vocab_bytes(int n_replicas, int64_t rows, int width, int classes, int dw_dtype, int piece) {
  return layout_of(n_replicas, rows, width, classes, dw_dtype, piece).total;
}

hipError_t hdet_launch_vocab_loss(const hdet_vocab_args& a, hipStream_t s) {
  const int n = a.n_replicas, d = a.width, V = a.classes;
  const int64_t M = a.rows;
  const vocab_layout l = layout_of(n, M, d, V, a.dw.dev ? a.dw_dtype : HDET_TYPE_BF16, a.piece);
  char* const ws = (char*)a.workspace_dev;
  float* const inv = (float*)(ws + l.count);
  hipLaunchKernelGGL(hdet_vocab_count_kernel, dim3(n), dim3(256), 0, s, a.labels_dev, M, V, inv, a.mean_loss_dev);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (M == 0) {
    if (a.dw.dev && (e = hdet_launch_zero_rows(a.dw, n, V, d, a.dw_dtype, s)) != hipSuccess) return e;
    return a.db_dev ? hdet_launch_partial_sum(nullptr, n, 0, V, 0, a.db_dev, a.db_stride, s) : hipSuccess;
  }
  float *const ref = (float*)(ws + l.ref), *const ra = (float*)(ws + l.a), *const zy = (float*)(ws + l.zy), *const z = (float*)(ws + l.z);
  double* const sum = (double*)(ws + l.sum);
  uint16_t *const dz = (uint16_t*)(ws + l.dz), *const h3 = (uint16_t*)(ws + l.h3);
  float* const part = (float*)(ws + l.part);
  const bool grads = a.dh.dev || a.dw.dev || a.db_dev;
  const uint16_t *h = (const uint16_t*)a.h.dev, *w = (const uint16_t*)a.w.dev;
  const int chunks = (int)((M + kRowChunk - 1) / kRowChunk);

  auto logits = [&](int v0, int cols) {
    hdet_bgemm_args g = {};
    g.a = h; g.lda = a.h.row_stride; g.a_s[0] = a.h.replica_stride;
    g.b = w + v0 * a.w.row_stride; g.ldb = a.w.row_stride; g.b_s[0] = a.w.replica_stride;
    g.c = z; g.ldc = l.pitch; g.c_s[0] = M * l.pitch;
    g.m = (int)M; g.n = cols; g.k = d;
    if (a.bias_dev) { g.bias = a.bias_dev + v0; g.bias_bs = a.bias_stride; }
    return hdet_launch_bgemm(g, true, true, a.bias_dev ? HDET_EPI_BIAS_F32 : HDET_EPI_F32, n, s);
  };
  for (int p = 0; p < l.pieces; ++p) {
    const int v0 = p * l.piece, cols = V - v0 < l.piece ? V - v0 : l.piece;
    if ((e = logits(v0, cols)) != hipSuccess) return e;
    hipLaunchKernelGGL(hdet_vocab_stat_kernel, dim3((unsigned)M, n), dim3(256), 0, s, z, l.pitch, M, cols, v0, a.labels_dev, ref, sum, zy);
  }
  hipLaunchKernelGGL(hdet_vocab_rows_kernel, dim3((unsigned)((M + 255) / 256), n), dim3(256), 0, s, ref, sum, zy, a.labels_dev, inv, M, V, ra, a.row_loss_dev);
  hipLaunchKernelGGL(hdet_vocab_mean_kernel, dim3(n), dim3(256), 0, s, a.row_loss_dev, inv, M, a.mean_loss_dev);
  if ((e = hipGetLastError()) != hipSuccess || !grads) return e;
  if (l.planes == 3 && a.dw.dev)
    hipLaunchKernelGGL(hdet_vocab_copy_kernel, dim3((unsigned)((M * d + 255) / 256), n), dim3(256), 0, s, h, a.h.row_stride, a.h.replica_stride, M, d, h3);
  for (int p = 0; p < l.pieces; ++p) {
    const int v0 = p * l.piece, cols = V - v0 < l.piece ? V - v0 : l.piece;
    if (l.pieces > 1 && (e = logits(v0, cols)) != hipSuccess) return e;
    const dim3 grid((unsigned)((l.pitch + 255) / 256), chunks, n);
    float* const to = a.db_dev ? part : nullptr;
    if (l.planes == 3) hipLaunchKernelGGL(hdet_vocab_grad_kernel<3>, grid, dim3(256), 0, s, z, l.pitch, M, cols, v0, V, a.labels_dev, ref, ra, inv, dz, to);
    else hipLaunchKernelGGL(hdet_vocab_grad_kernel<1>, grid, dim3(256), 0, s, z, l.pitch, M, cols, v0, V, a.labels_dev, ref, ra, inv, dz, to);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.db_dev && (e = hdet_launch_partial_sum(part, n, chunks, cols, l.pitch, a.db_dev + v0, a.db_stride, s)) != hipSuccess) return e;
    if (a.dh.dev) {
      hdet_bgemm_args g = {};
      g.a = dz; g.lda = l.pitch; g.a_s[0] = l.planes * M * l.pitch;
      g.b = w + v0 * a.w.row_stride; g.ldb = a.w.row_stride; g.b_s[0] = a.w.replica_stride;
      g.c = a.dh.dev; g.ldc = a.dh.row_stride; g.c_s[0] = a.dh.replica_stride;
      g.m = (int)M; g.n = d; g.k = cols;
      g.accum = (float*)(ws + l.acc); g.accum_ld = d; g.accum_bs = M * d;
      g.accum_first = p == 0; g.accum_last = p + 1 == l.pieces;
      if ((e = hdet_launch_bgemm(g, true, false, l.pieces > 1 ? HDET_EPI_ACCUM_BF16 : HDET_EPI_BF16, n, s)) != hipSuccess) return e;
    }
    if (a.dw.dev) {
      const bool f32 = l.planes == 3;
      hdet_bgemm_args g = {};
      g.a = dz; g.lda = l.pitch; g.a_s[0] = l.planes * M * l.pitch;
      g.b = f32 ? h3 : h; g.ldb = f32 ? d : a.h.row_stride; g.b_s[0] = f32 ? 3 * M * d : a.h.replica_stride;
      g.c = (char*)a.dw.dev + v0 * a.dw.row_stride * (f32 ? 4 : 2); g.ldc = a.dw.row_stride; g.c_s[0] = a.dw.replica_stride;
      g.m = cols; g.n = d; g.k = (int)(l.planes * M);
      if ((e = hdet_launch_bgemm(g, false, false, f32 ? HDET_EPI_F32 : HDET_EPI_BF16, n, s)) != hipSuccess) return e;
    }
  }
  return hipSuccess;
}
