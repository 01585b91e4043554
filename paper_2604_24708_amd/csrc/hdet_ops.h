// Launchers of the language-model operators (hdet_ops.hip checks arguments and calls them).
#pragma once

#include "hdet_internal.h"

// Blocks of 256 threads for `threads` of them a replica, which is blockIdx.y: a launch takes fewer than 2^32 along x, and a large matrix
// has more elements, or pieces of 8 of them
inline dim3 hdet_long_grid(int64_t threads, int n_replicas) {
  const int64_t blocks = (threads + 255) / 256, x = blocks < (1 << 23) ? blocks : 1 << 23;
  return dim3((unsigned)x, n_replicas, (unsigned)((blocks + x - 1) / x));
}
__device__ __forceinline__ int64_t hdet_long_thread() { return ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * 256 + threadIdx.x; }

// hdet_norm.hip
hipError_t hdet_launch_norm(const hdet_norm_args& a, hipStream_t s);
hipError_t hdet_launch_norm_backward(const hdet_norm_grad_args& a, hipStream_t s);
size_t hdet_norm_backward_bytes(int n_replicas, int64_t rows, int width);
hipError_t hdet_launch_quantise(const hdet_codes_args& a, hipStream_t s);
hipError_t hdet_launch_restore(const hdet_codes_args& a, hipStream_t s);
// Sums over the rows of a bfloat16 matrix, [width] per replica, in a fixed order; scratch: hdet_row_sum_bytes bytes.
size_t hdet_row_sum_bytes(int n_replicas, int64_t rows, int width);
hipError_t hdet_launch_row_sum(const hdet_rows& x, int n_replicas, int64_t rows, int width, float* out, int64_t out_stride, void* scratch, hipStream_t s);
// A bfloat16 matrix as `copies` matrices below each other in rows of `pitch` elements (a multiple of 8, at least width), zeros behind the
// last column and in rows whose label ([replica][row], or null: none) is negative
hipError_t hdet_launch_pad_rows(const hdet_rows& x, int n_replicas, int64_t rows, int width, const int32_t* labels, uint16_t* out, int64_t pitch, int copies, hipStream_t s);
// The second half of such a sum: out[z][j] = sum_p partial[z][p][j]
hipError_t hdet_launch_partial_sum(const float* partial, int n_replicas, int parts, int width, int64_t pitch, float* out, int64_t out_stride, hipStream_t s);

// hdet_gemm_codes.hip
hipError_t hdet_launch_codes_gemm(const hdet_linear_args& a, hipStream_t s);

// hdet_split.hip: products (input-gradient or weight-gradient order) of few tiles and a long contraction
struct hdet_split { int pieces; int64_t each; size_t bytes; };      // pieces of `each`, and the memory of their results (0: one piece, no split)
struct hdet_split_out {
  void* c; int dtype; int64_t ld, bs;                // result, HDET_TYPE_*, at any element
  const float* scale;                                // [replica] or null
  float* accum; int64_t accum_ld, accum_bs;          // as HDET_EPI_ACCUM_BF16, or null
  bool first, last;
};
hdet_split hdet_split_of(int batch, int64_t m, int64_t n, int64_t k);
// g: operands, m, n, k, padded; one batch level
hipError_t hdet_launch_split(const hdet_bgemm_args& g, bool a_kmajor, int batch, const hdet_split& sp, float* partial, const hdet_split_out& out, hipStream_t s);

// hdet_vocab.hip
hipError_t hdet_launch_zero_rows(const hdet_rows& m, int n_replicas, int64_t rows, int width, int dtype, hipStream_t s);
int hdet_vocab_kind(const hdet_vocab_args& a);                                       // HDET_TYPE_* of dw, HDET_VOCAB_* without one
size_t hdet_vocab_bytes(int n_replicas, int64_t rows, int width, int classes, int kind, int piece);
hipError_t hdet_launch_vocab_loss(const hdet_vocab_args& a, hipStream_t s);
