// The common norm of a model's gradient tensors, and the gradients times min(1, max_norm / norm) in the plane of the update.
//
//   norm_r = sqrt(sum over tensors and elements of g^2);  with shared gradients g is the replicas' mean;  out = g factor
//
// Bound by memory: every gradient is read twice, since its factor depends on all of them, and written once.  Tensors are cut into pieces of
// CHUNK elements; block b of G takes pieces b, b + G, b + 2 G .., so that all blocks together read neighbouring memory, whatever tensors they
// belong to, and sums in 64 bits and a fixed order.  The second kernel's blocks each add up the same partial sums (a few KB) instead of waiting for a
// third launch, and walk from the end, where the memory-side cache still holds what the first kernel read last.
//   us for the 870 million elements of a 12-layer transformer's four replicas: 1750, 520 for the norm and 1250 for the rest under the profiler, 5.3 TB/s
//   over both.  A run of pieces a block: 1950; 1825 without the numbers of blocks and the stores past the caches of hdet_launch_clip.
// A list of more than INLINE tensors is written to the workspace first, INLINE of them a launch (2 to 5 us each).

#include <math.h>

#include <algorithm>

#include "hdet_ops.h"
#include "hdet_elem.h"

namespace {

constexpr int THREADS = 256;
constexpr int CHUNK = 4096;                // elements of a piece: 4 x 4 a thread
constexpr int INLINE = 40;                 // tensors whose places fit a launch's arguments

struct tensor_place {
  const void* g;
  float* out;                              // null: g itself is scaled
  int64_t g_s, g_z, o_s, o_z;
  int64_t width, first;                    // elements of a row; first piece
  int64_t size;                            // rows * width
  int32_t bf16;
  int32_t whole;                           // rows are whole groups of 4 elements at boundaries of 4 (or there is one row)
};
struct tensor_list { tensor_place t[INLINE]; };
struct clip_args {
  const tensor_place* table;               // in the workspace, where the list does not fit the arguments
  double* partial;                         // [replica, or 1 shared][blocks]
  float* norm;
  int tensors, parts, n;
  int shared, scale;                       // scale: the second kernel writes gradients
  int stream;                              // .. past the caches
  int64_t chunks;                          // pieces in all
  double max_norm;
};

struct place_of {                          // a piece: its tensor, its first element
  const tensor_place* t;
  int64_t e0, row0, col0;
  int count;
};

// the tensor of piece c, given that it is `at` or a later one
__device__ __forceinline__ int tensor_of(const tensor_place* t, int tensors, int64_t c, int at) {
  if (at + 1 >= tensors || t[at + 1].first > c) return at;
  int lo = at + 1, hi = tensors;           // t[lo].first <= c < t[hi].first
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t[mid].first <= c) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ place_of piece(const tensor_place* t, int64_t c) {
  place_of p;
  p.t = t;
  p.e0 = (c - t->first) * CHUNK;
  p.row0 = p.e0 / t->width;
  p.col0 = p.e0 - p.row0 * t->width;
  const int64_t left = t->size - p.e0;
  p.count = left < CHUNK ? (int)left : CHUNK;
  return p;
}
// offset of element e0 + i of a piece in a matrix of row stride s
__device__ __forceinline__ int64_t offset_in(const place_of& p, int i, int64_t s) {
  const int64_t col = p.col0 + i;
  if (col < p.t->width) return p.row0 * s + col;
  if (p.t->width < (int64_t)1 << 30) {     // col < 2^30 + CHUNK
    const unsigned down = (unsigned)col / (unsigned)p.t->width;
    return (p.row0 + down) * s + ((unsigned)col - down * (unsigned)p.t->width);
  }
  return (p.row0 + 1) * s + (col - p.t->width);
}

// Four elements: 16 neighbouring bytes a lane of an fp32 tensor (eight, in two pieces of 16 that lie 32 apart: the same)
__device__ __forceinline__ hdet_f4 load4(const tensor_place& t, int64_t at) {
  return t.bf16 ? hdet_ld4((const uint16_t*)t.g + at) : hdet_ld4((const float*)t.g + at);
}
__device__ __forceinline__ float load1(const tensor_place& t, int64_t at) {
  return t.bf16 ? hdet_ld((const uint16_t*)t.g + at) : hdet_ld((const float*)t.g + at);
}

// Sum over the block's threads in a fixed order, the same in each
__device__ __forceinline__ double block_sum(double v, double* part) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

template <bool LISTED> __global__ __launch_bounds__(THREADS) void clip_norm_kernel(const clip_args g, const tensor_list list) {
  __shared__ double part[4];
  const tensor_place* const tensors = LISTED ? list.t : g.table;
  const int r = blockIdx.y;
  const double inv_n = 1.0 / g.n;
  double sum = 0.0;
  int at = 0;
  for (int64_t c = blockIdx.x; c < g.chunks; c += gridDim.x) {
    at = tensor_of(tensors, g.tensors, c, at);
    const tensor_place t = tensors[at];
    const place_of p = piece(&t, c);
    const int vecs = t.whole ? p.count >> 2 : 0;
    if (!g.shared) {
      const int64_t z = r * t.g_z;
      if (vecs == CHUNK / 4) {
        hdet_f4 x[CHUNK / 4 / THREADS];
#pragma unroll
        for (int u = 0; u < CHUNK / 4 / THREADS; ++u) x[u] = load4(t, z + offset_in(p, (threadIdx.x + u * THREADS) * 4, t.g_s));
#pragma unroll
        for (int u = 0; u < CHUNK / 4 / THREADS; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum = __builtin_fma((double)x[u].v[e], (double)x[u].v[e], sum);
        continue;
      }
      for (int i = threadIdx.x; i < vecs; i += THREADS) {
        const hdet_f4 x = load4(t, z + offset_in(p, i * 4, t.g_s));
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = __builtin_fma((double)x.v[e], (double)x.v[e], sum);
      }
      for (int i = vecs * 4 + threadIdx.x; i < p.count; i += THREADS) {
        const double x = load1(t, z + offset_in(p, i, t.g_s));
        sum = __builtin_fma(x, x, sum);
      }
    } else {
      for (int i = threadIdx.x; i < vecs; i += THREADS) {
        const int64_t o = offset_in(p, i * 4, t.g_s);
        double m[4] = {};
        for (int z = 0; z < g.n; ++z) {
          const hdet_f4 x = load4(t, z * t.g_z + o);
#pragma unroll
          for (int e = 0; e < 4; ++e) m[e] += x.v[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          m[e] *= inv_n;
          sum = __builtin_fma(m[e], m[e], sum);
        }
      }
      for (int i = vecs * 4 + threadIdx.x; i < p.count; i += THREADS) {
        const int64_t o = offset_in(p, i, t.g_s);
        double m = 0.0;
        for (int z = 0; z < g.n; ++z) m += load1(t, z * t.g_z + o);
        m *= inv_n;
        sum = __builtin_fma(m, m, sum);
      }
    }
  }
  sum = block_sum(sum, part);
  if (threadIdx.x == 0) g.partial[(int64_t)r * g.parts + blockIdx.x] = sum;
}

template <bool LISTED> __global__ __launch_bounds__(THREADS) void clip_scale_kernel(const clip_args g, const tensor_list list) {
  __shared__ double part[4];
  const tensor_place* const tensors = LISTED ? list.t : g.table;
  const int r = blockIdx.y;
  const double* const from = g.partial + (g.shared ? 0 : (int64_t)r * g.parts);
  double sum = 0.0;
  for (int i = threadIdx.x; i < g.parts; i += THREADS) sum += from[i];
  const double norm = sqrt(block_sum(sum, part));
  if (blockIdx.x == 0 && threadIdx.x == 0) g.norm[r] = (float)norm;
  if (!g.scale) return;
  const float factor = norm > g.max_norm && norm < INFINITY ? (float)(g.max_norm / norm) : 1.f;
  // from the end on: the last pieces are the ones that the first kernel has read last
  for (int64_t c = g.chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
    const int at = tensor_of(tensors, g.tensors, c, 0);
    const tensor_place t = tensors[at];
    if (!t.out && factor == 1.f) continue;
    const place_of p = piece(&t, c);
    const int vecs = t.whole ? p.count >> 2 : 0;
    const int64_t gz = r * t.g_z, oz = r * t.o_z;
    auto put4 = [&](int i, hdet_f4 x) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x.v[e] *= factor;
      if (t.out && g.stream) hdet_st4_stream(t.out + oz + offset_in(p, i, t.o_s), x);
      else if (t.out) hdet_st4(t.out + oz + offset_in(p, i, t.o_s), x);
      else if (t.bf16) hdet_st4((uint16_t*)t.g + gz + offset_in(p, i, t.g_s), x);
      else hdet_st4((float*)t.g + gz + offset_in(p, i, t.g_s), x);
    };
    if (vecs == CHUNK / 4) {
      hdet_f4 x[CHUNK / 4 / THREADS];
#pragma unroll
      for (int u = 0; u < CHUNK / 4 / THREADS; ++u) x[u] = load4(t, gz + offset_in(p, (threadIdx.x + u * THREADS) * 4, t.g_s));
#pragma unroll
      for (int u = 0; u < CHUNK / 4 / THREADS; ++u) put4((threadIdx.x + u * THREADS) * 4, x[u]);
      continue;
    }
    for (int i = threadIdx.x; i < vecs; i += THREADS) put4(i * 4, load4(t, gz + offset_in(p, i * 4, t.g_s)));
    for (int i = vecs * 4 + threadIdx.x; i < p.count; i += THREADS) {
      const float x = load1(t, gz + offset_in(p, i, t.g_s)) * factor;
      if (t.out) t.out[oz + offset_in(p, i, t.o_s)] = x;
      else if (t.bf16) hdet_st((uint16_t*)t.g + gz + offset_in(p, i, t.g_s), x);
      else hdet_st((float*)t.g + gz + offset_in(p, i, t.g_s), x);
    }
  }
}

// Part of a list that does not fit one launch's arguments, into the workspace
__global__ __launch_bounds__(THREADS) void clip_list_kernel(tensor_place* table, const tensor_list list, int count) {
  for (int i = threadIdx.x; i < count; i += THREADS) table[i] = list.t[i];
}

constexpr size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
int most_parts(int n) {
  const int b = 16 * hdet_compute_units() / n;
  return b < 1 ? 1 : b;
}
bool whole(const hdet_rows& m, int size, bool one_row) {
  return (uintptr_t)m.dev % (4 * size) == 0 && ((m.replica_stride | (one_row ? 0 : m.row_stride)) & 3) == 0;
}

}  // namespace

size_t hdet_clip_bytes(int n_replicas, int n_tensors) {
  // shared gradients take all blocks for one sum
  return up256(most_parts(1) * sizeof(double) + (size_t)n_replicas * sizeof(double)) + (n_tensors > INLINE ? up256((size_t)n_tensors * sizeof(tensor_place)) : 0);
}

hipError_t hdet_launch_clip(const hdet_clip_args& a, hipStream_t s) {
  const int n = a.n_replicas;
  clip_args g = {};
  std::vector<tensor_place> list;
  list.reserve(a.n_tensors);
  for (int i = 0; i < a.n_tensors; ++i) {
    const hdet_grad_tensor& q = a.tensors_host[i];
    if (q.rows == 0 || q.width == 0) continue;
    tensor_place t;
    t.g = q.grad.dev; t.g_s = q.grad.row_stride; t.g_z = q.grad.replica_stride;
    t.out = (float*)q.out.dev; t.o_s = q.out.row_stride; t.o_z = q.out.replica_stride;
    t.size = q.rows * q.width;
    t.width = q.width;
    // rows without gaps are one
    if (q.rows == 1 || (t.g_s == q.width && (!t.out || t.o_s == q.width))) t.width = t.size;
    const bool one = t.width == t.size;
    t.bf16 = q.dtype == HDET_TYPE_BF16;
    t.whole = (one || t.width % 4 == 0) && whole(q.grad, t.bf16 ? 2 : 4, one) && (!t.out || whole(q.out, 4, one));
    t.first = g.chunks;
    g.chunks += (t.size + CHUNK - 1) / CHUNK;
    g.scale |= t.out || a.max_norm < INFINITY;
    list.push_back(t);
  }
  g.tensors = (int)list.size();
  g.partial = (double*)a.workspace_dev;
  g.norm = a.norm_dev;
  g.n = n;
  g.shared = a.grad_mode == HDET_GRAD_SHARED;
  g.max_norm = a.max_norm;
  const int sums = g.shared ? 1 : n, most = most_parts(sums);
  g.parts = (int)(g.chunks < most ? g.chunks : most);
  tensor_list first = {};
  if (g.tensors > INLINE) {
    tensor_place* const table = (tensor_place*)((char*)a.workspace_dev + up256(most_parts(1) * sizeof(double) + (size_t)n * sizeof(double)));
    g.table = table;
    for (int i = 0; i < g.tensors; i += INLINE) {
      const int count = g.tensors - i < INLINE ? g.tensors - i : INLINE;
      for (int j = 0; j < count; ++j) first.t[j] = list[i + j];
      hipLaunchKernelGGL(clip_list_kernel, dim3(1), dim3(THREADS), 0, s, table + i, first, count);
    }
  } else {
    for (int j = 0; j < g.tensors; ++j) first.t[j] = list[j];
  }
  if (g.chunks > 0) {
    if (g.table) hipLaunchKernelGGL(clip_norm_kernel<false>, dim3(g.parts, sums), dim3(THREADS), 0, s, g, first);
    else hipLaunchKernelGGL(clip_norm_kernel<true>, dim3(g.parts, sums), dim3(THREADS), 0, s, g, first);
  }
  // more blocks than sums, so that what is left at the end is short (1825 -> 1785 us); outputs of more than the memory-side cache go past it (-> 1745)
  const int64_t blocks = g.scale ? std::min(g.chunks, (int64_t)4 * most_parts(n)) : 1;
  g.stream = (int64_t)n * g.chunks * CHUNK * 4 > (int64_t)256 << 20;
  if (g.table) hipLaunchKernelGGL(clip_scale_kernel<false>, dim3((unsigned)blocks, n), dim3(THREADS), 0, s, g, first);
  else hipLaunchKernelGGL(clip_scale_kernel<true>, dim3((unsigned)blocks, n), dim3(THREADS), 0, s, g, first);
  return hipGetLastError();
}
