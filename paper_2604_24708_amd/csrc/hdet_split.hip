// Products of few tiles and a long contraction, in pieces of it: the pieces are further batch items of one launch, their fp32 results are
// added by a second one.  (One block a compute unit walks 64 of the contraction in 0.4 us: a tile of 128 x 128 with 9600 of it alone took
// 62 us.)

#include "hdet_ops.h"
#include "hdet_elem.h"

// How a product is split: not at all from half a tile of 128 x 128 a compute unit on, else into as many pieces as there are units to take
// them, of 512 at least.  (us of the call, whole / split: loss of 2 x 1000 rows of 776, 5000 classes, 112 tiles, two pieces 184 / 169;  100
// rows of 96, 9600 classes, one tile 115 / 56)
hdet_split hdet_split_of(int batch, int64_t m, int64_t n, int64_t k) {
  hdet_split s = {1, k, 0};
  const int64_t tiles = ((m + 127) / 128) * ((n + 127) / 128) * batch, cus = hdet_compute_units();
  if (tiles < 1 || 2 * tiles > cus || k < 1536) return s;
  int64_t pieces = cus / tiles;
  if (pieces > k / 512) pieces = k / 512;
  s.each = ((k + pieces - 1) / pieces + 63) / 64 * 64;
  s.pieces = (int)((k + s.each - 1) / s.each);
  if (s.pieces > 1) s.bytes = (size_t)batch * s.pieces * m * ((n + 7) & ~7) * sizeof(float);
  return s;
}

namespace {
struct sum_args {
  const float* part;       // [batch][pieces][m][pitch]
  int pieces, m, n, pitch;
  hdet_split_out out;
};
}  // namespace

// Thread = 4 columns of a row; grid (ceil(m * pitch / 4 / 256), batch)
template <typename T>
__global__ __launch_bounds__(256) void hdet_split_sum_kernel(const sum_args a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, quads = a.pitch >> 2, row = i / quads;
  const int col = (int)(i - row * quads) * 4, z = blockIdx.y;
  if (row >= a.m || col >= a.n) return;
  const int64_t plane = (int64_t)a.m * a.pitch;
  const float* p = a.part + z * a.pieces * plane + row * a.pitch + col;
  hdet_f4v v = *reinterpret_cast<const hdet_f4v*>(p);
#pragma unroll 4
  for (int s = 1; s < a.pieces; ++s) v += *reinterpret_cast<const hdet_f4v*>(p + s * plane);
  if (a.out.accum) {
    hdet_f4v* const acc = reinterpret_cast<hdet_f4v*>(a.out.accum + z * a.out.accum_bs + row * a.out.accum_ld + col);
    if (!a.out.first) v += *acc;
    if (!a.out.last) {
      *acc = v;
      return;
    }
  }
  if (a.out.scale) v *= a.out.scale[z];
  T* const c = (T*)a.out.c + z * a.out.bs + row * a.out.ld + col;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (col + e < a.n) hdet_st(c + e, v[e]);
}

hipError_t hdet_launch_split(const hdet_bgemm_args& g_in, bool a_kmajor, int batch, const hdet_split& sp, float* partial, const hdet_split_out& out, hipStream_t s) {
  const int pitch = (g_in.n + 7) & ~7;
  const int64_t plane = (int64_t)g_in.m * pitch, a_step = a_kmajor ? sp.each : sp.each * g_in.lda, b_step = sp.each * g_in.ldb;
  hdet_bgemm_args g = g_in;
  g.ldc = pitch; g.c_s[0] = sp.pieces * plane; g.c_s[1] = plane; g.c_s[2] = 0;
  g.a_s[1] = a_step; g.b_s[1] = b_step; g.a_s[2] = g.b_s[2] = 0;
  g.n2 = 1; g.out_scale = nullptr;
  g.c = partial; g.k = (int)sp.each; g.n1 = sp.pieces;
  const int rest = (int)(g_in.k - (sp.pieces - 1) * sp.each);
  hipError_t e;
  g.k_last = rest;
  if (hdet_bgemm_dma_eligible(g, a_kmajor, false, HDET_EPI_SCALED_F32)) {
    if ((e = hdet_launch_bgemm(g, a_kmajor, false, HDET_EPI_SCALED_F32, batch * sp.pieces, s)) != hipSuccess) return e;
  } else {      // the general kernels: pieces of one length in a launch, the last one in another
    g.k_last = 0;
    g.n1 = sp.pieces - 1;
    if ((e = hdet_launch_bgemm(g, a_kmajor, false, HDET_EPI_SCALED_F32, batch * g.n1, s)) != hipSuccess) return e;
    g.a = g_in.a + g.n1 * a_step; g.b = g_in.b + g.n1 * b_step; g.c = partial + g.n1 * plane; g.k = rest; g.n1 = 1;
    if ((e = hdet_launch_bgemm(g, a_kmajor, false, HDET_EPI_SCALED_F32, batch, s)) != hipSuccess) return e;
  }
  const sum_args a = {partial, sp.pieces, g.m, g.n, pitch, out};
  const dim3 grid((unsigned)(((int64_t)g.m * (pitch >> 2) + 255) / 256), batch);
  if (out.dtype == HDET_TYPE_BF16) hipLaunchKernelGGL(hdet_split_sum_kernel<uint16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(hdet_split_sum_kernel<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
