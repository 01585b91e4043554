// Tiles and 32 x 32 blocks of the attention kernels: element types, LDS layout, matrix instructions.
//
// A tile is rows of D columns (a head, zeros behind its last column) of keys, values, queries or gradients, in LDS in chunks of 16 bytes; the
// chunks of row r are permuted by XOR with swz(r), so that the reads below touch disjoint banks: 16 bytes of each of 32 rows, and 4 rows x 32 bytes of
// the transposing read.  The first product of a block has the wavefront's own 32 rows as the accumulator's COLUMNS: a lane holds one of them and
// 16 entries of the other side, so that row reductions stay inside a lane and its partner lane + 32, and the accumulator, in bf16 or as it is, is the
// second product's operand: its rows are that product's contraction index.
#pragma once

#include "hdet_elem.h"
#include "hdet_lds.h"

namespace hdet_attend {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef int i4v __attribute__((ext_vector_type(4)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef short s8v __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// the largest of three numbers (NaN: of the others), without the compiler's quieting of each of them first
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ f16v all16(float x) {
  f16v z;
#pragma unroll
  for (int e = 0; e < 16; ++e) z[e] = x;
  return z;
}
// accumulator element e of lane l is row (e / 4) * 8 + (l / 32) * 4 + e % 4, column l % 32 of its 32 x 32 block
__device__ __forceinline__ int acc_row(int e, int lane) { return ((e >> 2) << 3) + ((lane >> 5) << 2) + (e & 3); }
// LDS of a wavefront's own: what its lanes have written is there for its other lanes
__device__ __forceinline__ void wave_fence() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Zeros for what is not finite among two bfloat16 numbers, or in a number
__device__ __forceinline__ unsigned finite_pair(unsigned x) {
  return ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
}
__device__ __forceinline__ unsigned finite_bits(unsigned x) { return (x & 0x7f800000u) == 0x7f800000u ? 0u : x; }

// (CLEAN: the second product takes zeros for what is not finite in the tile, which stays as it is for the first)
template <typename T, int D> struct shape;
// bf16: v_mfma_f32_32x32x16_bf16; the second product's other operand comes through the transposing LDS read
template <int D> struct shape<uint16_t, D> {
  typedef bf16x8 frag;
  static constexpr int E = 8, C = D / 8, NF = D / 16, ND = D / 32, TB = 64;
  static __device__ __forceinline__ int swz(int r) { return D == 64 ? ((r & 2) << 1) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3); }
  int k[NF], t[ND][2];                     // where a lane's fragments begin inside a tile (elements)
  __device__ __forceinline__ explicit shape(int lane) {
    const int row = lane & 31, p = lane & 15;
#pragma unroll
    for (int i = 0; i < NF; ++i) k[i] = row * D + (((2 * i + (lane >> 5)) ^ swz(row)) << 3);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int kr = ((lane >> 5) << 2) + (p >> 2) + 8 * u;
        t[dt][u] = kr * D + (((4 * dt + ((lane >> 4) & 1) * 2 + ((p & 3) >> 1)) ^ swz(kr)) << 3) + ((p & 1) << 2);
      }
  }
  // acc += (32 rows from `tile` on) (own rows)^T
  __device__ __forceinline__ f16v first(const uint16_t* tile, const frag (&own)[NF], f16v acc) const {
#pragma unroll
    for (int i = 0; i < NF; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const frag*>(tile + k[i]), own[i], acc, 0, 0, 0);
    return acc;
  }
  // the same with the own rows in LDS too
  __device__ __forceinline__ f16v first(const uint16_t* tile, const uint16_t* own, f16v acc) const {
#pragma unroll
    for (int i = 0; i < NF; ++i)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const frag*>(tile + k[i]), *reinterpret_cast<const frag*>(own + k[i]), acc, 0, 0, 0);
    return acc;
  }
  // a lane's 8 entries of column block dt of 16 rows
  template <bool CLEAN> __device__ __forceinline__ frag columns(const uint16_t* rows, int dt) const {
    const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4v __attribute__((address_space(3)))*)(rows + t[dt][0]));
    const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4v __attribute__((address_space(3)))*)(rows + t[dt][1]));
    const s8v both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    if (!CLEAN) return __builtin_bit_cast(frag, both);
    i4v words = __builtin_bit_cast(i4v, both);
#pragma unroll
    for (int i = 0; i < 4; ++i) words[i] = (int)finite_pair((unsigned)words[i]);
    __builtin_amdgcn_sched_barrier(0);     // one at a time: their temporaries would take the registers of the whole kernel
    return __builtin_bit_cast(frag, words);
  }
  // acc^T += (32 rows from `tile` on)^T x, x [row][own row] rounded to bf16
  template <bool CLEAN = false> __device__ __forceinline__ void second(const uint16_t* tile, const f16v& x, f16v (&acc)[ND]) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      frag f;
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = (__bf16)x[8 * j + i];
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(columns<CLEAN>(tile + 16 * j * D, dt), f, acc[dt], 0, 0, 0);
    }
  }
  // the same with x in two parts, 16 bits of it
  template <bool CLEAN = false> __device__ __forceinline__ void second_in_two(const uint16_t* tile, const f16v& x, f16v (&acc)[ND]) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      frag f, rest;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f[i] = (__bf16)x[8 * j + i];
        rest[i] = (__bf16)(x[8 * j + i] - (float)f[i]);
      }
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        const frag a = columns<CLEAN>(tile + 16 * j * D, dt);
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, f, acc[dt], 0, 0, 0);
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, rest, acc[dt], 0, 0, 0);
      }
    }
  }
  static __device__ __forceinline__ f16v product(const frag& a, const frag& b, const f16v& acc) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0); }
};
// fp32: v_mfma_f32_32x32x2_f32; a fragment is 4 columns, and step i of them contracts column i of both half-wavefronts' chunks
template <int D> struct shape<float, D> {
  typedef f4v frag;
  static constexpr int E = 4, C = D / 4, NF = D / 8, ND = D / 32, TB = 32;
  static __device__ __forceinline__ int swz(int r) { return r & 7; }
  int k[NF], t[ND][4];
  __device__ __forceinline__ explicit shape(int lane) {
    const int row = lane & 31;
#pragma unroll
    for (int i = 0; i < NF; ++i) k[i] = row * D + (((2 * i + (lane >> 5)) ^ swz(row)) << 2);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int r = ((lane >> 5) << 2) + u;
        t[dt][u] = r * D + (((8 * dt + (row >> 2)) ^ swz(r)) << 2) + (row & 3);
      }
  }
  __device__ __forceinline__ f16v first(const float* tile, const frag (&own)[NF], f16v acc) const {
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const frag a = *reinterpret_cast<const frag*>(tile + k[i]);
#pragma unroll
      for (int u = 0; u < 4; ++u) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[u], own[i][u], acc, 0, 0, 0);
    }
    return acc;
  }
  template <bool CLEAN = false> __device__ __forceinline__ void second(const float* tile, const f16v& x, f16v (&acc)[ND]) const {
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        float a = tile[(e >> 2) * 8 * D + t[dt][e & 3]];
        if (CLEAN) a = __uint_as_float(finite_bits(__float_as_uint(a)));
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, x[e], acc[dt], 0, 0, 0);
      }
  }
  template <bool CLEAN = false> __device__ __forceinline__ void second_in_two(const float* tile, const f16v& x, f16v (&acc)[ND]) const { second<CLEAN>(tile, x, acc); }
  static __device__ __forceinline__ f16v product(const frag& a, const frag& b, f16v acc) {
#pragma unroll
    for (int u = 0; u < 4; ++u) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[u], b[u], acc, 0, 0, 0);
    return acc;
  }
};

// Whether any of x, times a power of 2, is not finite
template <int N> __device__ __forceinline__ bool not_finite(const f16v (&x)[N], float times = 1.f) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) s = __builtin_fmaf(x[i][e] * times, 0.f, s);
  return s != 0.f;
}

// a descriptor in scalar registers (every lane has the same; the compiler does not always see it)
__device__ __forceinline__ hdet_rsrc scalar_rsrc(const void* p, uint32_t bytes) {
  hdet_rsrc r = make_rsrc(p, bytes);
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
  return r;
}
__device__ __forceinline__ bool finite_of(float x) { return fabsf(x) < INFINITY; }
// Weight of a pair of rows whose results are not finite: 0 where its score is minus infinity, otherwise more (1 will do)
template <typename T> __device__ __forceinline__ float pair_weight(const T* q, const T* k, int d, float scale, bool capped, int lane) {
  if (capped) return 1.f;
  float s = 0.f;
  for (int c = lane; c < d; c += 64) s = __builtin_fmaf(hdet_ld(q + c), hdet_ld(k + c), s);
  return hdet_wave_sum(s) * scale == -INFINITY ? 0.f : 1.f;
}
// What is not finite in rows from .. to - 1 of src, times weight(row, own row), is added to the rows of dst that attend them (seen(row, own row)): a
// wavefront's `have` rows
template <typename T, int D, typename U, typename F, typename G>
__device__ __forceinline__ void add_not_finite(const T* src, int64_t ld, int d, int from, int to, U* dst, int64_t dst_ld, int have, int lane, F seen, G weight) {
  typedef shape<T, D> S;
  constexpr int ROWS = 64 / S::C;
  for (int j = from; j < to; j += ROWS) {
    const int row = j + lane / S::C, col = lane % S::C * S::E;
    bool bad = false;
    if (row < to)
      for (int e = 0; e < S::E; ++e) bad = bad || (col + e < d && !finite_of(hdet_ld(src + row * ld + col + e)));
    const unsigned long long mask = __ballot(bad);
    if (!mask) continue;
    for (int i = 0; i < ROWS; ++i) {
      if (!(mask >> (i * S::C) & (S::C == 64 ? ~0ull : (1ull << (S::C & 63)) - 1))) continue;
      float x[D / 64];
      bool infinite = false;               // (a NaN has no weight)
#pragma unroll
      for (int u = 0; u < D / 64; ++u) {
        x[u] = lane + 64 * u < d ? hdet_ld(src + (j + i) * ld + lane + 64 * u) : 0.f;
        infinite = infinite || fabsf(x[u]) == INFINITY;
      }
      const bool weighted = __any(infinite);
      for (int own = 0; own < have; ++own) {
        if (!seen(j + i, own)) continue;
        const float w = weighted ? weight(j + i, own) : 1.f;
#pragma unroll
        for (int u = 0; u < D / 64; ++u)
          if (!finite_of(x[u])) {
            U* const to = dst + own * dst_ld + lane + 64 * u;
            hdet_st(to, hdet_ld(to) + x[u] * w);
          }
      }
    }
  }
}

// 16 bytes of a row of d elements from column col on, zeros behind the last, wherever the row lies: a load from within the row, moved into place (32
// sequences of 512, 4 heads of 50: forward 26 us, backward 79; element by element 46, 125)
typedef f4v f4v_any __attribute__((aligned(2)));
template <typename T> __device__ __forceinline__ f4v piece_of(const T* row, int col, int d) {
  constexpr int E = 16 / sizeof(T);
  f4v v = {0.f, 0.f, 0.f, 0.f};
  if (d >= E) {
    const int from = col + E <= d ? col : d - E;
    v = *reinterpret_cast<const f4v_any*>(row + from);
    if (from < col) {
      unsigned __int128 w;
      __builtin_memcpy(&w, &v, 16);
      w >>= (unsigned)((col - from) * (int)sizeof(T) * 8);
      __builtin_memcpy(&v, &w, 16);
    }
  } else {
    T x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = col + e < d ? row[col + e] : T(0);
    __builtin_memcpy(&v, x, 16);
  }
  return v;
}

// Tiles of ROWS rows of a matrix (row pitch ld, d columns) into LDS, by NW wavefronts.  WHOLE: 16-byte pieces straight from memory to LDS; else through
// registers.
template <typename T, int D, int ROWS, int NW, bool WHOLE> struct tile_loader {
  typedef shape<T, D> S;
  static constexpr int NI = ROWS * S::C / (64 * NW);       // pieces a lane
  static constexpr int STEP = 64 * NW / S::C;              // rows between them
  static constexpr bool EVEN = STEP % (sizeof(T) == 2 ? 16 : 8) == 0;      // swz does not see the step
  static constexpr int BYTES = ROWS * D * sizeof(T);
  const T* src;
  int64_t ld;
  int d, wave, lane;
  uint32_t off[EVEN ? 1 : NI];
  __device__ __forceinline__ tile_loader(const T* src_, int64_t ld_, int d_, int wave_, int lane_) : src(src_), ld(ld_), d(d_), wave(wave_), lane(lane_) {
#pragma unroll
    for (int u = 0; u < (EVEN ? 1 : NI); ++u) {
      const int id = (u * NW + wave) * 64 + lane, row = id / S::C, chunk = (id % S::C) ^ S::swz(row);
      // columns that there are not: an offset beyond any extent
      off[u] = chunk * S::E < d ? (uint32_t)((row * ld + chunk * S::E) * (int)sizeof(T)) : 0x80000000u;
    }
  }
  // rows row0 .. row0 + have - 1 (have <= 0: none), zeros behind them, to the LDS tile `at`
  __device__ __forceinline__ void load(int64_t row0, int have, T* at) const {
    if (have > ROWS) have = ROWS;
    if (WHOLE) {
      const hdet_rsrc rs = scalar_rsrc(src + (have > 0 ? row0 * ld : 0), have > 0 ? (uint32_t)(((have - 1) * ld + d) * (int)sizeof(T)) : 0u);
      const uint32_t to = __builtin_amdgcn_readfirstlane(lds_addr_of((const uint16_t*)at));
#pragma unroll
      for (int u = 0; u < NI; ++u)
        lds_load16(rs, to + (u * NW + wave) * 1024, EVEN ? off[0] + (uint32_t)(u * STEP * ld * (int)sizeof(T)) : off[EVEN ? 0 : u]);
    } else {
#pragma unroll 2
      for (int u = 0; u < NI; ++u) {
        const int id = (u * NW + wave) * 64 + lane, row = id / S::C, col = ((id % S::C) ^ S::swz(row)) * S::E;
        f4v v = {0.f, 0.f, 0.f, 0.f};
        if (row < have && col < d) v = piece_of(src + (row0 + row) * ld, col, d);
        *reinterpret_cast<f4v*>(at + id * S::E) = v;
      }
    }
  }
};

// Element (l % 32, l % 32) of an accumulator block
__device__ __forceinline__ float diagonal(const f16v& x, int lane) {
  float r = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) r = acc_row(e, lane) == (lane & 31) ? x[e] : r;
  const float o = other_half(r);
  return (lane >> 2 & 1) == lane >> 5 ? r : o;
}

// A lane's fragment i of its own row at p (null: zeros)
template <typename T, int D, bool WHOLE> __device__ __forceinline__ typename shape<T, D>::frag own_frag(const T* p, int i, int d, int lane) {
  typedef shape<T, D> S;
  const int col = (2 * i + (lane >> 5)) * S::E;
  typename S::frag f = {};
  if (WHOLE) {
    if (p && col < d) f = *reinterpret_cast<const typename S::frag*>(p + col);
  } else if (p && col < d) {
    const f4v v = piece_of(p, col, d);
    __builtin_memcpy(&f, &v, 16);
  }
  return f;
}

// A wavefront's results, [column][own row] in accumulators, to rows of dst (row pitch ld), the first `have` of 32 and d columns, through the
// wavefront's strip in LDS so that a store writes 16 bytes of a row
constexpr int STRIP = 32 * 36 * 4;         // bytes
template <typename T, int D, bool WHOLE>
__device__ __forceinline__ void store_rows(const f16v (&o)[D / 32], void* strip_, T* dst, int64_t ld, int have, int d, int lane, bool add = false) {
  typedef shape<T, D> S;
  constexpr int P = sizeof(T) == 2 ? 40 : 36, PER = 32 / S::E;
  T* const strip = (T*)strip_;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) {
    if (32 * dt >= d) break;
    wave_fence();
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4)
      hdet_st4(strip + (lane & 31) * P + acc_row(4 * e4, lane), hdet_f4{{o[dt][4 * e4], o[dt][4 * e4 + 1], o[dt][4 * e4 + 2], o[dt][4 * e4 + 3]}});
    wave_fence();
#pragma unroll
    for (int i = 0; i < PER / 2; ++i) {
      const int c = lane + 64 * i, row = c / PER, col = c % PER * S::E;
      if (row >= have) continue;
      T* const to = dst + row * ld + 32 * dt + col;
      if (WHOLE) {
        if (32 * dt + col >= d) continue;
        f4v x = *reinterpret_cast<const f4v*>(strip + row * P + col);
        if (sizeof(T) == 4 && add) x += *reinterpret_cast<const f4v*>(to);
        *reinterpret_cast<f4v*>(to) = x;
      } else if (!(sizeof(T) == 4 && add) && 32 * dt + col + S::E <= d) {
        *reinterpret_cast<f4v_any*>(to) = *reinterpret_cast<const f4v*>(strip + row * P + col);
      } else {
#pragma unroll
        for (int e = 0; e < S::E; ++e)
          if (32 * dt + col + e < d) to[e] = sizeof(T) == 4 && add ? (T)(to[e] + strip[row * P + col + e]) : strip[row * P + col + e];
      }
    }
  }
  wave_fence();
}

// tanh x - 1 = -2 / (e^2x + 1) on the hardware's exponential and reciprocal, off by 1.2e-7
__device__ __forceinline__ float tanh_less_1(float x2log2e) { return __builtin_amdgcn_rcpf(__builtin_fmaf(exp2_fast(x2log2e), -0.5f, -0.5f)); }
// tanh x to 1e-7 of itself: the same, and below 0.3, where it cancels, its series up to x^9
__device__ __forceinline__ float tanh_close(float x) {
  const float x2 = x * x;
  const float series = __builtin_fmaf(x * x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, 2.1869489e-2f, -5.3968254e-2f), 0.13333334f), -0.33333334f), x);
  return x2 < 0.09f ? series : 1.f + tanh_less_1(x * (2.f * kLog2e));
}

}  // namespace hdet_attend
