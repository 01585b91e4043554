// Product of two matrices in 8 bits, N replicas:  y = s_m t_o sum_k q[m][k] w[o][k] + b_o,  on v_mfma_i32_16x16x64_i8.  The sums of code
// products are whole numbers below 2^31 and exact; both scales and the bias come in as fp32 where a sum is complete.
//
//  * Tiles (hdet_codes_gemm_kernel): both operands are contiguous along k and their rows start at 16-byte boundaries, with zeros behind the
//    last column up to the next one, so every shape is made of whole 16-byte chunks.  Chunks go from global memory straight into LDS, a K
//    step of 128 bytes a row, NST steps in flight; a row's chunks are permuted by row / 2 so that the 128-bit fragment reads are free of
//    bank conflicts.  Rows past the matrix and chunks past k lie outside the buffer descriptor and arrive as zeros: no edge cases in the
//    loop.
//  * Few rows (hdet_codes_rows_kernel): the weights' stream is all there is; see there.

#include "hdet_ops.h"
#include "hdet_elem.h"
#include "hdet_lds.h"
#include "hdet_tiles.h"

namespace {

typedef int i4v __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned short us4 __attribute__((ext_vector_type(4)));

struct codes_args {
  const int8_t *x, *w;
  const float *x_scale, *w_scale, *bias;
  void* y;
  int64_t x_z, w_z, bias_z, y_z, x_ld, w_ld, y_ld;
  int m, n, kbytes;          // kbytes: k rounded up to whole chunks
};

// extent of the rows from `row0` on, as a descriptor takes it (offsets inside a tile stay below 2^31)
__device__ __forceinline__ uint32_t extent(int rows, int row0, int64_t ld, int kbytes) {
  const int64_t e = (int64_t)(rows - row0 - 1) * ld + kbytes;
  return e > 0x7fffffff ? 0x7fffffffu : (uint32_t)e;
}
__device__ __forceinline__ int swz(int r) { return (r >> 1) & 7; }

// Four consecutive results of one row, at any element
typedef f4 f4_any __attribute__((aligned(4)));
typedef hdet_u2v hdet_u2v_any __attribute__((aligned(2)));
template <typename OUT>
__device__ __forceinline__ void put4(OUT* y, int col, int n, f4 v) {
  if (col + 4 <= n) {
    if constexpr (sizeof(OUT) == 4) *reinterpret_cast<f4_any*>(y + col) = v;
    else *reinterpret_cast<hdet_u2v_any*>(y + col) = hdet_u2v{hdet_bf16_pack(v[0], v[1]), hdet_bf16_pack(v[2], v[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < n) hdet_st(y + col + e, v[e]);
  }
}

}  // namespace

template <typename OUT, int TM, int TN, int WGM, int WGN, int NST>
__global__ __launch_bounds__(64 * WGM * WGN, 160 * 1024 / (NST * (TM + TN) * 128) * (WGM * WGN / 4))
void hdet_codes_gemm_kernel(const codes_args g) {
  constexpr int THREADS = 64 * WGM * WGN, MB = TM / WGM / 16, NB = TN / WGN / 16;
  constexpr int STAGE = (TM + TN) * 128, NA = TM * 128 / (THREADS * 16), NBL = TN * 128 / (THREADS * 16), LPT = NA + NBL;
  __shared__ __attribute__((aligned(1024))) uint16_t S[NST * STAGE / 2];
  const int z = blockIdx.z, m0 = blockIdx.y * TM, n0 = blockIdx.x * TN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (wave / WGN) * (TM / WGM), wn = (wave % WGN) * (TN / WGN);
  const hdet_rsrc ra = make_rsrc(g.x + z * g.x_z + (int64_t)m0 * g.x_ld, extent(g.m, m0, g.x_ld, g.kbytes));
  const hdet_rsrc rb = make_rsrc(g.w + z * g.w_z + (int64_t)n0 * g.w_ld, extent(g.n, n0, g.w_ld, g.kbytes));
  const uint32_t s_addr = lds_addr_of(S);
  // chunk slot c = tid + i THREADS of a tile: row c / 8, chunk (c mod 8) ^ swz(row); THREADS / 8 rows apart the permutation is the same
  const int ck = ((tid & 7) ^ swz(tid >> 3)) * 16;
  const uint32_t off_a = (uint32_t)((tid >> 3) * g.x_ld + ck), off_b = (uint32_t)((tid >> 3) * g.w_ld + ck);
  auto issue = [&](int i, int s, int kt) {
    const bool ok = ck + kt * 128 < g.kbytes;
    if (i < NA) lds_load16(ra, s_addr + s * STAGE + (i * THREADS + wave * 64) * 16, ok ? off_a + (uint32_t)(kt * 128 + i * (THREADS / 8) * g.x_ld) : kAbsent);
    else lds_load16(rb, s_addr + s * STAGE + TM * 128 + ((i - NA) * THREADS + wave * 64) * 16, ok ? off_b + (uint32_t)(kt * 128 + (i - NA) * (THREADS / 8) * g.w_ld) : kAbsent);
  };
  static_assert(THREADS / 8 % 16 == 0, "the chunk permutation repeats every 16 rows");
  i4v acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = i4v{0, 0, 0, 0};
  const int nk = (g.kbytes + 127) / 128;
#pragma unroll
  for (int s = 0; s < NST; ++s)
#pragma unroll
    for (int i = 0; i < LPT; ++i) issue(i, s, s);
  wait_and_barrier<(NST - 1) * LPT>();
  const int8_t* const base = reinterpret_cast<const int8_t*>(S);
  i4v fa[2][MB], fb[2][NB];
  auto read_frag = [&](int set, int s, int ss, int idx) {
    const int r = lane & 15, ch = ((ss * 4 + (lane >> 4)) ^ swz(r)) * 16;
    if (idx < NB) fb[set][idx] = *reinterpret_cast<const i4v*>(base + s * STAGE + TM * 128 + (wn + idx * 16 + r) * 128 + ch);
    else if (idx < NB + MB) fa[set][idx - NB] = *reinterpret_cast<const i4v*>(base + s * STAGE + (wm + (idx - NB) * 16 + r) * 128 + ch);
  };
  constexpr int NM = MB * NB, NR = MB + NB, IPA = (NR + NM - 1) / NM, IPB = (NR + LPT + NM - 1) / NM;
  auto multiply = [&](int set, int q) { acc[q / NB][q % NB] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[set][q % NB], fa[set][q / NB], acc[q / NB][q % NB], 0, 0, 0); };
#pragma unroll
  for (int idx = 0; idx < NR; ++idx) read_frag(0, 0, 0, idx);
  for (int kt0 = 0; kt0 < nk; kt0 += NST) {
#pragma unroll
    for (int s = 0; s < NST; ++s) {
      const int kt = kt0 + s;
      if (kt >= nk) break;
#pragma unroll
      for (int q = 0; q < NM; ++q) {
        multiply(0, q);
#pragma unroll
        for (int u = 0; u < IPA; ++u) read_frag(1, s, 1, q * IPA + u);
        __builtin_amdgcn_sched_barrier(0);
      }
      // every wavefront has read all of this stage; the next one has landed
      wait_and_barrier<(NST - 2) * LPT>();
#pragma unroll
      for (int q = 0; q < NM; ++q) {
        multiply(1, q);
#pragma unroll
        for (int u = 0; u < IPB; ++u) {
          const int it = q * IPB + u;
          if (it < LPT) issue(it, s, kt + NST);
          else read_frag(0, (s + 1) % NST, 0, it - LPT);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  wait_and_barrier<0>();           // loads past the end have drained before the block gives its LDS up
  // accumulator element e of lane l: row l mod 16, column 4 (l / 16) + e of its block
  float sx[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int row = m0 + wm + i * 16 + (lane & 15);
    sx[i] = row < g.m ? g.x_scale[(int64_t)z * g.m + row] : 0.f;
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int col = n0 + wn + j * 16 + (lane >> 4) * 4;
    f4 sw, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool ok = col + e < g.n;
      sw[e] = ok ? g.w_scale[(int64_t)z * g.n + col + e] : 0.f;
      b[e] = ok && g.bias ? g.bias[z * g.bias_z + col + e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      const int row = m0 + wm + i * 16 + (lane & 15);
      f4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf((float)acc[i][j][e], sx[i] * sw[e], b[e]);
      if (row < g.m) put4<OUT>((OUT*)g.y + z * g.y_z + (int64_t)row * g.y_ld, col, g.n, v);
    }
  }
}

// Large products: blocks that walk over tiles of 256 x 256, so that a tile's end -- y is written there, as many bytes as the products of a
// K of 500 take to form -- lies under the next tile's loads.
//  * Eight wavefronts of 128 x 64 in two groups of four, one of each on every SIMD: while one group multiplies (32 instructions, 512
//    cycles), the other reads its next fragments and requests a later K step; the block's barriers hand the matrix cores over.  A K step of
//    128 bytes is two such turns: rows 0-63 of the wavefront, then rows 64-127 with the column fragments still in registers.  Two stages of
//    64 KiB; each turn waits for all but the newest eight of its loads.
//  * The next tile's first two K steps are requested in the last two of the tile before; its scales and bias come into LDS a tile ahead.
//  * Results leave from the registers.  Stores are always issued -- what does not exist lies outside the descriptor.  The next tile's first
//    two K steps are requested before them, and its first three turns wait for those loads, not for the stores.
//  * Rows and columns past the matrices are zeros in the loop, and their results are not stored.
// 8192^3 402 us = 2.7 POP/s, 8 x 8192 rows 1024 -> 4096 336 us = 1.6, 8 x 4096 rows 512 -> 2048 48 us = 1.4 (3.3 TB/s): what a tile stores
// bounds the short contractions.  Of those 336 us 71 go without the stores and 95 without the tile's end altogether.
template <typename OUT>
__global__ __launch_bounds__(512, 2) void hdet_codes_walk_kernel(const codes_args g, unsigned gx, unsigned gy, unsigned total, int tile_group) {
  constexpr int TM = 256, TN = 256, HALF = 128 * 128;             // bytes of half an operand tile
  constexpr int kStores = sizeof(OUT) == 4 ? 32 : 16;
  constexpr int kSideAt = 8 * HALF;                               // bias, column scales, row scales: [2][3][256]
  __shared__ __attribute__((aligned(1024))) uint16_t S[(8 * HALF + 2 * 3 * 256 * 4) / 2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = (wave % 4) * 64, hr = (wave / 4) * 64, wm = (wave / 4) * 128;
  // the lane's number outside the K loop, computed where it is used: kept over the tiles it would spill
  auto lane_now = [] {
    int x;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
    return x;
  };
  const uint32_t s_addr = lds_addr_of(S);
  const int8_t* const base = reinterpret_cast<const int8_t*>(S);
  const float* const side = reinterpret_cast<const float*>(base + kSideAt);
  // A fragment is rows order(i) + row_in(0 .. 15) of the wavefront's 64, so a lane of group cg = lane / 16 accumulates columns order(j) +
  // cg * kGroup + (0 .. 3), j = 0 .. 3, of y.  For bfloat16 results the order gives it 8 neighbours twice, so that one store of 16 bytes a
  // lane covers 64 bytes of each row; four fp32 results are 16 bytes as they are.
  constexpr bool kPlain = sizeof(OUT) == 4;
  constexpr int kGroup = kPlain ? 4 : 8;
  auto order = [](int j) { return kPlain ? j * 16 : (j >> 1) * 32 + (j & 1) * 4; };
  auto row_in = [](int r) { return kPlain ? r : ((r & 12) << 1) + (r & 3); };
  // the chunk permutation: by the bits in which a fragment's rows differ, but the lowest
  auto perm = [](int r) { return kPlain ? swz(r) : ((r >> 2) & 6) | ((r >> 1) & 1); };
  int nk = ((g.kbytes + 127) / 128 + 1) & ~1;                     // K steps of a tile, an even number from 4 on (steps beyond k are zeros)
  nk = nk < 4 ? 4 : nk;

  struct tile { int m0, n0, z; hdet_rsrc ra, rb; bool ok; };
  auto tile_at = [&](unsigned t) {
    tile r;
    const tile_id id = tile_of_index(t < total ? t : total - 1, gx, gy, total, tile_group);
    r.m0 = id.by * TM; r.n0 = id.bx * TN; r.z = id.bz;
    r.ok = t < total;
    r.ra = make_rsrc(g.x + r.z * g.x_z + (int64_t)r.m0 * g.x_ld, r.ok ? extent(g.m, r.m0, g.x_ld, g.kbytes) : 0u);
    r.rb = make_rsrc(g.w + r.z * g.w_z + (int64_t)r.n0 * g.w_ld, r.ok ? extent(g.n, r.n0, g.w_ld, g.kbytes) : 0u);
    return r;
  };
  const int ck = ((tid & 7) ^ perm(tid >> 3)) * 16;
  uint32_t off_a = (uint32_t)((tid >> 3) * g.x_ld + ck), off_b = (uint32_t)((tid >> 3) * g.w_ld + ck);
  // LDS, in units of 128 rows x 128 bytes: half h of A of stage s at 2 h + s (its rows 64 .. 127 are the tile's 128 .. 191 of that half), B
  // at 4 + 2 s
  auto load_a = [&](const hdet_rsrc& r, int h, int s, int kt) {
    const uint32_t at = s_addr + (2 * h + s) * HALF;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      lds_load16(r, at + (i * 512 + wave * 64) * 16, ck + kt * 128 < g.kbytes ? off_a + (uint32_t)(kt * 128 + (64 * h + 128 * i) * g.x_ld) : kAbsent);
  };
  auto load_b = [&](const hdet_rsrc& r, int s, int kt) {
    const uint32_t at = s_addr + (4 + 2 * s) * HALF;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      lds_load16(r, at + (i * 512 + wave * 64) * 16, ck + kt * 128 < g.kbytes ? off_b + (uint32_t)(kt * 128 + 64 * i * g.w_ld) : kAbsent);
  };
  auto load_side = [&](const tile& t, int slot) {
    const int ln = lane_now();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int q = wave + 8 * u, at = (q & 3) * 64 + ln;
      if (q < 12) {
        const float* src = q < 4 ? (g.bias ? g.bias + t.z * g.bias_z + t.n0 : nullptr) : q < 8 ? g.w_scale + (int64_t)t.z * g.n + t.n0 : g.x_scale + (int64_t)t.z * g.m + t.m0;
        const int count = q < 8 ? g.n - t.n0 : g.m - t.m0;
        lds_load4(make_rsrc(src, t.ok && src ? (uint32_t)count * 4u : 0u), s_addr + kSideAt + (slot * 3 * 256 + q * 64) * 4, (uint32_t)at * 4u);
      }
    }
  };
  i4v acc[8][4];
  i4v fa[2][4], fb[2][4];
  // fragment i of sub-step ss is order(i) rows behind fragment 0, whose chunk permutation it shares: two addresses an operand
  const int8_t *pa[2], *pb[2];
#pragma unroll
  for (int ss = 0; ss < 2; ++ss) {
    const int r = row_in(lane & 15), at = r * 128 + (((ss * 4 + (lane >> 4)) ^ perm(r)) << 4);
    pa[ss] = base + hr * 128 + at;
    pb[ss] = base + 4 * HALF + wn * 128 + at;
  }
  auto read_a = [&](int h, int s) {
#pragma unroll
    for (int ss = 0; ss < 2; ++ss)
#pragma unroll
      for (int i = 0; i < 4; ++i) fa[ss][i] = *reinterpret_cast<const i4v*>(pa[ss] + (2 * h + s) * HALF + order(i) * 128);
  };
  auto read_b = [&](int s) {
#pragma unroll
    for (int ss = 0; ss < 2; ++ss)
#pragma unroll
      for (int j = 0; j < 4; ++j) fb[ss][j] = *reinterpret_cast<const i4v*>(pb[ss] + 2 * s * HALF + order(j) * 128);
  };
  auto multiply = [&](int h, bool first) {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int ss = 0; ss < 2; ++ss)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[4 * h + i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[ss][j], fa[ss][i], first && ss == 0 ? i4v{0, 0, 0, 0} : acc[4 * h + i][j], 0, 0, 0);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto meet = [] {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto finish = [&](const tile& t, int slot) {
    __builtin_amdgcn_sched_barrier(0);
    const int ln = lane_now(), cg = ln >> 4, lr = row_in(ln & 15);
    const float* sd = side + slot * 3 * 256;
    f4 bias[4], sw[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bias[j] = *reinterpret_cast<const f4*>(sd + wn + order(j) + cg * kGroup);
      sw[j] = *reinterpret_cast<const f4*>(sd + 256 + wn + order(j) + cg * kGroup);
    }
    const auto rc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<OUT*>(g.y) + t.z * g.y_z + (int64_t)t.m0 * g.y_ld + t.n0, 0, 0x7fffffff, 0x00020000);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int tr = wm + (i >> 2) * 64 + order(i & 3) + lr;
      const bool row_ok = t.m0 + tr < g.m;
      const float sx = sd[512 + tr];
      f4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[j][e] = __builtin_fmaf((float)acc[i][j][e], sx * sw[j][e], bias[j][e]);
      if constexpr (sizeof(OUT) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int col = wn + j * 16 + cg * 4;
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(hdet_u4v, v[j]), rc, row_ok && t.n0 + col < g.n ? (uint32_t)((tr * (int)g.y_ld + col) * 4) : kAbsent, 0, 0);
        }
      } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int col = wn + u * 32 + cg * 8;
          const hdet_u4v o = {hdet_bf16_pack(v[2 * u][0], v[2 * u][1]), hdet_bf16_pack(v[2 * u][2], v[2 * u][3]),
                              hdet_bf16_pack(v[2 * u + 1][0], v[2 * u + 1][1]), hdet_bf16_pack(v[2 * u + 1][2], v[2 * u + 1][3])};
          __builtin_amdgcn_raw_buffer_store_b128(o, rc, row_ok && t.n0 + col < g.n ? (uint32_t)((tr * (int)g.y_ld + col) * 2) : kAbsent, 0, 0);
        }
      }
    }
  };

  unsigned t = blockIdx.x;
  tile cur = tile_at(t);
  int slot = 0;
  load_side(cur, 0);
  load_a(cur.ra, 0, 0, 0); load_b(cur.rb, 0, 0); load_a(cur.ra, 1, 0, 0);
  load_a(cur.ra, 0, 1, 1); load_b(cur.rb, 1, 1); load_a(cur.ra, 1, 1, 1);
  wait_and_barrier<8>();
  if (wave >= 4) meet();
  for (bool begun = false;; begun = true) {
    tile nxt;
    asm volatile("" : "+v"(off_a), "+v"(off_b));
    auto pair = [&](int kt0, bool first) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int kt = kt0 + s;
        const bool fs = first && s == 0;
        // all but the newest eight loads; in a tile's first three turns those are older than the stores of the tile before, which need not
        // be done
        auto wait = [&](bool early) {
          if (early && begun) wait_and_barrier<8 + kStores>();
          else wait_and_barrier<8>();
        };
        read_a(0, s);
        read_b(s);
        if (!fs) {                                               // (the first step's has been requested before the stores)
          if (first || kt + 1 < nk) load_a(cur.ra, 1, s ^ 1, kt + 1); else load_a(nxt.ra, 1, s ^ 1, 0);
        }
        wait(first);
        multiply(0, fs);
        meet();
        read_a(1, s);
        if (first || kt + 2 < nk) { load_a(cur.ra, 0, s, kt + 2); load_b(cur.rb, s, kt + 2); }
        else { load_a(nxt.ra, 0, s, kt + 2 - nk); load_b(nxt.rb, s, kt + 2 - nk); }
        if (first && s == 0) {
          t += gridDim.x;
          nxt = tile_at(t);
        }
        if (first && s == 1) load_side(nxt, slot ^ 1);
        wait(fs);
        multiply(1, fs);
        if (s == 0) meet();
      }
    };
    pair(0, true);
    for (int kt0 = 2; kt0 < nk; kt0 += 2) { meet(); pair(kt0, false); }
    // the first group ends its tile under the second's last products, the second at once
    if (wave < 4) meet();
    load_a(nxt.ra, 1, 1, 1);       // both groups have read what it goes over
    finish(cur, slot);
    if (wave >= 4) meet();
    if (t >= total) break;
    cur = nxt;
    slot ^= 1;
  }
  if (wave < 4) meet();
  wait_and_barrier<0>();
}

// Up to 16 rows.  The weights' stream is the work: a block takes 16 columns of y, its four wavefronts a quarter of k each, with fragments
// straight from global memory (16 rows of the weights, 64 bytes of each, an instruction) and no barrier in the loop; whole-number partial
// sums are added through LDS.  8 x 16 rows, 1024 -> 4096: 10.5 us, the weights at 3.2 TB/s; 8 x 1 row, 512 -> 2048: 4.0 us, a launch and
// its chain.
template <typename OUT>
__global__ __launch_bounds__(256) void hdet_codes_rows_kernel(const codes_args g) {
  __shared__ i4v part[4][64];
  const int z = blockIdx.z, n0 = blockIdx.x * 16, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(g.x + z * g.x_z), 0, (int)extent(g.m, 0, g.x_ld, g.kbytes), 0x00020000);
  const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(g.w + z * g.w_z + (int64_t)n0 * g.w_ld), 0, (int)extent(g.n, n0, g.w_ld, g.kbytes), 0x00020000);
  const int nk = (g.kbytes + 63) / 64, k0 = wave * nk / 4, k1 = (wave + 1) * nk / 4;
  const int r = lane & 15, kc = (lane >> 4) * 16;
  const int col = n0 + (lane >> 4) * 4;
  // what the end needs is requested before the loop
  float sx = 0.f;
  f4 sw = {0.f, 0.f, 0.f, 0.f}, b = {0.f, 0.f, 0.f, 0.f};
  if (wave == 0) {
    if (r < g.m) sx = g.x_scale[(int64_t)z * g.m + r];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < g.n) {
        sw[e] = g.w_scale[(int64_t)z * g.n + col + e];
        if (g.bias) b[e] = g.bias[z * g.bias_z + col + e];
      }
  }
  i4v acc = {0, 0, 0, 0};
#pragma unroll 8
  for (int k = k0; k < k1; ++k) {
    const int at = k * 64 + kc;
    const bool ok = at < g.kbytes;
    const i4v w = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(rb, ok ? (int)(r * g.w_ld) + at : (int)kAbsent, 0, 0));
    const i4v x = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(ra, ok ? (int)(r * g.x_ld) + at : (int)kAbsent, 0, 0));
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc, 0, 0, 0);
  }
  if (wave != 0) part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0 || r >= g.m) return;
  acc += part[1][lane] + part[2][lane] + part[3][lane];
  f4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf((float)acc[e], sx * sw[e], b[e]);
  put4<OUT>((OUT*)g.y + z * g.y_z + (int64_t)r * g.y_ld, col, g.n, v);
}

namespace {

template <typename OUT>
hipError_t launch_typed(const codes_args& g, int n_replicas, hipStream_t s) {
  const int size = sizeof(OUT);
  // Up to 16 rows; beyond, the tiles' shorter chain counts for more than their empty rows (8 x 64 rows, 1024 -> 4096: 24 us in blocks of 16
  // columns, 13 in tiles)
  if (g.m <= 16) {
    hipLaunchKernelGGL(hdet_codes_rows_kernel<OUT>, dim3((g.n + 15) / 16, 1, n_replicas), dim3(256), 0, s, g);
    return hipGetLastError();
  }
  const bool v8 = (reinterpret_cast<uintptr_t>(g.y) & 15) == 0 && ((g.n | g.y_ld | g.y_z) & (size == 2 ? 7 : 3)) == 0;
  if (v8 && g.y_ld < (1 << 20)) {
    const unsigned gx = (g.n + 255) / 256, gy = (g.m + 255) / 256, total = gx * gy * (unsigned)n_replicas, cus = (unsigned)hdet_compute_units();
    if (total >= cus) {
      hipLaunchKernelGGL(hdet_codes_walk_kernel<OUT>, dim3(total < cus ? total : cus), dim3(512), 0, s, g, gx, gy, total, tile_group_of(gx));
      return hipGetLastError();
    }
  }
  const dim3 grid((g.n + 127) / 128, (g.m + 127) / 128, n_replicas);
  hipLaunchKernelGGL((hdet_codes_gemm_kernel<OUT, 128, 128, 2, 2, 2>), grid, dim3(256), 0, s, g);
  return hipGetLastError();
}

}  // namespace

hipError_t hdet_launch_codes_gemm(const hdet_linear_args& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const codes_args g = {(const int8_t*)a.codes.dev, (const int8_t*)a.w_codes.dev, a.scale_dev, a.w_scale_dev, a.bias_dev, a.y.dev,
                        a.codes.replica_stride, a.w_codes.replica_stride, a.bias_stride, a.y.replica_stride,
                        a.codes.row_stride, a.w_codes.row_stride, a.y.row_stride, (int)a.rows, a.d_out, (a.d_in + 15) & ~15};
  return a.y_dtype == HDET_TYPE_BF16 ? launch_typed<uint16_t>(g, a.n_replicas, s) : launch_typed<float>(g, a.n_replicas, s);
}
