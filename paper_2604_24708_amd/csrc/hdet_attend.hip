// Attention under the masks of packed, prefixed, padded and cached sequences, and its backward pass.
//
//   z_ij = scale q_i . k_j, capped: cap tanh(z / cap), minus slope_h |pos_i - j|;  p_i = softmax over first_i <= j < end_i;  o_i = sum p_ij v_j
//   dv_j = sum_i p_ij do_i;  dz = p (do_i . v_j - do_i . o_i) (1 - tanh^2);  dq_i = scale sum_j dz k_j;  dk_j = scale sum_i dz q_i
//
// Every mask is a range of keys a query, so that a block of queries walks over the union of its ranges, tile by tile, and a 32 x 32 block of scores is
// outside, inside or across the ranges of its queries: only the last kind tests its pairs.
// In units of log2 throughout: p = 2^(z log2 e - m), one fma and one exponential a score.
//
// A pair that is not attended must leave no trace, but 0 times an infinity or a NaN does: the matrix cores multiply all of a block that lies across the
// ranges.  Results that came out finite are right; where one did not, the block walks its tiles a second time, and the second product takes zeros for
// what is not finite.  Scores and row dots are formed from the tiles as they are both times: a score of minus infinity has p = 0, that of an infinite
// entry under a cap is the cap, and the other columns of such rows are finite.  The entries left out are then added to the results of the rows that
// attend them (add_not_finite): values and output gradients times p, which is 0 for a score of minus infinity and more for any other; keys and queries
// times dz, which is 0 wherever an entry is infinite and its row's statistics are finite (p is 0, or the cap's derivative): NaN.

// Four kernels: attend (128 queries of a head a block), attend_few (few queries: the keys are divided over the chip), attend_dq and attend_dkv
// (backward; S = q k and dp are formed in both, since one kernel for all three gradients would add up dq with atomics, in an order that changes).  A
// wavefront owns 32 rows, as columns of the 32 x 32 products, so that a row's statistics lie in two lanes and a product's result is the next one's
// operand without a way through LDS.  Tiles of the other side (64 rows of bfloat16, 64 columns) come by direct loads to LDS, requested one stage ahead.
// (In attend_kernel the compiler waits for every load in flight before a block's first product, the next tile's among them, since it holds the queries'
// own loads for pending; in attend_dkv_kernel it does at the ranges of 32 queries, a load in the loop.)  The wavefronts of other blocks on the same CU
// cover the waits, so registers are what decides: 8 x 16 sequences of 256, 8 heads of 64, forward 4 wavefronts a SIMD 32 us; a variant with spills at
// that many: 2 to 3 times.
// Bound by the work between the two products of a block (16 exponentials a lane, sums, conversions) as much as by the products themselves, which wait
// for it: longer heads, more of the library's rate.  Reached, TFLOP/s (library's product: 1190 to 1270 bfloat16, 154 fp32): forward, 8192 queries and
// keys, heads of 64 910, of 128 950; of 128 causal, 278 to 304 us, 990 to 905 of the pairs that are attended; fp32 112 to 132; backward (5 products a
// pair), heads of 64 550 to 650.

#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "hdet_ops.h"
#include "hdet_attend_tiles.h"

using namespace hdet_attend;

namespace {

constexpr int THREADS = 256;
constexpr int NWV = THREADS / 64;
constexpr int WR = 32;                     // rows a wavefront owns
constexpr int RB = WR * NWV;               // rows a block owns

// n / d for any 32-bit n by a product and shifts (Granlund and Montgomery, Division by Invariant Integers using Multiplication, 1994): a division is
// some thirty instructions before a block's first load
struct divisor { unsigned d, mul, s1, s2; };
divisor divisor_of(unsigned d) {
  divisor v = {d, 0, 0, 0};
  if (d == 0) return v;
  unsigned l = 0;
  while (((uint64_t)1 << l) < d) ++l;
  v.mul = (unsigned)((((uint64_t)1 << 32) * (((uint64_t)1 << l) - d)) / d + 1);
  v.s1 = l < 1 ? l : 1;
  v.s2 = l > 1 ? l - 1 : 0;
  return v;
}
__device__ __forceinline__ unsigned over(unsigned n, const divisor& v) {
  const unsigned t = __umulhi(n, v.mul);
  return (t + ((n - t) >> v.s1)) >> v.s2;
}

struct attend_args {
  const void *q, *k, *v, *o, *dout;
  void *out, *dq, *dk, *dv;
  int64_t q_s, q_z, k_s, k_z, v_s, v_z, o_s, o_z, do_s, do_z, out_s, out_z, dq_s, dq_z, dk_s, dk_z, dv_s, dv_z;
  float* lse;                              // forward
  const float* lse_in;                     // backward
  float *lse2, *dot;                       // backward: [replica][head][row] lse log2 e (infinity for empty rows), minus sum_c do o
  int *lo, *hi, *pos_of;                   // backward: [replica][row] the rows' ranges and positions
  i4v* groups;                             // backward: [replica][sequence][32 queries] least and largest lo, least and largest hi
  float* part;                             // results of the splits
  float* lacks;                            // backward: the row dots' parts of dq's splits
  const float* slopes;
  int64_t slopes_z;
  const int32_t *pos, *first, *end;
  int n, seqs, q_len, kv_len, heads, kv_heads, group, d, causal, window;
  int splits;
  int run;                                 // dk and dv in fp32: the launch's number
  float scale, c, cap2, inv_cap;           // c = scale log2 e; cap2 = cap log2 e or 0
  bool close;                              // capped scores to fp32's last places, not to 1e-7 of the cap
  unsigned total;                          // blocks
  divisor by_nx, by_groups, by_own, by_heads, by_kv_heads, by_seqs, by_group;   // row blocks; total / nx, an eighth of that; ..
  bool heavy_first;
};

// Stages of two tiles (keys and values, or queries and output gradients) in LDS: one that is worked on, the other on its way.  (A third one, under the
// compiler's wait above: forward 167 -> 193 us at 8 x 16 sequences of 512, 16 heads of 64, for the blocks that the LDS then holds; with LDS for as many
// blocks, the same as two.)
constexpr int STAGES = 2;

struct key_range { int lo, hi, pos; };

// Keys that query i of sequence b attends: lo .. hi - 1, 0 .. -1 for none
__device__ __forceinline__ key_range range_of(const attend_args& g, int r, int b, int i) {
  const int64_t at = ((int64_t)r * g.seqs + b) * g.q_len + i;
  const int pos = g.pos ? g.pos[at] : i + g.kv_len - g.q_len;
  int lo = 0, hi = g.kv_len;
  if (g.first && g.first[at] > lo) lo = g.first[at];
  if (g.window) {
    const int64_t from = (int64_t)pos - g.window + 1;
    if (from > lo) lo = from > g.kv_len ? g.kv_len : (int)from;
  }
  if (g.end && g.end[at] < hi) hi = g.end[at];
  if (g.causal && pos < hi) hi = pos < 0 ? 0 : pos + 1 < hi ? pos + 1 : hi;
  if (hi <= lo) lo = hi = 0;
  return {lo, hi, pos};
}

// Block number -> row block x (of nx, the one with most work first) and (replica, sequence, head) grp.  Blocks reach the chip's 8 XCDs round-robin in
// launch order: every XCD works through a contiguous range of grp, so that the tiles which blocks share are in one L2; heavy_first: the longest row
// blocks of all grp first, then the next ones (few rounds of blocks: the last one's length counts more).
struct block_id { unsigned x, grp; };
__device__ __forceinline__ block_id place_block(unsigned lin, const attend_args& g) {
  const unsigned nx = g.by_nx.d, groups = g.by_groups.d, total = nx * groups;
  block_id b;
  if (g.heavy_first) {
    if ((groups & 7u) == 0u) {
      const unsigned j = lin >> 3;
      b.x = over(j, g.by_own);
      b.grp = (lin & 7u) * g.by_own.d + (j - b.x * g.by_own.d);
    } else {
      b.x = over(lin, g.by_groups);
      b.grp = lin - b.x * groups;
    }
  } else {
    if ((total & 7u) == 0u) lin = (lin & 7u) * (total >> 3) + (lin >> 3);
    b.grp = over(lin, g.by_nx);
    const unsigned turned = lin - b.grp * nx + b.grp + (b.grp >> 3) + (b.grp >> 6);
    b.x = turned - over(turned, g.by_nx) * nx;
  }
  return b;
}
// replica, sequence and head of a group
struct group_id { int r, b, h; };
__device__ __forceinline__ group_id place_group(unsigned grp, const attend_args& g, const divisor& heads) {
  const unsigned rb = over(grp, heads), r = over(rb, g.by_seqs);
  return {(int)r, (int)(rb - r * g.by_seqs.d), (int)(grp - rb * heads.d)};
}

// Least over the 32 rows of a wavefront
__device__ __forceinline__ int wave_min(int x) {
  x = min(x, __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, false));
  x = min(x, __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, false));
  x = min(x, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, false));
  x = min(x, __builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, false));
  return min(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16));
}
// The ranges of 32 queries: keys outside lo_min .. hi_max - 1 are outside for all, keys of lo_max .. hi_min - 1 inside for all
struct wave_range { int lo_min, lo_max, hi_min, hi_max; };
// `there`: the lane's row exists
__device__ __forceinline__ wave_range wave_range_of(const key_range& k, bool there) {
  const bool some = there && k.hi > k.lo;
  wave_range w;
  w.lo_min = wave_min(some ? k.lo : INT_MAX);
  w.hi_max = -wave_min(some ? -k.hi : 0);
  w.lo_max = -wave_min(some ? -k.lo : there ? -INT_MAX : 0);
  w.hi_min = wave_min(some ? k.hi : there ? 0 : INT_MAX);
  if (w.hi_max == 0) w.lo_max = INT_MAX;   // no keys at all are inside of no queries at all
  return w;
}
// Without arrays both ends of a range rise with the row: the same of rows i0 .. i0 + count - 1 of a sequence from the first and the last of them
__device__ __forceinline__ wave_range plain_range_of(const attend_args& g, int i0, int count) {
  if (i0 + count > g.q_len) count = g.q_len - i0;
  if (count <= 0) return {INT_MAX, INT_MAX, 0, 0};
  const key_range a = range_of(g, 0, 0, i0), b = range_of(g, 0, 0, i0 + count - 1);
  if (b.hi <= b.lo) return {INT_MAX, INT_MAX, 0, 0};                       // queries before the first key: the last one has most
  if (a.hi <= a.lo) return {0, INT_MAX, 0, b.hi};
  return {a.lo, b.lo, a.hi, b.hi};
}
// ... of a wavefront's 32 queries, the lanes' ranges given, and (lo, hi) of the block's 128 from q0 on, through LDS that nothing else uses before the
// next barrier but one
struct block_range { wave_range own; int lo, hi, pairs; };                // pairs: of the block's rows, about
__device__ __forceinline__ block_range block_range_of(const attend_args& g, const key_range& k, bool there, int q0, int w, int lane, int* ends) {
  block_range b;
  if (!g.pos && !g.first && !g.end) {
    b.own = plain_range_of(g, q0 + w * WR, WR);
    const wave_range all = plain_range_of(g, q0, RB);
    b.lo = all.lo_min;
    b.hi = all.hi_max;
    const key_range a = range_of(g, 0, 0, q0), z = range_of(g, 0, 0, min(q0 + RB, g.q_len) - 1);
    b.pairs = min((a.hi - a.lo + z.hi - z.lo) / 2, 1 << 20) * min(RB, g.q_len - q0);
  } else {
    b.own = wave_range_of(k, there);
    if (lane == 0) {
      ends[w] = b.own.lo_min;
      ends[NWV + w] = b.own.hi_max;
    }
    float pairs = there ? (float)(k.hi - k.lo) : 0.f;
    pairs = hdet_wave_sum(pairs) * 0.5f;   // (each row is in two lanes)
    if (lane == 0) ends[2 * NWV + w] = (int)fminf(pairs, 1e8f);
    __syncthreads();
    b.pairs = __builtin_amdgcn_readfirstlane(ends[8] + ends[9] + ends[10] + ends[11]);
    b.lo = __builtin_amdgcn_readfirstlane(min(min(ends[0], ends[1]), min(ends[2], ends[3])));
    b.hi = __builtin_amdgcn_readfirstlane(max(max(ends[4], ends[5]), max(ends[6], ends[7])));
  }
  return b;
}

// Whether any thread of the block's NW wavefronts says so; two barriers, and 4 NW bytes of LDS at `lds` that nothing else uses
template <int NW = NWV> __device__ __forceinline__ bool block_any(bool yes, int w, int lane, int* lds) {
  int any = __any(yes);
  __syncthreads();
  if (lane == 0) lds[w] = any;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) any |= lds[i];
  return any;
}

// Scores of a block from its raw products: x such that the score is (x + shift) mult log2 units (score_units).  With a cap x is tanh - 1, exact enough unless
// small scores are read off a very large cap (close).  dist(e): |position - key| of element e.
// EXTRA says how much of it is asked for: nothing (a product with c), a cap alone, anything.
enum { kPlain = 0, kCapped = 1, kGeneral = 2 };
struct score_units { float mult, shift; };
__device__ __forceinline__ score_units units_of(const attend_args& g, int extra) {
  return extra == kCapped ? score_units{g.cap2, 1.f} : extra == kPlain ? score_units{g.c, 0.f} : g.slopes || g.cap2 == 0.f ? score_units{1.f, 0.f} : score_units{g.cap2, g.close ? 0.f : 1.f};
}
template <int EXTRA, typename F> __device__ __forceinline__ void shape_scores(const attend_args& g, f16v& x, float slope2, F dist) {
  if (EXTRA == kCapped) {
    const float s = 2.f * kLog2e * g.scale * g.inv_cap;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = tanh_less_1(x[e] * s);
    return;
  }
  if (g.cap2 > 0.f && !g.close) {
    const float s = 2.f * kLog2e * g.scale * g.inv_cap;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = tanh_less_1(x[e] * s);
    if (g.slopes) {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = __builtin_fmaf(x[e], g.cap2, g.cap2);
    }
  } else if (g.cap2 > 0.f) {
    const float s = g.scale * g.inv_cap;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = tanh_close(x[e] * s);
    if (g.slopes) {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] *= g.cap2;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] *= g.c;
  }
  if (g.slopes) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = __builtin_fmaf(-slope2, dist(e), x[e]);
  }
}
// Backward: scores, in log2 units, from raw products; bend: the cap's derivative
template <int EXTRA, typename F> __device__ __forceinline__ void shape_scores_back(const attend_args& g, f16v& x, f16v& bend, float slope2, F dist) {
  if (EXTRA == kCapped || (g.cap2 > 0.f && !g.close)) {
    const float s = 2.f * kLog2e * g.scale * g.inv_cap;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float t = tanh_less_1(x[e] * s);
      bend[e] = -t * (t + 2.f);
      x[e] = __builtin_fmaf(t, g.cap2, g.cap2);
    }
  } else if (g.cap2 > 0.f) {
    const float s = g.scale * g.inv_cap;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float t = tanh_close(x[e] * s);
      bend[e] = __builtin_fmaf(-t, t, 1.f);
      x[e] = t * g.cap2;
    }
  } else {
    bend = all16(1.f);
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] *= g.c;
  }
  if (EXTRA == kGeneral && g.slopes) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = __builtin_fmaf(-slope2, dist(e), x[e]);
  }
}
__device__ __forceinline__ float distance(int pos, int key) { return (float)(pos < key ? (unsigned)key - (unsigned)pos : (unsigned)pos - (unsigned)key); }

// fp32 sums over keys are made in runs of 1024: a running sum over M keys rounds M times, at its own size, which takes it 0.3 x 2^-24 sqrt(M) off (8192
// keys: out off by 1.8e-6 of its norm, in runs by 6.6e-7).  What bfloat16 rounds elsewhere is far more.  What the runs before the present one have come
// to is kept
//   in registers, where there is one wavefront a SIMD all the same;
template <typename T> constexpr int key_run() { return sizeof(T) == 4 ? 1024 : 1 << 30; }
template <typename T, int D> struct runs_in_registers {
  f16v sum[D / 32];
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) sum[i] = all16(0.f);
  }
  // x and what is kept, times `scale`: KEEP: kept, and x is 0 from then on; else to x.  (Accumulator order: columns of the lane's row.)
  template <bool KEEP> __device__ __forceinline__ void join(f16v (&x)[D / 32], float scale, int) {
    if (sizeof(T) == 2) return;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float y = __builtin_fmaf(sum[i][e], scale, x[i][e]);
        sum[i][e] = y;
        x[i][e] = KEEP ? 0.f : y;
      }
  }
};
//   in the rows of the result, where registers would cost a wavefront (8 x 8192 queries and keys of 8 heads of 64, us: one sum 8160, in rows 8350, in
//   registers 8700).
template <typename T, int D> struct runs_in_rows {
  float* to;                               // the first of the wavefront's rows, `ld` apart
  int64_t ld;
  int d;
  bool some, any;                          // the lane's row takes part; there is something kept
  __device__ __forceinline__ void reset() { any = false; }
  template <bool KEEP> __device__ __forceinline__ void join(f16v (&x)[D / 32], float scale, int lane) {
    if (sizeof(T) == 2 || (!KEEP && !any)) return;
    asm volatile("" : "+v"(lane));         // addresses and tests are formed here, not held all the way
    float* const row = some ? to + (lane & 31) * ld : nullptr;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const int c = 32 * i + acc_row(4 * e4, lane);
        f4v y = {x[i][4 * e4], x[i][4 * e4 + 1], x[i][4 * e4 + 2], x[i][4 * e4 + 3]};
        if (row && c + 4 <= d) {
          f4v_any* const at = reinterpret_cast<f4v_any*>(row + c);
          if (any) y += *at * scale;
          if (KEEP) *at = y;
        } else if (row) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if (c + u >= d) continue;
            if (any) y[u] += row[c + u] * scale;
            if (KEEP) row[c + u] = y[u];
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) x[i][4 * e4 + u] = KEEP ? 0.f : y[u];
      }
    any = true;
  }
};
template <typename T, int D> __device__ __forceinline__ auto runs_of(void* to, int64_t ld, int d, bool some) {
  if constexpr (D == 64) return runs_in_rows<T, D>{(float*)to, ld, d, some, false};
  else return runs_in_registers<T, D>();
}

// Exponentials of up to 2^8 over the reference, all keys': as many powers of 2 that their sum is below 1, and what they are multiplied with stays in
// range.  (Values near the type's largest, whose mean is finite though the sum is not: taken on one more walk, since small values lose as many powers at
// fp32's other end.)
__device__ __forceinline__ float room_for(int keys) { return (float)(9 + 32 - __builtin_clz((unsigned)keys | 1u)); }

// Row statistics and results of a wavefront's 32 queries (columns of the accumulators) on its way over the keys
template <int D> struct running {
  f16v o[D / 32];
  float m, l;                              // reference of the exponentials (log2), this half-wavefront's sum
  float run_l, rescaled;                   // .. of the runs before; what those are to be multiplied by, since the reference has moved
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = all16(0.f);
    m = -INFINITY;
    l = run_l = 0.f;
    rescaled = 1.f;
  }
  // The end of a run: its results are kept; KEEP false: those of all runs
  template <bool KEEP, typename K> __device__ __forceinline__ void join(K& kept, int lane) {
    kept.template join<KEEP>(o, rescaled, lane);
    l = __builtin_fmaf(run_l, rescaled, l);
    rescaled = 1.f;
    if (!KEEP) return;
    run_l = l;
    l = 0.f;
  }
  __device__ __forceinline__ float ref() const { return m == -INFINITY ? 0.f : m; }
  // Exponentials of a block of scores times c.  Any reference will do that keeps them in fp32's range (bfloat16's is the same): FOLLOW takes the maximum, once
  // it has risen by more than 2^8 since (so that results are seldom rescaled); without it the reference stays, and where a score is more than 2^127
  // times larger, the sum says infinity.  room: of as many powers of 2 below it.
  template <bool FOLLOW> __device__ __forceinline__ void take(f16v& x, float c, float room) {
    if (FOLLOW) {
      float top = x[0];
#pragma unroll
      for (int e = 0; e < 16; e += 2) top = max3(top, x[e], x[e + 1]);
      top = fmaxf(top, other_half(top)) * c;
      if (__any(top > m + 8.f)) {
        const float next = fmaxf(m, top), keep = exp2_fast(m - (next == -INFINITY ? 0.f : next));
        m = next;
        l *= keep;
        rescaled *= keep;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[i][e] *= keep;
      }
    }
    const float r = -ref() - room;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      x[e] = exp2_fast(__builtin_fmaf(x[e], c, r));
      l += x[e];
    }
  }
};

// ---------------------------------------------------------------------------------------------
// forward: block = 128 queries of one (replica, sequence, head)
// ---------------------------------------------------------------------------------------------
template <typename T, int D, int EXTRA, bool WHOLE> constexpr int forward_waves() { return sizeof(T) == 2 ? (D == 64 ? (EXTRA ? 3 : 4) : 2) : D == 64 ? (WHOLE ? 3 : 2) : 1; }
template <typename T, int D, int EXTRA, bool WHOLE> __global__ __launch_bounds__(THREADS, (forward_waves<T, D, EXTRA, WHOLE>())) void attend_kernel(const attend_args g) {
  typedef shape<T, D> S;
  constexpr int TILE = S::TB * D, NB = S::TB / 32, LOADS = 2 * tile_loader<T, D, S::TB, NWV, WHOLE>::NI;
  __shared__ __attribute__((aligned(1024))) T smem[2 * STAGES * TILE];     // keys and values
  const unsigned lin = blockIdx.y * gridDim.x + blockIdx.x;
  if (lin >= g.total) return;
  const unsigned nx = g.by_nx.d;
  const block_id blk = place_block(lin, g);
  const group_id id = place_group(blk.grp, g, g.by_heads);
  const int h = id.h, b = id.b, r = id.r;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wq0 = (int)(nx - 1 - blk.x) * RB + w * WR, qi = wq0 + (lane & 31);
  const bool there = qi < g.q_len;
  const key_range range = there ? range_of(g, r, b, qi) : key_range{0, 0, 0};
  const int64_t col = (int64_t)h * g.d, kcol = (int64_t)over(h, g.by_group) * g.d, row0 = (int64_t)b * g.q_len + wq0;
  // (a row that attends nothing is not read: without keys there need be no queries)
  const T* const own = range.hi > range.lo ? (const T*)g.q + r * g.q_z + (row0 + (lane & 31)) * g.q_s + col : nullptr;
  typename S::frag fq[S::NF];
#pragma unroll
  for (int i = 0; i < S::NF; ++i) fq[i] = own_frag<T, D, WHOLE>(own, i, g.d, lane);
  const tile_loader<T, D, S::TB, NWV, WHOLE> keys((const T*)g.k + r * g.k_z + (int64_t)b * g.kv_len * g.k_s + kcol, g.k_s, g.d, w, lane);
  const tile_loader<T, D, S::TB, NWV, WHOLE> vals((const T*)g.v + r * g.v_z + (int64_t)b * g.kv_len * g.v_s + kcol, g.v_s, g.d, w, lane);
  const S at(lane);
  const float slope2 = EXTRA == kGeneral && g.slopes ? g.slopes[r * g.slopes_z + h] * kLog2e : 0.f;
  const score_units unit = units_of(g, EXTRA);
  // (the block's ends pass through the second stage, which is requested behind a barrier)
  const block_range br = block_range_of(g, range, there, wq0 - w * WR, w, lane, (int*)(smem + 2 * TILE));
  const wave_range wr = br.own;
  const int hi = br.hi, t0 = br.lo / S::TB, t1 = (hi + S::TB - 1) / S::TB; // hi = 0: none

  running<D> z;
  auto kept = runs_of<T, D>((T*)g.out + r * g.out_z + row0 * g.out_s + col, g.out_s, g.d, range.hi > range.lo);
  float room = 0.f;
  // (every request is as many loads, of zeros behind the last tile, so that a wait can count them)
  auto request = [&](int t, int slot) {
    T* const to = smem + slot * (2 * TILE);
    keys.load((int64_t)t * S::TB, t < t1 ? hi - t * S::TB : 0, to);
    vals.load((int64_t)t * S::TB, t < t1 ? hi - t * S::TB : 0, to + TILE);
  };
  auto walk = [&](auto clean) {
    z.reset();
    kept.reset();
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) request(t0 + i, i);
    int slot = 0, free = STAGES - 1;
    auto step = [&](int t, auto follow) {
      wait_and_barrier<(STAGES - 2) * LOADS>();
      request(t + STAGES - 1, free);
      T* const kt = smem + slot * (2 * TILE);
      T* const vt = kt + TILE;
      free = slot;
      slot = slot == STAGES - 1 ? 0 : slot + 1;
#pragma unroll 1
      for (int i = 0; i < NB; ++i) {
        const int kb = t * S::TB + 32 * i;
        if (kb >= wr.hi_max || kb + 32 <= wr.lo_min) continue;
        f16v x = at.first(kt + i * 32 * D, fq, all16(0.f));
        const int k0 = kb + ((lane >> 5) << 2);
        if (EXTRA) shape_scores<EXTRA>(g, x, slope2, [&](int e) { return distance(range.pos, k0 + acc_row(e, 0)); });
        if (!(kb >= wr.lo_max && kb + 32 <= wr.hi_min)) {
          const unsigned from = k0 - range.lo, len = range.hi - range.lo;
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = from + acc_row(e, 0) < len ? x[e] : -INFINITY;
        }
        z.template take<decltype(follow)::value>(x, unit.mult, decltype(clean)::value ? room : 0.f);
        at.template second<decltype(clean)::value>(vt + i * 32 * D, x, z.o);
      }
    };
    auto next_run = [&](int t) {
      if (sizeof(T) == 4 && __builtin_expect(t > t0 && (t - t0) % (key_run<T>() / S::TB) == 0, 0)) z.template join<true>(kept, lane);
    };
    // the reference follows the maximum until every row has met a key; all the way on the second walk, and where scores fall with the distance
    int t = t0;
    for (bool met = false; t < t1 && !met; ++t) {
      next_run(t);
      step(t, std::true_type());
      met = !(EXTRA == kGeneral && g.slopes) && !__any(range.hi > range.lo && z.m == -INFINITY);
    }
    for (; t < t1; ++t) {
      next_run(t);
      step(t, clean);
    }
    wait_and_barrier<0>();
    if (sizeof(T) == 4) z.template join<false>(kept, lane);
    z.l += other_half(z.l);
  };
  walk(std::false_type());
  int* const any = (int*)(smem + 2 * STAGES * TILE) - NWV;
  const bool again = block_any(there && z.l == z.l && (z.l == INFINITY || not_finite(z.o)), w, lane, any);
  while (again) {
    walk(std::true_type());
    if (room > 0.f || !block_any(there && z.l == z.l && not_finite(z.o), w, lane, any)) break;
    room = room_for(g.kv_len);
  }
  const bool some = range.hi > range.lo;
  const float inv = some ? 1.f / z.l : 0.f;
#pragma unroll
  for (int i = 0; i < S::ND; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) z.o[i][e] = some ? z.o[i][e] * inv : 0.f;
  if (g.lse && there && lane < 32) g.lse[((int64_t)r * g.heads + h) * g.seqs * g.q_len + row0 + lane] = some ? (z.ref() + room + unit.mult * unit.shift + log2f(z.l)) * kLn2 : -INFINITY;
  store_rows<T, D, WHOLE>(z.o, (char*)smem + w * STRIP, (T*)g.out + r * g.out_z + row0 * g.out_s + col, g.out_s, g.q_len - wq0, g.d, lane);
  if (again) {
    __threadfence_block();
    add_not_finite<T, D>(vals.src, g.v_s, g.d, wr.lo_min, wr.hi_max, (T*)g.out + r * g.out_z + row0 * g.out_s + col, g.out_s, min(WR, g.q_len - wq0), lane,
                         [&](int key, int i) { return key >= __builtin_amdgcn_readlane(range.lo, i) && key < __builtin_amdgcn_readlane(range.hi, i); },
                         [&](int key, int i) { return pair_weight((const T*)g.q + r * g.q_z + (row0 + i) * g.q_s + col, keys.src + key * g.k_s, g.d, g.scale, g.cap2 > 0.f, lane); });
  }
}

// ---------------------------------------------------------------------------------------------
// forward, few queries over many keys: a block takes 32 (query, head) pairs that share a key head, as one wavefront's rows, and a part of the keys, of
// which its wavefronts take every NW-th tile of 32, each through LDS of its own.  Their results are joined in LDS, those of the parts by a second launch.
// ---------------------------------------------------------------------------------------------
template <typename T, int D> constexpr int few_waves() { return sizeof(T) == 4 && D == 128 ? 2 : 4; }
template <typename T, int D, int EXTRA, bool WHOLE> __global__ __launch_bounds__((few_waves<T, D>() * 64)) void attend_few_kernel(const attend_args g) {
  typedef shape<T, D> S;
  constexpr int NW = few_waves<T, D>(), TILE = 32 * D, P = D + 4;
  __shared__ __attribute__((aligned(1024))) T smem[NW * 4 * TILE];
  unsigned lin = blockIdx.y * gridDim.x + blockIdx.x;
  if (lin >= g.total) return;
  if ((g.total & 7u) == 0u) lin = (lin & 7u) * (g.total >> 3) + (lin >> 3);
  const int pairs = g.group * g.q_len;
  const unsigned ncg = (pairs + 31) / 32, cg = lin % ncg, split = lin / ncg % g.splits, grp = lin / ncg / g.splits;
  const group_id id = place_group(grp, g, g.by_kv_heads);
  const int kh = id.h, b = id.b, r = id.r;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pair = cg * 32 + (lane & 31);
  const bool there = pair < pairs;
  const int h = kh * g.group + (there ? pair / g.q_len : 0), qi = there ? pair % g.q_len : 0;
  const key_range range = there ? range_of(g, r, b, qi) : key_range{0, 0, 0};
  const wave_range wr = wave_range_of(range, there);
  const int64_t row = (int64_t)b * g.q_len + qi, kcol = (int64_t)kh * g.d;
  const T* const own = range.hi > range.lo ? (const T*)g.q + r * g.q_z + row * g.q_s + (int64_t)h * g.d : nullptr;
  typename S::frag fq[S::NF];
#pragma unroll
  for (int i = 0; i < S::NF; ++i) fq[i] = own_frag<T, D, WHOLE>(own, i, g.d, lane);
  const tile_loader<T, D, 32, 1, WHOLE> keys((const T*)g.k + r * g.k_z + (int64_t)b * g.kv_len * g.k_s + kcol, g.k_s, g.d, 0, lane);
  const tile_loader<T, D, 32, 1, WHOLE> vals((const T*)g.v + r * g.v_z + (int64_t)b * g.kv_len * g.v_s + kcol, g.v_s, g.d, 0, lane);
  constexpr int IN_FLIGHT = 2 * tile_loader<T, D, 32, 1, WHOLE>::NI;
  const S at(lane);
  const float slope2 = EXTRA == kGeneral && g.slopes ? g.slopes[r * g.slopes_z + h] * kLog2e : 0.f;
  const score_units unit = units_of(g, EXTRA);
  // the union of the ranges in tiles, this block's part of them
  const int hi = wr.hi_max, lo = hi > 0 ? wr.lo_min : 0, t0 = lo / 32, t1 = (hi + 31) / 32, per = (t1 - t0 + g.splits - 1) / g.splits;
  const int ts = t0 + split * per, te = min(t1, ts + per);
  T* const mine = smem + w * (4 * TILE);

  running<D> z;
  runs_in_registers<T, D> kept;
  float room = 0.f;
  auto request = [&](int t, int stage) {
    const int have = t < te ? hi - t * 32 : 0;
    keys.load((int64_t)t * 32, have, mine + stage * (2 * TILE));
    vals.load((int64_t)t * 32, have, mine + stage * (2 * TILE) + TILE);
  };
  auto walk = [&](auto clean) {
    z.reset();
    kept.reset();
    int stage = 0;
    if (ts + w < te) request(ts + w, 0);
    auto step = [&](int t, auto follow) {
      wave_fence();                        // the other stage's tiles have been read
      request(t + NW, stage ^ 1);
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(IN_FLIGHT) : "memory");
      T* const kt = mine + stage * (2 * TILE);
      stage ^= 1;
      f16v x = at.first(kt, fq, all16(0.f));
      const int k0 = t * 32 + ((lane >> 5) << 2);
      if (EXTRA) shape_scores<EXTRA>(g, x, slope2, [&](int e) { return distance(range.pos, k0 + acc_row(e, 0)); });
      if (!(t * 32 >= wr.lo_max && t * 32 + 32 <= wr.hi_min)) {
        const unsigned from = k0 - range.lo, len = range.hi - range.lo;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = from + acc_row(e, 0) < len ? x[e] : -INFINITY;
      }
      z.template take<decltype(follow)::value>(x, unit.mult, decltype(clean)::value ? room : 0.f);
      at.template second<decltype(clean)::value>(kt + TILE, x, z.o);
    };
    auto next_run = [&](int t) {
      if (sizeof(T) == 4 && __builtin_expect(t > ts + w && (t - ts) % (NW * key_run<T>() / 32) == w, 0)) z.template join<true>(kept, lane);
    };
    int t = ts + w;
    for (bool met = false; t < te && !met; t += NW) {
      next_run(t);
      step(t, std::true_type());
      met = !(EXTRA == kGeneral && g.slopes) && !__any(range.hi > range.lo && z.m == -INFINITY);
    }
    for (; t < te; t += NW) {
      next_run(t);
      step(t, clean);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    if (sizeof(T) == 4) z.template join<false>(kept, lane);
    z.l += other_half(z.l);
  };
  walk(std::false_type());
  // (2^64 and 2^-9: for the sum over wavefronts and parts, 256 at most)
  const bool again = __any(there && z.l == z.l && (z.l > 0x1p64f || not_finite(z.o, 0x1p9f)));
  while (again) {
    walk(std::true_type());
    if (room > 0.f || !__any(there && z.l == z.l && not_finite(z.o, 0x1p9f))) break;
    room = room_for(g.kv_len);
  }

  // join the wavefronts
  float* const joint = (float*)smem;       // [wave][32][P], then [wave][32] references and sums
  float* const stats = joint + NW * 32 * P;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < S::ND; ++i)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4)
      *reinterpret_cast<f4v*>(joint + (w * 32 + (lane & 31)) * P + 32 * i + acc_row(4 * e4, lane)) = f4v{z.o[i][4 * e4], z.o[i][4 * e4 + 1], z.o[i][4 * e4 + 2], z.o[i][4 * e4 + 3]};
  if (again) {
    wave_fence();
    for (int t = ts + w; t < te; t += NW)
      add_not_finite<T, D>(vals.src, g.v_s, g.d, t * 32, min(t * 32 + 32, hi), joint + w * 32 * P, P, 32, lane,
                           [&](int key, int i) { return key >= __builtin_amdgcn_readlane(range.lo, i) && key < __builtin_amdgcn_readlane(range.hi, i); },
                           [&](int key, int i) {
                             const int64_t own_row = (int64_t)b * g.q_len + __builtin_amdgcn_readlane(qi, i);
                             return pair_weight((const T*)g.q + r * g.q_z + own_row * g.q_s + (int64_t)__builtin_amdgcn_readlane(h, i) * g.d, keys.src + key * g.k_s, g.d, g.scale,
                                                g.cap2 > 0.f, lane);
                           });
  }
  if (lane < 32) {
    stats[w * 64 + lane] = z.m + room;
    stats[w * 64 + 32 + lane] = z.l;
  }
  __syncthreads();
  for (int item = tid; item < 32 * (D / 4); item += NW * 64) {
    const int c_ = item / (D / 4), col = item % (D / 4) * 4, p = cg * 32 + c_;
    if (p >= pairs || col >= g.d) continue;
    float m = stats[c_];
#pragma unroll
    for (int i = 1; i < NW; ++i) m = fmaxf(m, stats[i * 64 + c_]);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float keep = exp2_fast(stats[i * 64 + c_] - ref);
      l = __builtin_fmaf(stats[i * 64 + 32 + c_], keep, l);
      const f4v x = *reinterpret_cast<const f4v*>(joint + (i * 32 + c_) * P + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(x[e], keep, o[e]);
    }
    if (g.splits > 1) {
      float* const to = g.part + ((int64_t)lin * 32 + c_) * (D + 2);
      if (col == 0) {
        to[0] = m + unit.mult * unit.shift;
        to[1] = l;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) to[2 + col + e] = o[e];
      continue;
    }
    const int oh = kh * g.group + p / g.q_len, oi = p % g.q_len;
    const key_range k = range_of(g, r, b, oi);
    const bool some = k.hi > k.lo;
    const float inv = some ? 1.f / l : 0.f;
    const int64_t orow = (int64_t)b * g.q_len + oi;
    T* const to = (T*)g.out + r * g.out_z + orow * g.out_s + (int64_t)oh * g.d + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < g.d) hdet_st(to + e, some ? o[e] * inv : 0.f);
    if (g.lse && col == 0) g.lse[((int64_t)r * g.heads + oh) * g.seqs * g.q_len + orow] = some ? (ref + unit.mult * unit.shift + log2f(l)) * kLn2 : -INFINITY;
  }
}

// A wavefront to a (query, head): the parts' results, times 2^(reference - the largest)
template <typename T, int D> __global__ __launch_bounds__(THREADS) void attend_join_kernel(const attend_args g) {
  const int pairs = g.group * g.q_len, ncg = (pairs + 31) / 32, lane = threadIdx.x & 63;
  const int64_t id = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * NWV + (threadIdx.x >> 6);
  if (id >= (int64_t)g.n * g.seqs * g.kv_heads * pairs) return;
  const int p = (int)(id % pairs);
  const int64_t grp = id / pairs;
  const int kh = (int)(grp % g.kv_heads), b = (int)(grp / g.kv_heads % g.seqs), r = (int)(grp / g.kv_heads / g.seqs);
  const float* const from = g.part + ((grp * g.splits * ncg + p / 32) * 32 + p % 32) * (D + 2);
  const int64_t step = (int64_t)ncg * 32 * (D + 2);
  const float own = lane < g.splits ? from[lane * step] : -INFINITY;
  const float m = hdet_wave_max(own), ref = m == -INFINITY ? 0.f : m, keep = exp2_fast(own - ref);
  const float l = hdet_wave_sum(lane < g.splits ? keep * from[lane * step + 1] : 0.f);
  float o[D / 64] = {};
  for (int i = 0; i < g.splits; ++i) {
    const float k = __shfl(keep, i);
#pragma unroll
    for (int u = 0; u < D / 64; ++u)
      if (lane + 64 * u < g.d) o[u] = __builtin_fmaf(k, from[i * step + 2 + lane + 64 * u], o[u]);
  }
  const int h = kh * g.group + p / g.q_len, qi = p % g.q_len;
  const key_range k = range_of(g, r, b, qi);
  const bool some = k.hi > k.lo;
  const float inv = some ? 1.f / l : 0.f;
  const int64_t row = (int64_t)b * g.q_len + qi;
  T* const to = (T*)g.out + r * g.out_z + row * g.out_s + (int64_t)h * g.d;
#pragma unroll
  for (int u = 0; u < D / 64; ++u)
    if (lane + 64 * u < g.d) hdet_st(to + lane + 64 * u, some ? o[u] * inv : 0.f);
  if (g.lse && lane == 0) g.lse[((int64_t)r * g.heads + h) * g.seqs * g.q_len + row] = some ? (ref + log2f(l)) * kLn2 : -INFINITY;
}

// ---------------------------------------------------------------------------------------------
// backward, step 1: dq, and what step 2 needs of the queries (row dots, statistics, ranges); block = 128 queries
// ---------------------------------------------------------------------------------------------
template <typename T, int D, int EXTRA, bool WHOLE> __global__ __launch_bounds__(THREADS, (sizeof(T) == 4 && D == 128 ? 1 : 2)) void attend_dq_kernel(const attend_args g) {
  typedef shape<T, D> S;
  constexpr int TILE = S::TB * D, NB = S::TB / 32, LOADS = 2 * tile_loader<T, D, S::TB, NWV, WHOLE>::NI;
  __shared__ __attribute__((aligned(1024))) T smem[2 * STAGES * TILE];     // keys and values
  unsigned lin = blockIdx.y * gridDim.x + blockIdx.x;
  if (lin >= g.total) return;
  const unsigned split = g.splits > 1 ? lin % g.splits : 0;
  if (g.splits > 1) lin /= g.splits;
  const unsigned nx = g.by_nx.d;
  const block_id blk = place_block(lin, g);
  const group_id id = place_group(blk.grp, g, g.by_heads);
  const int h = id.h, b = id.b, r = id.r;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wq0 = (int)(nx - 1 - blk.x) * RB + w * WR, qi = wq0 + (lane & 31);
  const bool there = qi < g.q_len;
  const key_range range = there ? range_of(g, r, b, qi) : key_range{0, 0, 0};
  const block_range br = block_range_of(g, range, there, wq0 - w * WR, w, lane, (int*)(smem + 2 * TILE));
  const wave_range wr = br.own;
  const int64_t rows = (int64_t)g.seqs * g.q_len, row0 = (int64_t)b * g.q_len + wq0, row = row0 + (lane & 31);
  const int64_t col = (int64_t)h * g.d, kcol = (int64_t)over(h, g.by_group) * g.d, stat = ((int64_t)r * g.heads + h) * rows + row;
  const bool some = range.hi > range.lo;
  const T* const own = some ? (const T*)g.q + r * g.q_z + row * g.q_s + col : nullptr;
  const T* const own_do = some ? (const T*)g.dout + r * g.do_z + row * g.do_s + col : nullptr;
  const T* const own_o = some ? (const T*)g.o + r * g.o_z + row * g.o_s + col : nullptr;
  typename S::frag fq[S::NF], fdo[S::NF];
  // minus the row's dot, from out as it is stored, summed as the products below sum: a row that attends one key has dz = 0 to the bit
  f16v both = all16(0.f);
#pragma unroll
  for (int i = 0; i < S::NF; ++i) {
    fq[i] = own_frag<T, D, WHOLE>(own, i, g.d, lane);
    fdo[i] = own_frag<T, D, WHOLE>(own_do, i, g.d, lane);
    both = S::product(own_frag<T, D, WHOLE>(own_o, i, g.d, lane), fdo[i], both);
  }
  float ndot = -diagonal(both, lane);
  const float lse2 = some ? g.lse_in[stat] * kLog2e : INFINITY;
  if (there && lane < 32 && split == 0) {
    g.lse2[stat] = lse2;
    if (h == 0) {
      g.lo[r * rows + row] = range.lo;
      g.hi[r * rows + row] = range.hi;
      g.pos_of[r * rows + row] = range.pos;
    }
  }
  // rows of the 32 that there are not: never inside
  if (h == 0 && lane == 0 && wq0 < g.q_len && split == 0)
    g.groups[((int64_t)r * g.seqs + b) * ((g.q_len + 31) / 32) + wq0 / 32] = i4v{wr.lo_min, wq0 + 32 > g.q_len ? INT_MAX : wr.lo_max, wr.hi_min, wr.hi_max};
  const tile_loader<T, D, S::TB, NWV, WHOLE> keys((const T*)g.k + r * g.k_z + (int64_t)b * g.kv_len * g.k_s + kcol, g.k_s, g.d, w, lane);
  const tile_loader<T, D, S::TB, NWV, WHOLE> vals((const T*)g.v + r * g.v_z + (int64_t)b * g.kv_len * g.v_s + kcol, g.v_s, g.d, w, lane);
  const S at(lane);
  const float slope2 = EXTRA == kGeneral && g.slopes ? g.slopes[r * g.slopes_z + h] * kLog2e : 0.f;
  const float c = EXTRA ? 1.f : g.c;
  const int hi = br.hi, first = br.lo / S::TB, last = (hi + S::TB - 1) / S::TB;
  // this block's part of the tiles
  // (rows of few keys, which form their dots first: the first part takes them all)
  const bool few_keys = sizeof(T) == 2 && br.pairs < 40 * min(RB, g.q_len - (wq0 - w * WR));
  const int parts = few_keys ? 1 : g.splits, share = hi > 0 ? (last - first + parts - 1) / parts : 0, t0 = first + split * share, t1 = hi > 0 ? min(last, t0 + share) : t0;

  f16v dq[S::ND];                          // [column][query]
  float* const part = g.part + (((int64_t)split * g.n + r) * g.heads + h) * rows * D + row0 * D;       // of a divided walk
  auto kept = runs_of<T, D>(g.splits > 1 ? (void*)part : (T*)g.dq + r * g.dq_z + row0 * g.dq_s + col, g.splits > 1 ? D : g.dq_s, g.d, some);
  // sum over the keys of p (dp - dot): what the dot lacks for out's rounding, since the p sum to 1
  float lack = 0.f;
  // (every request is as many loads, of zeros behind the last tile, so that a wait can count them)
  auto request = [&](int t, int slot) {
    T* const to = smem + slot * (2 * TILE);
    keys.load((int64_t)t * S::TB, t < t1 ? hi - t * S::TB : 0, to);
    vals.load((int64_t)t * S::TB, t < t1 ? hi - t * S::TB : 0, to + TILE);
  };
  // clean: zeros for keys that are not finite, in the second product; dots: no more than `lack`
  auto walk = [&](auto clean, auto dots) {
#pragma unroll
    for (int i = 0; i < S::ND; ++i) dq[i] = all16(0.f);
    lack = 0.f;
    kept.reset();
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) request(t0 + i, i);
    int slot = 0, free = STAGES - 1;
    for (int t = t0; t < t1; ++t) {
      if (sizeof(T) == 4 && __builtin_expect(t > t0 && (t - t0) % (key_run<T>() / S::TB) == 0, 0)) kept.template join<true>(dq, 1.f, lane);
      wait_and_barrier<(STAGES - 2) * LOADS>();
      request(t + STAGES - 1, free);
      T* const tiles = smem + slot * (2 * TILE);
      free = slot;
      slot = slot == STAGES - 1 ? 0 : slot + 1;
#pragma unroll 1
      for (int i = 0; i < NB; ++i) {
        const int key0 = t * S::TB + 32 * i;
        if (key0 >= wr.hi_max || key0 + 32 <= wr.lo_min) continue;
        const T* const kt = tiles + i * 32 * D;
        f16v x = at.first(kt, fq, all16(0.f)), dp = at.first(kt + TILE, fdo, all16(0.f)), bend;
        const int k0 = key0 + ((lane >> 5) << 2);
        if (EXTRA) shape_scores_back<EXTRA>(g, x, bend, slope2, [&](int e) { return distance(range.pos, k0 + acc_row(e, 0)); });
#pragma unroll
        for (int e = 0; e < 16; ++e) dp[e] = (dp[e] + ndot) * exp2_fast(__builtin_fmaf(x[e], c, -lse2));
        if (!(key0 >= wr.lo_max && key0 + 32 <= wr.hi_min)) {
          const unsigned from = k0 - range.lo, len = range.hi - range.lo;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const bool seen = from + acc_row(e, 0) < len;
            dp[e] = seen ? dp[e] : 0.f;
            if (EXTRA) bend[e] = seen ? bend[e] : 0.f;
          }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          lack += dp[e];
          if (EXTRA) dp[e] *= bend[e];
        }
        if (!decltype(dots)::value) at.template second_in_two<decltype(clean)::value>(kt, dp, dq);
      }
    }
    wait_and_barrier<0>();
    if (sizeof(T) == 4) kept.template join<false>(dq, 1.f, lane);
  };
  // Few keys a row: a dot that is off by out's rounding is off by as much in all of them, and the sum of dz k does not average that away (two keys: dq off by 2.4 times its
  // own rounding): the dots first, then.  Many: it does (1.1 to 1.3 times), with dz in two bfloat16 parts (1.5 in one).
  if (few_keys && split == 0) {
    walk(std::false_type(), std::true_type());
    ndot -= lack + other_half(lack);
    __syncthreads();
  }
  walk(std::false_type(), std::false_type());
  const bool again = block_any(some && finite_of(lse2) && not_finite(dq), w, lane, (int*)(smem + 2 * STAGES * TILE) - NWV);
  if (again) walk(std::true_type(), std::false_type());
  lack += other_half(lack);
  if (there && lane < 32) {
    if (g.splits == 1) g.dot[stat] = ndot - lack;
    else g.lacks[(int64_t)split * g.n * g.heads * rows + stat] = split == 0 ? ndot - lack : -lack;
  }
#pragma unroll
  for (int i = 0; i < S::ND; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) dq[i][e] = some ? dq[i][e] * g.scale : 0.f;               // (a row that attends nothing has not asked for the second walk)
  char* const strip = (char*)smem + w * STRIP;
  auto put = [&](auto to, int64_t ld, auto wh) {
    typedef std::remove_pointer_t<decltype(to)> U;
    store_rows<U, D, decltype(wh)::value>(dq, strip, to, ld, g.q_len - wq0, g.d, lane);
    if (!again) return;
    __threadfence_block();
    add_not_finite<T, D>(keys.src, g.k_s, g.d, max(wr.lo_min, t0 * S::TB), min(wr.hi_max, t1 * S::TB), to, ld, min(WR, g.q_len - wq0), lane,
                         [&](int key, int i) { return key >= __builtin_amdgcn_readlane(range.lo, i) && key < __builtin_amdgcn_readlane(range.hi, i); },
                         [](int, int) { return 0.f; });
  };
  if (g.splits == 1) put((T*)g.dq + r * g.dq_z + row0 * g.dq_s + col, g.dq_s, std::integral_constant<bool, WHOLE>());
  else put(part, (int64_t)D, std::false_type());
}

// dq and the row dots from the splits' parts, [split][replica][head][row]
template <typename T, int D> __global__ __launch_bounds__(THREADS) void attend_dq_join_kernel(const attend_args g) {
  const int64_t rows = (int64_t)g.seqs * g.q_len, all = rows * g.heads * g.n, i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * THREADS + threadIdx.x, stat = i / D;
  const int col = (int)(i % D);
  if (stat >= all) return;
  if (col == 0) {
    float dot = 0.f;
    for (int s = 0; s < g.splits; ++s) dot += g.lacks[(int64_t)s * all + stat];
    g.dot[stat] = dot;
  }
  if (col >= g.d) return;
  float dq = 0.f;
  for (int s = 0; s < g.splits; ++s) dq += g.part[((int64_t)s * all + stat) * D + col];
  const int64_t row = stat % rows;
  const int h = (int)(stat / rows % g.heads), r = (int)(stat / rows / g.heads);
  hdet_st((T*)g.dq + r * g.dq_z + row * g.dq_s + (int64_t)h * g.d + col, dq);
}

// ---------------------------------------------------------------------------------------------
// backward, step 2: dk and dv; block = 128 keys of a key head, walks over the query tiles of the heads that share it
// ---------------------------------------------------------------------------------------------
// bfloat16 heads of more than 64 columns: two wavefronts to 32 keys, one to either half of a query tile, and the own keys and values in LDS, since in
// registers they leave room for one wavefront a SIMD (the backward pass of 2 x 8192 tokens, 8 query and 2 key heads of 128, in undivided walks: 1610
// us, in registers 2231; 8 x 4 x 1024 tokens of 8 and 8: 440, 530)
template <typename T, int D> constexpr bool dkv_paired() { return sizeof(T) == 2 && D == 128; }
template <typename T, int D> constexpr int dkv_threads() { return dkv_paired<T, D>() ? 512 : 256; }
template <typename T, int D, int EXTRA, bool TWO> constexpr int dkv_waves() { return sizeof(T) == 2 ? (D == 64 && !EXTRA && !TWO ? 3 : 2) : D == 64 ? 2 : 1; }
// Query tiles that one launch sums up: in fp32 1024 rows, and the next launch adds its sums to what the one before has written, since a running sum
// over all rows of the heads that share a key head rounds once a row (4 heads of 1088 rows: dk and dv off by 1.3e-6 of their norms, in runs by
// 7.9e-7; 2 x 8192 tokens of 4 heads and one key head: the backward pass in undivided walks 3400 -> 3780 us)
template <typename T, int D> constexpr int run_tiles() { return sizeof(T) == 2 ? 1 << 28 : 1024 / shape<T, D>::TB; }
// TWO: dk and dv from dz and p in two bfloat16 parts each
template <typename T, int D, int EXTRA, bool WHOLE, bool TWO> __global__ __launch_bounds__((dkv_threads<T, D>()), (dkv_waves<T, D, EXTRA, TWO>())) void attend_dkv_kernel(const attend_args g) {
  typedef shape<T, D> S;
  constexpr int TILE = S::TB * D, NB = S::TB / 32, STATS = 5 * S::TB;      // lse2, dot, lo, hi, position
  constexpr bool PAIRED = dkv_paired<T, D>();
  constexpr int NW = dkv_threads<T, D>() / 64, LOADS = 2 * tile_loader<T, D, S::TB, NW, WHOLE>::NI + 2, RING = 2 * STAGES * TILE;
  __shared__ __attribute__((aligned(1024))) T smem[RING + (PAIRED ? 2 * RB * D : 0)];        // queries and output gradients; own keys and values
  __shared__ __attribute__((aligned(16))) int stats[STAGES * STATS];
  __shared__ int ends[2 * NW];
  unsigned lin = blockIdx.y * gridDim.x + blockIdx.x;
  if (lin >= g.total) return;
  const unsigned split = g.splits > 1 ? lin % g.splits : 0;
  if (g.splits > 1) lin /= g.splits;
  const block_id blk = place_block(lin, g);
  const group_id id = place_group(blk.grp, g, g.by_kv_heads);
  const int kh = id.h, b = id.b, r = id.r;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = PAIRED ? w >> 2 : 0, k0 = blk.x * RB, wk0 = k0 + (w & 3) * WR, key = wk0 + (lane & 31);
  const int n_groups = (g.q_len + 31) / 32;
  const i4v* const groups = g.groups + ((int64_t)r * g.seqs + b) * n_groups;
  // first and last group of queries that attend any of the block's keys
  const bool plain = !g.pos && !g.first && !g.end;
  int first = INT_MAX, last = -1;
  if (plain) {
    const int64_t off = (int64_t)g.kv_len - g.q_len, from = g.causal && k0 > off ? k0 - off : 0, to = g.window ? (int64_t)k0 + RB + g.window - 2 - off : INT_MAX;
    if (from < g.q_len && to >= 0) {       // (no queries: none)
      first = (int)from / 32;
      last = (int)(to < g.q_len ? to : g.q_len - 1) / 32;
    }
  } else {
    for (int i = tid; i < n_groups; i += NW * 64) {
      const i4v x = groups[i];
      if (x[0] < k0 + RB && x[3] > k0) {
        first = min(first, i);
        last = i;
      }
    }
    first = min(wave_min(first), wave_min(__shfl_xor(first, 32)));
    last = -min(wave_min(-last), wave_min(-__shfl_xor(last, 32)));
    if (lane == 0) {
      ends[w] = first;
      ends[NW + w] = last;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      first = min(first, ends[i]);
      last = max(last, ends[NW + i]);
    }
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);
  }
  const int t0 = last < 0 ? 0 : first / NB, tiles = last < 0 ? 0 : last / NB + 1 - t0;
  // this block's part of all heads' tiles
  const int share = (tiles * g.group + g.splits - 1) / g.splits, end = min(tiles * g.group, (int)(split + 1) * share), begin = split * share + g.run * run_tiles<T, D>(),
            all = min(end, begin + run_tiles<T, D>());
  if (g.run && begin >= all) return;
  // (without queries keys and values need not be there)
  const bool there = key < g.kv_len && g.q_len > 0;
  const int64_t kcol = (int64_t)kh * g.d, row0 = (int64_t)b * g.kv_len + wk0, rows = (int64_t)g.seqs * g.q_len, q_row0 = (int64_t)b * g.q_len;
  typename S::frag fk[PAIRED ? 1 : S::NF], fv[PAIRED ? 1 : S::NF];
  T* const own_k = smem + RING + (w & 3) * WR * D;
  T* const own_v = own_k + RB * D;
  if constexpr (PAIRED) {
    const T* const from_k = (const T*)g.k + r * g.k_z + ((int64_t)b * g.kv_len + k0) * g.k_s + kcol;
    const T* const from_v = (const T*)g.v + r * g.v_z + ((int64_t)b * g.kv_len + k0) * g.v_s + kcol;
#pragma unroll
    for (int i = 0; i < RB / S::TB; ++i) {
      const int have = g.q_len > 0 ? g.kv_len - k0 - i * S::TB : 0;
      tile_loader<T, D, S::TB, NW, WHOLE>(from_k, g.k_s, g.d, w, lane).load(i * S::TB, have, smem + RING + i * TILE);
      tile_loader<T, D, S::TB, NW, WHOLE>(from_v, g.v_s, g.d, w, lane).load(i * S::TB, have, smem + RING + RB * D + i * TILE);
    }
  }
  // (again before a second walk, whose registers then leave the first walk's alone)
  auto load_own = [&] {
    if constexpr (!PAIRED) {
      const T* const from_k = there ? (const T*)g.k + r * g.k_z + (row0 + (lane & 31)) * g.k_s + kcol : nullptr;
      const T* const from_v = there ? (const T*)g.v + r * g.v_z + (row0 + (lane & 31)) * g.v_s + kcol : nullptr;
#pragma unroll
      for (int i = 0; i < S::NF; ++i) {
        fk[i] = own_frag<T, D, WHOLE>(from_k, i, g.d, lane);
        fv[i] = own_frag<T, D, WHOLE>(from_v, i, g.d, lane);
      }
    }
  };
  load_own();
  const S at(lane);
  const float c = EXTRA ? 1.f : g.c;
  tile_loader<T, D, S::TB, NW, WHOLE> qs((const T*)g.q + r * g.q_z + q_row0 * g.q_s, g.q_s, g.d, w, lane);
  tile_loader<T, D, S::TB, NW, WHOLE> dos((const T*)g.dout + r * g.do_z + q_row0 * g.do_s, g.do_s, g.d, w, lane);
  const T *const q_at = qs.src, *const do_at = dos.src;
  f16v dk[S::ND], dv[S::ND];               // [column][key]
  auto request = [&](int j, int slot) {    // tile j of all heads' tiles
    const int h = kh * g.group + (tiles ? j / tiles : 0), t = t0 + (tiles ? j % tiles : 0), q0 = t * S::TB, have = j < all ? min(g.q_len - q0, S::TB) : 0;
    qs.src = q_at + (int64_t)h * g.d;
    dos.src = do_at + (int64_t)h * g.d;
    T* const to = smem + slot * (2 * TILE);
    qs.load(q0, have, to);
    dos.load(q0, have, to + TILE);
    // statistics: a wavefront an array, all of them the positions; zeros behind the last row
    const int64_t row = q_row0 + q0, stat = ((int64_t)r * g.heads + h) * rows + row;
    const int array = w & 3;
    const void* const from = array == 0 ? (const void*)(g.lse2 + stat) : array == 1 ? (const void*)(g.dot + stat) : array == 2 ? (const void*)(g.lo + r * rows + row) : (const void*)(g.hi + r * rows + row);
    int* const st = stats + slot * STATS;
    if (lane < S::TB) {
      lds_load4(scalar_rsrc(from, have * 4), __builtin_amdgcn_readfirstlane(lds_addr_of((const uint16_t*)(st + array * S::TB))), lane * 4);
      lds_load4(scalar_rsrc(g.pos_of + r * rows + row, have * 4), __builtin_amdgcn_readfirstlane(lds_addr_of((const uint16_t*)(st + 4 * S::TB))), lane * 4);
    }
  };
  auto walk = [&](auto clean) {
#pragma unroll
    for (int i = 0; i < S::ND; ++i) dk[i] = dv[i] = all16(0.f);
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) request(begin + i, i);
    int slot = 0, free = STAGES - 1;
    for (int j = begin; j < all; ++j) {
      wait_and_barrier<(STAGES - 2) * LOADS>();
      request(j + STAGES - 1, free);
      T* const at_tiles = smem + slot * (2 * TILE);
      const int* const at_stats = stats + slot * STATS;
      free = slot;
      slot = slot == STAGES - 1 ? 0 : slot + 1;
      const int h = kh * g.group + j / tiles, t = t0 + j % tiles;
      const float slope2 = EXTRA == kGeneral && g.slopes ? g.slopes[r * g.slopes_z + h] * kLog2e : 0.f;
#pragma unroll 1
      for (int i = half; i < (PAIRED ? half + 1 : NB); ++i) {
        const int gi = t * NB + i;
        if (gi >= n_groups) continue;
        wave_range gr;
        if (plain) {
          gr = plain_range_of(g, gi * 32, 32);
          if (gi * 32 + 32 > g.q_len) gr.lo_max = INT_MAX;                 // the rows that there are not
        } else {
          const i4v x = groups[gi];
          gr = wave_range{x[0], x[1], x[2], x[3]};
        }
        if (gr.lo_min >= wk0 + 32 || gr.hi_max <= wk0) continue;
        const T* const qt = at_tiles + i * 32 * D;
        const int* const st = at_stats + 32 * i + ((lane >> 5) << 2);
        f16v x, dp, bend;
        if constexpr (PAIRED) {
          x = at.first(qt, own_k, all16(0.f));
          dp = at.first(qt + TILE, own_v, all16(0.f));
        } else {
          x = at.first(qt, fk, all16(0.f));
          dp = at.first(qt + TILE, fv, all16(0.f));
        }
        if (EXTRA) shape_scores_back<EXTRA>(g, x, bend, slope2, [&](int e) { return distance(st[4 * S::TB + acc_row(e, 0)], key); });
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const f4v l2 = *reinterpret_cast<const f4v*>(st + 8 * e4), nd = *reinterpret_cast<const f4v*>(st + S::TB + 8 * e4);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int e = 4 * e4 + u;
            x[e] = exp2_fast(__builtin_fmaf(x[e], c, -l2[u]));
            dp[e] = (dp[e] + nd[u]) * x[e];
            if (EXTRA) dp[e] *= bend[e];
          }
        }
        const bool inside = wk0 >= gr.lo_max && wk0 + 32 <= gr.hi_min;
        if (!inside) {
#pragma unroll
          for (int e4 = 0; e4 < 4; ++e4) {
            const i4v lo = *reinterpret_cast<const i4v*>(st + 2 * S::TB + 8 * e4), hi = *reinterpret_cast<const i4v*>(st + 3 * S::TB + 8 * e4);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const bool seen = key >= lo[u] && key < hi[u];
              x[4 * e4 + u] = seen ? x[4 * e4 + u] : 0.f;
              dp[4 * e4 + u] = seen ? dp[4 * e4 + u] : 0.f;
            }
          }
        }
        constexpr bool CLEAN = decltype(clean)::value;
        if (TWO) {
          at.template second_in_two<CLEAN>(qt + TILE, x, dv);
          at.template second_in_two<CLEAN>(qt, dp, dk);
        } else {
          at.template second<CLEAN>(qt + TILE, x, dv);
          at.template second<CLEAN>(qt, dp, dk);
        }
      }
    }
    wait_and_barrier<0>();
  };
  walk(std::false_type());
  const bool again = block_any<NW>(there && (not_finite(dk) || not_finite(dv)), w, lane, (int*)(smem + RING) - NW);
  if (again) {
    load_own();
    walk(std::true_type());
  }
  if constexpr (PAIRED) {
    // the two halves' sums, as they lie in the lanes
    f4v* const part = reinterpret_cast<f4v*>(smem) + (w & 3) * (2 * S::ND * 4 * 64) + lane;
    __syncthreads();
    if (half == 1) {
#pragma unroll
      for (int i = 0; i < S::ND; ++i)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          part[(i * 4 + e4) * 64] = f4v{dk[i][4 * e4], dk[i][4 * e4 + 1], dk[i][4 * e4 + 2], dk[i][4 * e4 + 3]};
          part[((S::ND + i) * 4 + e4) * 64] = f4v{dv[i][4 * e4], dv[i][4 * e4 + 1], dv[i][4 * e4 + 2], dv[i][4 * e4 + 3]};
        }
    }
    __syncthreads();
    if (half == 0) {
#pragma unroll
      for (int i = 0; i < S::ND; ++i)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const f4v a = part[(i * 4 + e4) * 64], c = part[((S::ND + i) * 4 + e4) * 64];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            dk[i][4 * e4 + u] += a[u];
            dv[i][4 * e4 + u] += c[u];
          }
        }
    }
    __syncthreads();
    if (half == 1) return;
  }
#pragma unroll
  for (int i = 0; i < S::ND; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) dk[i][e] *= g.scale;
  char* const strip = (char*)smem + w * STRIP;
  auto put = [&](auto to_k, auto to_v, int64_t k_s, int64_t v_s, auto wh) {
    typedef std::remove_pointer_t<decltype(to_k)> U;
    store_rows<U, D, decltype(wh)::value>(dk, strip, to_k, k_s, g.kv_len - wk0, g.d, lane, sizeof(T) == 4 && g.run);
    store_rows<U, D, decltype(wh)::value>(dv, strip, to_v, v_s, g.kv_len - wk0, g.d, lane, sizeof(T) == 4 && g.run);
    if (!again) return;
    __threadfence_block();
    for (int h = 0; h < g.group; ++h) {
      // the rows of this block's tiles of the head
      const int from = (t0 + min(max(begin - h * tiles, 0), tiles)) * S::TB, to = min(g.q_len, (t0 + min(max(all - h * tiles, 0), tiles)) * S::TB);
      const int64_t head = (int64_t)(kh * g.group + h) * g.d;
      auto seen = [&](int q, int i) { return wk0 + i >= g.lo[r * rows + q_row0 + q] && wk0 + i < g.hi[r * rows + q_row0 + q]; };
      add_not_finite<T, D>(do_at + head, g.do_s, g.d, from, to, to_v, v_s, min(WR, g.kv_len - wk0), lane, seen, [&](int q, int i) {
        return pair_weight(q_at + q * g.q_s + head, (const T*)g.k + r * g.k_z + (row0 + i) * g.k_s + kcol, g.d, g.scale, g.cap2 > 0.f, lane);
      });
      add_not_finite<T, D>(q_at + head, g.q_s, g.d, from, to, to_k, k_s, min(WR, g.kv_len - wk0), lane, seen, [](int, int) { return 0.f; });
    }
  };
  if (g.splits == 1) {
    put((T*)g.dk + r * g.dk_z + row0 * g.dk_s + kcol, (T*)g.dv + r * g.dv_z + row0 * g.dv_s + kcol, g.dk_s, g.dv_s, std::integral_constant<bool, WHOLE>());
  } else {
    float* const to = g.part + (((int64_t)split * g.by_groups.d + blk.grp) * g.kv_len + wk0) * (2 * D);
    put(to, to + D, 2 * D, 2 * D, std::false_type());
  }
}

// dk and dv from the splits' parts, [split][replica, sequence, key head][key][dk | dv]
template <typename T, int D> __global__ __launch_bounds__(THREADS) void attend_dkv_join_kernel(const attend_args g) {
  const int64_t rows = (int64_t)g.n * g.seqs * g.kv_heads * g.kv_len, i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * THREADS + threadIdx.x, row = i / D;
  const int col = (int)(i % D);
  if (row >= rows || col >= g.d) return;
  float dk = 0.f, dv = 0.f;
  for (int s = 0; s < g.splits; ++s) {
    dk += g.part[((int64_t)s * rows + row) * (2 * D) + col];
    dv += g.part[((int64_t)s * rows + row) * (2 * D) + D + col];
  }
  const int64_t grp = row / g.kv_len, key = row % g.kv_len;
  const int kh = (int)(grp % g.kv_heads), b = (int)(grp / g.kv_heads % g.seqs), r = (int)(grp / g.kv_heads / g.seqs);
  const int64_t at = (int64_t)b * g.kv_len + key, c = (int64_t)kh * g.d + col;
  hdet_st((T*)g.dk + r * g.dk_z + at * g.dk_s + c, dk);
  hdet_st((T*)g.dv + r * g.dv_z + at * g.dv_s + c, dv);
}

// ---------------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------------
template <typename A> attend_args common_args(const A& a) {
  attend_args g = {};
  g.q = a.q.dev; g.q_s = a.q.row_stride; g.q_z = a.q.replica_stride;
  g.k = a.k.dev; g.k_s = a.k.row_stride; g.k_z = a.k.replica_stride;
  g.v = a.v.dev; g.v_s = a.v.row_stride; g.v_z = a.v.replica_stride;
  g.slopes = a.slopes_dev; g.slopes_z = a.slopes_stride;
  g.pos = a.positions_dev; g.first = a.first_dev; g.end = a.end_dev;
  g.n = a.n_replicas; g.seqs = a.seqs; g.q_len = a.q_len; g.kv_len = a.kv_len; g.heads = a.heads; g.kv_heads = a.kv_heads; g.group = a.heads / a.kv_heads;
  g.d = a.head_dim; g.causal = a.causal; g.window = a.window; g.splits = 1;
  g.scale = (float)a.scale; g.c = (float)(a.scale * 1.4426950408889634); g.cap2 = (float)(a.softcap * 1.4426950408889634);
  // (scale / cap beyond fp32 is as good at 1e37: products from 1e-36 on are at the cap with either, and one of 0 stays 0)
  g.inv_cap = a.softcap > 0 ? (float)std::min(1.0 / a.softcap, 1e37 / std::max(fabs(a.scale), 1e-30)) : 0.f;
  g.by_heads = divisor_of(a.heads); g.by_kv_heads = divisor_of(a.kv_heads); g.by_seqs = divisor_of(a.seqs); g.by_group = divisor_of(g.group);
  // bfloat16 inputs: a score off by 1e-7 of a cap up to 1000 moves p by no more than 2^-13 of itself, where its rounding takes 2^-9
  g.close = a.dtype == HDET_TYPE_F32 || a.softcap > 1000.0;
  return g;
}
// whole 16-byte pieces, and a tile within 31 bits
bool whole(const hdet_rows& m, int size, int d) {
  const int64_t mask = 16 / size - 1;
  return ((uintptr_t)m.dev & 15) == 0 && ((m.row_stride | m.replica_stride | d) & mask) == 0 && m.row_stride < (int64_t)1 << 23;
}
// `nx` row blocks of each group
void set_blocks(attend_args& g, unsigned nx, unsigned groups) {
  g.total = nx * groups;
  g.by_nx = divisor_of(nx);
  g.by_groups = divisor_of(groups);
  g.by_own = divisor_of(groups >> 3);
  // longest row blocks first while there are few rounds of them
  g.heavy_first = nx && g.total <= (nx >= 8 ? 16u : 8u) * (unsigned)hdet_compute_units();
}
dim3 grid_of(unsigned blocks) {
  const unsigned x = blocks < (1u << 20) ? blocks : 1u << 20;
  return dim3(x, (blocks + x - 1) / x);
}
// what scores need: more than a product with a constant, also where a scale of 0 or below turns the maximum around, or is 0 in fp32 (0 times a masked
// score's infinity)
template <typename A> int extra(const A& a, const attend_args& g) {
  return a.slopes_dev || !(g.c > 0.f) || (a.softcap > 0 && g.close) ? kGeneral : a.softcap > 0 ? kCapped : kPlain;
}

// f(type, D, EXTRA, WHOLE); rows that are not whole pieces take the general scores too
template <typename F> void with_shape(int dtype, int d, int ex, bool wh, F f) {
  typedef std::integral_constant<int, kPlain> plain;
  typedef std::integral_constant<int, kGeneral> general;
  auto with_flags = [&](auto t, auto dd) {
    typedef std::integral_constant<int, sizeof(t) == 2 ? kCapped : kGeneral> capped;
    if (!wh) f(t, dd, general(), std::false_type());
    else if (ex == kGeneral) f(t, dd, general(), std::true_type());
    else if (ex == kCapped) f(t, dd, capped(), std::true_type());
    else f(t, dd, plain(), std::true_type());
  };
  auto with_d = [&](auto t) {
    if (d <= 64) with_flags(t, std::integral_constant<int, 64>());
    else with_flags(t, std::integral_constant<int, 128>());
  };
  if (dtype == HDET_TYPE_BF16) with_d(uint16_t());
  else with_d(float());
}

// Parts of the keys for few queries, 0: the queries fill the chip.  Up to 16 queries: always a part at least.  More: where blocks of 32 rows, whose
// four wavefronts divide the keys, are no more than fit the chip at once, a block's way being four times as short (us; 128 queries a block, 32):
//   blocks of 32   8 x 8 x 512 keys, 64 columns 256: 12.1, 9.4     fp32 45, 17       16 x 8 x 1024 512: 19.6, 13.8
//                  8 x 8 x 2048 512: 33.5, 18.0      8 x 8 x 4096 1024: 62, 43.5
//   128 columns    8 x 512 128: 15.9, 11.2      32 x 512 queries of 8192 keys 512: 194, 108     16 x 2048 1024: 47, 61
// (Under 128 keys two or more of the four wavefronts have nothing: 32 keys of 16 x 4, fp32, 7.8, 9.4.  With more blocks the join, 64 to 128 KB of LDS
// a block and four times the tiles cost more: 6 x 333 keys of 8 x 128 13, 33.)
int few_splits(int n, int seqs, int q_len, int kv_len, int heads, int kv_heads, int head_dim, int window) {
  const int64_t pairs = (int64_t)(heads / kv_heads) * q_len, groups = (int64_t)n * seqs * kv_heads, cus = hdet_compute_units();
  if (pairs == 0 || groups == 0) return 0;
  const int64_t seen = (int64_t)window + (q_len < RB ? q_len : RB), keys = window && seen < kv_len ? seen : kv_len, few = groups * ((pairs + 31) / 32);
  if (q_len > 16 && (keys < 128 || few > (keys < 1024 ? cus : keys < 2048 ? 2 * cus : 4 * cus) / (head_dim > 64 && keys >= 1024 ? 2 : 1))) return 0;
  int64_t s = (2 * cus + few - 1) / few, most = keys < 1024 ? 1 : (keys + 255) / 256;
  if (s > most) s = most;
  return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}
constexpr size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// Parts of a block's walk in the backward pass, of `tiles` tiles: where there are fewer blocks than CUs, two tiles at least a part; up to two blocks
// a CU of eight tiles at least and, of up to 64 columns, four of sixteen, since one or two blocks leave a CU waiting (the backward pass, us: 8 x 8 x
// 1024 tokens, 8 heads of 64 over 2: 128, 100; 4096 of 8 x 64: 235, 166; 8192 of 4 x 64: 453, 220; 4096 of 8 over 2 x 128: 303, 234; fp32 2 x 2048 of
// 8 x 128: 954, 604.  Four blocks a CU of 128 columns: 2 x 2048 of 16 x 128 272, 305).
int parts_of(int64_t blocks, int64_t tiles, int head_dim) {
  if (blocks == 0) return 1;
  const int64_t cus = hdet_compute_units();
  int64_t s = std::max(std::min(cus / blocks, tiles / 2), std::min(2 * cus / blocks, tiles / 8));
  if (head_dim <= 64) s = std::max(s, std::min(4 * cus / blocks, tiles / 16));
  return (int)(s < 1 ? 1 : s > 16 ? 16 : s);
}
// Keys (queries) that 128 queries (keys) see of a sequence of `len`, without arrays of ranges
int within(int window, int len) { return window && window < len - RB ? window + RB : len; }
// .. and parts of two tiles at least
int dkv_most(int window, int q_len, int group) { return (int)std::max<int64_t>(1, (int64_t)((within(window, q_len) + 63) / 64) * group / 2); }
// .. over the keys for dq; over the query tiles of the heads that share a key head for dk and dv
int dq_splits(int n, int seqs, int q_len, int kv_len, int heads, int head_dim) {
  return parts_of((int64_t)n * seqs * heads * ((q_len + RB - 1) / RB), kv_len < 512 ? 1 : (kv_len + 63) / 64, head_dim);
}
int dkv_splits(int n, int seqs, int q_len, int kv_len, int heads, int kv_heads, int head_dim) {
  return parts_of((int64_t)n * seqs * kv_heads * ((kv_len + RB - 1) / RB), (int64_t)((q_len + 63) / 64) * (heads / kv_heads), head_dim);
}

struct backward_layout { size_t lse2, dot, lo, hi, pos, groups, lacks, part, total; };
backward_layout layout_of(int n, int seqs, int q_len, int kv_len, int heads, int kv_heads, int d) {
  const size_t rows = (size_t)n * seqs * q_len;
  const size_t wide = d <= 64 ? 64 : 128, keys = (size_t)n * seqs * kv_len;
  const size_t q_parts = dq_splits(n, seqs, q_len, kv_len, heads, d), k_parts = dkv_splits(n, seqs, q_len, kv_len, heads, kv_heads, d);
  // (the parts of dq have been joined when those of dk and dv are made)
  const size_t dq_part = q_parts > 1 ? q_parts * rows * heads * wide * 4 : 0, dkv_part = k_parts > 1 ? k_parts * keys * kv_heads * 2 * wide * 4 : 0;
  backward_layout l;
  l.lse2 = 0;
  l.dot = l.lse2 + up256(rows * heads * 4);
  l.lo = l.dot + up256(rows * heads * 4);
  l.hi = l.lo + up256(rows * 4);
  l.pos = l.hi + up256(rows * 4);
  l.groups = l.pos + up256(rows * 4);
  l.lacks = l.groups + up256((size_t)n * seqs * ((q_len + 31) / 32) * 16);
  l.part = l.lacks + (q_parts > 1 ? up256(q_parts * rows * heads * 4) : 0);
  l.total = rows ? l.part + up256(dq_part > dkv_part ? dq_part : dkv_part) : 0;
  return l;
}

}  // namespace

size_t hdet_attend_bytes(int n, int seqs, int q_len, int kv_len, int heads, int kv_heads, int head_dim) {
  const int s = few_splits(n, seqs, q_len, kv_len, heads, kv_heads, head_dim, 0);   // (a window: no more parts)
  if (s <= 1) return 0;
  const size_t ncg = ((size_t)(heads / kv_heads) * q_len + 31) / 32;
  return up256((size_t)n * seqs * kv_heads * ncg * s * 32 * ((head_dim <= 64 ? 64 : 128) + 2) * 4);
}
size_t hdet_attend_backward_bytes(int n, int seqs, int q_len, int kv_len, int heads, int kv_heads, int head_dim) {
  return layout_of(n, seqs, q_len, kv_len, heads, kv_heads, head_dim).total;
}

hipError_t hdet_launch_attend(const hdet_attention_args& a, hipStream_t s) {
  attend_args g = common_args(a);
  const int size = a.dtype == HDET_TYPE_BF16 ? 2 : 4;
  g.out = a.out.dev; g.out_s = a.out.row_stride; g.out_z = a.out.replica_stride;
  g.lse = a.lse_dev;
  if ((int64_t)a.seqs * a.q_len == 0) return hipSuccess;
  const bool wh = whole(a.q, size, a.head_dim) && whole(a.k, size, a.head_dim) && whole(a.v, size, a.head_dim) && whole(a.out, size, a.head_dim);
  const int splits = few_splits(a.n_replicas, a.seqs, a.q_len, a.kv_len, a.heads, a.kv_heads, a.head_dim, a.window);
  if (splits) {
    const int64_t pairs = (int64_t)g.group * a.q_len, groups = (int64_t)a.n_replicas * a.seqs * a.kv_heads;
    g.splits = splits;
    g.part = (float*)a.workspace_dev;
    g.total = (unsigned)(groups * ((pairs + 31) / 32) * splits);
    with_shape(a.dtype, a.head_dim, extra(a, g), wh, [&](auto t, auto d, auto ex, auto w) {
      typedef decltype(t) T;
      hipLaunchKernelGGL((attend_few_kernel<T, d, ex, w>), grid_of(g.total), dim3(few_waves<T, d>() * 64), 0, s, g);
      if (splits > 1) hipLaunchKernelGGL((attend_join_kernel<T, d>), grid_of((unsigned)((groups * pairs + NWV - 1) / NWV)), dim3(THREADS), 0, s, g);
    });
    return hipGetLastError();
  }
  const unsigned nx = (a.q_len + RB - 1) / RB;
  set_blocks(g, nx, (unsigned)a.n_replicas * a.seqs * a.heads);
  with_shape(a.dtype, a.head_dim, extra(a, g), wh, [&](auto t, auto d, auto ex, auto w) {
    hipLaunchKernelGGL((attend_kernel<decltype(t), d, ex, w>), grid_of(g.total), dim3(THREADS), 0, s, g);
  });
  return hipGetLastError();
}

hipError_t hdet_launch_attend_backward(const hdet_attention_grad_args& a, hipStream_t s) {
  attend_args g = common_args(a);
  const int size = a.dtype == HDET_TYPE_BF16 ? 2 : 4;
  g.o = a.out.dev; g.o_s = a.out.row_stride; g.o_z = a.out.replica_stride;
  g.dout = a.dout.dev; g.do_s = a.dout.row_stride; g.do_z = a.dout.replica_stride;
  g.dq = a.dq.dev; g.dq_s = a.dq.row_stride; g.dq_z = a.dq.replica_stride;
  g.dk = a.dk.dev; g.dk_s = a.dk.row_stride; g.dk_z = a.dk.replica_stride;
  g.dv = a.dv.dev; g.dv_s = a.dv.row_stride; g.dv_z = a.dv.replica_stride;
  g.lse_in = a.lse_dev;
  const backward_layout l = layout_of(a.n_replicas, a.seqs, a.q_len, a.kv_len, a.heads, a.kv_heads, a.head_dim);
  char* const w8 = (char*)a.workspace_dev;
  g.lse2 = (float*)(w8 + l.lse2); g.dot = (float*)(w8 + l.dot);
  g.lo = (int*)(w8 + l.lo); g.hi = (int*)(w8 + l.hi); g.pos_of = (int*)(w8 + l.pos); g.groups = (i4v*)(w8 + l.groups);
  g.part = (float*)(w8 + l.part);
  g.lacks = (float*)(w8 + l.lacks);
  bool wh = true;
  for (const hdet_rows* m : {&a.q, &a.k, &a.v, &a.out, &a.dout, &a.dq, &a.dk, &a.dv}) wh = wh && (!m->dev || whole(*m, size, a.head_dim));
  // few queries: dk and dv are made of few dz and p, whose rounding in one part shows (two queries of 4 heads to a key head: dk off by up to 1.7 times its own rounding; many
  // queries: 1.42 times; 8 x 16 x 256 queries in two parts: the backward pass 125 -> 152 us)
  const bool two = a.dtype == HDET_TYPE_BF16 && (int64_t)g.group * a.q_len <= 192;
  const unsigned nq = (a.q_len + RB - 1) / RB, nk = (a.kv_len + RB - 1) / RB;
  with_shape(a.dtype, a.head_dim, extra(a, g), wh, [&](auto t, auto d, auto ex, auto w) {
    typedef decltype(t) T;
    set_blocks(g, nq, (unsigned)a.n_replicas * a.seqs * a.heads);
    // (a window shortens the walks: no more parts than the workspace has)
    g.splits = dq_splits(a.n_replicas, a.seqs, a.q_len, within(a.window, a.kv_len), a.heads, a.head_dim);
    g.total *= g.splits;
    if (g.total) hipLaunchKernelGGL((attend_dq_kernel<T, d, ex, w>), grid_of(g.total), dim3(THREADS), 0, s, g);
    if (g.total && g.splits > 1)
      hipLaunchKernelGGL((attend_dq_join_kernel<T, d>), grid_of((unsigned)(((int64_t)a.n_replicas * a.seqs * a.q_len * a.heads * d + THREADS - 1) / THREADS)), dim3(THREADS), 0, s, g);
    set_blocks(g, nk, (unsigned)a.n_replicas * a.seqs * a.kv_heads);
    g.splits = std::min(dkv_splits(a.n_replicas, a.seqs, a.q_len, a.kv_len, a.heads, a.kv_heads, a.head_dim), dkv_most(a.window, a.q_len, g.group));
    g.total *= g.splits;
    // query tiles of a part: 128 keys are seen by window + 127 queries in a row, where that is all the mask says
    constexpr int tb = shape<T, d>::TB;
    int64_t tiles = (a.q_len + tb - 1) / tb;
    if (a.causal && a.window && !a.positions_dev && !a.first_dev && !a.end_dev) tiles = std::min(tiles, ((int64_t)a.window + RB - 2 + tb - 1) / tb + 1);
    const int64_t share = (tiles * g.group + g.splits - 1) / g.splits;
    for (g.run = 0; g.total && (g.run == 0 || (int64_t)g.run * run_tiles<T, d>() < share); ++g.run) {
      if (two) hipLaunchKernelGGL((attend_dkv_kernel<T, d, ex, w, sizeof(T) == 2>), grid_of(g.total), dim3(dkv_threads<T, d>()), 0, s, g);
      else hipLaunchKernelGGL((attend_dkv_kernel<T, d, ex, w, false>), grid_of(g.total), dim3(dkv_threads<T, d>()), 0, s, g);
    }
    if (g.total && g.splits > 1)
      hipLaunchKernelGGL((attend_dkv_join_kernel<T, d>), grid_of((unsigned)(((int64_t)a.n_replicas * a.seqs * a.kv_heads * a.kv_len * d + THREADS - 1) / THREADS)), dim3(THREADS), 0, s, g);
  });
  return hipGetLastError();
}
