// Output layer with its softmax cross-entropy in pieces of the vocabulary, N replicas:
//
//   z = h W^T + b,  loss = log sum exp z - z_label,  dz = (softmax(z) - onehot) / c,  dh = dz W,  dW = dz^T h,  db = sum_rows dz
//
// No more than `piece` classes of z and dz exist at a time: a first round forms each row's reference and sum of exponentials, a second
// forms z again, dz from it, and with dz the piece's share of dh (added up in fp32) and its rows of dW and db.
//
//  * Where h and W are made of whole 16-byte chunks -- copies are made of rows that are not -- z never leaves the matrix cores' registers:
//    one product leaves reference and sum of each tile's part of a row, a second dz (hdet_bgemm_walk_kernel).  Rows of whole chunks at
//    other boundaries take z through memory in fp32, by pieces that are smaller by as much.
//  * Exponentials are exp2(z log2(e) - r) with r the whole number next to max log2(e): tiles and pieces refer to each other by exact powers
//    of two.  The label's z is taken times the same fp32 log2(e): 64 bits of it there would leave 1.3e-8 of the logit's size in the loss
//    (-4e-5 for a row certain of a label at 3008).
//  * dz is held as c dz = softmax - onehot and the products' results are divided by c: at a label it is next to -1, which a bfloat16 holds
//    to 2^-9 of itself, where (softmax - onehot) / c lies anywhere between two powers of two (dh against 64 bits: 2.9e-3 of its norm with
//    the division before the rounding).
//  * dz leaves as bfloat16 -- what the matrix cores multiply -- for dh and a bfloat16 dW, whose own rounding is as coarse.  An fp32 dW
//    takes dz in three bfloat16 parts, 24 bits: they stand below each other as rows, beside three copies of h, and make one product of
//    three times the rows.  (Two fp16 parts take two thirds of that product -- 4 x 8192 rows of 1024, 32000 classes: the call 9.3 ms for
//    10.8 -- but hold nothing below about 2^-40: the gradient of a class that is never likely came out as 0.)
//  * Bound by the products and by the exponentials and stores at their tiles' ends.  8 x 4096 rows of 512, 32000 classes, bf16 dW, us:
//    statistics 1086 (1.0 PFLOP/s), dz 1318 (0.8), dh 818 (1.3), dW 880 (1.2).

#include <type_traits>

#include "hdet_ops.h"
#include "hdet_elem.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;
constexpr int kRowChunk = 128;                          // rows of a block's column sums in tiles
constexpr size_t kSmallRoom = (size_t)64 << 20;         // z and dz take that much where they pass through memory, if not all of them fits what dz alone takes
// Most that z takes in a call for the losses alone (us, rows one element off a 16-byte boundary, 64 / 128 / 256 MB: 8 x 4096 rows of 512,
// 32000 classes 7677 / 5859 / 6561, 4 x 8192 of 1024, 32000 8922 / 8088 / 8958, 4096 of 1024, 50000 1709 / 1664 / 1764)
constexpr size_t kLossRoom = (size_t)128 << 20;
constexpr size_t kPieceBytes = (size_t)1 << 30;         // most that dz of a piece takes where the caller does not say

// Memory of a call, in the order it is carved.  What a member names: [replica][...].
struct vocab_layout {
  int piece, pieces;        // classes at a time where z stays in registers
  int small_piece;          // ... where it goes through memory
  int planes;               // bfloat16 parts of dz
  int64_t bias_pitch;
  int64_t width8;           // a row of h and W in whole 16-byte pieces
  int h_copies;             // copies of h in such rows, zeros in those that do not count: as many below each other as dz has parts;
                            // without dw one where h's own rows are no whole pieces
  size_t inv, labels, ref, a, sum, zy, bias, dz, h, w, acc, part, split, split_bytes, total;
};
size_t up(size_t x) { return (x + 255) & ~(size_t)255; }
int64_t up8(int64_t x) { return (x + 7) & ~(int64_t)7; }
// rows of a block of hdet_vocab_grad_kernel: 128, fewer until there are two blocks a compute unit
int rows_each(int n, int64_t rows, int cols) {
  int each = 128;
  while (each > 4 && (rows + each - 1) / each * ((cols + 1023) / 1024) * n < 2 * hdet_compute_units()) each >>= 1;
  return each;
}
// Whether z goes through memory also where it could stay in the matrix cores' registers: up to a tile of 256 x 256 on every fourth compute
// unit, where a tile's long way from the first load to the last store (12 us for its statistics, 18 for dz in three parts) counts for more
// than the passes over z, and up to 8192 classes, whose rows the statistics walk one block each.  us of the call, registers / memory
// (tiles):  4 x 128 rows of 64, 512 classes, fp32 dW (8) 51 / 37;  3 x 159 of 896, 523 (9) 78 / 49;  4 x 256 of 1024, 2048 (32) 101 / 75;
// 1024 of 512, 4096 (64) 100 / 85;  256 of 512, 16384 (64) 95 / 107;  100 of 90, 9600 (38) 63 / 66;  2 x 512 of 256, 8192 (128) 85 / 169
bool small_call(int n, int64_t rows, int classes) {
  return classes <= 8192 && 4 * ((rows + 255) / 256 * ((classes + 255) / 256) * n) <= hdet_compute_units();
}

// Classes at a time.  A piece's dW is one product with the rows as its contraction: it wants whole rounds of 256 x 256 tiles over the
// compute units, and every piece costs about a twelfth of a round in launches, first loads and passes over the sum of dh.  us, by classes a
// piece (rounds of each):
//   8 x 4096 rows of 512, 32000 classes, bf16 dW: 1536 (3/8) 4876, 2048 (1/2) 4484, 4096 (1) 4161, 6400 (1.6) 4110, 8192 (2) 4028,
//     16384 (4) 3947, 32000 3860
//   4 x 8192 rows of 1024, 32000 classes, fp32 dW: 2048 (1/2) 12739, 4096 (1) 10972, 6400 (1.6) 11420, 8192 (2) 10720, 32000 10439
//   4096 rows of 1024, 50000 classes, bf16: 2048 (1/8) 2689, 4096 (1/4) 1883, 8192 (1/2) 1697, 16384 (1) 1550, 32000 (2) 1558, 50000 1684
// Between the two stands kPieceBytes.
// Without a dW nothing wants rounds: pieces alike, as few as fit.
int chosen_piece(int n, size_t class_bytes, int width, int classes, size_t piece_bytes, bool dw) {
  const int64_t tiles = (int64_t)((width + 255) / 256) * n, cus = hdet_compute_units(), columns = (classes + 255) / 256;
  int64_t most = (int64_t)(piece_bytes / class_bytes) / 256;      // columns of tiles that fit
  if (most < 4) most = 4;
  if (most >= columns) most = columns;
  if (!dw) {
    const int64_t pieces = (columns + most - 1) / most;
    return pieces == 1 ? classes : (int)((columns + pieces - 1) / pieces) * 256;
  }
  int64_t best = most;
  double least = 1e30;
  for (int64_t pieces = (columns + most - 1) / most; pieces <= columns && pieces <= 4 * ((columns + most - 1) / most) + 4; ++pieces) {
    const int64_t c = (columns + pieces - 1) / pieces, count = (columns + c - 1) / c;
    const double time = (double)count * ((double)((c * tiles + cus - 1) / cus) + 0.08);
    if (time < least) { least = time; best = c; }
  }
  return best >= columns ? classes : (int)best * 256;
}

// kind: HDET_TYPE_* of dw, or one of HDET_VOCAB_*.  Pieces are made for plan_planes parts of dz that take piece_bytes at most, for a call
// with dw or without.
vocab_layout layout_in(int n, int64_t rows, int width, int classes, int kind, int plan_planes, int piece, size_t piece_bytes = kPieceBytes, bool for_dw = true) {
  vocab_layout l;
  const size_t all = (size_t)n * rows;
  if (piece <= 0) {
    piece = chosen_piece(n, all * 2 * plan_planes, width, classes, piece_bytes, for_dw);
  } else {      // whole tiles of 256 classes, or whole groups of 8 where the caller wants fewer
    if (piece > classes) piece = classes;
    if (piece < classes) piece = piece >= 256 ? piece / 256 * 256 : piece >= 8 ? piece / 8 * 8 : 8;
    if (piece > classes) piece = classes;
  }
  l.piece = piece;
  l.pieces = (classes + piece - 1) / piece;
  size_t room = all * up8(l.piece) * 2 * plan_planes;                               // dz
  const size_t a_class = all * (4 + 2 * plan_planes), small = kSmallRoom;           // z and dz
  const size_t whole = a_class * up8(l.piece);
  if (room < (whole < small ? whole : small)) room = whole < small ? whole : small;
  if (room < a_class * 8) room = a_class * 8;
  const size_t stats = all * 8 * ((size_t)(classes + 255) / 256);                   // the first round's, before there is a dz
  if (room < stats) room = stats;
  size_t fit = room / a_class / 8 * 8;
  l.small_piece = fit < (size_t)l.piece ? (int)fit : l.piece;
  const bool dw = kind >= 0, losses = kind == HDET_VOCAB_LOSSES;
  l.planes = dw ? plan_planes : 1;
  if (!dw) {                                                                        // what is left of that room: z, and one part of dz
    room = all * up8(l.small_piece) * (losses ? 4 : 6);
    if (!losses && room < all * up8(l.piece) * 2) room = all * up8(l.piece) * 2;
    if (losses && room > kLossRoom) room = kLossRoom > all * 32 ? kLossRoom : all * 32;
    if (room < stats) room = stats;
    if (losses && room / (all * 4) / 8 * 8 < (size_t)l.small_piece) l.small_piece = (int)(room / (all * 4) / 8 * 8);
  }
  l.bias_pitch = up8(classes);
  l.width8 = up8(width);
  l.h_copies = dw ? l.planes : l.width8 != width ? 1 : 0;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += up(bytes); return here; };
  l.inv = take((size_t)n * 4);
  l.labels = take(all * 4);
  l.ref = take(all * 4);
  l.a = take(all * 4);
  l.sum = take(all * 8);
  l.zy = take(all * 4);
  l.bias = take((size_t)n * l.bias_pitch * 4);
  l.dz = take(room);
  l.h = take(all * l.h_copies * l.width8 * 2);
  l.w = take(l.width8 != width ? (size_t)n * classes * l.width8 * 2 : 0);
  l.acc = take(!losses && (l.pieces > 1 || l.small_piece < l.piece) ? all * l.width8 * 4 : 0);
  size_t part = (size_t)n * ((rows + kRowChunk - 1) / kRowChunk) * up8(l.piece);
  for (const int cols : {l.small_piece, classes - (classes + l.small_piece - 1) / l.small_piece * l.small_piece + l.small_piece}) {
    const int each = rows_each(n, rows, cols);
    const size_t want = (size_t)n * ((rows + each - 1) / each) * up8(cols);
    if (want > part) part = want;
  }
  l.part = take(losses ? 0 : part * 4);
  // results of pieces of a long contraction: the most that a piece of either kind may take
  l.split_bytes = 0;
  for (const int cols : {l.piece, classes - (l.pieces - 1) * l.piece, l.small_piece, classes - (classes + l.small_piece - 1) / l.small_piece * l.small_piece + l.small_piece})
    for (const hdet_split& sp : {hdet_split_of(n, rows, width, cols), hdet_split_of(n, cols, width, dw ? l.planes * rows : 0)})
      if (!losses && sp.bytes > l.split_bytes) l.split_bytes = sp.bytes;
  l.split = take(l.split_bytes);
  l.total = at;
  return l;
}

// Memory that is enough for a call with a dw of either type is enough without: pieces as large as the smaller of the two allows, at the
// least those of one of the calls with dw, whose own layout less what only dw needs fits it.
vocab_layout layout_of(int n, int64_t rows, int width, int classes, int kind, int piece) {
  if (kind >= 0) return layout_in(n, rows, width, classes, kind, kind == HDET_TYPE_F32 ? 3 : 1, piece);
  int planes = 1, eighths = 8;
  bool for_dw = false;
  auto with = [&](int kind) { return layout_in(n, rows, width, classes, kind, planes, piece, kPieceBytes / 8 * eighths, for_dw); };
  vocab_layout l = with(HDET_VOCAB_NO_DW);
  if (l.pieces > 1 || (size_t)n * rows * 10 * up8(classes) > kSmallRoom) {      // (else one piece for all three of them)
    const size_t f32 = layout_in(n, rows, width, classes, HDET_TYPE_F32, 3, piece).total, bf16 = layout_in(n, rows, width, classes, HDET_TYPE_BF16, 1, piece).total;
    const size_t most = f32 < bf16 ? f32 : bf16;
    while (l.total > most && --eighths > 2) l = with(HDET_VOCAB_NO_DW);
    if (l.total > most) {
      planes = bf16 == most ? 1 : 3;
      eighths = 8;
      for_dw = true;
      l = with(HDET_VOCAB_NO_DW);
    }
  }
  return kind == HDET_VOCAB_NO_DW ? l : with(kind);
}

struct prep_args {
  const int32_t* labels; int32_t* labels_out;
  const float* bias; int64_t bias_z; float* bias_out; int64_t bias_pitch;
  const uint16_t* h; int64_t h_s, h_z; uint16_t* h_out; int width, copies;      // rows of whole 16-byte pieces
  float* inv;
  int64_t rows;
  int classes;
};

}  // namespace

// What a call starts with, [replica] on blockIdx.y: labels that name no class become -1; 1 / rows that count; bias in rows padded with
// -inf; copies of h below each other, zeros in rows that do not count (their dz is 0 and would take a NaN or infinity of h into dW's sum).
__global__ __launch_bounds__(1024) void hdet_vocab_prep_kernel(const prep_args a) {
  const int z = blockIdx.y;
  const int64_t t = (int64_t)blockIdx.x * 1024 + threadIdx.x, step = (int64_t)gridDim.x * 1024;
  const int32_t* lab = a.labels + z * a.rows;
  for (int64_t i = t; i < a.rows; i += step) a.labels_out[z * a.rows + i] = (unsigned)lab[i] < (unsigned)a.classes ? lab[i] : -1;
  if (a.bias_out)
    for (int64_t i = t; i < a.bias_pitch; i += step) a.bias_out[z * a.bias_pitch + i] = i >= a.classes ? -INFINITY : a.bias ? a.bias[z * a.bias_z + i] : 0.f;
  if (a.h_out) {
    const int64_t pieces = a.width / 8, all = a.rows * pieces;
    hdet_u4v* const out = reinterpret_cast<hdet_u4v*>(a.h_out) + z * a.copies * all;
    for (int64_t i = t; i < all; i += step) {
      const int64_t row = i / pieces;
      hdet_u4v v = *reinterpret_cast<const hdet_u4v*>(a.h + z * a.h_z + row * a.h_s + i % pieces * 8);
      if ((unsigned)lab[row] >= (unsigned)a.classes) v = hdet_u4v{0u, 0u, 0u, 0u};
      for (int q = 0; q < a.copies; ++q) out[q * all + i] = v;
    }
  }
  if (blockIdx.x != 0) return;
  __shared__ int part[16];
  int n = 0;
  for (int64_t i = threadIdx.x; i < a.rows; i += 1024) n += (unsigned)lab[i] < (unsigned)a.classes ? 1 : 0;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) n += part[w];
    a.inv[z] = 1.f / (float)(n > 1 ? n : 1);
  }
}

// Reference and sum of a row over the classes so far, and its label's logit; after the last piece its loss.  Block = one row of a piece;
// grid (rows, replicas).
__global__ __launch_bounds__(256) void hdet_vocab_stat_kernel(const float* z, int64_t pitch, int64_t rows, int cols, int v0, const int32_t* labels, float* ref,
                                                              double* sum, float* zy, bool last, float* a_out, float* row_loss) {
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
    const int y = labels[at] - v0;
    float top = r, ly = (unsigned)y < (unsigned)cols ? p[y] : 0.f;
    double all = (double)((part[0] + part[1]) + (part[2] + part[3]));
    if (v0 != 0) {
      const float r0 = ref[at];
      top = fmaxf(r0, r);
      // a side without classes has the sum 0 (or NaN) and no reference
      all = (r0 == -INFINITY ? sum[at] : sum[at] * (double)__builtin_amdgcn_exp2f(r0 - top)) + (r == -INFINITY ? all : all * (double)__builtin_amdgcn_exp2f(r - top));
      if ((unsigned)y >= (unsigned)cols) ly = zy[at];
    }
    ref[at] = top;
    if (last) {      // the row's loss and the factor of its exponentials in dz
      const bool counts = labels[at] >= 0;
      a_out[at] = counts ? (float)(1.0 / all) : 0.f;
      row_loss[at] = counts ? (float)(((double)top + log2(all) - (double)ly * (double)kLog2e) * kLn2) : 0.f;
    } else {
      sum[at] = all;
      zy[at] = ly;
    }
  }
}

// What it leaves after the last piece, from the column tiles' references and sums ([replica][tile][row]); lse: log2 of the sum of exp2(z
// log2(e)).  Rows that do not count: loss and factor 0.
// Block = 64 rows x 4 phases; phase q takes tiles q, q + 4, ..., the phases are added in their order, in 64 bits.
__global__ __launch_bounds__(256) void hdet_vocab_merge_kernel(const float2* part, int tiles, int64_t rows, const int32_t* labels, float* ref, float* a, double* lse, float* row_loss) {
  __shared__ float refs[4][64];
  __shared__ double sums[4][64];
  const int lane = threadIdx.x & 63, q = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * 64 + lane, at = blockIdx.y * rows + row;
  float mx = -INFINITY;
  double s = 0.0;
  if (row < rows) {
    const float2* p = part + (int64_t)blockIdx.y * tiles * rows + row;
#pragma unroll 8
    for (int t = q; t < tiles; t += 4) {
      const float2 v = p[(int64_t)t * rows];
      const float mn = fmaxf(mx, v.x);
      if (v.x != -INFINITY) s = s * (double)__builtin_amdgcn_exp2f(mx - mn) + (double)(v.y * __builtin_amdgcn_exp2f(v.x - mn));
      else s += v.y;
      mx = mn;
    }
  }
  refs[q][lane] = mx;
  sums[q][lane] = s;
  __syncthreads();
  if (q != 0 || row >= rows) return;
  float r[4];
  double p[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) { r[w] = refs[w][lane]; p[w] = sums[w][lane]; }
  const float top = fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3]));
  double sum = 0.0;
#pragma unroll
  for (int w = 0; w < 4; ++w) sum += r[w] == -INFINITY && p[w] == 0.0 && top != -INFINITY ? 0.0 : p[w] * (double)__builtin_amdgcn_exp2f(r[w] - top);
  const bool counts = labels[at] >= 0;
  ref[at] = top;
  a[at] = counts ? (float)(1.0 / sum) : 0.f;
  lse[at] = (double)top + log2(sum);
  if (!counts) row_loss[at] = 0.f;
}

// Row losses where no gradients are wanted: the label's logit by itself.  A wavefront a row; grid (ceil(rows / 4), replicas).
__global__ __launch_bounds__(256) void hdet_vocab_label_kernel(const uint16_t* h, int64_t h_s, int64_t h_z, const uint16_t* w, int64_t w_s, int64_t w_z, const float* bias,
                                                               int64_t bias_pitch, const int32_t* labels, const double* lse, int64_t rows, int width, float* row_loss) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), at = blockIdx.y * rows + row;
  const int lane = threadIdx.x & 63;
  if (row >= rows) return;
  const int y = labels[at];
  if (y < 0) return;
  const uint16_t *p = h + blockIdx.y * h_z + row * h_s, *q = w + blockIdx.y * w_z + y * w_s;
  float s = 0.f;
  for (int c = lane * 8; c < width; c += 512) {
    const hdet_f8 u = hdet_ld8(p + c), v = hdet_ld8(q + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = __builtin_fmaf(u.v[e], v.v[e], s);
  }
  s = hdet_wave_sum(s) + bias[blockIdx.y * bias_pitch + y];
  if (lane == 0) row_loss[at] = (float)((lse[at] - (double)s * (double)kLog2e) * kLn2);
}

// c dz of a piece from z, in PLANES bfloat16 parts, and its sums over `each` rows.  Thread = 4 columns; grid (ceil(pitch / 1024), row
// blocks, replicas).
template <int PLANES>
__global__ __launch_bounds__(256) void hdet_vocab_grad_kernel(const float* z, int64_t pitch, int64_t rows, int each, int cols, int v0, const int32_t* labels, const float* ref,
                                                              const float* a, uint16_t* dz, float* part, int64_t part_pitch) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4, zr = blockIdx.z;
  if (c >= pitch) return;
  const int64_t r0 = (int64_t)blockIdx.y * each, r1 = r0 + each < rows ? r0 + each : rows;
  hdet_f4v sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r) {
    const int64_t at = zr * rows + r;
    const hdet_f4v x = *reinterpret_cast<const hdet_f4v*>(z + at * pitch + c);
    const float f = a[at], rf = ref[at];
    const int y = labels[at] - v0 - c;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = f != 0.f ? __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], kLog2e, -rf)) * f : 0.f;      // (rows that do not count: 0 whatever z is)
      if (e == y) v[e] -= 1.f;
      if (c + e >= cols) v[e] = 0.f;
      sum[e] += v[e];
    }
    uint16_t* p = dz + ((int64_t)zr * PLANES * rows + r) * pitch + c;
#pragma unroll
    for (int q = 0; q < PLANES; ++q) {
      const hdet_u2v b = {hdet_bf16_pack(v[0], v[1]), hdet_bf16_pack(v[2], v[3])};
      *reinterpret_cast<hdet_u2v*>(p + q * rows * pitch) = b;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] -= __uint_as_float(e & 1 ? b[e >> 1] & 0xffff0000u : b[e >> 1] << 16);
    }
  }
  if (part && c < part_pitch) *reinterpret_cast<hdet_f4v*>(part + ((int64_t)zr * gridDim.y + blockIdx.y) * part_pitch + c) = sum;
}

// db of a piece from its column sums, 64 columns x 4 phases a block; the last block column, where row_loss is given: the mean loss.  Grid
// (blocks, replicas).
__global__ __launch_bounds__(256) void hdet_vocab_sums_kernel(const float* part, int parts, int cols, int64_t pitch, float* db, int64_t db_z, const float* inv, const float* row_loss,
                                                              int64_t rows, float* mean) {
  __shared__ double sum[4];
  __shared__ float s[4][64];
  const int z = blockIdx.y, lane = threadIdx.x & 63, ph = threadIdx.x >> 6;
  if (row_loss && blockIdx.x + 1 == gridDim.x) {
    double x = 0.0;
    for (int64_t i = threadIdx.x; i < rows; i += 256) x += (double)row_loss[z * rows + i];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
    if (lane == 0) sum[ph] = x;
    __syncthreads();
    if (threadIdx.x == 0) mean[z] = (float)((sum[0] + sum[1] + sum[2] + sum[3]) * (double)inv[z]);
    return;
  }
  const int col = blockIdx.x * 64 + lane;
  float x = 0.f;
  if (col < cols) {
    const float* p = part + (int64_t)z * parts * pitch + col;
#pragma unroll 4
    for (int i = ph; i < parts; i += 4) x += p[i * pitch];
  }
  s[ph][lane] = x;
  __syncthreads();
  if (ph == 0 && col < cols) db[z * db_z + col] = ((s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane])) * inv[z];
}

// zeros in a matrix of `size`-byte elements (2 or 4).  Grid: hdet_long_grid(rows * width).
__global__ __launch_bounds__(256) void hdet_zero_rows_kernel(void* m, int64_t row_s, int64_t rep_s, int64_t rows, int width, int size) {
  const int64_t i = hdet_long_thread();
  if (i >= rows * width) return;
  const int64_t at = blockIdx.y * rep_s + i / width * row_s + i % width;
  if (size == 2) ((uint16_t*)m)[at] = 0;
  else ((float*)m)[at] = 0.f;
}

hipError_t hdet_launch_zero_rows(const hdet_rows& m, int n_replicas, int64_t rows, int width, int dtype, hipStream_t s) {
  hipLaunchKernelGGL(hdet_zero_rows_kernel, hdet_long_grid(rows * width, n_replicas), dim3(256), 0, s, m.dev, m.row_stride, m.replica_stride, rows, width,
                     dtype == HDET_TYPE_BF16 ? 2 : 4);
  return hipGetLastError();
}

size_t hdet_vocab_bytes(int n_replicas, int64_t rows, int width, int classes, int kind, int piece) {
  return rows == 0 ? 0 : layout_of(n_replicas, rows, width, classes, kind, piece).total;
}
int hdet_vocab_kind(const hdet_vocab_args& a) { return a.dw.dev ? a.dw_dtype : a.dh.dev || a.db_dev ? HDET_VOCAB_NO_DW : HDET_VOCAB_LOSSES; }

hipError_t hdet_launch_vocab_loss(const hdet_vocab_args& a, hipStream_t s) {
  const int n = a.n_replicas, d = a.width, V = a.classes;
  const int64_t M = a.rows;
  hipError_t e;
  if (M == 0) {      // no rows: the sums over none of them
    if ((e = hdet_launch_partial_sum(nullptr, n, 0, 1, 0, a.mean_loss_dev, 1, s)) != hipSuccess) return e;
    if (a.dw.dev && (e = hdet_launch_zero_rows(a.dw, n, V, d, a.dw_dtype, s)) != hipSuccess) return e;
    return a.db_dev ? hdet_launch_partial_sum(nullptr, n, 0, V, 0, a.db_dev, a.db_stride, s) : hipSuccess;
  }
  const vocab_layout l = layout_of(n, M, d, V, hdet_vocab_kind(a), a.piece);
  char* const ws = (char*)a.workspace_dev;
  float *const inv = (float*)(ws + l.inv), *const ref = (float*)(ws + l.ref), *const ra = (float*)(ws + l.a), *const zy = (float*)(ws + l.zy), *const part = (float*)(ws + l.part);
  float* const bias = (float*)(ws + l.bias);
  int32_t* const labels = (int32_t*)(ws + l.labels);
  double* const sum = (double*)(ws + l.sum);
  // operands of the products: the caller's, or copies in rows of whole pieces
  const int copies = l.h_copies;
  hdet_rows h = a.h, w = a.w, hk = a.h;              // hk: what stands beside all parts of dz
  if (copies) hk = {ws + l.h, l.width8, copies * M * l.width8};
  if (l.width8 != d) {
    h = hk;
    w = {ws + l.w, l.width8, V * l.width8};
  }
  const uint16_t *hp = (const uint16_t*)h.dev, *wp = (const uint16_t*)w.dev;
  const bool grads = hdet_vocab_kind(a) != HDET_VOCAB_LOSSES;

  // z = h W^T + bias of the classes from v0 on; in tiles: bias padded
  auto product = [&](int v0, int cols, bool tiles) {
    hdet_bgemm_args g = {};
    g.a = hp; g.lda = h.row_stride; g.a_s[0] = h.replica_stride;
    g.b = wp + v0 * w.row_stride; g.ldb = w.row_stride; g.b_s[0] = w.replica_stride;
    g.m = (int)M; g.n = cols; g.k = l.width8 != d ? (int)l.width8 : d; g.n1 = g.n2 = 1;      // (zeros behind a copy's rows)
    g.bias = tiles ? bias + v0 : a.bias_dev ? a.bias_dev + v0 : nullptr;
    g.bias_bs = tiles ? l.bias_pitch : a.bias_stride;
    g.padded = tiles;
    g.xent.labels = labels; g.xent.row_loss = a.row_loss_dev; g.xent.row_ref = ref; g.xent.row_a = ra; g.xent.row_lse = sum;
    g.xent.invb = 1.f; g.xent.label0 = v0;
    return g;
  };
  const bool tiles = !small_call(n, M, V) && hdet_vocab_tiles_eligible(product(0, V, true));
  const int piece = tiles ? l.piece : l.small_piece, pieces = (V + piece - 1) / piece;
  const int64_t pitch = up8(piece);

  bool copied;
  {
    // (copies of rows that are no whole pieces take a launch of their own)
    const bool copy = copies && l.width8 == d && ((a.h.row_stride | a.h.replica_stride) & 7) == 0 && (reinterpret_cast<uintptr_t>(a.h.dev) & 15) == 0;
    const prep_args p = {a.labels_dev, labels, a.bias_dev, a.bias_stride, tiles ? bias : nullptr, l.bias_pitch, (const uint16_t*)a.h.dev, a.h.row_stride, a.h.replica_stride,
                         copy ? (uint16_t*)(ws + l.h) : nullptr, d, copies, inv, M, V};
    int64_t work = M > l.bias_pitch ? M : l.bias_pitch;
    if (copy && M * d / 8 > work) work = M * d / 8;
    copied = copy;
    int64_t blocks = (work + 1023) / 1024;
    if (blocks > 1024) blocks = 1024;
    hipLaunchKernelGGL(hdet_vocab_prep_kernel, dim3((unsigned)blocks, n), dim3(1024), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (copies && !copied && (e = hdet_launch_pad_rows(a.h, n, M, d, labels, (uint16_t*)(ws + l.h), l.width8, copies, s)) != hipSuccess) return e;
  if (l.width8 != d && (e = hdet_launch_pad_rows(a.w, n, V, d, nullptr, (uint16_t*)(ws + l.w), l.width8, 1, s)) != hipSuccess) return e;
  float* const z = (float*)(ws + l.dz);
  uint16_t* const dz = (uint16_t*)(ws + l.dz + (tiles ? 0 : (size_t)n * M * pitch * 4));
  auto logits = [&](int v0, int cols) {
    hdet_bgemm_args g = product(v0, cols, false);
    g.c = z; g.ldc = pitch; g.c_s[0] = M * pitch;
    return hdet_launch_bgemm(g, true, true, a.bias_dev ? HDET_EPI_BIAS_F32 : HDET_EPI_F32, n, s);
  };

  // first round: every row's reference and sum
  if (tiles) {
    hdet_bgemm_args g = product(0, V, true);
    float2* const stats = (float2*)(ws + l.dz);
    g.xent.part = stats;
    if ((e = hdet_launch_vocab_stat(g, n, s)) != hipSuccess) return e;
    hipLaunchKernelGGL(hdet_vocab_merge_kernel, dim3((unsigned)((M + 63) / 64), n), dim3(256), 0, s, stats, (V + 255) / 256, M, labels, ref, ra, sum, a.row_loss_dev);
    if (!grads)
      hipLaunchKernelGGL(hdet_vocab_label_kernel, dim3((unsigned)((M + 3) / 4), n), dim3(256), 0, s, hp, h.row_stride, h.replica_stride, wp, w.row_stride, w.replica_stride,
                         bias, l.bias_pitch, labels, sum, M, (int)l.width8, a.row_loss_dev);
  } else {
    for (int p = 0; p < pieces; ++p) {
      const int v0 = p * piece, cols = V - v0 < piece ? V - v0 : piece;
      if ((e = logits(v0, cols)) != hipSuccess) return e;
      hipLaunchKernelGGL(hdet_vocab_stat_kernel, dim3((unsigned)M, n), dim3(256), 0, s, z, pitch, M, cols, v0, labels, ref, sum, zy, p + 1 == pieces, ra, a.row_loss_dev);
    }
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;

  // second round: dz of a piece and what comes of it
  for (int p = 0; p < pieces && grads; ++p) {
    const int v0 = p * piece, cols = V - v0 < piece ? V - v0 : piece;
    const int64_t part_pitch = (cols + 3) & ~3;
    const int each = tiles ? kRowChunk : rows_each(n, M, cols), chunks = (int)((M + each - 1) / each);
    if (tiles) {
      hdet_bgemm_args g = product(v0, cols, true);
      g.c = dz; g.ldc = pitch; g.c_s[0] = l.planes * M * pitch;
      g.colsum = a.db_dev ? part : nullptr;
      if ((e = hdet_launch_vocab_grad(g, l.planes, n, s)) != hipSuccess) return e;
    } else {
      if (pieces > 1 && (e = logits(v0, cols)) != hipSuccess) return e;
      const dim3 grid((unsigned)((pitch + 1023) / 1024), chunks, n);
      float* const to = a.db_dev ? part : nullptr;
      if (l.planes == 3) hipLaunchKernelGGL(hdet_vocab_grad_kernel<3>, grid, dim3(256), 0, s, z, pitch, M, each, cols, v0, labels, ref, ra, dz, to, part_pitch);
      else hipLaunchKernelGGL(hdet_vocab_grad_kernel<1>, grid, dim3(256), 0, s, z, pitch, M, each, cols, v0, labels, ref, ra, dz, to, part_pitch);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const bool last = p + 1 == pieces;
    if (a.db_dev || last) {
      const unsigned blocks = (a.db_dev ? (cols + 63) / 64 : 0) + (last ? 1 : 0);
      hipLaunchKernelGGL(hdet_vocab_sums_kernel, dim3(blocks, n), dim3(256), 0, s, part, chunks, cols, part_pitch, a.db_dev + v0, a.db_stride, inv,
                         last ? a.row_loss_dev : nullptr, M, a.mean_loss_dev);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.dh.dev) {
      hdet_bgemm_args g = {};
      g.a = dz; g.lda = pitch; g.a_s[0] = l.planes * M * pitch;
      g.b = wp + v0 * w.row_stride; g.ldb = w.row_stride; g.b_s[0] = w.replica_stride;
      g.c = a.dh.dev; g.ldc = a.dh.row_stride; g.c_s[0] = a.dh.replica_stride;
      g.m = (int)M; g.n = d; g.k = cols;
      g.accum = (float*)(ws + l.acc); g.accum_ld = l.width8; g.accum_bs = M * l.width8;
      g.accum_first = p == 0; g.accum_last = last; g.out_scale = inv;
      g.padded = true;
      const hdet_split sp = hdet_split_of(n, M, d, cols);
      if (sp.pieces > 1) {
        if ((e = hdet_launch_split(g, true, n, sp, (float*)(ws + l.split), {g.c, HDET_TYPE_BF16, g.ldc, g.c_s[0], inv, g.accum, g.accum_ld, g.accum_bs, p == 0, last}, s)) != hipSuccess)
          return e;
      } else if ((e = hdet_launch_bgemm(g, true, false, HDET_EPI_ACCUM_BF16, n, s)) != hipSuccess) {
        return e;
      }
    }
    if (a.dw.dev) {
      const bool f32 = l.planes == 3;
      hdet_bgemm_args g = {};
      g.a = dz; g.lda = pitch; g.a_s[0] = l.planes * M * pitch;
      g.b = (const uint16_t*)hk.dev; g.ldb = hk.row_stride; g.b_s[0] = hk.replica_stride;
      g.c = (char*)a.dw.dev + v0 * a.dw.row_stride * (f32 ? 4 : 2); g.ldc = a.dw.row_stride; g.c_s[0] = a.dw.replica_stride;
      g.m = cols; g.n = d; g.k = (int)(l.planes * M); g.out_scale = inv;
      g.padded = true;
      const hdet_split sp = hdet_split_of(n, cols, d, l.planes * M);
      if (sp.pieces > 1) {
        if ((e = hdet_launch_split(g, false, n, sp, (float*)(ws + l.split), {g.c, a.dw_dtype, g.ldc, g.c_s[0], inv, nullptr, 0, 0, true, true}, s)) != hipSuccess) return e;
      } else if ((e = hdet_launch_bgemm(g, false, false, f32 ? HDET_EPI_SCALED_F32 : HDET_EPI_SCALED_BF16, n, s)) != hipSuccess) {
        return e;
      }
    }
  }
  if (!grads) {
    hipLaunchKernelGGL(hdet_vocab_sums_kernel, dim3(1, n), dim3(256), 0, s, part, 0, 0, 0, a.db_dev, 0, inv, a.row_loss_dev, M, a.mean_loss_dev);
    return hipGetLastError();
  }
  return hipSuccess;
}
