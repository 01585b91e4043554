// C entry points of the language-model operators: argument checks, and the order of the launches.

#include "hdet_ops.h"

#include <limits.h>
#include <math.h>

#include <algorithm>
#include <functional>
#include <initializer_list>

namespace {

// rows a replica: what the launches' grids and 32-bit row numbers hold
constexpr int64_t kMaxRows = (int64_t)1 << 21;
constexpr int64_t kMaxKeys = (int64_t)1 << 28;             // keys a replica: 32-bit key numbers with room to add a tile
constexpr int64_t kMaxHeadColumns = (int64_t)1 << 20;      // columns of all heads of a row

struct argument_checks {
  std::string why;
  bool ok() const { return why.empty(); }
  void need(bool cond, const char* msg) { if (why.empty() && !cond) why = msg; }
  void common(int n, int64_t rows) {
    need(n >= 1 && n <= HDET_MAX_REPLICAS, "n_replicas out of range");
    need(rows >= 0 && rows <= kMaxRows, "rows must be in 0 .. 2^21 per replica");
  }
  void type(int dtype, const char* msg) { need(dtype == HDET_TYPE_F32 || dtype == HDET_TYPE_BF16, msg); }
  // a matrix of rows x width elements of `size` bytes; `out`: no two elements share memory
  void matrix(const char* name, const hdet_rows& m, int n, int64_t rows, int64_t width, int size, bool required, bool out) {
    if (!ok()) return;
    const std::string s(name);
    if (!m.dev) {
      if (required && rows > 0) why = s + " is required";
      return;
    }
    if (reinterpret_cast<uintptr_t>(m.dev) % size) why = s + " is not aligned to its elements";
    else if (m.row_stride < 0 || m.replica_stride < 0 || m.row_stride > (int64_t)1 << 32 || m.replica_stride > (int64_t)1 << 44) why = s + ": strides out of range";
    else if (rows > 1 && m.row_stride < width) why = s + ": row_stride is less than a row";
    else if (out && n > 1 && m.replica_stride < (rows - 1) * m.row_stride + width) {
      // replicas may also lie between each other's rows
      if (rows > 1 && !(m.replica_stride >= width && m.row_stride >= (n - 1) * m.replica_stride + width)) why = s + ": replicas overlap";
      else if (rows <= 1 && m.replica_stride < width) why = s + ": replicas overlap";
    }
  }
  void codes(const char* name, const hdet_rows& m, int n, int64_t rows, int64_t width, bool required, bool out) {
    matrix(name, m, n, rows, (width + 15) / 16 * 16, 1, required, out);
    if (!ok() || !m.dev) return;
    const std::string s(name);
    if (reinterpret_cast<uintptr_t>(m.dev) & 15 || (m.row_stride | m.replica_stride) & 15) why = s + ": rows must start 16-byte aligned (strides multiples of 16)";
    else if (m.row_stride >= (int64_t)1 << 22) why = s + ": row_stride must be less than 2^22";
  }
  // [count] fp32 a replica, `stride` apart
  void vector(const char* name, const void* p, int n, int64_t count, int64_t stride, bool required, bool out) {
    if (!ok()) return;
    const std::string s(name);
    if (!p) {
      if (required && count > 0) why = s + " is required";
    } else if (reinterpret_cast<uintptr_t>(p) & 3) why = s + " is not aligned to its elements";
    else if (stride < 0 || (out && n > 1 && stride < count)) why = s + ": stride is less than a vector";
  }
  void workspace(const void* p, size_t have, size_t want) {
    if (!ok() || !want) return;
    if (!p || have < want) why = "workspace is too small: " + std::to_string(want) + " bytes are needed";
    else if (reinterpret_cast<uintptr_t>(p) & 15) why = "workspace must be 16-byte aligned";
  }
};

// Runs one entry: f(argument_checks) checks, g() launches.  Nothing thrown leaves it.
template <typename F, typename G>
int entry(const char* name, F check, G launch) {
  try {
    argument_checks c;
    check(c);
    if (!c.ok()) {
      hdet_set_global_error(std::string(name) + ": " + c.why);
      return HDET_EINVAL;
    }
    const hipError_t e = launch();
    if (e == hipSuccess) return HDET_OK;
    hdet_set_global_error(std::string(name) + ": " + hipGetErrorString(e));
    return HDET_EHIP;
  } catch (...) {
    return HDET_EINVAL;        // out of host memory while a message was made
  }
}

int element(int dtype) { return dtype == HDET_TYPE_BF16 ? 2 : 4; }

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
// Workspace of the linear layer's gradients, of what the results that are wanted need: X (for dw) and W (for dx) in bfloat16, and dy where
// its rows are no whole 16-byte pieces, in rows of whole pieces; partial sums of dy, results of pieces of a long contraction.  (X over W,
// which dx is done with by then: 57.9 -> 60.7 us for 3 x 515 rows of 776 -> 1501, 44.7 -> 46.5 for 3 x 500 of 512 -> 1536, 1192 -> 1199 for
// 8 x 8192 of 1024 -> 4096.)
struct linear_layout { int64_t pitch, dy_pitch; hdet_split for_dx, for_dw; size_t x, w, dy, sum, part, total; };
linear_layout linear_layout_of(int n, int64_t rows, int d_in, int d_out, bool dx, bool dw, bool db) {
  linear_layout l;
  l.pitch = (d_in + 7) & ~7;
  l.dy_pitch = (d_out + 7) & ~7;
  l.for_dx = hdet_split_of(n, rows, d_in, d_out);
  l.for_dw = hdet_split_of(n, d_out, d_in, rows);
  l.x = 0;
  l.w = l.x + (dw ? up256((size_t)n * rows * l.pitch * 2) : 0);
  l.dy = l.w + (dx ? up256((size_t)n * d_out * l.pitch * 2) : 0);
  l.sum = l.dy + ((dx || dw) && l.dy_pitch != d_out ? up256((size_t)n * rows * l.dy_pitch * 2) : 0);
  l.part = l.sum + (db ? up256(hdet_row_sum_bytes(n, rows, d_out)) : 0);
  const size_t part_x = dx ? l.for_dx.bytes : 0, part_w = dw ? l.for_dw.bytes : 0;
  l.total = rows == 0 ? 0 : l.part + (part_x > part_w ? part_x : part_w);
  return l;
}
linear_layout linear_layout_of(const hdet_linear_grad_args& a) {
  return linear_layout_of(a.n_replicas, a.rows, a.d_in, a.d_out, a.dx.dev != nullptr, a.dw.dev != nullptr, a.db_dev != nullptr);
}
void linear_sizes(argument_checks& c, int n, int64_t rows, int d_in, int d_out) {
  c.common(n, rows);
  c.need(d_in >= 1 && d_in <= HDET_MAX_CODES_WIDTH, "d_in must be in 1 .. HDET_MAX_CODES_WIDTH");
  c.need(d_out >= 1 && d_out <= kMaxRows, "d_out must be in 1 .. 2^21");
}
void vocab_sizes(argument_checks& c, int n, int64_t rows, int width, int classes, int piece) {
  c.common(n, rows);
  c.need(width >= 1 && width <= HDET_MAX_CODES_WIDTH, "width must be in 1 .. HDET_MAX_CODES_WIDTH");
  c.need(classes >= 1 && classes <= kMaxRows, "classes must be in 1 .. 2^21");
  c.need(piece >= 0, "piece must be 0 or a number of classes");
}

// Sizes that both passes of the rotation check
template <typename A> void rotary_sizes(argument_checks& c, const A& a) {
  c.common(a.n_replicas, a.rows);
  c.type(a.dtype, "dtype must be HDET_TYPE_F32 or HDET_TYPE_BF16");
  c.need(a.head_dim >= 1 && a.head_dim <= HDET_MAX_ROTARY_DIM, "head_dim must be in 1 .. HDET_MAX_ROTARY_DIM");
  if (!c.ok()) return;
  c.need(a.q_heads >= 1 && (int64_t)a.q_heads * a.head_dim <= kMaxHeadColumns, "q_heads must be 1 or more, q_heads * head_dim up to 2^20");
  c.need(!a.k.dev || (a.k_heads >= 1 && (int64_t)a.k_heads * a.head_dim <= kMaxHeadColumns), "k_heads must be 1 or more, k_heads * head_dim up to 2^20");
  c.need(a.rotated >= 0 && a.rotated <= a.head_dim && a.rotated % 2 == 0, "rotated must be even and in 0 .. head_dim");
  c.need(a.layout == HDET_ROTARY_HALVES || a.layout == HDET_ROTARY_PAIRS, "layout must be HDET_ROTARY_HALVES or HDET_ROTARY_PAIRS");
  c.need(a.period >= 0, "period must be 0 or a number of rows");
  c.need(a.eps >= 0.0 && a.eps < 1e30, "eps must be a number from 0 on");
  c.need(a.magnitude > -1e30 && a.magnitude < 1e30, "magnitude must be finite");
  c.need(a.rotated == 0 || a.rows == 0 || a.freq_dev, "freq_dev is required");
  c.need(reinterpret_cast<uintptr_t>(a.freq_dev) % 8 == 0, "freq_dev is not aligned to its elements");
  c.need(reinterpret_cast<uintptr_t>(a.positions_dev) % 4 == 0, "positions_dev is not aligned to its elements");
  if (!c.ok()) return;
  c.vector("q_gain_dev", a.q_gain_dev, a.n_replicas, a.head_dim, a.q_gain_stride, false, false);
  if (a.k.dev) c.vector("k_gain_dev", a.k_gain_dev, a.n_replicas, a.head_dim, a.k_gain_stride, false, false);
}

void attention_sizes(argument_checks& c, int n, int seqs, int q_len, int kv_len, int heads, int kv_heads, int head_dim) {
  c.need(seqs >= 0 && q_len >= 0 && kv_len >= 0, "seqs, q_len and kv_len must be 0 or more");
  if (!c.ok()) return;
  c.need(n >= 1 && n <= HDET_MAX_REPLICAS, "n_replicas out of range");
  c.need((int64_t)seqs * q_len <= kMaxRows, "seqs * q_len must be in 0 .. 2^21 per replica");
  c.need(kv_len <= kMaxKeys && (int64_t)seqs * kv_len <= kMaxKeys, "seqs * kv_len must be in 0 .. 2^28 per replica");
  c.need(head_dim >= 1 && head_dim <= HDET_MAX_ATTENTION_DIM, "head_dim must be in 1 .. HDET_MAX_ATTENTION_DIM");
  c.need(kv_heads >= 1 && heads >= 1 && heads % (kv_heads < 1 ? 1 : kv_heads) == 0, "heads must be a multiple of kv_heads");
  c.need((int64_t)heads * head_dim <= kMaxHeadColumns, "heads * head_dim must be up to 2^20");
  if (!c.ok()) return;
  // the kernels count their blocks in 32 bits
  const int64_t pairs = (int64_t)n * seqs * (q_len > 0 ? q_len : 1) * heads, blocks = (int64_t)n * seqs * kv_heads * (((int64_t)kv_len + 127) / 128);
  c.need(seqs <= kMaxKeys && pairs <= (int64_t)1 << 31 && blocks <= (int64_t)1 << 31, "too many sequences and heads: n_replicas * seqs * q_len * heads must be up to 2^31");
}
// What both passes of attention check
template <typename A> void attention_arguments(argument_checks& c, const A& a) {
  attention_sizes(c, a.n_replicas, a.seqs, a.q_len, a.kv_len, a.heads, a.kv_heads, a.head_dim);
  c.type(a.dtype, "dtype must be HDET_TYPE_F32 or HDET_TYPE_BF16");
  c.need(a.window >= 0, "window must be 0 or a number of keys");
  c.need(a.scale > -1e30 && a.scale < 1e30, "scale must be finite");
  c.need(a.softcap >= 0.0 && a.softcap < 1e30 && (a.softcap == 0.0 || a.softcap > 1e-30), "softcap must be 0 or a number above it");
  if (!c.ok()) return;
  const int n = a.n_replicas, size = element(a.dtype);
  const int64_t rows = (int64_t)a.seqs * a.q_len, keys = (int64_t)a.seqs * a.kv_len, wide = (int64_t)a.heads * a.head_dim, narrow = (int64_t)a.kv_heads * a.head_dim;
  c.matrix("q", a.q, n, rows, wide, size, keys > 0, false);
  c.matrix("k", a.k, n, keys, narrow, size, rows > 0, false);
  c.matrix("v", a.v, n, keys, narrow, size, rows > 0, false);
  c.vector("slopes_dev", a.slopes_dev, n, a.heads, a.slopes_stride, false, false);
  c.vector("positions_dev", a.positions_dev, n, rows, rows, false, false);
  c.vector("first_dev", a.first_dev, n, rows, rows, false, false);
  c.vector("end_dev", a.end_dev, n, rows, rows, false, false);
}

// A matrix of a call: its place and its extent
struct extent { hdet_rows m; int64_t rows, width; int size; };
bool same_place(const extent& a, const extent& b, int n) {
  return a.m.dev == b.m.dev && a.size == b.size && a.rows == b.rows && a.width == b.width && (a.rows <= 1 || a.m.row_stride == b.m.row_stride) &&
         (n <= 1 || a.m.replica_stride == b.m.replica_stride);
}
// Whether two of n replicas' matrices share memory.  Exact where their strides agree, as those of slices of one matrix do: row j of replica z + dz of b lies dz replica strides
// and dj row strides from row j - dj of replica z of a; otherwise only matrices that start at the same place do.
bool share_memory(const extent& a, const extent& b, int n) {
  if (!a.m.dev || !b.m.dev || a.rows == 0 || b.rows == 0 || a.width == 0 || b.width == 0) return false;
  if (a.m.dev == b.m.dev) return true;
  const int64_t row_a = a.m.row_stride * a.size, row_b = b.m.row_stride * b.size, row = a.rows > 1 ? row_a : row_b;
  const int64_t rep_a = a.m.replica_stride * a.size, rep_b = b.m.replica_stride * b.size, rep = n > 1 ? rep_a : 0;
  if ((a.rows > 1 && b.rows > 1 && row_a != row_b) || (n > 1 && rep_a != rep_b)) return false;
  const int64_t wide_a = a.width * a.size, wide_b = b.width * b.size, from = (int64_t)((uintptr_t)b.m.dev - (uintptr_t)a.m.dev);
  // from first to last element they lie apart
  if (from >= (n - 1) * rep + (a.rows - 1) * row + wide_a || -from >= (n - 1) * rep + (b.rows - 1) * row + wide_b) return false;
  for (int64_t dz = 1 - n; dz < n; ++dz) {
    // some dj in 1 - a.rows .. b.rows - 1 with -wide_b < x + dj row < wide_a
    const int64_t x = from + dz * rep;
    if (a.rows == 1 && b.rows == 1) {
      if (-wide_b < x && x < wide_a) return true;
      continue;
    }
    const int64_t low = -wide_b - x;                                       // dj row above this; the first dj that is
    const int64_t dj = std::max((low >= 0 ? low / row : -((-low + row - 1) / row)) + 1, 1 - a.rows);
    if (dj < b.rows && x + dj * row < wide_a) return true;
  }
  return false;
}
// Outputs that share memory with an input or another output
void written_apart(argument_checks& c, int n, std::initializer_list<extent> outputs, std::initializer_list<extent> inputs, bool any) {
  for (auto o = outputs.begin(); any && c.ok() && o != outputs.end(); ++o) {
    auto meets = [&](const extent& x) { return share_memory(*o, x, n); };
    c.need(std::none_of(inputs.begin(), inputs.end(), meets) && std::none_of(o + 1, outputs.end(), meets), "an output lies over an input or another output");
  }
}
// An output that shares memory with an input and is not the whole of it
void in_place_or_apart(argument_checks& c, int n, const extent& output, const extent& input) {
  c.need(same_place(output, input, n) || !share_memory(output, input, n), "an output lies over its own input with other strides, or over a part of it");
}

void clip_sizes(argument_checks& c, int n, int tensors) {
  c.need(n >= 1 && n <= HDET_MAX_REPLICAS, "n_replicas out of range");
  c.need(tensors >= 0 && tensors <= HDET_MAX_GRAD_TENSORS, "n_tensors must be in 0 .. HDET_MAX_GRAD_TENSORS");
}

}  // namespace

extern "C" int hdet_rmsnorm(const hdet_norm_args* a, void* stream) {
  return entry("hdet_rmsnorm", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    const int n = a->n_replicas;
    c.common(n, a->rows);
    c.need(a->width >= 1 && a->width <= HDET_MAX_NORM_WIDTH, "width must be in 1 .. HDET_MAX_NORM_WIDTH");
    c.type(a->dtype, "dtype must be HDET_TYPE_F32 or HDET_TYPE_BF16");
    c.need(a->eps >= 0.0 && a->eps < 1e30, "eps must be a number from 0 on");
    if (!c.ok()) return;
    const int size = element(a->dtype);
    c.matrix("x", a->x, n, a->rows, a->width, size, true, false);
    c.matrix("resid", a->resid, n, a->rows, a->width, size, false, false);
    c.matrix("total", a->total, n, a->rows, a->width, size, false, true);
    c.matrix("y", a->y, n, a->rows, a->width, size, false, true);
    c.codes("codes", a->codes, n, a->rows, a->width, false, true);
    c.vector("scale_dev", a->scale_dev, n, a->rows, a->rows, a->codes.dev != nullptr, true);
    c.vector("rstd_dev", a->rstd_dev, n, a->rows, a->rows, false, true);
    c.vector("gain_dev", a->gain_dev, n, a->width, a->gain_stride, true, false);
  }, [&] { return hdet_launch_norm(*a, (hipStream_t)stream); });
}

extern "C" int hdet_rmsnorm_backward_workspace(int32_t n_replicas, int64_t rows, int32_t width, size_t* bytes) {
  return entry("hdet_rmsnorm_backward_workspace", [&](argument_checks& c) {
    c.common(n_replicas, rows);
    c.need(width >= 1 && width <= HDET_MAX_NORM_WIDTH, "width must be in 1 .. HDET_MAX_NORM_WIDTH");
    c.need(bytes != nullptr, "bytes is null");
  }, [&] { *bytes = hdet_norm_backward_bytes(n_replicas, rows, width); return hipSuccess; });
}

extern "C" int hdet_rmsnorm_backward(const hdet_norm_grad_args* a, void* stream) {
  return entry("hdet_rmsnorm_backward", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    const int n = a->n_replicas;
    c.common(n, a->rows);
    c.need(a->width >= 1 && a->width <= HDET_MAX_NORM_WIDTH, "width must be in 1 .. HDET_MAX_NORM_WIDTH");
    c.type(a->dtype, "dtype must be HDET_TYPE_F32 or HDET_TYPE_BF16");
    if (!c.ok()) return;
    const int size = element(a->dtype);
    c.matrix("total", a->total, n, a->rows, a->width, size, true, false);
    c.matrix("dy", a->dy, n, a->rows, a->width, size, true, false);
    c.matrix("dtotal", a->dtotal, n, a->rows, a->width, size, false, false);
    c.matrix("dx", a->dx, n, a->rows, a->width, size, true, true);
    c.vector("rstd_dev", a->rstd_dev, n, a->rows, a->rows, true, false);
    c.vector("gain_dev", a->gain_dev, n, a->width, a->gain_stride, true, false);
    c.vector("dgain_dev", a->dgain_dev, n, a->width, a->dgain_stride, false, true);
    if (c.ok() && a->dgain_dev) c.workspace(a->workspace_dev, a->workspace_bytes, hdet_norm_backward_bytes(n, a->rows, a->width));
  }, [&] { return hdet_launch_norm_backward(*a, (hipStream_t)stream); });
}

static int codes_entry(const char* name, const hdet_codes_args* a, void* stream, bool restore) {
  return entry(name, [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    const int n = a->n_replicas;
    c.common(n, a->rows);
    const int most = restore ? HDET_MAX_CODES_WIDTH : HDET_MAX_NORM_WIDTH;
    c.need(a->width >= 1 && a->width <= most, restore ? "width must be in 1 .. HDET_MAX_CODES_WIDTH" : "width must be in 1 .. HDET_MAX_NORM_WIDTH");
    c.type(a->dtype, "dtype must be HDET_TYPE_F32 or HDET_TYPE_BF16");
    if (!c.ok()) return;
    c.matrix("values", a->values, n, a->rows, a->width, element(a->dtype), true, restore);
    c.codes("codes", a->codes, n, a->rows, a->width, true, !restore);
    c.vector("scale_dev", a->scale_dev, n, a->rows, a->rows, true, !restore);
  }, [&] { return restore ? hdet_launch_restore(*a, (hipStream_t)stream) : hdet_launch_quantise(*a, (hipStream_t)stream); });
}
extern "C" int hdet_quantise_rows(const hdet_codes_args* a, void* stream) { return codes_entry("hdet_quantise_rows", a, stream, false); }
extern "C" int hdet_restore_rows(const hdet_codes_args* a, void* stream) { return codes_entry("hdet_restore_rows", a, stream, true); }

extern "C" int hdet_quantised_linear(const hdet_linear_args* a, void* stream) {
  return entry("hdet_quantised_linear", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    const int n = a->n_replicas;
    linear_sizes(c, n, a->rows, a->d_in, a->d_out);
    c.type(a->y_dtype, "y_dtype must be HDET_TYPE_F32 or HDET_TYPE_BF16");
    if (!c.ok()) return;
    c.codes("codes", a->codes, n, a->rows, a->d_in, true, false);
    c.codes("w_codes", a->w_codes, n, a->d_out, a->d_in, true, false);
    c.vector("scale_dev", a->scale_dev, n, a->rows, a->rows, true, false);
    c.vector("w_scale_dev", a->w_scale_dev, n, a->d_out, a->d_out, true, false);
    c.vector("bias_dev", a->bias_dev, n, a->d_out, a->bias_stride, false, false);
    c.matrix("y", a->y, n, a->rows, a->d_out, element(a->y_dtype), true, true);
  }, [&] { return hdet_launch_codes_gemm(*a, (hipStream_t)stream); });
}

extern "C" int hdet_quantised_linear_backward_workspace(int32_t n_replicas, int64_t rows, int32_t d_in, int32_t d_out, size_t* bytes) {
  return entry("hdet_quantised_linear_backward_workspace", [&](argument_checks& c) {
    linear_sizes(c, n_replicas, rows, d_in, d_out);
    c.need(bytes != nullptr, "bytes is null");
  }, [&] { *bytes = linear_layout_of(n_replicas, rows, d_in, d_out, true, true, true).total; return hipSuccess; });
}

extern "C" int hdet_quantised_linear_backward(const hdet_linear_grad_args* a, void* stream) {
  return entry("hdet_quantised_linear_backward", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    const int n = a->n_replicas;
    linear_sizes(c, n, a->rows, a->d_in, a->d_out);
    if (!c.ok()) return;
    c.matrix("dy", a->dy, n, a->rows, a->d_out, 2, true, false);
    c.codes("codes", a->codes, n, a->rows, a->d_in, a->dw.dev != nullptr, false);
    c.codes("w_codes", a->w_codes, n, a->d_out, a->d_in, a->dx.dev != nullptr, false);
    c.vector("scale_dev", a->scale_dev, n, a->rows, a->rows, a->dw.dev != nullptr, false);
    c.vector("w_scale_dev", a->w_scale_dev, n, a->d_out, a->d_out, a->dx.dev != nullptr, false);
    c.matrix("dx", a->dx, n, a->rows, a->d_in, 2, false, true);
    c.matrix("dw", a->dw, n, a->d_out, a->d_in, 4, false, true);
    c.vector("db_dev", a->db_dev, n, a->d_out, a->db_stride, false, true);
    if (c.ok()) c.workspace(a->workspace_dev, a->workspace_bytes, linear_layout_of(*a).total);
  }, [&]() -> hipError_t {
    const hipStream_t s = (hipStream_t)stream;
    const int n = a->n_replicas;
    const int64_t M = a->rows;
    hipError_t e;
    if (M == 0) {
      if (a->dw.dev && (e = hdet_launch_zero_rows(a->dw, n, a->d_out, a->d_in, HDET_TYPE_F32, s)) != hipSuccess) return e;
      return a->db_dev ? hdet_launch_row_sum(a->dy, n, 0, a->d_out, a->db_dev, a->db_stride, nullptr, s) : hipSuccess;
    }
    const linear_layout l = linear_layout_of(*a);
    char* const ws = (char*)a->workspace_dev;
    auto restored = [&](const hdet_rows& codes, const float* scale, int64_t rows, size_t at) {
      hdet_codes_args r = {};
      r.n_replicas = n; r.dtype = HDET_TYPE_BF16; r.rows = rows; r.width = (int32_t)l.pitch;      // with the zeros behind a row's codes
      r.values = {ws + at, l.pitch, rows * l.pitch};
      r.codes = codes; r.scale_dev = const_cast<float*>(scale);
      return hdet_launch_restore(r, s);
    };
    if (a->db_dev && (e = hdet_launch_row_sum(a->dy, n, M, a->d_out, a->db_dev, a->db_stride, ws + l.sum, s)) != hipSuccess) return e;
    hdet_rows dy = a->dy;
    if (l.dy_pitch != a->d_out && (a->dx.dev || a->dw.dev)) {
      if ((e = hdet_launch_pad_rows(a->dy, n, M, a->d_out, nullptr, (uint16_t*)(ws + l.dy), l.dy_pitch, 1, s)) != hipSuccess) return e;
      dy = {ws + l.dy, l.dy_pitch, M * l.dy_pitch};
    }
    // a result of any alignment takes an epilogue that writes at any element where the operands allow the fast path
    auto product = [&](hdet_bgemm_args& g, bool a_kmajor, int epi, int any_epi, const hdet_split& sp) {
      g.padded = true;
      if (sp.pieces > 1)
        return hdet_launch_split(g, a_kmajor, n, sp, (float*)(ws + l.part), {g.c, a_kmajor ? HDET_TYPE_BF16 : HDET_TYPE_F32, g.ldc, g.c_s[0], nullptr, nullptr, 0, 0, true, true}, s);
      g.accum = (float*)ws; g.accum_ld = 4; g.accum_first = g.accum_last = true;      // (one piece: never touched)
      g.n1 = g.n2 = 1;
      const bool any = !hdet_bgemm_dma_eligible(g, a_kmajor, false, epi) && hdet_bgemm_dma_eligible(g, a_kmajor, false, any_epi);
      return hdet_launch_bgemm(g, a_kmajor, false, any ? any_epi : epi, n, s);
    };
    if (a->dx.dev) {
      if ((e = restored(a->w_codes, a->w_scale_dev, a->d_out, l.w)) != hipSuccess) return e;
      hdet_bgemm_args g = {};
      g.a = (const uint16_t*)dy.dev; g.lda = dy.row_stride; g.a_s[0] = dy.replica_stride;
      g.b = (const uint16_t*)(ws + l.w); g.ldb = l.pitch; g.b_s[0] = a->d_out * l.pitch;
      g.c = a->dx.dev; g.ldc = a->dx.row_stride; g.c_s[0] = a->dx.replica_stride;
      g.m = (int)M; g.n = a->d_in; g.k = a->d_out;
      if ((e = product(g, true, HDET_EPI_BF16, HDET_EPI_ACCUM_BF16, l.for_dx)) != hipSuccess) return e;
    }
    if (a->dw.dev) {
      if ((e = restored(a->codes, a->scale_dev, M, l.x)) != hipSuccess) return e;
      hdet_bgemm_args g = {};
      g.a = (const uint16_t*)dy.dev; g.lda = dy.row_stride; g.a_s[0] = dy.replica_stride;
      g.b = (const uint16_t*)(ws + l.x); g.ldb = l.pitch; g.b_s[0] = M * l.pitch;
      g.c = a->dw.dev; g.ldc = a->dw.row_stride; g.c_s[0] = a->dw.replica_stride;
      g.m = a->d_out; g.n = a->d_in; g.k = (int)M;
      if ((e = product(g, false, HDET_EPI_F32, HDET_EPI_SCALED_F32, l.for_dw)) != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

extern "C" int hdet_vocab_loss_workspace(int32_t n_replicas, int64_t rows, int32_t width, int32_t classes, int32_t dw_dtype, int32_t piece, size_t* bytes) {
  return entry("hdet_vocab_loss_workspace", [&](argument_checks& c) {
    vocab_sizes(c, n_replicas, rows, width, classes, piece);
    if (dw_dtype != HDET_VOCAB_NO_DW && dw_dtype != HDET_VOCAB_LOSSES) c.type(dw_dtype, "dw_dtype must be HDET_TYPE_F32, HDET_TYPE_BF16, HDET_VOCAB_NO_DW or HDET_VOCAB_LOSSES");
    c.need(bytes != nullptr, "bytes is null");
  }, [&] { *bytes = hdet_vocab_bytes(n_replicas, rows, width, classes, dw_dtype, piece); return hipSuccess; });
}

extern "C" int hdet_vocab_loss(const hdet_vocab_args* a, void* stream) {
  return entry("hdet_vocab_loss", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    const int n = a->n_replicas;
    vocab_sizes(c, n, a->rows, a->width, a->classes, a->piece);
    c.type(a->dw_dtype, "dw_dtype must be HDET_TYPE_F32 or HDET_TYPE_BF16");
    if (!c.ok()) return;
    c.matrix("h", a->h, n, a->rows, a->width, 2, true, false);
    c.matrix("w", a->w, n, a->classes, a->width, 2, true, false);
    c.vector("bias_dev", a->bias_dev, n, a->classes, a->bias_stride, false, false);
    c.vector("labels_dev", a->labels_dev, n, a->rows, a->rows, true, false);
    c.vector("row_loss_dev", a->row_loss_dev, n, a->rows, a->rows, true, true);
    c.vector("mean_loss_dev", a->mean_loss_dev, n, 1, 1, true, true);
    c.matrix("dh", a->dh, n, a->rows, a->width, 2, false, true);
    c.matrix("dw", a->dw, n, a->classes, a->width, element(a->dw_dtype), false, true);
    c.vector("db_dev", a->db_dev, n, a->classes, a->db_stride, false, true);
    if (c.ok()) c.workspace(a->workspace_dev, a->workspace_bytes, hdet_vocab_bytes(n, a->rows, a->width, a->classes, hdet_vocab_kind(*a), a->piece));
  }, [&] { return hdet_launch_vocab_loss(*a, (hipStream_t)stream); });
}

extern "C" int hdet_head_rotary(const hdet_rotary_args* a, void* stream) {
  return entry("hdet_head_rotary", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    rotary_sizes(c, *a);
    if (!c.ok()) return;
    const int n = a->n_replicas, size = element(a->dtype);
    c.matrix("q", a->q, n, a->rows, (int64_t)a->q_heads * a->head_dim, size, true, false);
    c.matrix("q_out", a->q_out, n, a->rows, (int64_t)a->q_heads * a->head_dim, size, true, true);
    const extent q = {a->q, a->rows, (int64_t)a->q_heads * a->head_dim, size}, q_out = {a->q_out, q.rows, q.width, size};
    if (c.ok()) in_place_or_apart(c, n, q_out, q);
    if (!a->k.dev) return;
    c.matrix("k", a->k, n, a->rows, (int64_t)a->k_heads * a->head_dim, size, true, false);
    c.matrix("k_out", a->k_out, n, a->rows, (int64_t)a->k_heads * a->head_dim, size, true, true);
    if (!c.ok()) return;
    const extent k = {a->k, a->rows, (int64_t)a->k_heads * a->head_dim, size}, k_out = {a->k_out, k.rows, k.width, size};
    in_place_or_apart(c, n, k_out, k);
    written_apart(c, n, {q_out}, {k, k_out}, true);
    written_apart(c, n, {k_out}, {q}, true);
  }, [&] { return hdet_launch_rotary(*a, (hipStream_t)stream); });
}

extern "C" int hdet_head_rotary_backward_workspace(int32_t n_replicas, int64_t rows, int32_t head_dim, int32_t q_heads, int32_t k_heads, size_t* bytes) {
  return entry("hdet_head_rotary_backward_workspace", [&](argument_checks& c) {
    c.common(n_replicas, rows);
    c.need(head_dim >= 1 && head_dim <= HDET_MAX_ROTARY_DIM, "head_dim must be in 1 .. HDET_MAX_ROTARY_DIM");
    c.need(q_heads >= 1 && k_heads >= 0 && (int64_t)q_heads * head_dim <= kMaxHeadColumns && (int64_t)k_heads * head_dim <= kMaxHeadColumns,
           "q_heads must be 1 or more, k_heads 0 or more, heads * head_dim up to 2^20");
    c.need(bytes != nullptr, "bytes is null");
  }, [&] { *bytes = hdet_rotary_backward_bytes(n_replicas, rows, head_dim, q_heads, k_heads); return hipSuccess; });
}

extern "C" int hdet_head_rotary_backward(const hdet_rotary_grad_args* a, void* stream) {
  return entry("hdet_head_rotary_backward", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    rotary_sizes(c, *a);
    if (!c.ok()) return;
    const int n = a->n_replicas, size = element(a->dtype);
    const int64_t wide = (int64_t)a->q_heads * a->head_dim, narrow = (int64_t)a->k_heads * a->head_dim;
    const bool keys = a->dk_out.dev != nullptr;
    c.need(keys || !a->k.dev, "dk_out is required with k");
    c.need(!keys || (a->k_heads >= 1 && narrow <= kMaxHeadColumns), "k_heads must be 1 or more, k_heads * head_dim up to 2^20");
    c.matrix("q", a->q, n, a->rows, wide, size, a->q_gain_dev != nullptr, false);
    c.matrix("dq_out", a->dq_out, n, a->rows, wide, size, true, false);
    c.matrix("dq", a->dq, n, a->rows, wide, size, true, true);
    c.need(a->q_gain_dev || !a->dq_gain_dev, "dq_gain_dev needs q_gain_dev");
    c.vector("dq_gain_dev", a->dq_gain_dev, n, a->head_dim, a->dq_gain_stride, false, true);
    if (keys) {
      c.matrix("k", a->k, n, a->rows, narrow, size, a->k_gain_dev != nullptr, false);
      c.matrix("dk_out", a->dk_out, n, a->rows, narrow, size, true, false);
      c.matrix("dk", a->dk, n, a->rows, narrow, size, true, true);
      c.vector("k_gain_dev", a->k_gain_dev, n, a->head_dim, a->k_gain_stride, false, false);
    }
    c.need(!a->dk_gain_dev || (keys && a->k_gain_dev), "dk_gain_dev needs dk_out and k_gain_dev");
    c.vector("dk_gain_dev", a->dk_gain_dev, n, a->head_dim, a->dk_gain_stride, false, true);
    if (!c.ok()) return;
    // (q and k are read where there are gains)
    const hdet_rows none = {};
    const extent q = {a->q_gain_dev ? a->q : none, a->rows, wide, size}, dq_out = {a->dq_out, a->rows, wide, size}, dq = {a->dq, a->rows, wide, size};
    const extent k = {a->k_gain_dev && keys ? a->k : none, a->rows, narrow, size}, dk_out = {a->dk_out, a->rows, narrow, size}, dk = {keys ? a->dk : none, a->rows, narrow, size};
    in_place_or_apart(c, n, dq, dq_out);
    in_place_or_apart(c, n, dq, q);
    in_place_or_apart(c, n, dk, dk_out);
    in_place_or_apart(c, n, dk, k);
    written_apart(c, n, {dq}, {k, dk_out, dk}, true);
    written_apart(c, n, {dk}, {q, dq_out}, true);
    if (c.ok() && (a->dq_gain_dev || a->dk_gain_dev))
      c.workspace(a->workspace_dev, a->workspace_bytes, hdet_rotary_backward_bytes(n, a->rows, a->head_dim, a->q_heads, keys ? a->k_heads : 0));
  }, [&] { return hdet_launch_rotary_backward(*a, (hipStream_t)stream); });
}

extern "C" int hdet_rotary_frequencies(int32_t rotated, double base, int32_t stretch, double factor, double context, double slow, double fast, double* freq_host) {
  return entry("hdet_rotary_frequencies", [&](argument_checks& c) {
    c.need(rotated >= 0 && rotated <= HDET_MAX_ROTARY_DIM && rotated % 2 == 0, "rotated must be even and in 0 .. HDET_MAX_ROTARY_DIM");
    c.need(base > 0.0 && base < 1e30, "base must be a number above 0");
    c.need(stretch >= HDET_STRETCH_POSITIONS && stretch <= HDET_STRETCH_PARTS, "stretch must be one of HDET_STRETCH_*");
    c.need(factor > 0.0 && factor < 1e30, "factor must be a number above 0");
    c.need(stretch != HDET_STRETCH_BASE || rotated != 2 || factor == 1.0, "HDET_STRETCH_BASE needs more than one pair");
    c.need(stretch != HDET_STRETCH_PARTS || (context > 0.0 && context < 1e30 && slow > 0.0 && slow < fast && fast < 1e30),
           "HDET_STRETCH_PARTS needs a context above 0 and 0 < slow < fast");
    c.need(freq_host != nullptr || rotated == 0, "freq_host is null");
  }, [&] {
    if (stretch == HDET_STRETCH_BASE && rotated > 2) base *= pow(factor, (double)rotated / (rotated - 2));
    for (int t = 0; t < rotated / 2; ++t) {
      const double f = pow(base, -2.0 * t / rotated);
      double keep = stretch == HDET_STRETCH_BASE ? 1.0 : 0.0;      // the part of the unstretched frequency
      if (stretch == HDET_STRETCH_PARTS) keep = std::min(1.0, std::max(0.0, (context * f / (2.0 * M_PI) - slow) / (fast - slow)));
      freq_host[t] = f * (keep + (1.0 - keep) / factor);
    }
    return hipSuccess;
  });
}

extern "C" int hdet_attention_workspace(int32_t n_replicas, int32_t seqs, int32_t q_len, int32_t kv_len, int32_t heads, int32_t kv_heads, int32_t head_dim, size_t* bytes) {
  return entry("hdet_attention_workspace", [&](argument_checks& c) {
    attention_sizes(c, n_replicas, seqs, q_len, kv_len, heads, kv_heads, head_dim);
    c.need(bytes != nullptr, "bytes is null");
  }, [&] { *bytes = hdet_attend_bytes(n_replicas, seqs, q_len, kv_len, heads, kv_heads, head_dim); return hipSuccess; });
}

extern "C" int hdet_attention(const hdet_attention_args* a, void* stream) {
  return entry("hdet_attention", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    attention_arguments(c, *a);
    if (!c.ok()) return;
    const int n = a->n_replicas, size = element(a->dtype);
    const int64_t rows = (int64_t)a->seqs * a->q_len, keys = (int64_t)a->seqs * a->kv_len, wide = (int64_t)a->heads * a->head_dim, narrow = (int64_t)a->kv_heads * a->head_dim;
    c.matrix("out", a->out, n, rows, wide, size, true, true);
    c.vector("lse_dev", a->lse_dev, n, rows * a->heads, rows * a->heads, false, true);
    written_apart(c, n, {{a->out, rows, wide, size}}, {{a->q, rows, wide, size}, {a->k, keys, narrow, size}, {a->v, keys, narrow, size}}, rows * a->kv_len > 0);
    c.workspace(a->workspace_dev, a->workspace_bytes, hdet_attend_bytes(n, a->seqs, a->q_len, a->kv_len, a->heads, a->kv_heads, a->head_dim));
  }, [&] { return hdet_launch_attend(*a, (hipStream_t)stream); });
}

extern "C" int hdet_attention_backward_workspace(int32_t n_replicas, int32_t seqs, int32_t q_len, int32_t kv_len, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                                 size_t* bytes) {
  return entry("hdet_attention_backward_workspace", [&](argument_checks& c) {
    attention_sizes(c, n_replicas, seqs, q_len, kv_len, heads, kv_heads, head_dim);
    c.need(bytes != nullptr, "bytes is null");
  }, [&] { *bytes = hdet_attend_backward_bytes(n_replicas, seqs, q_len, kv_len, heads, kv_heads, head_dim); return hipSuccess; });
}

extern "C" int hdet_attention_backward(const hdet_attention_grad_args* a, void* stream) {
  return entry("hdet_attention_backward", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    attention_arguments(c, *a);
    if (!c.ok()) return;
    const int n = a->n_replicas, size = element(a->dtype);
    const int64_t rows = (int64_t)a->seqs * a->q_len, keys = (int64_t)a->seqs * a->kv_len, wide = (int64_t)a->heads * a->head_dim, narrow = (int64_t)a->kv_heads * a->head_dim;
    c.matrix("out", a->out, n, rows, wide, size, keys > 0, false);
    c.matrix("dout", a->dout, n, rows, wide, size, keys > 0, false);
    c.vector("lse_dev", a->lse_dev, n, rows * a->heads, rows * a->heads, keys > 0, false);
    c.matrix("dq", a->dq, n, rows, wide, size, true, true);
    c.matrix("dk", a->dk, n, keys, narrow, size, true, true);
    c.matrix("dv", a->dv, n, keys, narrow, size, true, true);
    written_apart(c, n, {{a->dq, rows, wide, size}, {a->dk, keys, narrow, size}, {a->dv, keys, narrow, size}},
                  {{a->q, rows, wide, size}, {a->k, keys, narrow, size}, {a->v, keys, narrow, size}, {a->out, rows, wide, size}, {a->dout, rows, wide, size}}, rows * a->kv_len > 0);
    c.workspace(a->workspace_dev, a->workspace_bytes, hdet_attend_backward_bytes(n, a->seqs, a->q_len, a->kv_len, a->heads, a->kv_heads, a->head_dim));
  }, [&] { return hdet_launch_attend_backward(*a, (hipStream_t)stream); });
}

extern "C" int hdet_clip_gradients_workspace(int32_t n_replicas, int32_t n_tensors, size_t* bytes) {
  return entry("hdet_clip_gradients_workspace", [&](argument_checks& c) {
    clip_sizes(c, n_replicas, n_tensors);
    c.need(bytes != nullptr, "bytes is null");
  }, [&] { *bytes = hdet_clip_bytes(n_replicas, n_tensors); return hipSuccess; });
}

extern "C" int hdet_clip_gradients(const hdet_clip_args* a, void* stream) {
  return entry("hdet_clip_gradients", [&](argument_checks& c) {
    c.need(a != nullptr, "args is null");
    if (!c.ok()) return;
    clip_sizes(c, a->n_replicas, a->n_tensors);
    c.need(a->n_tensors == 0 || a->tensors_host, "tensors_host is null");
    c.need(a->grad_mode == HDET_GRAD_PER_REPLICA || a->grad_mode == HDET_GRAD_SHARED, "grad_mode must be HDET_GRAD_PER_REPLICA or HDET_GRAD_SHARED");
    c.need(a->max_norm >= 0.0, "max_norm must be a number from 0 on, or infinity");
    if (!c.ok()) return;
    const int n = a->n_replicas;
    c.vector("norm_dev", a->norm_dev, n, 1, 1, true, true);
    struct start { const void* at; int tensor; bool written; };
    std::vector<start> starts;
    for (int i = 0; i < a->n_tensors && c.ok(); ++i) {
      const hdet_grad_tensor& t = a->tensors_host[i];
      c.type(t.dtype, "dtype of a tensor must be HDET_TYPE_F32 or HDET_TYPE_BF16");
      c.need(t.rows >= 0 && t.width >= 0 && (t.width == 0 || t.rows <= ((int64_t)1 << 40) / t.width), "rows * width of a tensor must be in 0 .. 2^40");
      if (!c.ok() || t.rows == 0 || t.width == 0) continue;
      const bool in_place = !t.out.dev;
      c.matrix("grad", t.grad, n, t.rows, t.width, element(t.dtype), true, in_place && a->max_norm < INFINITY);
      c.matrix("out", t.out, n, t.rows, t.width, 4, false, true);
      starts.push_back({t.grad.dev, i, in_place && a->max_norm < INFINITY});
      if (in_place || !c.ok()) continue;
      starts.push_back({t.out.dev, i, true});
      in_place_or_apart(c, n, {t.out, t.rows, t.width, 4}, {t.grad, t.rows, t.width, element(t.dtype)});
    }
    if (!c.ok()) return;
    // the second pass reads every gradient while others' outputs are written
    std::sort(starts.begin(), starts.end(), [](const start& x, const start& y) { return std::less<const void*>()(x.at, y.at); });
    for (size_t i = 0, j; i < starts.size(); i = j) {
      bool written = false, several = false;
      for (j = i; j < starts.size() && starts[j].at == starts[i].at; ++j) {
        written |= starts[j].written;
        several |= starts[j].tensor != starts[i].tensor;
      }
      c.need(!(written && several), "a tensor is written where another one starts");
    }
    c.workspace(a->workspace_dev, a->workspace_bytes, hdet_clip_bytes(n, a->n_tensors));
  }, [&] { return hdet_launch_clip(*a, (hipStream_t)stream); });
}
