// C entry points of the language-model operators: argument checks, and the order of the launches.

#include "hdet_ops.h"

#include <limits.h>

namespace {

// rows a replica: what the launches' grids and 32-bit row numbers hold
constexpr int64_t kMaxRows = (int64_t)1 << 21;

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
