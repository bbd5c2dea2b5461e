// C ABI of the operators that produce gradients (include/lionmuon_grad.h):
// validation, then one launcher each.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdint>
#include <exception>
#include <initializer_list>
#include <string>

#include "error.h"
#include "grad.h"
#include "lionmuon_grad.h"

namespace {

using lm::CkptView;
using lm::Elem;
using lm::GroupArgs;
using lm::MatView;
using lm::NormArgs;
using lm::set_error;

static_assert(LM_CHECKPOINT_BLOCK == lm::kCkptBlock, "one block length");

constexpr int64_t kMaxLd = int64_t(1) << 22;      // elements between rows
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxGroupedRows = int64_t(1) << 30;   // of a product: rows of a tile past it still fit an int

// A rejected argument; the entry points turn it into a status.
struct Bad {
  lm_status status;
  std::string msg;
};
[[noreturn]] void refuse(const char* name, const char* msg) {
  throw Bad{LM_ERR_INVALID_ARGUMENT, *name ? std::string(name) + ": " + msg : std::string(msg)};
}
// (the message is put together for a refusal only)
inline void need(bool ok, const char* name, const char* msg) {
  if (!ok) refuse(name, msg);
}
inline void need(bool ok, const char* msg) { need(ok, "", msg); }

size_t elem_bytes(int32_t dtype) { return dtype == LM_F32 ? 4 : 2; }

void check_shape(const char* name, int64_t rows, int64_t cols, int64_t ld, int32_t dtype, uint32_t reserved) {
  need(dtype == LM_F32 || dtype == LM_BF16 || dtype == LM_F16, name, "unknown dtype");
  need(reserved == 0, name, "reserved must be 0");
  need(rows >= 0 && cols >= 0, name, "negative size");
  need(rows <= kMaxRows, name, "too many rows");
  need(ld >= cols, name, "ld must be at least cols");
  need(ld < kMaxLd, name, "rows must be less than 2^22 elements apart");
}

void check(const char* name, const lm_matrix* m) {
  need(m != nullptr, name, "null descriptor");
  check_shape(name, m->rows, m->cols, m->ld, m->dtype, m->reserved);
  if (m->rows == 0 || m->cols == 0) return;
  need(m->data != nullptr, name, "null data");
  need(reinterpret_cast<uintptr_t>(m->data) % elem_bytes(m->dtype) == 0, name, "misaligned data");
}

void check(const char* name, const lm_stack* m) {
  need(m != nullptr, name, "null descriptor");
  check_shape(name, m->rows, m->cols, m->ld, m->dtype, m->reserved);
  need(m->count >= 0 && m->count <= kMaxRows, name, "bad count");
  if (m->count == 0 || m->rows == 0 || m->cols == 0) return;
  need(m->data != nullptr, name, "null data");
  need(reinterpret_cast<uintptr_t>(m->data) % elem_bytes(m->dtype) == 0, name, "misaligned data");
  need(m->count == 1 || m->stride >= (m->rows - 1) * m->ld + m->cols, name, "stride smaller than a matrix");
  need(m->count == 1 || m->stride <= (int64_t(1) << 62) / (m->count * 4), name, "stride too large");
}

void check(const char* name, const lm_checkpoint* c) {
  need(c != nullptr, name, "null descriptor");
  need(c->rows >= 0 && c->cols >= 0, name, "negative size");
  need(c->rows <= kMaxRows, name, "too many rows");
  need(c->ld_codes >= c->cols && c->ld_codes % 16 == 0, name, "ld_codes must be a multiple of 16 and at least cols");
  need(c->ld_codes <= kMaxLd, name, "rows must be at most 2^22 bytes apart");
  need(c->ld_scales >= (c->cols + LM_CHECKPOINT_BLOCK - 1) / LM_CHECKPOINT_BLOCK, name, "ld_scales smaller than a row of scales");
  need(c->ld_scales <= kMaxLd, name, "rows of scales must be at most 2^22 bytes apart");
  if (c->rows == 0 || c->cols == 0) return;
  need(c->codes != nullptr && c->scales != nullptr, name, "null data");
  need(reinterpret_cast<uintptr_t>(c->codes) % 16 == 0, name, "codes must be 16-byte aligned");
}

void same_shape(const char* what, const lm_matrix* a, int64_t rows, int64_t cols) {
  need(a->rows == rows && a->cols == cols, what, "wrong shape");
}

// Memory of an argument: rows of `width` bytes, `pitch` bytes apart.
struct Span {
  const char* name;
  uintptr_t lo, hi, pitch, width;
};
Span span(const char* name, const void* p, int64_t rows, int64_t pitch, int64_t width) {
  Span s{name, 0, 0, 0, 0};
  if (!p || rows <= 0 || width <= 0) return s;
  s.lo = reinterpret_cast<uintptr_t>(p);
  s.hi = s.lo + uintptr_t(rows - 1) * uintptr_t(pitch) + uintptr_t(width);
  s.pitch = uintptr_t(pitch);
  s.width = uintptr_t(width);
  return s;
}
Span span(const char* name, const lm_matrix* m) {
  if (!m) return span(name, nullptr, 0, 0, 0);
  const int64_t b = int64_t(elem_bytes(m->dtype));
  return span(name, m->data, m->rows, m->ld * b, m->cols * b);
}
Span span(const char* name, const lm_stack* m) {
  const int64_t b = int64_t(elem_bytes(m->dtype));
  if (m->count <= 0 || m->rows <= 0 || m->cols <= 0) return span(name, nullptr, 0, 0, 0);
  const int64_t all = (m->count == 1 ? 0 : (m->count - 1) * m->stride) + (m->rows - 1) * m->ld + m->cols;
  return span(name, m->data, 1, 0, all * b);
}
Span codes_span(const char* name, const lm_checkpoint* c) {
  if (!c) return span(name, nullptr, 0, 0, 0);
  return span(name, c->codes, c->rows, c->ld_codes, (c->cols + 15) / 16 * 16);
}
Span scales_span(const char* name, const lm_checkpoint* c) {
  if (!c) return span(name, nullptr, 0, 0, 0);
  return span(name, c->scales, c->rows, c->ld_scales, (c->cols + LM_CHECKPOINT_BLOCK - 1) / LM_CHECKPOINT_BLOCK);
}
// Column ranges of one buffer (two views with the same distance between rows,
// side by side) do not overlap although their spans do.
bool overlap(const Span& a, const Span& b) {
  if (a.lo >= a.hi || b.lo >= b.hi || a.hi <= b.lo || b.hi <= a.lo) return false;
  if (a.pitch != 0 && a.pitch == b.pitch) {
    const uintptr_t d = (b.lo > a.lo ? b.lo - a.lo : a.pitch - (a.lo - b.lo) % a.pitch) % a.pitch;
    if (d >= a.width && d + b.width <= a.pitch) return false;
  }
  return true;
}
[[noreturn]] void overlapping(const Span& a, const Span& b) {
  throw Bad{LM_ERR_INVALID_ARGUMENT, std::string(a.name) + " and " + b.name + " overlap"};
}
void apart(std::initializer_list<Span> outputs, std::initializer_list<Span> inputs) {
  for (auto o = outputs.begin(); o != outputs.end(); ++o) {
    for (auto p = outputs.begin(); p != o; ++p)
      if (overlap(*o, *p)) overlapping(*o, *p);
    for (const Span& i : inputs)
      if (overlap(*o, i)) overlapping(*o, i);
  }
}
bool same_place(const lm_matrix* a, const lm_matrix* b) { return a && b && a->data == b->data && a->ld == b->ld; }

MatView view(const lm_matrix* m) { return m ? MatView{m->data, m->ld} : MatView{}; }
CkptView view(const lm_checkpoint* c) {
  return c ? CkptView{static_cast<uint8_t*>(c->codes), static_cast<uint8_t*>(c->scales), c->ld_codes, c->ld_scales} : CkptView{};
}

void check_workspace(const void* ws, size_t bytes, size_t wanted) {
  need((ws == nullptr) == (bytes == 0), "workspace and workspace_bytes must both be set or both be 0");
  need(reinterpret_cast<uintptr_t>(ws) % 256 == 0, "workspace must be 256-byte aligned");
  if (bytes < wanted)
    throw Bad{LM_ERR_WORKSPACE_TOO_SMALL, "workspace holds " + std::to_string(bytes) + " bytes of " + std::to_string(wanted)};
}

// Runs an entry point's body: a rejected argument, a failed launch and a failed
// host allocation become statuses, and no exception leaves the library.
template <class F>
lm_status guarded(const char* what, F body) noexcept {
  try {
    const hipError_t e = body();
    if (e == hipSuccess) return LM_OK;
    return set_error(LM_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  } catch (const Bad& b) {
    try {
      return set_error(b.status, b.msg);
    } catch (...) {
      return b.status;
    }
  } catch (...) {
    return LM_ERR_OUT_OF_MEMORY;
  }
}

Elem elem(int32_t dtype) { return static_cast<Elem>(dtype); }

// Checks shared by the grouped products; T rows.
void check_group(const lm_stack* w, const int32_t* offsets, int64_t rows) {
  need(w->rows >= 1 && w->cols >= 1, "n and k must be at least 1");
  need(w->count >= 1, "there must be at least one expert");
  need(offsets != nullptr && reinterpret_cast<uintptr_t>(offsets) % 4 == 0, "offsets: null or misaligned");
  if (w->count > LM_GROUPED_MAX_EXPERTS) throw Bad{LM_ERR_UNSUPPORTED, "too many experts"};
  need(rows < kMaxGroupedRows, "too many rows");
}
void need_half(const char* name, int32_t dtype) {
  if (dtype == LM_F32) throw Bad{LM_ERR_UNSUPPORTED, std::string(name) + ": products take bf16 or fp16"};
}
void check_grid(bool fits) {
  if (!fits) throw Bad{LM_ERR_UNSUPPORTED, "too many tiles for one launch"};
}

size_t partial_bytes(int64_t rows, int64_t count, int64_t n, int64_t k) {
  return size_t(lm::weight_grad_partials(rows, count, n, k, lm::current_cus())) * size_t(n) * size_t(k) * 4u;
}

}  // namespace

extern "C" {

lm_status lionmuon_checkpoint(const lm_matrix* x, const lm_checkpoint* out, hipStream_t stream) {
  return guarded("lionmuon_checkpoint", [&]() -> hipError_t {
    check("x", x);
    check("out", out);
    need(out->rows == x->rows && out->cols == x->cols, "out: wrong shape");
    apart({codes_span("codes", out), scales_span("scales", out)}, {span("x", x)});
    if (x->rows == 0 || x->cols == 0) return hipSuccess;
    return lm::launch_checkpoint(elem(x->dtype), view(x), view(out), x->rows, x->cols, stream);
  });
}

lm_status lionmuon_checkpoint_restore(const lm_checkpoint* c, const lm_matrix* out, hipStream_t stream) {
  return guarded("lionmuon_checkpoint_restore", [&]() -> hipError_t {
    check("checkpoint", c);
    check("out", out);
    same_shape("out", out, c->rows, c->cols);
    apart({span("out", out)}, {codes_span("codes", c), scales_span("scales", c)});
    if (c->rows == 0 || c->cols == 0) return hipSuccess;
    return lm::launch_restore(elem(out->dtype), view(c), view(out), c->rows, c->cols, stream);
  });
}

lm_status lionmuon_activation(const lm_matrix* a, int32_t kind, const lm_matrix* h,
                              const lm_checkpoint* kept, hipStream_t stream) {
  return guarded("lionmuon_activation", [&]() -> hipError_t {
    check("a", a);
    check("h", h);
    need(kind == LM_ACT_GELU || kind == LM_ACT_SWIGLU, "unknown kind");
    need(a->rows == h->rows && a->cols == h->cols * (kind == LM_ACT_SWIGLU ? 2 : 1), "h: wrong shape");
    need(a->dtype == h->dtype, "a and h must have one type");
    if (kept) {
      check("checkpoint", kept);
      need(kept->rows == a->rows && kept->cols == a->cols, "checkpoint: wrong shape");
    }
    apart({span("h", h), codes_span("codes", kept), scales_span("scales", kept)}, {span("a", a)});
    if (h->rows == 0 || h->cols == 0) return hipSuccess;
    return lm::launch_activation(elem(a->dtype), kind, view(a), view(h), view(kept), h->rows, h->cols, stream);
  });
}

lm_status lionmuon_activation_grad(const lm_matrix* dh, const lm_matrix* a,
                                   const lm_checkpoint* kept, int32_t kind, const lm_matrix* da,
                                   const lm_matrix* h, hipStream_t stream) {
  return guarded("lionmuon_activation_grad", [&]() -> hipError_t {
    check("dh", dh);
    check("da", da);
    need(kind == LM_ACT_GELU || kind == LM_ACT_SWIGLU, "unknown kind");
    need((a == nullptr) != (kept == nullptr), "either a or its checkpoint");
    const int64_t wide = dh->cols * (kind == LM_ACT_SWIGLU ? 2 : 1);
    same_shape("da", da, dh->rows, wide);
    need(da->dtype == dh->dtype, "dh and da must have one type");
    if (a) {
      check("a", a);
      same_shape("a", a, dh->rows, wide);
      need(a->dtype == dh->dtype, "a and dh must have one type");
    } else {
      check("checkpoint", kept);
      need(kept->rows == dh->rows && kept->cols == wide, "checkpoint: wrong shape");
    }
    if (h) {
      check("h", h);
      same_shape("h", h, dh->rows, dh->cols);
      need(h->dtype == dh->dtype, "h and dh must have one type");
    }
    apart({span("da", da), span("h", h)},
          {span("dh", dh), span("a", a), codes_span("codes", kept), scales_span("scales", kept)});
    if (dh->rows == 0 || dh->cols == 0) return hipSuccess;
    return lm::launch_activation_grad(elem(dh->dtype), kind, view(dh), view(a), view(kept), view(da), view(h), dh->rows, dh->cols, stream);
  });
}

lm_status lionmuon_rmsnorm(const lm_matrix* x, const lm_matrix* residual, const float* weight,
                           double eps, const lm_matrix* y, const lm_matrix* sum, float* rstd,
                           const lm_checkpoint* kept, hipStream_t stream) {
  return guarded("lionmuon_rmsnorm", [&]() -> hipError_t {
    check("x", x);
    need(x->cols >= 1, "rows must have at least one element");
    if (x->cols > LM_RMSNORM_MAX_COLS)
      throw Bad{LM_ERR_UNSUPPORTED, "rows of more than " + std::to_string(LM_RMSNORM_MAX_COLS) + " elements"};
    need(weight != nullptr && reinterpret_cast<uintptr_t>(weight) % 4 == 0, "weight: null or misaligned");
    need(reinterpret_cast<uintptr_t>(rstd) % 4 == 0, "rstd: misaligned");
    need(eps >= 0.0 && std::isfinite(eps), "eps must be finite and >= 0");
    need(sum == nullptr || residual != nullptr, "sum needs a residual");
    const lm_matrix* others[] = {residual, y, sum};
    const char* names[] = {"residual", "y", "sum"};
    for (int i = 0; i < 3; ++i) {
      if (!others[i]) continue;
      check(names[i], others[i]);
      same_shape(names[i], others[i], x->rows, x->cols);
      need(others[i]->dtype == x->dtype, names[i], "wrong type");
    }
    if (kept) {
      check("checkpoint", kept);
      need(kept->rows == x->rows && kept->cols == x->cols, "checkpoint: wrong shape");
    }
    const bool in_place = same_place(sum, residual);
    const Span w = span("weight", weight, 1, 0, x->cols * 4);
    apart({span("y", y), span("sum", sum), span("rstd", rstd, 1, 0, x->rows * 4), codes_span("codes", kept), scales_span("scales", kept)},
          {span("x", x), span("residual", in_place ? nullptr : residual), w});
    if (x->rows == 0) return hipSuccess;
    NormArgs n;
    n.x = view(x);
    n.residual = view(residual);
    n.y = view(y);
    n.sum = view(sum);
    n.kept = view(kept);
    n.weight = weight;
    n.rstd = rstd;
    n.rows = x->rows;
    n.cols = int32_t(x->cols);
    n.eps = float(eps);
    return lm::launch_rmsnorm(elem(x->dtype), n, stream);
  });
}

lm_status lionmuon_rmsnorm_workspace_bytes(int64_t rows, int64_t cols, size_t* out_bytes) {
  return guarded("lionmuon_rmsnorm_workspace_bytes", [&]() -> hipError_t {
    need(out_bytes != nullptr, "null output");
    need(rows >= 0 && rows <= kMaxRows && cols >= 1, "bad size");
    if (cols > LM_RMSNORM_MAX_COLS)
      throw Bad{LM_ERR_UNSUPPORTED, "rows of more than " + std::to_string(LM_RMSNORM_MAX_COLS) + " elements"};
    *out_bytes = size_t(lm::rmsnorm_grad_groups(rows, cols)) * size_t(cols) * 4u;
    return hipSuccess;
  });
}

lm_status lionmuon_rmsnorm_grad(const lm_matrix* dy, const lm_matrix* s,
                                const lm_checkpoint* kept, const float* weight,
                                const float* rstd, const lm_matrix* residual_grad,
                                const lm_matrix* dx, float* dweight, int32_t accumulate,
                                void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return guarded("lionmuon_rmsnorm_grad", [&]() -> hipError_t {
    check("dy", dy);
    need(dy->cols >= 1, "rows must have at least one element");
    if (dy->cols > LM_RMSNORM_MAX_COLS)
      throw Bad{LM_ERR_UNSUPPORTED, "rows of more than " + std::to_string(LM_RMSNORM_MAX_COLS) + " elements"};
    need((s == nullptr) != (kept == nullptr), "either s or its checkpoint");
    need(weight != nullptr && reinterpret_cast<uintptr_t>(weight) % 4 == 0, "weight: null or misaligned");
    need((rstd != nullptr || dy->rows == 0) && reinterpret_cast<uintptr_t>(rstd) % 4 == 0, "rstd: null or misaligned");
    need(reinterpret_cast<uintptr_t>(dweight) % 4 == 0, "dweight: misaligned");
    need(accumulate == 0 || accumulate == 1, "accumulate must be 0 or 1");
    const lm_matrix* others[] = {s, residual_grad, dx};
    const char* names[] = {"s", "residual_grad", "dx"};
    for (int i = 0; i < 3; ++i) {
      if (!others[i]) continue;
      check(names[i], others[i]);
      same_shape(names[i], others[i], dy->rows, dy->cols);
      need(others[i]->dtype == dy->dtype, names[i], "wrong type");
    }
    if (kept) {
      check("checkpoint", kept);
      need(kept->rows == dy->rows && kept->cols == dy->cols, "checkpoint: wrong shape");
    }
    const size_t wanted = dweight ? size_t(lm::rmsnorm_grad_groups(dy->rows, dy->cols)) * size_t(dy->cols) * 4u : 0;
    check_workspace(workspace, workspace_bytes, wanted);
    const bool in_place = same_place(dx, residual_grad);
    apart({span("dx", dx), span("dweight", dweight, 1, 0, dy->cols * 4), span("workspace", workspace, 1, 0, int64_t(wanted))},
          {span("dy", dy), span("s", s), span("residual_grad", in_place ? nullptr : residual_grad), codes_span("codes", kept),
           scales_span("scales", kept), span("weight", weight, 1, 0, dy->cols * 4), span("rstd", rstd, 1, 0, dy->rows * 4)});
    if (!dx && !dweight) return hipSuccess;
    if (dy->rows == 0 && !dweight) return hipSuccess;
    NormArgs n;
    n.dy = view(dy);
    n.s = view(s);
    n.kept = view(kept);
    n.residual_grad = view(residual_grad);
    n.dx = view(dx);
    n.weight = weight;
    n.rstd = const_cast<float*>(rstd);
    n.dweight = dweight;
    n.partial = static_cast<float*>(workspace);
    n.rows = dy->rows;
    n.cols = int32_t(dy->cols);
    n.accumulate = accumulate;
    return lm::launch_rmsnorm_grad(elem(dy->dtype), n, stream);
  });
}

lm_status lionmuon_grouped_product(const lm_matrix* x, const lm_stack* w, const int32_t* offsets,
                                   const lm_matrix* y, hipStream_t stream) {
  return guarded("lionmuon_grouped_product", [&]() -> hipError_t {
    check("x", x);
    check("w", w);
    check("y", y);
    check_group(w, offsets, x->rows);
    need(x->cols == w->cols, "x: its columns must be w's");
    same_shape("y", y, x->rows, w->rows);
    need_half("x", x->dtype);
    need(w->dtype == x->dtype && y->dtype == x->dtype, "x, w and y must have one type");
    check_grid(lm::row_product_fits(x->rows, w->count, w->rows));
    apart({span("y", y)}, {span("x", x), span("w", w), span("offsets", offsets, 1, 0, (w->count + 1) * 4)});
    if (x->rows == 0) return hipSuccess;
    GroupArgs g;
    g.a = x->data;
    g.lda = x->ld;
    g.b = w->data;
    g.ldb = w->ld;
    g.b_stride = w->count == 1 ? 0 : w->stride;
    g.c = y->data;
    g.ldc = y->ld;
    g.offsets = offsets;
    g.rows = x->rows;
    g.experts = int32_t(w->count);
    g.n = int32_t(w->rows);
    g.k = int32_t(w->cols);
    g.cus = lm::current_cus();
    return lm::launch_grouped_product(elem(x->dtype), g, stream);
  });
}

lm_status lionmuon_grouped_input_grad(const lm_matrix* dy, const lm_stack* w,
                                      const int32_t* offsets, const lm_matrix* dx,
                                      hipStream_t stream) {
  return guarded("lionmuon_grouped_input_grad", [&]() -> hipError_t {
    check("dy", dy);
    check("w", w);
    check("dx", dx);
    check_group(w, offsets, dy->rows);
    need(dy->cols == w->rows, "dy: its columns must be w's rows");
    same_shape("dx", dx, dy->rows, w->cols);
    need_half("dy", dy->dtype);
    need(w->dtype == dy->dtype && dx->dtype == dy->dtype, "dy, w and dx must have one type");
    check_grid(lm::row_product_fits(dy->rows, w->count, w->cols));
    apart({span("dx", dx)}, {span("dy", dy), span("w", w), span("offsets", offsets, 1, 0, (w->count + 1) * 4)});
    if (dy->rows == 0) return hipSuccess;
    GroupArgs g;
    g.a = dy->data;
    g.lda = dy->ld;
    g.b = w->data;
    g.ldb = w->ld;
    g.b_stride = w->count == 1 ? 0 : w->stride;
    g.c = dx->data;
    g.ldc = dx->ld;
    g.offsets = offsets;
    g.rows = dy->rows;
    g.experts = int32_t(w->count);
    g.n = int32_t(w->rows);
    g.k = int32_t(w->cols);
    g.cus = lm::current_cus();
    return lm::launch_grouped_input_grad(elem(dy->dtype), g, stream);
  });
}

lm_status lionmuon_grouped_workspace_bytes(int64_t rows, int64_t count, int64_t n, int64_t k,
                                           size_t* out_bytes) {
  return guarded("lionmuon_grouped_workspace_bytes", [&]() -> hipError_t {
    need(out_bytes != nullptr, "null output");
    need(rows >= 0 && rows < kMaxGroupedRows && count >= 1 && n >= 1 && k >= 1 && n < kMaxLd && k < kMaxLd, "bad size");
    if (count > LM_GROUPED_MAX_EXPERTS) throw Bad{LM_ERR_UNSUPPORTED, "too many experts"};
    *out_bytes = partial_bytes(rows, count, n, k);
    return hipSuccess;
  });
}

lm_status lionmuon_grouped_weight_grad(const lm_matrix* dy, const lm_matrix* x,
                                       const lm_checkpoint* kept, const int32_t* offsets,
                                       const lm_stack* dw, int32_t accumulate, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream) {
  return guarded("lionmuon_grouped_weight_grad", [&]() -> hipError_t {
    check("dy", dy);
    check("dw", dw);
    check_group(dw, offsets, dy->rows);
    need((x == nullptr) != (kept == nullptr), "either x or its checkpoint");
    need(accumulate == 0 || accumulate == 1, "accumulate must be 0 or 1");
    need(dy->cols == dw->rows, "dy: its columns must be dw's rows");
    need(dw->dtype == LM_F32, "dw must be fp32");
    need(dw->rows < kMaxLd, "n too large");
    need_half("dy", dy->dtype);
    if (x) {
      check("x", x);
      same_shape("x", x, dy->rows, dw->cols);
      need(x->dtype == dy->dtype, "x and dy must have one type");
    } else {
      check("checkpoint", kept);
      need(kept->rows == dy->rows && kept->cols == dw->cols, "checkpoint: wrong shape");
      if (dy->dtype != LM_BF16)
        throw Bad{LM_ERR_UNSUPPORTED, "dy must be bf16 with a checkpoint (fp16 does not hold its values)"};
    }
    check_grid(lm::weight_grad_fits(dw->count, dw->rows, dw->cols));
    const size_t wanted = partial_bytes(dy->rows, dw->count, dw->rows, dw->cols);
    check_workspace(workspace, workspace_bytes, wanted);
    apart({span("dw", dw), span("workspace", workspace, 1, 0, int64_t(wanted))},
          {span("dy", dy), span("x", x), codes_span("codes", kept), scales_span("scales", kept),
           span("offsets", offsets, 1, 0, (dw->count + 1) * 4)});
    GroupArgs g;
    g.a = dy->data;
    g.lda = dy->ld;
    if (x) {
      g.b = x->data;
      g.ldb = x->ld;
    }
    g.kept = view(kept);
    g.c = dw->data;
    g.ldc = dw->ld;
    g.c_stride = dw->count == 1 ? 0 : dw->stride;
    g.offsets = offsets;
    g.rows = dy->rows;
    g.experts = int32_t(dw->count);
    g.n = int32_t(dw->rows);
    g.k = int32_t(dw->cols);
    g.accumulate = accumulate;
    g.partial = static_cast<float*>(workspace);
    g.cus = lm::current_cus();
    return lm::launch_grouped_weight_grad(elem(dy->dtype), g, stream);
  });
}

}  // extern "C"
