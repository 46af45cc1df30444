// Checks of a call's arguments, for entry points with many tensors.
#pragma once

#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "mtf_internal.h"

namespace mtf {

inline int64_t numel(const mtf_tensor& t) {
  int64_t n = 1;
  for (int i = 0; i < t.ndim; ++i) n *= t.dims[i].size;
  return n;
}

// What the tensors of one call are checked against, one after the other; `st` keeps the first thing found wrong.
struct Arguments {
  const char* what;
  const mtf_layout_t* layout;
  const char* of_name = "logits";      // the tensor whose dims the others are held to
  mtf_status st = MTF_OK;
  struct Range { uintptr_t lo, hi; bool out; };
  std::vector<Range> ranges;

  Arguments(const char* w, const mtf_layout_t* L) : what(w), layout(L) {
    ranges.reserve(16);
    if (!L) st = fail(MTF_ERR_INVALID_ARG, "%s: NULL layout", w);
  }
  bool ok() const { return st == MTF_OK; }
  template <typename... A>
  void wrong(mtf_status s, const char* fmt, A... a) {
    if (!ok()) return;
    const std::string f = std::string("%s: ") + fmt;
    st = fail(s, f.c_str(), what, a...);
  }
  void not_across_ranks(const char* dim) {
    if (ok() && layout->bound_dim >= 0 && layout->world > 1 && layout->mesh_dim_of(dim) == layout->bound_dim)
      wrong(MTF_ERR_UNSUPPORTED, "the dimension '%s' is split across ranks; what is taken along it would need a combine across ranks, which is not built", dim);
  }
  void memory(const void* p, int64_t bytes, int align, bool out, const char* name) {
    if (!ok()) return;
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    if (lo % (uintptr_t)align) return wrong(align == 16 ? MTF_ERR_UNSUPPORTED : MTF_ERR_INVALID_ARG, "%s must be %d-byte aligned", name, align);
    const Range r = {lo, lo + (uintptr_t)bytes, out};
    for (auto& o : ranges)
      if ((out || o.out) && r.lo < o.hi && o.lo < r.hi) return wrong(MTF_ERR_INVALID_ARG, "%s overlaps another tensor of the call", name);
    ranges.push_back(r);
  }
  // Whether dims are in order under a layout without rules: nearly every call's, and the checks below, which copy the names, then have nothing to find.
  bool in_order(const mtf_tensor* t) const {
    if (!layout->rules.empty() || t->ndim < 0 || t->ndim > kMaxTensorDims || (t->ndim > 0 && !t->dims)) return false;
    for (int i = 0; i < t->ndim; ++i) {
      const mtf_dim& d = t->dims[i];
      if (!d.name || !d.name[0] || d.size <= 0) return false;
      for (int j = 0; j < i; ++j)
        if (!strcmp(t->dims[j].name, d.name)) return false;
    }
    return true;
  }
  // a tensor whose own dims are legal under the layout; not NULL, with data (unless it is a description alone)
  bool there(const mtf_tensor* t, const char* name, bool data = true) {
    if (!ok()) return false;
    if (!t || (data && !t->data)) { wrong(MTF_ERR_INVALID_ARG, "%s is NULL or has no data", name); return false; }
    if (in_order(t)) return true;
    std::vector<Dim> d;
    if ((st = mtf::read_dims(t->ndim, t->dims, &d, name)) != MTF_OK) return false;
    return (st = mtf::check_tensor(layout, d)) == MTF_OK;
  }
  // dims [first, first + n) of `of`, then `more` further dims
  void dims_like(const mtf_tensor* t, const mtf_tensor* of, int first, int n, int more, const char* name) {
    if (!ok()) return;
    if (t->ndim != n + more) return wrong(MTF_ERR_SIZE_MISMATCH, "%s has %d dims, not %d", name, (int)t->ndim, n + more);
    for (int i = 0; i < n; ++i)
      if (strcmp(t->dims[i].name, of->dims[first + i].name) || t->dims[i].size != of->dims[first + i].size)
        return wrong(MTF_ERR_SIZE_MISMATCH, "%s: dimension %d is not that of the %s ('%s', %lld)", name, i, of_name, of->dims[first + i].name, (long long)of->dims[first + i].size);
  }
  // Whether it has exactly these dims of a tensor that is legal, and so is legal itself: nearly every tensor of a call that is in order, and
  // the checks above then have nothing to find.
  static bool alike(const mtf_tensor* t, const mtf_tensor* of, int first, int n) {
    if (!t || !t->data || t->ndim != n || !t->dims) return false;
    for (int i = 0; i < n; ++i) {
      const mtf_dim &d = t->dims[i], &o = of->dims[first + i];
      if (d.size != o.size || !d.name || (d.name != o.name && strcmp(d.name, o.name))) return false;
    }
    return true;
  }
  void f32(const mtf_tensor* t, const char* name) {
    if (ok() && t->dtype != MTF_F32) wrong(MTF_ERR_UNSUPPORTED, "%s must be f32", name);
  }
  // f32 tensor of dims [first, first + n) of the logits
  const float* values(const mtf_tensor* t, const mtf_tensor* logits, int first, int n, const char* name, bool out) {
    if (!alike(t, logits, first, n)) {
      if (!there(t, name)) return nullptr;
      dims_like(t, logits, first, n, 0, name);
    }
    f32(t, name);
    memory(t->data, ok() ? numel(*t) * 4 : 0, 4, out, name);
    return reinterpret_cast<const float*>(t->data);
  }
  const float* per_token(const mtf_tensor* t, const mtf_tensor* logits, const char* name, bool out = false) {
    return ok() ? values(t, logits, 0, logits->ndim - 1, name, out) : nullptr;
  }
  float* token_out(const mtf_tensor* t, const mtf_tensor* logits, const char* name) { return const_cast<float*>(per_token(t, logits, name, true)); }
  const int32_t* ids(const int32_t* p, int64_t n, const char* name) {
    if (!ok()) return nullptr;
    if (!p) { wrong(MTF_ERR_INVALID_ARG, "%s is NULL", name); return nullptr; }
    memory(p, n * 4, 4, false, name);
    return p;
  }
};

// Nothing may leave a C entry by an exception: what the checks allocate can fail.
template <typename F>
mtf_status guarded(const char* what, F body) {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return fail(MTF_ERR_INVALID_ARG, "%s: out of host memory", what);
  } catch (...) {
    return fail(MTF_ERR_INVALID_ARG, "%s: an argument check failed", what);
  }
}

}  // namespace mtf
