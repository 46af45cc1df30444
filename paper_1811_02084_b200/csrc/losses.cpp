// Entry points of the losses on stored logits beyond cross-entropy: distillation from a teacher's words, the clipped policy
// loss and the preference loss on pairs.  Validation only; the arithmetic runs in loss_rows.cu.
#include <cmath>
#include <cstring>
#include <new>

#include "losses.h"

using mtf::Dim;
using mtf::fail;
using mtf::LossRows;

namespace {

int64_t numel(const mtf_tensor& t) {
  int64_t n = 1;
  for (int i = 0; i < t.ndim; ++i) n *= t.dims[i].size;
  return n;
}

// What the tensors of one call are checked against, one after the other; `st` keeps the first thing found wrong.
struct Arguments {
  const char* what;
  const mtf_layout_t* layout;
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
  // a tensor whose own dims are legal under the layout; not NULL, with data
  bool there(const mtf_tensor* t, const char* name) {
    if (!ok()) return false;
    if (!t || !t->data) { wrong(MTF_ERR_INVALID_ARG, "%s is NULL or has no data", name); return false; }
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
        return wrong(MTF_ERR_SIZE_MISMATCH, "%s: dimension %d is not that of the logits ('%s', %lld)", name, i, of->dims[first + i].name, (long long)of->dims[first + i].size);
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

// logits, and the gradient where the call has one
void take_logits(Arguments& c, const mtf_tensor* logits, bool with_gradient, const mtf_tensor* dlogits, LossRows* a) {
  if (!c.there(logits, "logits")) return;
  if (logits->ndim < 2) return c.wrong(MTF_ERR_INVALID_ARG, "logits have the dims [*tokens, vocab]");
  if (logits->dtype != MTF_BF16 && logits->dtype != MTF_F32) return c.wrong(MTF_ERR_INVALID_ARG, "unknown type of the logits");
  const int64_t V = logits->dims[logits->ndim - 1].size, rows = numel(*logits) / V, bytes = numel(*logits) * (logits->dtype == MTF_BF16 ? 2 : 4);
  if (V > 0x7fffff00LL || rows > 0x7fffffffLL) return c.wrong(MTF_ERR_UNSUPPORTED, "at most 2^31 tokens and words");
  c.not_across_ranks(logits->dims[logits->ndim - 1].name);
  a->z = logits->data;
  a->V = (int)V;
  a->rows = rows;
  a->bf16 = logits->dtype == MTF_BF16;
  if (with_gradient) {
    if (!Arguments::alike(dlogits, logits, 0, logits->ndim)) {
      if (!c.there(dlogits, "dlogits")) return;
      c.dims_like(dlogits, logits, 0, logits->ndim, 0, "dlogits");
    }
    if (dlogits->dtype != logits->dtype) c.wrong(MTF_ERR_INVALID_ARG, "dlogits must have the type of the logits");
    a->d = dlogits->data;
  }
  if (!with_gradient || dlogits->data != logits->data) c.memory(logits->data, bytes, 16, false, "logits");
  if (with_gradient) c.memory(dlogits->data, bytes, 16, true, "dlogits");
}

void take_weight(Arguments& c, const mtf_tensor* logits, const mtf_tensor* weight, LossRows* a) {
  if (weight) a->weight = c.per_token(weight, logits, "weight");
}

void take_distill(Arguments& c, const mtf_tensor* logits, const int32_t* teacher_ids, const mtf_tensor* teacher, const int32_t* targets, const mtf_tensor* weight,
                  const mtf_distill_params* hp, LossRows* a) {
  if (!c.ok()) return;
  if (!hp) return c.wrong(MTF_ERR_INVALID_ARG, "NULL params");
  if (!(hp->temperature > 0.f) || !std::isfinite(hp->temperature) || !(hp->soft_weight >= 0.f) || !std::isfinite(hp->soft_weight) || !(hp->hard_weight >= 0.f) ||
      !std::isfinite(hp->hard_weight))
    return c.wrong(MTF_ERR_INVALID_ARG, "temperature must be above 0, soft_weight and hard_weight at least 0, all finite");
  // (factors of an exponent: temperature, 1 / temperature and temperature^2 all have to be ordinary numbers)
  if (hp->temperature < 1e-4f || hp->temperature > 1e4f) return c.wrong(MTF_ERR_UNSUPPORTED, "temperatures from 1e-4 to 1e4");
  a->temperature = hp->temperature;
  a->soft = hp->soft_weight;
  a->hard = hp->hard_weight;
  if (!c.there(teacher, "teacher_logits")) return;
  if (teacher->dtype != MTF_BF16 && teacher->dtype != MTF_F32) return c.wrong(MTF_ERR_INVALID_ARG, "unknown type of teacher_logits");
  c.dims_like(teacher, logits, 0, logits->ndim - 1, 1, "teacher_logits");
  if (!c.ok()) return;
  const int64_t slots = teacher->dims[teacher->ndim - 1].size;
  if (slots > mtf::kMaxTeacher) return c.wrong(MTF_ERR_UNSUPPORTED, "at most %d slots a token, got %lld", mtf::kMaxTeacher, (long long)slots);
  c.not_across_ranks(teacher->dims[teacher->ndim - 1].name);
  a->teacher_bf16 = teacher->dtype == MTF_BF16;
  a->slots = (int)slots;
  c.memory(teacher->data, a->rows * slots * (a->teacher_bf16 ? 2 : 4), a->teacher_bf16 ? 2 : 4, false, "teacher_logits");
  a->teacher = teacher->data;
  a->teacher_ids = c.ids(teacher_ids, a->rows * slots, "teacher_ids");
  if (targets || a->hard != 0.f) a->targets = c.ids(targets, a->rows, "targets");
  take_weight(c, logits, weight, a);
}

float* take_stats(Arguments& c, const mtf_tensor* logits, const mtf_tensor* stats, bool out) {
  if (!c.there(stats, "stats")) return nullptr;
  c.f32(stats, "stats");
  c.dims_like(stats, logits, 0, logits->ndim - 1, 1, "stats");
  if (!c.ok()) return nullptr;
  if (stats->dims[stats->ndim - 1].size != 2) { c.wrong(MTF_ERR_SIZE_MISMATCH, "stats hold two values per token"); return nullptr; }
  c.not_across_ranks(stats->dims[stats->ndim - 1].name);
  c.memory(stats->data, numel(*stats) * 4, 4, out, "stats");
  return reinterpret_cast<float*>(stats->data);
}

void take_policy(Arguments& c, const mtf_tensor* logits, const int32_t* targets, const mtf_tensor* old_logp, const mtf_tensor* ref_logp, const mtf_tensor* advantage,
                 const mtf_tensor* weight, const mtf_policy_params* hp, LossRows* a) {
  if (!c.ok()) return;
  if (!hp) return c.wrong(MTF_ERR_INVALID_ARG, "NULL params");
  if (!(hp->clip_low >= 0.f) || !(hp->clip_low <= 1.f) || !(hp->clip_high >= 0.f) || !(hp->kl_weight >= 0.f) || !std::isfinite(hp->kl_weight))
    return c.wrong(MTF_ERR_INVALID_ARG, "clip_low from 0 to 1, clip_high and kl_weight at least 0, kl_weight finite");
  if (hp->kl_weight != 0.f && !ref_logp) return c.wrong(MTF_ERR_INVALID_ARG, "kl_weight needs ref_logp");
  a->clip_low = hp->clip_low;
  a->clip_high = hp->clip_high;
  a->kl_weight = hp->kl_weight;
  a->targets = c.ids(targets, a->rows, "targets");
  a->old_logp = c.per_token(old_logp, logits, "old_logp");
  if (ref_logp) a->ref_logp = c.per_token(ref_logp, logits, "ref_logp");
  a->advantage = c.per_token(advantage, logits, "advantage");
  take_weight(c, logits, weight, a);
}

// one value per answer: [2, *pairs]
float* per_sequence(Arguments& c, const mtf_tensor* t, const mtf_tensor* logits, const char* name, bool out) {
  return c.ok() ? const_cast<float*>(c.values(t, logits, 0, logits->ndim - 2, name, out)) : nullptr;
}
// one value per pair: [*pairs]
float* per_pair(Arguments& c, const mtf_tensor* t, const mtf_tensor* logits, const char* name, bool out) {
  if (!c.ok()) return nullptr;
  if (logits->ndim > 3) return const_cast<float*>(c.values(t, logits, 1, logits->ndim - 3, name, out));
  if (!c.there(t, name)) return nullptr;      // one pair, without dims of its own
  c.f32(t, name);
  if (c.ok() && numel(*t) != 1) c.wrong(MTF_ERR_SIZE_MISMATCH, "%s holds one value per pair", name);
  c.memory(t->data, 4, 4, out, name);
  return reinterpret_cast<float*>(t->data);
}

void take_pairs(Arguments& c, const mtf_tensor* logits, LossRows* a) {
  if (!c.ok()) return;
  if (logits->ndim < 3 || logits->dims[0].size != 2) return c.wrong(MTF_ERR_INVALID_ARG, "logits have the dims [2, *pairs, length, vocab]");
  a->length = logits->dims[logits->ndim - 2].size;
  a->pairs = a->rows / a->length / 2;
  c.not_across_ranks(logits->dims[0].name);
  c.not_across_ranks(logits->dims[logits->ndim - 2].name);
}

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

}  // namespace

extern "C" {

mtf_status mtf_distill_forward(const mtf_layout_t* layout, const mtf_tensor* logits, const int32_t* teacher_ids, const mtf_tensor* teacher_logits,
                               const int32_t* targets, const mtf_tensor* weight, const mtf_distill_params* params, mtf_tensor* stats, mtf_tensor* loss, void* stream) {
  return guarded("distill_forward", [&] {
    Arguments c("distill_forward", layout);
    LossRows a;
    take_logits(c, logits, false, nullptr, &a);
    take_distill(c, logits, teacher_ids, teacher_logits, targets, weight, params, &a);
    a.lse = take_stats(c, logits, stats, true);
    a.loss = c.token_out(loss, logits, "loss");
    return c.ok() ? mtf::launch_loss_rows(mtf::LOSS_DISTILL, mtf::LOSS_FORWARD, a, stream) : c.st;
  });
}

mtf_status mtf_distill_backward(const mtf_layout_t* layout, const mtf_tensor* logits, const int32_t* teacher_ids, const mtf_tensor* teacher_logits,
                                const int32_t* targets, const mtf_tensor* weight, const mtf_distill_params* params, const mtf_tensor* stats,
                                const mtf_tensor* dloss, mtf_tensor* dlogits, void* stream) {
  return guarded("distill_backward", [&] {
    Arguments c("distill_backward", layout);
    LossRows a;
    take_logits(c, logits, true, dlogits, &a);
    take_distill(c, logits, teacher_ids, teacher_logits, targets, weight, params, &a);
    a.lse = take_stats(c, logits, stats, false);
    if (dloss) a.dloss = c.per_token(dloss, logits, "dloss");
    return c.ok() ? mtf::launch_loss_rows(mtf::LOSS_DISTILL, mtf::LOSS_BACKWARD, a, stream) : c.st;
  });
}

mtf_status mtf_distill_step(const mtf_layout_t* layout, const mtf_tensor* logits, const int32_t* teacher_ids, const mtf_tensor* teacher_logits, const int32_t* targets,
                            const mtf_tensor* weight, const mtf_distill_params* params, mtf_tensor* loss, mtf_tensor* dlogits, void* stream) {
  return guarded("distill_step", [&] {
    Arguments c("distill_step", layout);
    LossRows a;
    take_logits(c, logits, true, dlogits, &a);
    take_distill(c, logits, teacher_ids, teacher_logits, targets, weight, params, &a);
    a.loss = c.token_out(loss, logits, "loss");
    return c.ok() ? mtf::launch_loss_rows(mtf::LOSS_DISTILL, mtf::LOSS_STEP, a, stream) : c.st;
  });
}

mtf_status mtf_policy_forward(const mtf_layout_t* layout, const mtf_tensor* logits, const int32_t* targets, const mtf_tensor* old_logp, const mtf_tensor* ref_logp,
                              const mtf_tensor* advantage, const mtf_tensor* weight, const mtf_policy_params* params, mtf_tensor* lse, mtf_tensor* logp,
                              mtf_tensor* dlogp, mtf_tensor* loss, void* stream) {
  return guarded("policy_forward", [&] {
    Arguments c("policy_forward", layout);
    LossRows a;
    take_logits(c, logits, false, nullptr, &a);
    take_policy(c, logits, targets, old_logp, ref_logp, advantage, weight, params, &a);
    a.lse = c.token_out(lse, logits, "lse");
    a.logp = c.token_out(logp, logits, "logp");
    a.dlogp = c.token_out(dlogp, logits, "dlogp");
    a.loss = c.token_out(loss, logits, "loss");
    return c.ok() ? mtf::launch_loss_rows(mtf::LOSS_POLICY, mtf::LOSS_FORWARD, a, stream) : c.st;
  });
}

mtf_status mtf_policy_backward(const mtf_layout_t* layout, const mtf_tensor* logits, const int32_t* targets, const mtf_tensor* lse, const mtf_tensor* dlogp,
                               const mtf_tensor* dloss, mtf_tensor* dlogits, void* stream) {
  return guarded("policy_backward", [&] {
    Arguments c("policy_backward", layout);
    LossRows a;
    take_logits(c, logits, true, dlogits, &a);
    if (c.ok()) a.targets = c.ids(targets, a.rows, "targets");
    a.lse = const_cast<float*>(c.per_token(lse, logits, "lse"));
    a.dlogp = const_cast<float*>(c.per_token(dlogp, logits, "dlogp"));
    if (dloss) a.dloss = c.per_token(dloss, logits, "dloss");
    return c.ok() ? mtf::launch_loss_rows(mtf::LOSS_POLICY, mtf::LOSS_BACKWARD, a, stream) : c.st;
  });
}

mtf_status mtf_policy_step(const mtf_layout_t* layout, const mtf_tensor* logits, const int32_t* targets, const mtf_tensor* old_logp, const mtf_tensor* ref_logp,
                           const mtf_tensor* advantage, const mtf_tensor* weight, const mtf_policy_params* params, mtf_tensor* logp, mtf_tensor* loss,
                           mtf_tensor* dlogits, void* stream) {
  return guarded("policy_step", [&] {
    Arguments c("policy_step", layout);
    LossRows a;
    take_logits(c, logits, true, dlogits, &a);
    take_policy(c, logits, targets, old_logp, ref_logp, advantage, weight, params, &a);
    a.logp = c.token_out(logp, logits, "logp");
    a.loss = c.token_out(loss, logits, "loss");
    return c.ok() ? mtf::launch_loss_rows(mtf::LOSS_POLICY, mtf::LOSS_STEP, a, stream) : c.st;
  });
}

mtf_status mtf_preference_forward(const mtf_layout_t* layout, const mtf_tensor* logits, const int32_t* targets, const mtf_tensor* weight, const mtf_tensor* ref_logp,
                                  const mtf_preference_params* params, mtf_tensor* lse, mtf_tensor* logp, mtf_tensor* seq_logp, mtf_tensor* dseq, mtf_tensor* loss,
                                  void* stream) {
  return guarded("preference_forward", [&] {
    Arguments c("preference_forward", layout);
    LossRows a;
    mtf::PreferencePairs p;
    take_logits(c, logits, false, nullptr, &a);
    take_pairs(c, logits, &a);
    if (c.ok() && !params) c.wrong(MTF_ERR_INVALID_ARG, "NULL params");
    if (c.ok()) {
      if (params->kind < MTF_PREFERENCE_SIGMOID || params->kind > MTF_PREFERENCE_SQUARED) c.wrong(MTF_ERR_INVALID_ARG, "unknown kind %d", (int)params->kind);
      if (!(params->beta > 0.f) || !std::isfinite(params->beta)) c.wrong(MTF_ERR_INVALID_ARG, "beta must be above 0 and finite");
      if (!(params->smoothing >= 0.f) || !(params->smoothing <= 0.5f) || (params->smoothing != 0.f && params->kind != MTF_PREFERENCE_SIGMOID))
        c.wrong(MTF_ERR_INVALID_ARG, "smoothing from 0 to 0.5, and 0 unless the kind is sigmoid");
      p.kind = params->kind;
      p.beta = params->beta;
      p.smoothing = params->smoothing;
    }
    if (c.ok()) a.targets = c.ids(targets, a.rows, "targets");
    if (c.ok()) take_weight(c, logits, weight, &a);
    p.ref = per_sequence(c, ref_logp, logits, "ref_logp", false);
    a.lse = c.token_out(lse, logits, "lse");
    a.logp = c.token_out(logp, logits, "logp");
    p.seq = per_sequence(c, seq_logp, logits, "seq_logp", true);
    p.dseq = per_sequence(c, dseq, logits, "dseq", true);
    p.loss = per_pair(c, loss, logits, "loss", true);
    if (!c.ok()) return c.st;
    p.z = a.z;
    p.V = a.V;
    p.bf16 = a.bf16;
    p.targets = a.targets;
    p.lse = a.lse;
    p.logp = a.logp;
    p.weight = a.weight;
    p.pairs = a.pairs;
    p.length = a.length;
    const mtf_status st = mtf::launch_loss_rows(mtf::LOSS_LOGP, mtf::LOSS_FORWARD, a, stream);
    return st == MTF_OK ? mtf::launch_preference_pairs(p, stream) : st;
  });
}

mtf_status mtf_preference_backward(const mtf_layout_t* layout, const mtf_tensor* logits, const int32_t* targets, const mtf_tensor* weight, const mtf_tensor* lse,
                                   const mtf_tensor* dseq, const mtf_tensor* dloss, mtf_tensor* dlogits, void* stream) {
  return guarded("preference_backward", [&] {
    Arguments c("preference_backward", layout);
    LossRows a;
    take_logits(c, logits, true, dlogits, &a);
    take_pairs(c, logits, &a);
    if (c.ok()) a.targets = c.ids(targets, a.rows, "targets");
    if (c.ok()) take_weight(c, logits, weight, &a);
    a.lse = const_cast<float*>(c.per_token(lse, logits, "lse"));
    a.dseq = per_sequence(c, dseq, logits, "dseq", false);
    if (dloss) a.dloss = per_pair(c, dloss, logits, "dloss", false);
    return c.ok() ? mtf::launch_loss_rows(mtf::LOSS_LOGP, mtf::LOSS_BACKWARD, a, stream) : c.st;
  });
}

}  // extern "C"
