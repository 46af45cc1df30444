// Entry points of answering: a paged cache of keys and values, attention of one new token over it, beam search's selection and the reordering
// behind it.  Validation only; the arithmetic runs in cache_rows.cu, attention_decode.cu and beam_select.cu.
#include <cmath>

#include "answer.h"
#include "arguments.h"

using mtf::Arguments;
using mtf::CachePool;
using mtf::Dim;
using mtf::guarded;
using mtf::numel;

namespace {

// (sizes whose product no memory holds would wrap around in what follows)
void holds(Arguments& c, const mtf_tensor* t, const char* name) {
  if (!c.ok()) return;
  int64_t n = 1;
  for (int i = 0; i < t->ndim; ++i) {
    if (t->dims[i].size > (1LL << 46) / n) return c.wrong(MTF_ERR_UNSUPPORTED, "%s has more than 2^46 values", name);
    n *= t->dims[i].size;
  }
}

bool same(const mtf_dim& a, const mtf_dim& b) { return a.size == b.size && (a.name == b.name || !strcmp(a.name, b.name)); }

// The pools of a cache and their places in memory; `heads`: the name of the heads' dimension (NULL: whichever is not the slots').
struct TakenCache {
  const mtf_tensor* k = nullptr;
  const mtf_dim* heads = nullptr;
  CachePool p;
};
void take_cache(Arguments& c, const mtf_cache* cache, long long sequences, bool written, TakenCache* t) {
  if (!c.ok()) return;
  if (!cache) return c.wrong(MTF_ERR_INVALID_ARG, "NULL cache");
  const mtf_tensor *k = cache->k, *v = cache->v;
  if (!c.there(k, "the cache's k") || !c.there(v, "the cache's v")) return;
  holds(c, k, "the cache's k");
  holds(c, v, "the cache's v");
  if (!c.ok()) return;
  if (k->ndim != 4 || v->ndim != 4) return c.wrong(MTF_ERR_INVALID_ARG, "the cache's k and v have the dims [page, slot, heads, d] or [page, heads, slot, d]");
  if (k->dtype != MTF_BF16 && k->dtype != MTF_E4M3) return c.wrong(MTF_ERR_UNSUPPORTED, "the cache must be bf16 or e4m3");
  if (v->dtype != k->dtype) return c.wrong(MTF_ERR_INVALID_ARG, "the cache's k and v must be of one type");
  for (int i = 0; i < 3; ++i)
    if (!same(k->dims[i], v->dims[i])) return c.wrong(MTF_ERR_SIZE_MISMATCH, "the cache's k and v differ in dimension %d ('%s')", i, k->dims[i].name);
  const char* const slot = cache->slot ? cache->slot : "slot";
  const int at = !strcmp(k->dims[1].name, slot) ? 1 : !strcmp(k->dims[2].name, slot) ? 2 : 0;
  if (!at) return c.wrong(MTF_ERR_UNKNOWN_DIM, "neither the second nor the third dimension of the cache's k is the slots' ('%s')", slot);
  t->k = k;
  t->heads = &k->dims[3 - at];
  CachePool& p = t->p;
  p.e4m3 = k->dtype == MTF_E4M3;
  const int64_t pages = k->dims[0].size, slots = k->dims[at].size, heads = t->heads->size, dk = k->dims[3].size, dv = v->dims[3].size;
  const int step = p.e4m3 ? 16 : 8;
  if (dk % step || dv % step || dk > mtf::kMaxCacheWidth || dv > mtf::kMaxCacheWidth)
    return c.wrong(MTF_ERR_UNSUPPORTED, "rows of the cache have a multiple of %d values, at most %d; these have %lld and %lld", step, mtf::kMaxCacheWidth, (long long)dk, (long long)dv);
  if (pages > 0x7fffffffLL || slots > 0x7fffffffLL || heads > 0x7fffffffLL || slots * heads > (1LL << 24) || pages * slots * heads > 0x7fffffffLL)
    return c.wrong(MTF_ERR_UNSUPPORTED, "at most 2^31 rows in a cache, and 2^24 in a page");
  if (cache->table_pages < 1) return c.wrong(MTF_ERR_INVALID_ARG, "table_pages must be at least 1");
  if (cache->table_pages > (1LL << 30) || cache->table_pages * slots > (1LL << 30) || sequences > 0x7fffffffLL) return c.wrong(MTF_ERR_UNSUPPORTED, "at most 2^30 positions a sequence, 2^31 sequences");
  c.not_across_ranks(k->dims[0].name);
  c.not_across_ranks(k->dims[at].name);
  c.not_across_ranks(k->dims[3].name);
  c.not_across_ranks(v->dims[3].name);
  p.dk = (int)dk;
  p.dv = (int)dv;
  p.heads = (int)heads;
  p.slots = (int)slots;
  p.pages = (int)pages;
  p.rows_page = (int)(slots * heads);
  p.row_slot = at == 1 ? (int)heads : 1;
  p.row_head = at == 1 ? 1 : (int)slots;
  p.per_sequence = (int)cache->table_pages;
  p.sequences = sequences;
  p.k = k->data;
  p.v = v->data;
  const int64_t rows = pages * slots * heads, bytes = p.e4m3 ? 1 : 2;
  c.memory(k->data, rows * dk * bytes, 16, written, "the cache's k");
  c.memory(v->data, rows * dv * bytes, 16, written, "the cache's v");
  if (!p.e4m3 && (cache->k_scale || cache->v_scale)) return c.wrong(MTF_ERR_INVALID_ARG, "scales belong to an e4m3 cache");
  if (p.e4m3) {
    const char* const of = c.of_name;
    c.of_name = "cache's k";
    p.ks = const_cast<float*>(c.values(cache->k_scale, k, 0, 3, "the cache's k_scale", written));
    if (c.ok()) p.vs = const_cast<float*>(c.values(cache->v_scale, k, 0, 3, "the cache's v_scale", written));
    c.of_name = of;
  }
  if (!c.ok()) return;
  p.table = c.ids(cache->table, sequences * cache->table_pages, "the cache's table");
}

// The layout has to keep apart all dimensions that an operation walks over, those of several tensors together.
void together(Arguments& c, std::initializer_list<std::pair<const mtf_tensor*, int>> of) {
  if (!c.ok() || c.layout->rules.empty()) return;
  std::vector<Dim> all;
  for (const auto& t : of)
    for (int i = t.second; i < t.first->ndim; ++i) {
      bool known = false;
      for (const Dim& d : all) known |= d.name == t.first->dims[i].name;
      if (!known) all.push_back({t.first->dims[i].name, t.first->dims[i].size});
    }
  c.st = mtf::check_tensor(c.layout, all);
}

// dense rows [*sequences, length, heads, d] of k, and v's like them
void take_dense(Arguments& c, const mtf_tensor* kk, const mtf_tensor* vv, long long* sequences, mtf::CacheRows* r) {
  if (!c.there(kk, "kk") || !c.there(vv, "vv")) return;
  if (kk->ndim < 4) return c.wrong(MTF_ERR_INVALID_ARG, "kk and vv have the dims [*sequences, length, heads, d]");
  holds(c, kk, "kk");
  holds(c, vv, "vv");
  c.of_name = "kk";
  c.dims_like(vv, kk, 0, kk->ndim - 1, 1, "vv");
  if (!c.ok()) return;
  if (kk->dtype != MTF_BF16 && kk->dtype != MTF_F32) return c.wrong(MTF_ERR_UNSUPPORTED, "kk and vv must be bf16 or f32");
  if (vv->dtype != kk->dtype) return c.wrong(MTF_ERR_INVALID_ARG, "kk and vv must be of one type");
  long long n = 1;
  for (int i = 0; i < kk->ndim - 3; ++i) n *= kk->dims[i].size;
  *sequences = n;
  r->k = kk->data;
  r->v = vv->data;
  r->bf16 = kk->dtype == MTF_BF16;
  r->length = kk->dims[kk->ndim - 3].size;
  const int64_t heads = kk->dims[kk->ndim - 2].size;
  if (n > 0x7fffffffLL || r->length > 0x7fffffffLL || n * r->length > 0x7fffffffLL || heads > 0x7fffffffLL || n * r->length * heads > 0x7fffffffLL)
    return c.wrong(MTF_ERR_UNSUPPORTED, "at most 2^31 rows");
}
void dense_fits(Arguments& c, const mtf_tensor* kk, const mtf_tensor* vv, const mtf_cache* cache, const TakenCache& t, bool written) {
  if (!c.ok()) return;
  const int last = kk->ndim - 1;
  if (!same(kk->dims[last - 1], *t.heads)) return c.wrong(MTF_ERR_SIZE_MISMATCH, "kk's heads are not those of the cache ('%s', %lld)", t.heads->name, (long long)t.heads->size);
  if (!same(kk->dims[last], cache->k->dims[3]) || !same(vv->dims[last], cache->v->dims[3])) return c.wrong(MTF_ERR_SIZE_MISMATCH, "the last dimensions of kk and vv are not those of the cache");
  const int bytes = kk->dtype == MTF_BF16 ? 2 : 4;
  c.memory(kk->data, numel(*kk) * bytes, 16, written, "kk");
  c.memory(vv->data, numel(*vv) * bytes, 16, written, "vv");
  together(c, {{kk, 0}, {cache->k, 0}, {cache->v, 0}});
}

mtf_status cache_rows(const char* what, const mtf_layout_t* layout, const mtf_tensor* kk, const mtf_tensor* vv, const int32_t* starts, const int32_t* counts,
                      const mtf_cache* cache, bool write, void* stream) {
  return guarded(what, [&] {
    Arguments c(what, layout);
    TakenCache t;
    mtf::CacheRows r;
    long long sequences = 0;
    take_dense(c, kk, vv, &sequences, &r);
    take_cache(c, cache, sequences, write, &t);
    dense_fits(c, kk, vv, cache, t, !write);
    if (c.ok() && starts) r.starts = c.ids(starts, sequences, "starts");
    if (c.ok() && counts) r.counts = c.ids(counts, sequences, "counts");
    if (!c.ok()) return c.st;
    return write ? mtf::launch_cache_write(t.p, r, stream) : mtf::launch_cache_read(t.p, r, stream);
  });
}

// q [*sequences, heads, d_k] or [*sequences, heads, group, d_k]
void take_queries(Arguments& c, const mtf_tensor* q, const mtf_cache* cache, TakenCache* t, int* group, bool data) {
  if (!c.ok()) return;
  if (!c.there(q, "q", data)) return;
  holds(c, q, "q");
  if (!c.ok()) return;
  if (q->ndim < 3) return c.wrong(MTF_ERR_INVALID_ARG, "q has the dims [*sequences, heads, d_k] or [*sequences, heads, group, d_k]");
  // the heads' place is known from the cache, whose checks want the number of sequences: by name first
  if (!cache || !cache->k || !cache->k->dims || cache->k->ndim != 4) return c.wrong(MTF_ERR_INVALID_ARG, "the cache's k is NULL or has other dims than [page, slot, heads, d] or [page, heads, slot, d]");
  const char* const slot = cache->slot ? cache->slot : "slot";
  const mtf_dim* heads = nullptr;
  for (int i = 1; i < 3; ++i)
    if (cache->k->dims[i].name && strcmp(cache->k->dims[i].name, slot)) heads = &cache->k->dims[i];
  const int last = q->ndim - 1;
  int at = -1;
  if (heads)
    for (int i = last - 1; i >= last - 2 && i >= 1; --i)
      if (!strcmp(q->dims[i].name, heads->name)) at = i;
  if (at < 0) return c.wrong(MTF_ERR_SIZE_MISMATCH, "q has the dims [*sequences, heads, d_k] or [*sequences, heads, group, d_k], with the cache's name for heads");
  long long n = 1;
  for (int i = 0; i < at; ++i) n *= q->dims[i].size;
  const int64_t g = at == last - 2 ? q->dims[last - 1].size : 1;
  if (g > 4096) return c.wrong(MTF_ERR_UNSUPPORTED, "at most 4096 heads of queries to a head of the cache");
  *group = (int)g;
  take_cache(c, cache, n, false, t);
  if (!c.ok()) return;
  if (!same(q->dims[at], *t->heads) || !same(q->dims[last], cache->k->dims[3])) return c.wrong(MTF_ERR_SIZE_MISMATCH, "q's heads or last dimension are not those of the cache");
  if (q->dtype != MTF_BF16) return c.wrong(MTF_ERR_UNSUPPORTED, "q must be bf16");
  if (n * t->heads->size * g > 0x7fffffffLL) return c.wrong(MTF_ERR_UNSUPPORTED, "at most 2^31 heads of queries");
  together(c, {{q, 0}, {cache->k, 0}, {cache->v, 0}});
}

}  // namespace

extern "C" {

mtf_status mtf_cache_write(const mtf_layout_t* layout, const mtf_tensor* kk, const mtf_tensor* vv, const int32_t* starts, const int32_t* counts, const mtf_cache* cache,
                           void* stream) {
  return cache_rows("cache_write", layout, kk, vv, starts, counts, cache, true, stream);
}

mtf_status mtf_cache_read(const mtf_layout_t* layout, const mtf_cache* cache, const int32_t* starts, const int32_t* counts, mtf_tensor* kk, mtf_tensor* vv, void* stream) {
  return cache_rows("cache_read", layout, kk, vv, starts, counts, cache, false, stream);
}

mtf_status mtf_attention_decode(const mtf_layout_t* layout, const mtf_tensor* q, const mtf_cache* cache, const int32_t* lengths, float scale, mtf_tensor* o, void* workspace,
                                size_t workspace_bytes, void* stream) {
  return guarded("attention_decode", [&] {
    Arguments c("attention_decode", layout);
    TakenCache t;
    mtf::DecodeCall d;
    take_queries(c, q, cache, &t, &d.group, true);
    if (!c.there(o, "o")) return c.st;
    holds(c, o, "o");
    c.of_name = "q";
    c.dims_like(o, q, 0, q->ndim - 1, 1, "o");
    if (c.ok() && !same(o->dims[o->ndim - 1], cache->v->dims[3])) c.wrong(MTF_ERR_SIZE_MISMATCH, "o's last dimension is not that of the cache's v");
    if (c.ok() && o->dtype != MTF_BF16) c.wrong(MTF_ERR_UNSUPPORTED, "o must be bf16");
    if (c.ok() && !std::isfinite(scale * 1.5f)) c.wrong(MTF_ERR_INVALID_ARG, "scale must be finite, and in powers of two, too");
    if (!c.ok()) return c.st;
    c.memory(q->data, numel(*q) * 2, 16, false, "q");
    c.memory(o->data, numel(*o) * 2, 16, true, "o");
    d.lengths = c.ids(lengths, t.p.sequences, "lengths");
    if (!c.ok()) return c.st;
    const size_t need = mtf::attention_decode_workspace(t.p, d.group);
    if (need) {
      if (!workspace || workspace_bytes < need) return mtf::fail(MTF_ERR_WORKSPACE_TOO_SMALL, "attention_decode: needs %zu workspace bytes, got %zu", need, workspace ? workspace_bytes : (size_t)0);
      c.memory(workspace, (int64_t)need, 16, true, "workspace");
      if (!c.ok()) return c.st;
    }
    d.q = q->data;
    d.o = o->data;
    d.scale = scale;
    d.workspace = workspace;
    return mtf::launch_attention_decode(t.p, d, stream);
  });
}

mtf_status mtf_attention_decode_workspace_bytes(const mtf_layout_t* layout, const mtf_tensor* q, const mtf_cache* cache, size_t* bytes) {
  return guarded("attention_decode_workspace_bytes", [&] {
    Arguments c("attention_decode_workspace_bytes", layout);
    TakenCache t;
    int group = 1;
    if (c.ok() && !bytes) c.wrong(MTF_ERR_INVALID_ARG, "NULL result");
    take_queries(c, q, cache, &t, &group, false);
    if (!c.ok()) return c.st;
    *bytes = mtf::attention_decode_workspace(t.p, group);
    return MTF_OK;
  });
}

mtf_status mtf_beam_select(const mtf_layout_t* layout, const mtf_tensor* logits, const mtf_tensor* scores, const int32_t* finished, int32_t end_id, int32_t* parents,
                           int32_t* tokens, mtf_tensor* new_scores, int32_t* new_finished, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded("beam_select", [&] {
    Arguments c("beam_select", layout);
    mtf::BeamSelect b;
    if (!c.there(logits, "logits")) return c.st;
    holds(c, logits, "logits");
    const int last = logits->ndim - 1;
    if (last < 1) c.wrong(MTF_ERR_INVALID_ARG, "logits have the dims [*sentences, beam, vocab]");
    if (c.ok() && logits->dtype != MTF_BF16 && logits->dtype != MTF_F32) c.wrong(MTF_ERR_UNSUPPORTED, "logits must be bf16 or f32");
    if (!c.ok()) return c.st;
    const int64_t V = logits->dims[last].size, beams = logits->dims[last - 1].size, rows = numel(*logits) / V, sentences = rows / beams;
    if (rows > 0x7ff00000LL || beams * V > 0x7fffff00LL) c.wrong(MTF_ERR_UNSUPPORTED, "at most 2^31 beams, and 2^31 words of a sentence's beams");
    if (c.ok() && beams > mtf::kMaxBeams) c.wrong(MTF_ERR_UNSUPPORTED, "at most %d beams, got %lld", mtf::kMaxBeams, (long long)beams);
    c.not_across_ranks(logits->dims[last].name);
    c.not_across_ranks(logits->dims[last - 1].name);
    if (c.ok() && (end_id < 0 || end_id >= V)) c.wrong(MTF_ERR_INVALID_ARG, "end_id outside [0, vocab)");
    c.memory(logits->data, numel(*logits) * (logits->dtype == MTF_BF16 ? 2 : 4), 16, false, "logits");
    b.scores = c.per_token(scores, logits, "scores");
    if (finished) b.finished = c.ids(finished, rows, "finished");
    if (!c.there(new_scores, "new_scores")) return c.st;
    c.f32(new_scores, "new_scores");
    c.dims_like(new_scores, logits, 0, last - 1, 1, "new_scores");
    if (!c.ok()) return c.st;
    const int64_t slots = new_scores->dims[last - 1].size, out = sentences * slots;
    c.not_across_ranks(new_scores->dims[last - 1].name);
    if (slots > mtf::kMaxSlots || slots > beams * V) c.wrong(MTF_ERR_UNSUPPORTED, "at most %d slots, and not more than there are words of beams; got %lld", mtf::kMaxSlots, (long long)slots);
    c.memory(new_scores->data, out * 4, 4, true, "new_scores");
    auto result = [&](int32_t* p, const char* name) {
      if (c.ok() && !p) c.wrong(MTF_ERR_INVALID_ARG, "%s is NULL", name);
      c.memory(p, out * 4, 4, true, name);
      return p;
    };
    b.parents = result(parents, "parents");
    b.tokens = result(tokens, "tokens");
    if (new_finished) b.new_finished = result(new_finished, "new_finished");
    if (!c.ok()) return c.st;
    const size_t need = mtf::beam_select_workspace(sentences, (int)beams, (int)V, logits->dtype == MTF_BF16);
    if (!workspace || workspace_bytes < need) return mtf::fail(MTF_ERR_WORKSPACE_TOO_SMALL, "beam_select: needs %zu workspace bytes, got %zu", need, workspace ? workspace_bytes : (size_t)0);
    c.memory(workspace, (int64_t)need, 16, true, "workspace");
    if (!c.ok()) return c.st;
    b.logits = logits->data;
    b.bf16 = logits->dtype == MTF_BF16;
    b.vocab = (int)V;
    b.beams = (int)beams;
    b.slots = (int)slots;
    b.sentences = sentences;
    b.end_id = end_id;
    b.new_scores = reinterpret_cast<float*>(new_scores->data);
    b.workspace = workspace;
    return mtf::launch_beam_select(b, stream);
  });
}

mtf_status mtf_beam_select_workspace_bytes(const mtf_layout_t* layout, const mtf_tensor* logits, int64_t slots, size_t* bytes) {
  return guarded("beam_select_workspace_bytes", [&] {
    Arguments c("beam_select_workspace_bytes", layout);
    if (c.ok() && (!logits || !bytes)) c.wrong(MTF_ERR_INVALID_ARG, "NULL argument");
    if (!c.ok()) return c.st;
    std::vector<Dim> d;
    if ((c.st = mtf::read_dims(logits->ndim, logits->dims, &d, "logits")) != MTF_OK || (c.st = mtf::check_tensor(layout, d)) != MTF_OK) return c.st;
    holds(c, logits, "logits");
    const int last = logits->ndim - 1;
    if (last < 1) c.wrong(MTF_ERR_INVALID_ARG, "logits have the dims [*sentences, beam, vocab]");
    else if (logits->dims[last - 1].size * logits->dims[last].size > 0x7fffff00LL || numel(*logits) / logits->dims[last].size > 0x7ff00000LL)
      c.wrong(MTF_ERR_UNSUPPORTED, "at most 2^31 beams, and 2^31 words of a sentence's beams");
    else if (logits->dims[last - 1].size > mtf::kMaxBeams || slots > mtf::kMaxSlots) c.wrong(MTF_ERR_UNSUPPORTED, "at most %d beams and %d slots", mtf::kMaxBeams, mtf::kMaxSlots);
    else if (slots < 1) c.wrong(MTF_ERR_INVALID_ARG, "at least one slot");
    if (!c.ok()) return c.st;
    const int64_t beams = logits->dims[last - 1].size, V = logits->dims[last].size;
    *bytes = mtf::beam_select_workspace(numel(*logits) / V / beams, (int)beams, (int)V, logits->dtype == MTF_BF16);
    return MTF_OK;
  });
}

mtf_status mtf_beam_reorder(const mtf_layout_t* layout, const char* beam, const int32_t* parents, const mtf_tensor* states, mtf_tensor* out, void* stream) {
  return guarded("beam_reorder", [&] {
    Arguments c("beam_reorder", layout);
    if (c.ok() && !beam) c.wrong(MTF_ERR_INVALID_ARG, "NULL name of the beams' dimension");
    if (!c.there(states, "states") || !c.there(out, "out")) return c.st;
    holds(c, states, "states");
    holds(c, out, "out");
    if (!c.ok()) return c.st;
    int at = -1;
    for (int i = 0; i < states->ndim; ++i)
      if (!strcmp(states->dims[i].name, beam)) at = i;
    if (at < 0) return mtf::fail(MTF_ERR_UNKNOWN_DIM, "beam_reorder: the states have no dimension '%s'", beam);
    if (states->dtype != MTF_F32 && states->dtype != MTF_BF16 && states->dtype != MTF_E4M3) c.wrong(MTF_ERR_INVALID_ARG, "unknown type of the states");
    if (c.ok() && out->dtype != states->dtype) c.wrong(MTF_ERR_INVALID_ARG, "out must have the type of the states");
    if (c.ok() && out->ndim != states->ndim) c.wrong(MTF_ERR_SIZE_MISMATCH, "out has %d dims, not %d", (int)out->ndim, (int)states->ndim);
    if (!c.ok()) return c.st;
    long long groups = 1, bytes = states->dtype == MTF_F32 ? 4 : states->dtype == MTF_BF16 ? 2 : 1;
    const long long size = bytes;
    for (int i = 0; i < states->ndim; ++i) {
      if (strcmp(out->dims[i].name, states->dims[i].name) || (i != at && out->dims[i].size != states->dims[i].size)) {
        c.wrong(MTF_ERR_SIZE_MISMATCH, "dimension %d of out is not that of the states ('%s', %lld)", i, states->dims[i].name, (long long)states->dims[i].size);
        return c.st;
      }
      if (i < at) groups *= states->dims[i].size;
      if (i > at) bytes *= states->dims[i].size;
    }
    const int64_t beams = states->dims[at].size, slots = out->dims[at].size;
    c.not_across_ranks(beam);
    if (groups > 0x7fffffffLL || slots > 0x7fffffffLL || beams > 0x7fffffffLL || groups * slots > 0x7fffffffLL) c.wrong(MTF_ERR_UNSUPPORTED, "at most 2^31 beams");
    c.memory(states->data, numel(*states) * size, (int)size, false, "states");
    c.memory(out->data, numel(*out) * size, (int)size, true, "out");
    c.ids(parents, groups * slots, "parents");
    if (!c.ok()) return c.st;
    return mtf::launch_beam_reorder(parents, states->data, out->data, groups, (int)beams, (int)slots, bytes, stream);
  });
}

mtf_status mtf_cache_reorder(const mtf_layout_t* layout, const mtf_cache* cache, int64_t sentences, int64_t beams, int64_t slots, const int32_t* parents,
                             const int32_t* lengths, const int32_t* fresh, int32_t* new_table, int32_t* new_lengths, void* stream) {
  return guarded("cache_reorder", [&] {
    Arguments c("cache_reorder", layout);
    TakenCache t;
    mtf::CacheReorder r;
    if (c.ok() && (sentences < 1 || beams < 1 || slots < 1)) c.wrong(MTF_ERR_INVALID_ARG, "sentences, beams and slots are at least 1");
    if (c.ok() && (sentences > 0x7fffffffLL || beams > 0x7fffffffLL || slots > 0x7fffffffLL || sentences * beams > 0x7fffffffLL || sentences * slots > 0x7fffffffLL))
      c.wrong(MTF_ERR_UNSUPPORTED, "at most 2^31 beams");
    take_cache(c, cache, c.ok() ? sentences * beams : 0, true, &t);
    if (!c.ok()) return c.st;
    together(c, {{cache->k, 0}, {cache->v, 0}});
    r.parents = c.ids(parents, sentences * slots, "parents");
    r.lengths = c.ids(lengths, sentences * beams, "lengths");
    r.fresh = c.ids(fresh, sentences * slots, "fresh");
    if (c.ok() && (!new_table || !new_lengths)) c.wrong(MTF_ERR_INVALID_ARG, "new_table or new_lengths is NULL");
    c.memory(new_table, sentences * slots * t.p.per_sequence * 4, 4, true, "new_table");
    c.memory(new_lengths, sentences * slots * 4, 4, true, "new_lengths");
    if (!c.ok()) return c.st;
    r.table = new_table;
    r.new_lengths = new_lengths;
    r.groups = sentences;
    r.beams = (int)beams;
    r.out = (int)slots;
    return mtf::launch_cache_reorder(t.p, r, stream);
  });
}

}  // extern "C"
