// What the entry points of answering (answer.cpp: paged caches, attention of one new token, beam search) hand to their kernels.
#pragma once

#include <cstdint>

#include "mtf_internal.h"

namespace mtf {

constexpr int kMaxCacheWidth = 256;   // d_k, d_v
constexpr int kMaxSlots = 64;         // of beam selection: the best of a sentence
constexpr int kMaxBeams = 64;

// The pools of a paged cache: rows of d values, row (page, slot, head) at page * rows_page + slot * row_slot + head * row_head.
struct CachePool {
  void *k = nullptr, *v = nullptr;
  float *ks = nullptr, *vs = nullptr;          // e4m3: a scale a row
  int e4m3 = 0;
  int dk = 0, dv = 0, heads = 0, slots = 0;    // slots of a page
  int pages = 0;
  int rows_page = 0, row_slot = 0, row_head = 0;
  const int32_t* table = nullptr;              // [sequence, per_sequence]
  int per_sequence = 0;
  long long sequences = 0;
};

// New or dense rows [sequence, length, heads, d]; row i of a sequence is position start + i, its first `counts` rows are meant.
struct CacheRows {
  void *k = nullptr, *v = nullptr;
  int bf16 = 0;
  long long length = 0;
  const int32_t *starts = nullptr, *counts = nullptr;   // NULL: 0, length
};
mtf_status launch_cache_write(const CachePool& c, const CacheRows& r, void* stream);
mtf_status launch_cache_read(const CachePool& c, const CacheRows& r, void* stream);

struct CacheReorder {
  const int32_t *parents = nullptr, *lengths = nullptr, *fresh = nullptr;   // [group, out], [group, beams], [group, out]
  int32_t *table = nullptr, *new_lengths = nullptr;                         // [group, out, per_sequence], [group, out]
  long long groups = 0;
  int beams = 0, out = 0;
};
mtf_status launch_cache_reorder(const CachePool& c, const CacheReorder& r, void* stream);
// out[g, i, :] = in[g, parents[g, i], :], rows of `bytes`
mtf_status launch_beam_reorder(const int32_t* parents, const void* in, void* out, long long groups, int beams, int slots, long long bytes, void* stream);

struct DecodeCall {
  const void* q = nullptr;                     // bf16 [sequence, heads, group, dk]
  void* o = nullptr;                           // bf16 [sequence, heads, group, dv]
  const int32_t* lengths = nullptr;
  int group = 1;
  float scale = 1.f;
  void* workspace = nullptr;
};
size_t attention_decode_workspace(const CachePool& c, int group);
mtf_status launch_attention_decode(const CachePool& c, const DecodeCall& d, void* stream);

struct BeamSelect {
  const void* logits = nullptr;                // [sentence, beams, vocab]
  int bf16 = 0, vocab = 0, beams = 0, slots = 0;
  long long sentences = 0;
  const float* scores = nullptr;
  const int32_t* finished = nullptr;
  int end_id = 0;
  int32_t *parents = nullptr, *tokens = nullptr, *new_finished = nullptr;   // [sentence, slots]; new_finished may be NULL
  float* new_scores = nullptr;
  void* workspace = nullptr;
};
size_t beam_select_workspace(long long sentences, int beams, int vocab, int bf16);
mtf_status launch_beam_select(const BeamSelect& b, void* stream);

}  // namespace mtf
