// What the entry points of the losses on stored logits (losses.cpp) hand to their kernels (loss_rows.cu).
#pragma once

#include <cstdint>

#include "mtf_internal.h"

namespace mtf {

constexpr int kMaxTeacher = 512;      // slots of a teacher's list

// One row of logits per token.  Pointers that an operator does not use are NULL.
struct LossRows {
  const void* z = nullptr;            // logits [rows, V]
  void* d = nullptr;                  // their gradient; may be z
  long long rows = 0;
  int V = 0;
  int bf16 = 0;
  const int32_t* targets = nullptr;
  const float* weight = nullptr;      // 0: the row is not read
  float* lse = nullptr;               // one per row (distillation: two), written by the forward pass, read by the backward pass
  float* logp = nullptr;
  float* loss = nullptr;
  // policy
  const float *old_logp = nullptr, *ref_logp = nullptr, *advantage = nullptr;
  float* dlogp = nullptr;             // written by the forward pass, read by the backward pass
  float clip_low = 0.f, clip_high = 0.f, kl_weight = 0.f;
  // preference, backward: row r belongs to sequence r / length, of pair (r / length) % pairs
  const float* dseq = nullptr;
  long long length = 1, pairs = 1;
  // distillation
  const int32_t* teacher_ids = nullptr;
  const void* teacher = nullptr;
  int teacher_bf16 = 0, slots = 0;
  float temperature = 1.f, soft = 0.f, hard = 0.f;
  double inv_tau = 1.0;               // 1 / temperature where the softened term is on
  int reverse = 0;                    // rows from the last to the first
  const float* dloss = nullptr;       // backward: one per row (preference: per pair); NULL = 1
};

enum LossOp { LOSS_LOGP = 0, LOSS_POLICY = 1, LOSS_DISTILL = 2 };
enum LossPass { LOSS_FORWARD = 1, LOSS_BACKWARD = 2, LOSS_STEP = 3 };

mtf_status launch_loss_rows(LossOp op, LossPass pass, const LossRows& a, void* stream);

struct PreferencePairs {
  const void* z = nullptr;            // logits
  int V = 0, bf16 = 0;
  const int32_t* targets = nullptr;
  const float *logp = nullptr, *weight = nullptr, *ref = nullptr;
  float *lse = nullptr, *seq = nullptr, *dseq = nullptr, *loss = nullptr;
  long long pairs = 0, length = 0;
  int kind = 0;
  float beta = 0.f, smoothing = 0.f;
};
mtf_status launch_preference_pairs(const PreferencePairs& a, void* stream);

}  // namespace mtf
