// Losses on stored logits beyond cross-entropy: one row of logits per token, a few numbers worked out per row, and the row's gradient.
//   distillation   a tau^2 KL(q || softmax(z / tau)) + g (lse - z_y), q = softmax over a teacher's list of words / tau
//   policy         clipped ratio of exp(logp - old_logp) times the advantage, and a KL term, logp = z_y - lse
//   preference     logp per token; a second kernel adds a sequence's up and takes the loss of a pair
// Every gradient is a row of  k0 exp((z - m0) / tau)  (+ k1 exp(z - m1))  with a few entries (the label, the teacher's words) changed.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "launch.cuh"
#include "losses.h"

namespace {

using mtf::LossRows;
using mtf::kMaxTeacher;

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T> struct Piece;      // 16 bytes of a row
template <> struct Piece<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void get(const uint4& u, float* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(w[e] << 16);
      f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
      w[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float one(const void* p, long long i) { return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]); }
  static __device__ __forceinline__ void set(void* p, long long i, float v) { reinterpret_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v); }
};
template <> struct Piece<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void get(const uint4& u, float* f) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float one(const void* p, long long i) { return reinterpret_cast<const float*>(p)[i]; }
  static __device__ __forceinline__ void set(void* p, long long i, float v) { reinterpret_cast<float*>(p)[i] = v; }
};

// A row's whole pieces and the elements in front of and behind them (at most 14 in all: vocabularies that are no multiple of a piece
// leave rows that start anywhere).
struct RowSpan {
  int head, pieces, tail;
};
template <typename T>
__device__ __forceinline__ RowSpan row_span(long long row, int V) {
  constexpr int n = Piece<T>::kN;
  RowSpan s;
  const int off = (int)((row * V) % n);
  s.head = min(V, (n - off) % n);
  s.pieces = (V - s.head) / n;
  s.tail = V - s.head - s.pieces * n;
  return s;
}
__device__ __forceinline__ int edge_element(const RowSpan& s, int i, int V) { return i < s.head ? i : V - s.tail + (i - s.head); }

// Running maximum and sums of exponentials relative to it.  The maximum starts at the lowest finite number, so that entries of
// -infinity add nothing and need no care, and a row of them alone leaves sums of 0.
template <int NT>
struct RunningSum {
  float m = kLowest, s0 = 0.f, s1 = 0.f;      // s0: exponents times a0, s1: times a1 (NT = 2)
  template <int N>
  __device__ __forceinline__ void add(const float* f, float a0, float a1) {
    float pm = f[0];
#pragma unroll
    for (int e = 1; e < N; ++e) pm = fmaxf(pm, f[e]);
    if (pm > m) {
      s0 *= ex2((m - pm) * a0);
      if (NT == 2) s1 *= ex2((m - pm) * a1);
      m = pm;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      s0 += ex2((f[e] - m) * a0);
      if (NT == 2) s1 += ex2((f[e] - m) * a1);
    }
  }
  __device__ __forceinline__ void join(float m2, float t0, float t1, float a0, float a1) {
    const float mx = fmaxf(m, m2);
    s0 = s0 * ex2((m - mx) * a0) + t0 * ex2((m2 - mx) * a0);
    if (NT == 2) s1 = s1 * ex2((m - mx) * a1) + t1 * ex2((m2 - mx) * a1);
    m = mx;
  }
};

struct RowResult {
  float m;                     // the exponentials' shift in both sums
  double s0, s1;
};

// What a row's gradient is made of: k0 exp2((z - m0) a0) (+ k1 exp2((z - m1) a1)), and the entries that differ.
struct RowGrad {
  float k0, m0, k1, m1;
  int zero;                    // the whole row is 0
  int fix_id;                  // LOGP, POLICY: the label's entry and its value
  float fix;
};

struct Scratch {
  float m[kThreads / 32], s0[kThreads / 32], s1[kThreads / 32];
  RowGrad g;
};
// the teacher's list, and behind it the label
struct Slots {
  double q[kMaxTeacher + 1];
  int id[kMaxTeacher + 1];
  float z[kMaxTeacher + 1];
  float fix[kMaxTeacher + 1];      // the entry's gradient
  int first[kMaxTeacher + 1];      // of the slots with this id it is the first, which writes
  double red[2][kThreads / 32];
};

__device__ __forceinline__ double warp_add(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// sum (or maximum) over the block, the same in every thread; red: a slot per warp
template <bool kMax>
__device__ __forceinline__ double block_all(double v, double* red) {
  v = kMax ? warp_max(v) : warp_add(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  double r = red[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) r = kMax ? fmax(r, red[w]) : r + red[w];
  return r;
}

// One block per row: the statistics in one walk over the row, the gradient in another.
template <typename T, int OP, int PASS, int NT>
__global__ void __launch_bounds__(kThreads) loss_rows_kernel(const LossRows a, int* __restrict__ bad) {
  using P = Piece<T>;
  mtf::chain_wait_only();
  __shared__ Scratch sc;
  extern __shared__ __align__(16) unsigned char dyn[];
  Slots& sl = *reinterpret_cast<Slots*>(dyn);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = blockIdx.x;
  const int V = a.V;
  const RowSpan sp = row_span<T>(row, V);
  const char* const zr = reinterpret_cast<const char*>(a.z) + row * V * (long long)sizeof(T);
  char* const dr = reinterpret_cast<char*>(a.d) + row * V * (long long)sizeof(T);
  const uint4* const z16 = reinterpret_cast<const uint4*>(zr + sp.head * (int)sizeof(T));
  uint4* const d16 = reinterpret_cast<uint4*>(dr + sp.head * (int)sizeof(T));
  const bool soft_on = OP == mtf::LOSS_DISTILL && a.soft != 0.f, hard_on = OP == mtf::LOSS_DISTILL && a.hard != 0.f;
  // the first sum is the softened one wherever there is one
  const float tau = soft_on ? a.temperature : 1.f;
  const float a0 = kLog2e / tau, a1 = kLog2e;

  const float w = a.weight ? a.weight[row] : 1.f;
  // a row whose factor is 0 is not looked at: neither its label nor anything else of it
  bool skip = w == 0.f;
  float scale = 1.f;           // of the gradient (backward)
  if (PASS == mtf::LOSS_BACKWARD && !skip) {
    long long at = row;
    if (OP == mtf::LOSS_DISTILL) scale = w;
    else if (a.dseq) { scale = w * a.dseq[row / a.length]; at = (row / a.length) % a.pairs; }
    else scale = a.dlogp[row];
    if (a.dloss && scale != 0.f) scale *= a.dloss[at];
    skip = scale == 0.f;
  }
  int label = 0;
  if (!skip && (OP != mtf::LOSS_DISTILL || hard_on)) {
    label = a.targets[row];
    if (label < 0 || label >= V) { skip = true; if (tid == 0) atomicExch(bad, 1); }
  }
  if (skip) {
    if ((PASS & mtf::LOSS_FORWARD) && tid == 0) {
      if (a.loss) a.loss[row] = 0.f;
      if (a.logp) a.logp[row] = 0.f;
      if (a.dlogp) a.dlogp[row] = 0.f;
      if (a.lse) {
        if (OP == mtf::LOSS_DISTILL) { a.lse[2 * row] = 0.f; a.lse[2 * row + 1] = 0.f; }
        else a.lse[row] = 0.f;
      }
    }
    if (PASS & mtf::LOSS_BACKWARD) {
      for (int p = tid; p < sp.pieces; p += kThreads) d16[p] = make_uint4(0u, 0u, 0u, 0u);
      if (tid < sp.head + sp.tail) P::set(dr, edge_element(sp, tid, V), 0.f);
    }
    return;
  }

  // ---- statistics -------------------------------------------------------------------------------------------------
  RowResult r;
  r.m = 0.f; r.s0 = 1.0; r.s1 = 1.0;
  if (PASS & mtf::LOSS_FORWARD) {
    RunningSum<NT> rs;
    for (int p = tid; p < sp.pieces; p += kThreads) {
      float f[P::kN];
      P::get(z16[p], f);
      rs.template add<P::kN>(f, a0, a1);
    }
    if (tid < sp.head + sp.tail) {
      const float f = P::one(zr, edge_element(sp, tid, V));
      rs.template add<1>(&f, a0, a1);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, rs.m, o), t0 = __shfl_xor_sync(0xffffffffu, rs.s0, o);
      const float t1 = NT == 2 ? __shfl_xor_sync(0xffffffffu, rs.s1, o) : 0.f;
      rs.join(m2, t0, t1, a0, a1);
    }
    if (lane == 0) { sc.m[warp] = rs.m; sc.s0[warp] = rs.s0; sc.s1[warp] = rs.s1; }
    __syncthreads();
    r.m = kLowest;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) r.m = fmaxf(r.m, sc.m[i]);
    r.s0 = r.s1 = 0.0;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) {
      r.s0 += (double)(sc.s0[i] * ex2((sc.m[i] - r.m) * a0));
      if (NT == 2) r.s1 += (double)(sc.s1[i] * ex2((sc.m[i] - r.m) * a1));
    }
    if (NT == 1) r.s1 = r.s0;
  }

  // ---- the row's numbers, in 64 bits: they are differences of values near each other ------------------------------------
  if (OP != mtf::LOSS_DISTILL) {
    if (tid == 0) {
      RowGrad g = {};
      g.fix_id = label;
      double c, logp;
      const double zy = (double)P::one(zr, label);
      if (PASS & mtf::LOSS_FORWARD) {
        const double log_s = log(r.s0);
        logp = (zy - (double)r.m) - log_s;
        if (a.lse) a.lse[row] = (float)((double)r.m + log_s);
        if (a.logp) a.logp[row] = (float)logp;
        c = 0.0;
        if (OP == mtf::LOSS_POLICY) {
          const double adv = (double)a.advantage[row], ratio = exp(logp - (double)a.old_logp[row]);
          const double plain = ratio * adv, clipped = fmin(fmax(ratio, 1.0 - (double)a.clip_low), 1.0 + (double)a.clip_high) * adv;
          const bool cut = plain > clipped;             // (not so for NaN, which both results then show)
          double loss = cut ? -clipped : -plain, dl = cut ? 0.0 : -plain;
          if (a.kl_weight != 0.f) {
            const double e = (double)a.ref_logp[row] - logp, em1 = expm1(e);
            loss += (double)a.kl_weight * (em1 - e);
            dl -= (double)a.kl_weight * em1;
          }
          a.loss[row] = (float)((double)w * loss);
          c = (double)w * dl;
          if (a.dlogp) a.dlogp[row] = (float)c;
        }
        g.k0 = (float)(-c / r.s0);
        g.m0 = r.m;
      } else {
        const float lse = a.lse[row];
        logp = zy - (double)lse;
        c = (double)scale;
        g.k0 = -scale;
        g.m0 = lse;
      }
      g.zero = c == 0.0;
      g.fix = (float)(-c * expm1(logp));
      sc.g = g;
    }
  } else {
    const int K = a.slots;
    double lse0, lse1;           // of z / tau, of z
    if (PASS & mtf::LOSS_FORWARD) {
      lse0 = (double)r.m / (double)tau + log(r.s0);
      lse1 = (double)r.m + log(r.s1);
      if (tid == 0 && a.lse) {
        a.lse[2 * row] = (float)(soft_on ? lse0 : 0.0);
        a.lse[2 * row + 1] = (float)(hard_on ? lse1 : 0.0);
      }
    } else {
      lse0 = (double)a.lse[2 * row];
      lse1 = (double)a.lse[2 * row + 1];
    }
    // the teacher's distribution over its used slots
    double best = -INFINITY;
    if (soft_on) {
      for (int k = tid; k < K; k += kThreads) {
        int id = a.teacher_ids[row * K + k];
        if (id < -1 || id >= V) { atomicExch(bad, 1); id = -1; }
        double t = -INFINITY;
        if (id >= 0) {
          t = (double)(a.teacher_bf16 ? Piece<__nv_bfloat16>::one(a.teacher, row * K + k) : Piece<float>::one(a.teacher, row * K + k)) / (double)tau;
          sl.z[k] = P::one(zr, id);
        }
        sl.id[k] = id;
        sl.q[k] = t;
        best = fmax(best, t != t ? INFINITY : t);      // (NaN: every difference to the maximum is NaN)
      }
      best = block_all<true>(best, sl.red[0]);
    }
    const bool any = soft_on && best != -INFINITY;
    double sum = 0.0;
    if (any)
      for (int k = tid; k < K; k += kThreads) sum += exp(sl.q[k] - best);
    sum = block_all<false>(sum, sl.red[1]);
    const double log_norm = any ? best + log(sum) : 0.0;
    double kl = 0.0;
    if (any)
      for (int k = tid; k < K; k += kThreads) {
        const double t = sl.q[k] - log_norm, q = exp(t);
        if (q != 0.0) kl += q * (t - ((double)sl.z[k] / (double)tau - lse0));      // (a word of probability 0 adds nothing, whatever the student says to it)
        sl.q[k] = q;
      }
    if (PASS & mtf::LOSS_FORWARD) {
      kl = block_all<false>(kl, sl.red[0]);
      if (tid == 0) {
        double loss = any ? (double)a.soft * (double)tau * (double)tau * kl : 0.0;
        if (hard_on) loss += (double)a.hard * (lse1 - (double)P::one(zr, label));
        a.loss[row] = (float)((double)w * loss);
      }
    }
    if (PASS & mtf::LOSS_BACKWARD) {
      const double g = PASS == mtf::LOSS_BACKWARD ? (double)scale : (double)w;
      const double cs = any ? g * (double)a.soft * (double)tau : 0.0, ch = hard_on ? g * (double)a.hard : 0.0;
      if (tid == 0) {
        RowGrad gr = {};
        if (PASS == mtf::LOSS_STEP) {
          gr.m0 = gr.m1 = r.m;
          gr.k0 = (float)(NT == 2 ? cs / r.s0 : (cs + ch) / r.s0);
          gr.k1 = (float)(ch / r.s1);
        } else {
          gr.m0 = (float)(soft_on ? lse0 * (double)tau : lse1);
          gr.m1 = (float)lse1;
          gr.k0 = (float)(NT == 2 ? cs : cs + ch);
          gr.k1 = (float)ch;
        }
        gr.zero = cs == 0.0 && ch == 0.0;
        sc.g = gr;
        sl.id[K] = hard_on ? label : -1;
        sl.q[K] = 0.0;
        if (hard_on) sl.z[K] = P::one(zr, label);
      }
      if (!any)
        for (int k = tid; k < K; k += kThreads) sl.id[k] = -1;
      __syncthreads();
      // the entries that differ; of slots with one id the first takes care of all
      for (int k = tid; k <= K; k += kThreads) {
        const int id = sl.id[k];
        bool first = id >= 0;
        double q = 0.0;
        for (int j = 0; first && j <= K; ++j)
          if (sl.id[j] == id) {
            first = j >= k;
            q += sl.q[j];
          }
        sl.first[k] = first;
        if (!first) continue;
        const double z = (double)sl.z[k];
        double v = 0.0;
        if (any) v += cs * (exp(z / (double)tau - lse0) - q);
        if (hard_on) v += ch * (exp(z - lse1) - (id == label ? 1.0 : 0.0));
        sl.fix[k] = (float)v;
      }
    }
  }
  if (!(PASS & mtf::LOSS_BACKWARD)) return;
  __syncthreads();

  // ---- gradient -------------------------------------------------------------------------------------------------------
  const RowGrad g = sc.g;
  if (g.zero) {
    for (int p = tid; p < sp.pieces; p += kThreads) d16[p] = make_uint4(0u, 0u, 0u, 0u);
    if (tid < sp.head + sp.tail) P::set(dr, edge_element(sp, tid, V), 0.f);
    return;
  }
  auto value = [&](float z) {
    float v = g.k0 * ex2((z - g.m0) * a0);
    if (NT == 2) v += g.k1 * ex2((z - g.m1) * a1);
    return v;
  };
  for (int p = tid; p < sp.pieces; p += kThreads) {
    float f[P::kN];
    P::get(z16[p], f);
#pragma unroll
    for (int e = 0; e < P::kN; ++e) f[e] = value(f[e]);
    d16[p] = P::put(f);
  }
  if (tid < sp.head + sp.tail) {
    const int e = edge_element(sp, tid, V);
    P::set(dr, e, value(P::one(zr, e)));
  }
  __syncthreads();
  if (OP != mtf::LOSS_DISTILL) {
    if (tid == 0) P::set(dr, g.fix_id, g.fix);
  } else {
    for (int k = tid; k <= a.slots; k += kThreads)
      if (sl.first[k]) P::set(dr, sl.id[k], sl.fix[k]);
  }
}

// One block per pair: both sequences' log-probabilities added up in a fixed order, in 64 bits, then the loss of the pair and its
// derivative by each of the two sums.
__global__ void __launch_bounds__(kThreads) preference_pairs_kernel(const mtf::PreferencePairs a) {
  mtf::chain_wait();
  __shared__ double red[kThreads / 32];
  const long long b = blockIdx.x;
  double s[2];
  for (int i = 0; i < 2; ++i) {
    const long long at = (i * a.pairs + b) * a.length;
    double v = 0.0;
    for (long long t = threadIdx.x; t < a.length; t += kThreads) {
      const float w = a.weight ? a.weight[at + t] : 1.f;
      if (w != 0.f) v += (double)w * (double)a.logp[at + t];
    }
    s[i] = block_all<false>(v, red);
  }
  if (threadIdx.x) return;
  const double margin = (s[0] - (double)a.ref[b]) - (s[1] - (double)a.ref[a.pairs + b]), beta = (double)a.beta, h = beta * margin;
  double loss, d;
  if (a.kind == MTF_PREFERENCE_SIGMOID) {
    // -log sigmoid(h) = max(-h, 0) + log1p(exp(-|h|))
    const double tail = log1p(exp(-fabs(h))), eps = (double)a.smoothing;
    loss = (1.0 - eps) * (fmax(-h, 0.0) + tail) + eps * (fmax(h, 0.0) + tail);
    d = beta * (eps - 1.0 / (1.0 + exp(h)));
  } else if (a.kind == MTF_PREFERENCE_HINGE) {
    loss = fmax(1.0 - h, 0.0);
    d = h < 1.0 ? -beta : 0.0;
  } else {
    const double off = margin - 0.5 / beta;
    loss = off * off;
    d = 2.0 * off;
  }
  if (h != h) loss = d = h;      // (the comparisons above lose a NaN)
  a.seq[b] = (float)s[0];
  a.seq[a.pairs + b] = (float)s[1];
  a.dseq[b] = (float)d;
  a.dseq[a.pairs + b] = (float)-d;
  a.loss[b] = (float)loss;
}

template <typename T, int OP, int PASS, int NT>
void launch(const LossRows& a, int* bad, cudaStream_t st) {
  const size_t smem = OP == mtf::LOSS_DISTILL ? sizeof(Slots) : 0;
  mtf::launch_chained(loss_rows_kernel<T, OP, PASS, NT>, (unsigned)a.rows, kThreads, smem, st, a, bad);
}

template <typename T>
void dispatch(mtf::LossOp op, mtf::LossPass pass, int sums, const LossRows& a, int* bad, cudaStream_t st) {
  using namespace mtf;
  if (op == LOSS_DISTILL) {
    if (pass == LOSS_FORWARD) { if (sums == 2) launch<T, LOSS_DISTILL, LOSS_FORWARD, 2>(a, bad, st); else launch<T, LOSS_DISTILL, LOSS_FORWARD, 1>(a, bad, st); }
    else if (pass == LOSS_BACKWARD) { if (sums == 2) launch<T, LOSS_DISTILL, LOSS_BACKWARD, 2>(a, bad, st); else launch<T, LOSS_DISTILL, LOSS_BACKWARD, 1>(a, bad, st); }
    else { if (sums == 2) launch<T, LOSS_DISTILL, LOSS_STEP, 2>(a, bad, st); else launch<T, LOSS_DISTILL, LOSS_STEP, 1>(a, bad, st); }
  } else if (pass == LOSS_BACKWARD) {
    launch<T, LOSS_LOGP, LOSS_BACKWARD, 1>(a, bad, st);
  } else if (op == LOSS_LOGP) {
    launch<T, LOSS_LOGP, LOSS_FORWARD, 1>(a, bad, st);
  } else if (pass == LOSS_FORWARD) {
    launch<T, LOSS_POLICY, LOSS_FORWARD, 1>(a, bad, st);
  } else {
    launch<T, LOSS_POLICY, LOSS_STEP, 1>(a, bad, st);
  }
}

}  // namespace

namespace mtf {

static mtf_status after(const char* what) {
  count_launch();
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
  return MTF_OK;
}

mtf_status launch_loss_rows(LossOp op, LossPass pass, const LossRows& a, void* stream) {
  const int sums = op == LOSS_DISTILL && a.soft != 0.f && a.hard != 0.f && a.temperature != 1.f ? 2 : 1;
  if (a.bf16) dispatch<__nv_bfloat16>(op, pass, sums, a, bad_index_flag(), (cudaStream_t)stream);
  else dispatch<float>(op, pass, sums, a, bad_index_flag(), (cudaStream_t)stream);
  return after("loss_rows_kernel");
}

mtf_status launch_preference_pairs(const PreferencePairs& a, void* stream) {
  launch_chained(preference_pairs_kernel, (unsigned)a.pairs, kThreads, 0, (cudaStream_t)stream, a);
  return after("preference_pairs_kernel");
}

}  // namespace mtf
