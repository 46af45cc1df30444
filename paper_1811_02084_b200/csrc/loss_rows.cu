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
#include "per_device.h"

namespace {

using mtf::LossRows;
using mtf::kMaxTeacher;

__device__ int g_bad_id = 0;         // an id outside [0, V) was seen
__device__ int g_loss_status = 0;    // a wait was given up
// Testing hooks (mtf_debug_wait_test): how many cycles a wait may take, and a barrier that waits for a signal more than is sent.
constexpr long long kWaitCycles = 4000000000LL;
__constant__ long long g_wait_limit = kWaitCycles;
constexpr int kNumbersHeld = 1, kSumsHeld = 2;
__constant__ int g_withhold = 0;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two f32 values side by side: one instruction works on both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ f32x2 pair(float v) { return pair(v, v); }
__device__ __forceinline__ float2 both(f32x2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) { f32x2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// 2^y of both on the special-function unit, ...
__device__ __forceinline__ f32x2 ex2_unit(f32x2 y) {
  const float2 f = both(y);
  return pair(ex2(f.x), ex2(f.y));
}
// ... and on the arithmetic pipes, for y below 127 (40 is the most that the sums and gradients come with) or NaN: y = i + f, i whole, |f| <= 1/2, and 2^f as the polynomial of degree 5 through
// (0, 1) with the smallest largest relative error on [-1/2, 1/2] (found by linear programming: 9e-8; 1.7e-7 with f32 coefficients and sums).
// Below -127 the result is exactly 0.  A NaN may come out as a number.
__device__ __forceinline__ f32x2 ex2_fma(f32x2 y) {
  float2 c = both(y);
  y = pair(fmaxf(c.x, -127.f), fmaxf(c.y, -127.f));
  const f32x2 whole = add2(y, pair(12582912.f));                  // 1.5 * 2^23: the sum's low bits are i
  const f32x2 f = fma2(add2(whole, pair(-12582912.f)), pair(-1.f), y);
  f32x2 v = fma2(f, pair(0.0013264727f), pair(0.009671513f));
  v = fma2(f, v, pair(0.055507336f));
  v = fma2(f, v, pair(0.24022242f));
  v = fma2(f, v, pair(0.693147f));
  v = fma2(f, v, pair(1.f));
  const float2 w = both(whole);
  c = both(v);
  return pair(__uint_as_float(__float_as_uint(c.x) + (__float_as_uint(w.x) << 23)), __uint_as_float(__float_as_uint(c.y) + (__float_as_uint(w.y) << 23)));
}

template <typename T> struct Piece;      // 16 bytes of a row: kN values, two by two
template <> struct Piece<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void get(const uint4& u, f32x2* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = pair(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  // the largest value of N pieces (NaN only if there is nothing else)
  template <int N>
  static __device__ __forceinline__ float largest(const uint4* u) {
    uint32_t m = max2(max2(u[0].x, u[0].y), max2(u[0].z, u[0].w));
#pragma unroll
    for (int i = 1; i < N; ++i) m = max2(m, max2(max2(u[i].x, u[i].y), max2(u[i].z, u[i].w)));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint4 put(const f32x2* f) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 v = both(f[e]);
      const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
      w[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float one(const void* p, long long i) { return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]); }
  static __device__ __forceinline__ void set(void* p, long long i, float v) { reinterpret_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v); }
};
template <> struct Piece<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void get(const uint4& u, f32x2* f) {
    f[0] = pair(__uint_as_float(u.x), __uint_as_float(u.y));
    f[1] = pair(__uint_as_float(u.z), __uint_as_float(u.w));
  }
  template <int N>
  static __device__ __forceinline__ float largest(const uint4* u) {
    float m = kLowest;
#pragma unroll
    for (int i = 0; i < N; ++i)
      m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(u[i].x), __uint_as_float(u[i].y)), fmaxf(__uint_as_float(u[i].z), __uint_as_float(u[i].w))));
    return m;
  }
  static __device__ __forceinline__ uint4 put(const f32x2* f) {
    const float2 a = both(f[0]), b = both(f[1]);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
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
  const int off = (int)(((uint32_t)row * (uint32_t)V) & (n - 1));
  s.head = min(V, (n - off) & (n - 1));
  s.pieces = (int)((uint32_t)(V - s.head) / n);
  s.tail = V - s.head - s.pieces * n;
  return s;
}
__device__ __forceinline__ int edge_element(const RowSpan& s, int i, int V) { return i < s.head ? i : V - s.tail + (i - s.head); }

// How a row's exponentials are formed; NT of the kernels below.
//   one       2^(z a0 - b0)
//   two       and 2^(z a1 - b1): a temperature and none, a0 being the softened one
//   powers    of one exponential t = 2^(z a0 - b0): t^soft for the temperature hard / soft, and t^hard without one
// The special-function unit takes an exponential every 8 cycles a scheduler and bounds the walks: a power in place of a second one takes
// 8192 x 32768 bf16 logits at temperature 1.5 in one call from 321 to 231 us, 2000 x 131072 in a forward call from 105 to 80 (temperatures that are no
// such quotient take 321 and 105).
constexpr int kOne = 1, kTwo = 2;
constexpr int powers(int soft, int hard) { return 16 * soft + hard; }
__host__ __device__ constexpr bool is_powers(int nt) { return nt >= 16; }
__host__ __device__ constexpr int soft_power(int nt) { return is_powers(nt) ? nt / 16 : 1; }
__host__ __device__ constexpr int hard_power(int nt) { return is_powers(nt) ? nt % 16 : 1; }

// The first exponential, and the second if it is one of its own, of pair e of a piece.  Where there are two the arithmetic pipes take over every
// other softened one of the sums and every fourth of the gradient, whose factors want more of them.  (Of the sums only softened ones: a NaN may
// come out as a number there, and the other exponential of its entry shows it.  A gradient's factors are NaN where its row has one.)
template <int NT, bool kGradient>
__device__ __forceinline__ void exponentials(int e, f32x2 z, float a0, float nb0, float a1, float nb1, f32x2& e0, f32x2& e1) {
  const f32x2 y = fma2(z, pair(a0), pair(nb0));
  const bool fma = NT == kTwo && (kGradient ? (e & 3) == 3 : (e & 1) == 1);
  e0 = fma ? ex2_fma(y) : ex2_unit(y);
  if (NT == kTwo) e1 = ex2_unit(fma2(z, pair(a1), pair(nb1)));
}
// t^n
template <int N>
__device__ __forceinline__ f32x2 power(f32x2 t) {
  if constexpr (N == 1) return t;
  else if constexpr (N % 2 == 0) return power<N / 2>(mul2(t, t));
  else return mul2(t, power<N - 1>(t));
}

__device__ __forceinline__ float reference(float m, float a) { return __fmul_rn(m, a); }
// What a row's exponents are formed from: the factors a0 and a1 (powers: that of the highest power), and the size `huge` from which on logits have no room for the products (they would
// be rounded by a whole exponent and more).  A row without an entry between -huge and huge, or with one above (a row that is masked as a whole by
// the type's lowest value, say), is worked out from differences instead.
struct Factors {
  float a0, a1, huge;
  __host__ __device__ __forceinline__ Factors(float a0_, float a1_) : a0(a0_), a1(a1_), huge(16777216.f / (a0_ > a1_ ? a0_ : a1_)) {}
  __device__ __forceinline__ bool is_huge(float m) const { return !(fabsf(m) < huge); }
};

// a maximum over the warp: f32 values in the order of whole numbers
__device__ __forceinline__ float warp_max(float v) {
  int i = __float_as_int(v);
  i = __reduce_max_sync(0xffffffffu, i >= 0 ? i : i ^ 0x7fffffff);
  return __int_as_float(i >= 0 ? i : i ^ 0x7fffffff);
}
__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Sums of exponentials relative to a reference m, an entry of the row: sums of 2^(z a - b) with b = fl(m a), the one rounding of which every use
// of the sums allows for.  m starts at -huge (far lower entries, infinity among them, add nothing) and is raised to the largest entry seen only
// where that lies 2^40 above it: an f32 sum has room for that, and nearly every entry is spared the rescaling (with a maximum that is always
// exact some thread of a warp has to rescale at nearly every step, and holds up the others).
template <int NT>
struct RunningSum {
  float m, limit, nb0, nb1;
  f32x2 p0 = 0ull, p1 = 0ull;      // p0: exponents times a0, p1: times a1 (two temperatures); two partial sums each
  __device__ __forceinline__ explicit RunningSum(const Factors& F) : m(-F.huge), limit(-F.huge), nb0(reference(F.huge, F.a0)), nb1(reference(F.huge, F.a1)) {}
  __device__ __forceinline__ void raise(float pm, const Factors& F) {
    if (pm > limit) {
      const float b0 = reference(pm, F.a0), b1 = reference(pm, F.a1);
      p0 = mul2(p0, pair(ex2(soft_power(NT) * (-nb0 - b0))));
      if (NT == kTwo) p1 = mul2(p1, pair(ex2(-nb1 - b1)));
      if (is_powers(NT)) p1 = mul2(p1, pair(ex2(hard_power(NT) * (-nb0 - b0))));
      m = pm;
      limit = pm + 40.f / (NT != kOne ? fmaxf(F.a0, F.a1) : F.a0);
      nb0 = -b0;
      nb1 = -b1;
    }
  }
  template <typename T, int N>
  __device__ __forceinline__ void add_below(const uint4* u, const Factors& F) {      // entries that the reference has been raised for
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f32x2 f[Piece<T>::kN / 2];
      Piece<T>::get(u[i], f);
#pragma unroll
      for (int e = 0; e < Piece<T>::kN / 2; ++e) {
        f32x2 e0, e1;
        exponentials<NT, false>(e, f[e], F.a0, nb0, F.a1, nb1, e0, e1);
        if (is_powers(NT)) {
          const f32x2 soft = power<soft_power(NT)>(e0);
          p0 = add2(p0, soft);
          p1 = fma2(soft, power<hard_power(NT) - soft_power(NT)>(e0), p1);
        } else {
          p0 = add2(p0, e0);
          if (NT == kTwo) p1 = add2(p1, e1);
        }
      }
    }
  }
  template <typename T, int N>
  __device__ __forceinline__ void add(const uint4* u, const Factors& F) {
    raise(Piece<T>::template largest<N>(u), F);
    add_below<T, N>(u, F);
  }
  __device__ __forceinline__ void add_one(float f, const Factors& F) {
    raise(f, F);
    const float y = fmaf(f, F.a0, nb0);
    p0 = add2(p0, pair(ex2(soft_power(NT) * y), 0.f));
    if (NT != kOne) p1 = add2(p1, pair(ex2(NT == kTwo ? fmaf(f, F.a1, nb1) : hard_power(NT) * y), 0.f));
  }
  __device__ __forceinline__ void of_warp(float& t_m, float& t_0, float& t_1, const Factors& F) const;
};

// what a sum (of powers n) relative to m is multiplied by to be relative to mx >= m
__device__ __forceinline__ float to_reference(float m, float mx, float a, int n, const Factors& F) {
  return ex2(n * (F.is_huge(mx) ? (m - mx) * a : reference(m, a) - reference(mx, a)));
}
// the lanes' references and sums joined, the same in every lane
template <int NT>
__device__ __forceinline__ void warp_join(float& m, float& s0, float& s1, const Factors& F) {
  const float mx = warp_max(m);
  s0 = warp_add(s0 * to_reference(m, mx, F.a0, soft_power(NT), F));
  if (NT != kOne) s1 = warp_add(s1 * to_reference(m, mx, NT == kTwo ? F.a1 : F.a0, hard_power(NT), F));
  m = mx;
}
template <int NT>
__device__ __forceinline__ void RunningSum<NT>::of_warp(float& t_m, float& t_0, float& t_1, const Factors& F) const {
  t_m = m;
  t_0 = both(p0).x + both(p0).y;
  t_1 = both(p1).x + both(p1).y;
  warp_join<NT>(t_m, t_0, t_1, F);
}

// What a row's gradient is made of: k0 2^(z a0 + nb0) (+ k1 2^(z a1 + nb1)), or with huge logits k0 2^((z - m0) a0) (+ ...); k0 t^soft + k1 t^hard
// with t the first of the two exponentials.
struct RowGrad {
  float k0, nb0, k1, nb1, m0, m1;
  int zero;                    // the whole row is 0
  int huge;
};
// What else a row comes to, in 64 bits.
struct RowNumbers {
  double c;                    // LOGP, POLICY: derivative by the label's log-probability
  double plain, clipped, em1;  // POLICY: both sides of the limit, and exp(ref - logp) - 1
  double cs, ch;               // distillation: factors of the two distributions in the gradient
  double lse0, lse1;           // log-sum-exp of z / tau and of z
};

// A teacher's list: arrays of `slots`, rounded up to 4.
struct Slots {
  double* q;                   // its distribution
  int* id;                     // -1: empty
  float* z;                    // the student's logit; later the entry's gradient
  static __host__ __device__ int room(int slots) { return (slots + 3) & ~3; }
  static __host__ __device__ size_t bytes(int slots) { return (size_t)room(slots) * 16; }
  __device__ Slots(unsigned char* at, int slots) : q(reinterpret_cast<double*>(at)), id(reinterpret_cast<int*>(q + room(slots))), z(reinterpret_cast<float*>(id + room(slots))) {}
};

__device__ __forceinline__ double warp_add(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// (The rows' numbers are long stretches of code that run once a row beside the walks, at the rate at which their instructions come in: one
// copy each of the functions that they call more than once.)
__device__ __noinline__ double exp64(double x) { return exp(x); }
__device__ __noinline__ double log64(double x) { return log(x); }

// ---- what a row is worked out from, apart from the walks over its logits -------------------------------------------------------
template <int OP> __device__ __forceinline__ bool soft_on(const LossRows& a) { return OP == mtf::LOSS_DISTILL && a.soft != 0.f; }
template <int OP> __device__ __forceinline__ bool hard_on(const LossRows& a) { return OP == mtf::LOSS_DISTILL && a.hard != 0.f; }

struct RowIn {
  float w, scale;              // factors of the loss and (backward) of the gradient
  int label;
  bool skip, bad;              // nothing to be done but zeros; the label is out of range
};
// A row whose factor is 0 is not looked at: neither its label nor anything else of it.
template <int OP, int PASS>
__device__ __forceinline__ RowIn row_in(const LossRows& a, long long row) {
  // (all loads at once; what a row's factor of 0 leaves out is loaded and not looked at)
  RowIn r;
  const bool wants_label = OP != mtf::LOSS_DISTILL || hard_on<OP>(a);
  r.w = a.weight ? a.weight[row] : 1.f;
  r.label = wants_label ? a.targets[row] : 0;
  r.scale = 1.f;
  if (PASS == mtf::LOSS_BACKWARD) {
    long long at = row;
    if (OP == mtf::LOSS_DISTILL) r.scale = r.w;
    else if (a.dseq) {
      const unsigned seq = (unsigned)row / (unsigned)a.length;
      at = seq % (unsigned)a.pairs;
      const float d = a.dseq[seq];
      r.scale = r.w == 0.f ? 0.f : r.w * d;
    } else {
      r.scale = a.dlogp[row];
    }
    const float f = a.dloss ? a.dloss[at] : 1.f;
    if (r.scale != 0.f) r.scale *= f;
  }
  r.skip = r.w == 0.f || (PASS == mtf::LOSS_BACKWARD && r.scale == 0.f);
  r.bad = !r.skip && wants_label && (r.label < 0 || r.label >= a.V);
  r.skip |= r.bad;
  return r;
}

// by one thread: the results of a row that is skipped
template <int OP>
__device__ __forceinline__ void zero_results(const LossRows& a, long long row) {
  if (a.loss) a.loss[row] = 0.f;
  if (a.logp) a.logp[row] = 0.f;
  if (a.dlogp) a.dlogp[row] = 0.f;
  if (!a.lse) return;
  if (OP == mtf::LOSS_DISTILL) { a.lse[2 * row] = 0.f; a.lse[2 * row + 1] = 0.f; }
  else a.lse[row] = 0.f;
}

struct RowInputs {
  float zy, old, ref, adv;
  float best;                  // the teacher's largest logit
  float zr;                    // the largest of the student's logits to the teacher's words, or 0
  double kl, sum;              // the teacher's sum_k q_k (log q_k - (z_k - zr) / tau), and sum_k q_k: 1, or 0 without a used slot
};
// The first slots of a teacher's list as they are loaded, kB a lane.
constexpr int kB = 4;
struct Fetched {
  int id[kB];
  float t[kB];
};
__device__ __forceinline__ void fetch_slots(const LossRows& a, long long row, int first, int lane, bool on, Fetched& f) {
#pragma unroll
  for (int i = 0; i < kB; ++i) {
    const int k = first + lane + 32 * i;
    f.id[i] = -1;
    f.t[i] = 0.f;
    if (on && k < a.slots) {
      f.id[i] = a.teacher_ids[row * a.slots + k];
      f.t[i] = a.teacher_bf16 ? Piece<__nv_bfloat16>::one(a.teacher, row * a.slots + k) : Piece<float>::one(a.teacher, row * a.slots + k);
    }
  }
}

// By one warp, before anything of the row is overwritten; all lanes return the same.  The teacher's list (f: its first slots) goes to `sl`; its
// distribution is for teacher() to work out.
template <typename T, int OP>
__device__ __forceinline__ RowInputs row_inputs(const LossRows& a, long long row, const char* zr, int label, Fetched& f, const Slots& sl, int lane, bool report) {
  RowInputs r = {};
  if (OP != mtf::LOSS_DISTILL || hard_on<OP>(a)) r.zy = Piece<T>::one(zr, label);
  if (OP == mtf::LOSS_POLICY) {
    r.old = a.old_logp[row];
    r.adv = a.advantage[row];
    if (a.kl_weight != 0.f) r.ref = a.ref_logp[row];
  }
  if (OP != mtf::LOSS_DISTILL) return r;
  const int K = a.slots;
  float best = -INFINITY, top = -INFINITY;      // of the logits as they are: f32 values
  for (int first = 0; first < K; first += 32 * kB) {
    float z[kB];
    if (first) fetch_slots(a, row, first, lane, soft_on<OP>(a), f);
#pragma unroll
    for (int i = 0; i < kB; ++i) {
      if (f.id[i] < -1 || f.id[i] >= a.V) { if (report) atomicExch(&g_bad_id, 1); f.id[i] = -1; }
      z[i] = f.id[i] >= 0 ? Piece<T>::one(zr, f.id[i]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kB; ++i) {
      const int k = first + lane + 32 * i;
      if (k >= Slots::room(K)) continue;
      const float t = f.id[i] >= 0 ? f.t[i] : -INFINITY;
      sl.id[k] = f.id[i];
      sl.z[k] = z[i];
      sl.q[k] = (double)t;
      best = fmaxf(best, t != t ? INFINITY : t);      // (NaN: every difference to the maximum is NaN)
      if (f.id[i] >= 0) top = fmaxf(top, z[i]);
    }
  }
  best = warp_max(best);
  top = warp_max(top);
  r.best = best;
  r.zr = top != -INFINITY ? top : 0.f;
  r.sum = best != -INFINITY ? 1.0 : 0.0;
  __syncwarp();
  return r;
}
// Its distribution over the used slots, to sl.q.
__device__ __forceinline__ void teacher(const LossRows& a, RowInputs& r, const Slots& sl, int lane) {
  const int K = a.slots;
  double sum = 0.0, kl = 0.0;
  if (r.sum != 0.0) {
#pragma unroll 1
    for (int k = lane; k < K; k += 32) {
      const double d = (sl.q[k] - (double)r.best) * a.inv_tau, e = exp64(d);
      sum += e;
      if (e != 0.0) kl += e * (d - ((double)sl.z[k] - (double)r.zr) * a.inv_tau);      // (a word of probability 0 adds nothing, whatever the student says to it)
      sl.q[k] = e;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
      kl += __shfl_xor_sync(0xffffffffu, kl, o);
    }
    const double inv = 1.0 / sum;
    r.kl = kl * inv - log64(sum);
    for (int k = lane; k < K; k += 32) sl.q[k] *= inv;
  } else {
    for (int k = lane; k < K; k += 32) sl.id[k] = -1;
  }
  __syncwarp();
}

// what log(s) + m / tau is off by as log-sum-exp of z / tau, s being relative to m: the rounding of the reference
__device__ __forceinline__ double reference_off(float m, float af, int n, const Factors& F) {
  return F.is_huge(m) ? 0.0 : ((double)reference(m, af) - (double)m * (double)af) * n * 0.6931471805599453;
}

// First what the gradient's walk waits for: the row's factors, from its reference m and sums.  (POLICY: the ratio is
// exp(z_y - m - old) / s, so that the logarithm can wait, too.)
template <int OP, int PASS, int NT>
__device__ __forceinline__ RowGrad row_gradient(const LossRows& a, long long row, const RowIn& in, const RowInputs& x, float m, float s0, float s1, const Factors& F,
                                                RowNumbers& r) {
  const float a0 = F.a0, a1 = F.a1;
  RowGrad g = {};
  r = {};
  const double w = (double)in.w;
  g.m0 = g.m1 = m;
  double c0, c1 = 0.0;         // factors of the two distributions in the gradient
  if (OP != mtf::LOSS_DISTILL) {
    r.c = (double)in.scale;
    if (PASS & mtf::LOSS_FORWARD) {
      r.c = 0.0;
      if (OP == mtf::LOSS_POLICY) {
        const double base = ((double)x.zy - (double)m) - reference_off(m, a0, 1, F), adv = (double)x.adv;
        const double ratio = exp64(base - (double)x.old) / (double)s0;
        r.plain = ratio * adv;
        r.clipped = fmin(fmax(ratio, 1.0 - (double)a.clip_low), 1.0 + (double)a.clip_high) * adv;
        double dl = r.plain > r.clipped ? 0.0 : -r.plain;             // (NaN: not cut, and both results show it)
        if (a.kl_weight != 0.f) {
          r.em1 = exp64((double)x.ref - base) * (double)s0 - 1.0;
          dl -= (double)a.kl_weight * r.em1;
        }
        r.c = w * dl;
      }
    }
    c0 = -r.c;
  } else {
    const double f = PASS == mtf::LOSS_BACKWARD ? (double)in.scale : w;
    r.cs = x.sum != 0.0 ? f * (double)a.soft * (double)a.temperature : 0.0;
    r.ch = hard_on<OP>(a) ? f * (double)a.hard : 0.0;
    c0 = NT != kOne ? r.cs : r.cs + r.ch;
    c1 = r.ch;
  }
  if (PASS == mtf::LOSS_FORWARD) return g;
  g.zero = c0 == 0.0 && (NT == kOne || c1 == 0.0);
  if (PASS == mtf::LOSS_STEP) {
    g.huge = F.is_huge(m);
    g.nb0 = -reference(m, a0);
    g.nb1 = -reference(m, a1);
    g.k0 = (float)c0 / s0;
    g.k1 = NT != kOne ? (float)c1 / s1 : 0.f;
    return g;
  }
  // from the stored log-sum-exps: 2^(z a - b) for exp of z / tau - lse, the rest of the exponent goes to the factor
  if (OP == mtf::LOSS_DISTILL) {
    r.lse0 = (double)a.lse[2 * row];
    r.lse1 = (double)a.lse[2 * row + 1];
  } else {
    r.lse0 = r.lse1 = (double)a.lse[row];
  }
  const double l0 = soft_on<OP>(a) ? r.lse0 * (double)a.temperature : OP == mtf::LOSS_DISTILL ? r.lse1 : r.lse0;
  g.m0 = (float)l0;
  g.m1 = NT == kOne ? g.m0 : (float)r.lse1;
  g.huge = F.is_huge(g.m0) || F.is_huge(g.m1);
  g.nb0 = -reference(is_powers(NT) ? g.m1 : g.m0, a0);      // (powers: t^hard is the probability, and nothing above it overflows or is lost below)
  g.nb1 = -reference(g.m1, a1);
  g.k0 = (float)(g.huge ? c0 : c0 * exp2((-(double)g.nb0 - l0 * (double)a0) * soft_power(NT)));
  g.k1 = (float)(g.huge || NT == kOne ? c1 : c1 * exp2(NT == kTwo ? -(double)g.nb1 - r.lse1 * (double)a1 : (-(double)g.nb0 - r.lse1 * (double)a0) * hard_power(NT)));
  return g;
}

// Then the rest.  write: this thread stores the results per row.
template <int OP, int PASS, int NT>
__device__ __forceinline__ void row_results(const LossRows& a, long long row, const RowIn& in, const RowInputs& x, float m, float s0, float s1, bool write, const Factors& F,
                                            RowNumbers& r) {
  const double w = (double)in.w;
  double logp = 0.0;           // of the label
  double above = 0.0;          // log-sum-exp of z / tau less zr / tau
  if (PASS & mtf::LOSS_FORWARD) {
    const double inv_tau = OP == mtf::LOSS_DISTILL ? a.inv_tau : 1.0, l0 = reference_off(m, F.a0, soft_power(NT), F) + log64((double)s0);
    const double l1 = NT == kOne ? l0 : reference_off(m, NT == kTwo ? F.a1 : F.a0, hard_power(NT), F) + log64((double)s1);
    r.lse0 = (double)m * inv_tau + l0;
    r.lse1 = NT == kOne ? r.lse0 : (double)m + l1;      // (one sum: tau is 1, or only one of the two is used)
    if (NT == kTwo && isnan(s1)) r.lse0 = r.lse1;       // (of two sums the softened one may have lost a NaN: see exponentials)
    if (s0 == 0.f) r.lse0 = r.lse1 = nan("");           // (no finite logit: the reference's own exponential is 1 in any other row's sums)
    logp = ((double)x.zy - (double)m) - l1;
    above = ((double)m - (double)x.zr) * inv_tau + l0;
  }
  if (OP != mtf::LOSS_DISTILL) {
    if (PASS & mtf::LOSS_FORWARD) {
      const float hi = (float)logp;
      // (preference: until the pairs' kernel has added the log-probabilities up, lse holds what rounding logp to f32 leaves over)
      if (write && a.lse) a.lse[row] = OP == mtf::LOSS_LOGP && isfinite(hi) ? (float)(logp - (double)hi) : (float)r.lse0;
      if (write && a.logp) a.logp[row] = hi;
      if (OP == mtf::LOSS_POLICY) {
        double loss = r.plain > r.clipped ? -r.clipped : -r.plain;
        if (a.kl_weight != 0.f) loss += (double)a.kl_weight * (r.em1 - ((double)x.ref - logp));
        if (write) a.loss[row] = (float)(w * loss);
        if (write && a.dlogp) a.dlogp[row] = (float)r.c;
      }
    }
    return;
  }
  if (PASS & mtf::LOSS_FORWARD) {
    double loss = 0.0;
    // (differences first: in a row of the type's lowest values the log-sum-exp has no digits left for anything else)
    if (x.sum != 0.0) loss = (double)a.soft * (double)a.temperature * (double)a.temperature * (x.kl + above);
    if (hard_on<OP>(a)) loss -= (double)a.hard * logp;
    if (write) {
      a.loss[row] = (float)(w * loss);
      if (a.lse) {
        a.lse[2 * row] = (float)(soft_on<OP>(a) ? r.lse0 : 0.0);
        a.lse[2 * row + 1] = (float)(hard_on<OP>(a) ? r.lse1 : 0.0);
      }
    }
  }
}

// one entry of a row's gradient as a walk writes it: for the row's edges, for rows with huge logits and for the entries that differ
template <int NT>
__device__ __forceinline__ float gradient_of(float z, const RowGrad& g, const Factors& F) {
  const float y = fmaf(z, F.a0, g.nb0);
  // (a stored log-sum-exp of that size is off by more than whole exponents: no probability above 1 comes of it; NaN stays)
  auto below = [](float d) { return d > 0.f ? 0.f : d; };
  float v = g.k0 * ex2(soft_power(NT) * (g.huge ? below((z - g.m0) * F.a0) : y));
  if (NT == kTwo) v += g.k1 * ex2(g.huge ? below((z - g.m1) * F.a1) : fmaf(z, F.a1, g.nb1));
  if (is_powers(NT)) v += g.k1 * ex2(hard_power(NT) * (g.huge ? below((z - g.m1) * F.a0) : y));
  return v;
}

// Slots with one id, by one warp: the first takes the others' share, and they get the id -1.  Up to 32 slots are compared at once.  For more, `seen`: two tables of kSeenBits bits, 0 before and
// behind (slot_values clears them); an id whose bit comes up twice in the first has it set in the second, and only such ids are searched for.
// (All pairs compared: 8192 rows of 32768 with 64 words 210 us in place of 196, with 256 592 in place of 334.)
constexpr int kSeenBits = 8192, kSeenWords = 2 * kSeenBits / 32;
__device__ __forceinline__ unsigned seen_bit(int id) { return ((unsigned)id ^ (unsigned)id >> 13) % kSeenBits; }
__device__ __forceinline__ void join_slots(const Slots& sl, int K, unsigned* seen, int lane) {
  if (K <= 32) {
    const int id = lane < K ? sl.id[lane] : -1;
    const unsigned same = __match_any_sync(0xffffffffu, id >= 0 ? id : -1 - lane);
    const bool first = (same & ((1u << lane) - 1u)) == 0u;
    __syncwarp();
    if (lane < K && !first) sl.id[lane] = -1;
    if (lane < K && first && (same & (same - 1u))) {
      double q = sl.q[lane];
      for (unsigned m = same & (same - 1u); m; m &= m - 1) q += sl.q[__ffs(m) - 1];
      sl.q[lane] = q;
    }
    __syncwarp();
    return;
  }
  bool twice = false;
#pragma unroll 1
  for (int k = lane; k < K; k += 32)
    if (sl.id[k] >= 0) {
      const unsigned bit = seen_bit(sl.id[k]), mask = 1u << (bit & 31);
      if (atomicOr(seen + (bit >> 5), mask) & mask) {
        atomicOr(seen + kSeenWords / 2 + (bit >> 5), mask);
        twice = true;
      }
    }
  if (!__any_sync(0xffffffffu, twice)) return;
  __syncwarp();
#pragma unroll 1
  for (int base = 0; base < K; base += 32) {
    const int k = base + lane, id = k < K ? sl.id[k] : -1;
    const unsigned bit = seen_bit(id);
    unsigned todo = __ballot_sync(0xffffffffu, id >= 0 && ((seen[kSeenWords / 2 + (bit >> 5)] >> (bit & 31)) & 1u));
    for (; todo; todo &= todo - 1) {
      const int first = base + __ffs(todo) - 1, wanted = sl.id[first];
      if (wanted < 0) continue;                      // (joined to an earlier one by now)
      double q = sl.q[first];
      for (int from = base; from < K; from += 32) {
        const int j = from + lane;
        const bool same = j > first && j < K && sl.id[j] == wanted;
        for (unsigned m = __ballot_sync(0xffffffffu, same); m; m &= m - 1) q += sl.q[from + __ffs(m) - 1];
        if (same) sl.id[j] = -1;
      }
      if (lane == 0) sl.q[first] = q;
      __syncwarp();
    }
  }
}
// The entries of a distillation row's gradient that differ from the walk's, by one warp: their values take the place of sl.z.  True: a slot has the
// label's entry, too.
template <int NT>
__device__ __forceinline__ bool slot_values(const LossRows& a, const RowGrad& g, const RowNumbers& r, const Slots& sl, unsigned* seen, int label, int lane, const Factors& F) {
  const int K = a.slots;
  join_slots(sl, K, seen, lane);
  bool has_label = false;
#pragma unroll 1
  for (int k = lane; k < K; k += 32) {
    const int id = sl.id[k];
    if (id < 0) continue;
    if (K > 32) seen[seen_bit(id) >> 5] = seen[kSeenWords / 2 + (seen_bit(id) >> 5)] = 0u;
    const bool is_label = r.ch != 0.0 && id == label;
    has_label |= is_label;
    sl.z[k] = (float)((double)gradient_of<NT>(sl.z[k], g, F) - r.cs * sl.q[k] - (is_label ? r.ch : 0.0));
  }
  __syncwarp();
  return __any_sync(0xffffffffu, has_label);
}
// ... behind the walk's stores, by threads `at` of n.  owned(id): this block writes that entry; label_alone: the label's entry is no slot's.
template <typename T, typename O>
__device__ __forceinline__ void write_slots(const LossRows& a, float fix, const Slots& sl, int label, bool label_alone, char* dr, int at, int n, O owned) {
  for (int k = at; k < a.slots; k += n) {
    const int id = sl.id[k];
    if (id >= 0 && owned(id)) Piece<T>::set(dr, id, sl.z[k]);
  }
  if (at == 0 && label_alone && owned(label)) Piece<T>::set(dr, label, fix);
}
// the label's entry (distillation: where no slot has it)
template <int OP, int NT>
__device__ __forceinline__ float label_value(const RowGrad& g, const RowNumbers& r, float zy, const Factors& F) {
  return (float)((double)gradient_of<NT>(zy, g, F) + (OP == mtf::LOSS_DISTILL ? -r.ch : r.c));
}

template <typename T, int NT>
struct GradValues {
  float k0 = 0.f, nb0 = 0.f, k1 = 0.f, nb1 = 0.f;
  __device__ __forceinline__ void set(const RowGrad& g) { k0 = g.k0; nb0 = g.nb0; k1 = g.k1; nb1 = g.nb1; }
  template <int kPair = 0>     // the first pair's number (of pieces of two pairs the second of two is numbered on)
  __device__ __forceinline__ uint4 piece(const uint4& u, const Factors& F) const {
    f32x2 f[Piece<T>::kN / 2];
    Piece<T>::get(u, f);
#pragma unroll
    for (int e = 0; e < Piece<T>::kN / 2; ++e) {
      f32x2 e0, e1;
      exponentials<NT, true>(kPair + e, f[e], F.a0, nb0, F.a1, nb1, e0, e1);
      if (is_powers(NT)) f[e] = mul2(power<soft_power(NT)>(e0), fma2(power<hard_power(NT) - soft_power(NT)>(e0), pair(k1), pair(k0)));      // (k0 and k1 have one sign)
      else f[e] = NT == kTwo ? fma2(e1, pair(k1), mul2(e0, pair(k0))) : mul2(e0, pair(k0));
    }
    return Piece<T>::put(f);
  }
};
// pieces [first, last) of a row with huge logits, by threads `at` of n
template <typename T, int NT>
__device__ __noinline__ void huge_pieces(const uint4* from, uint4* to, int first, int last, int at, int n, const RowGrad& g, const Factors& F) {
  for (int p = first + at; p < last; p += n) {
    f32x2 f[Piece<T>::kN / 2];
    Piece<T>::get(from[p], f);
    for (int e = 0; e < Piece<T>::kN / 2; ++e) f[e] = pair(gradient_of<NT>(both(f[e]).x, g, F), gradient_of<NT>(both(f[e]).y, g, F));
    to[p] = Piece<T>::put(f);
  }
}

// A row's part that one block works on: pieces [begin, end), and the row's edges with the first part.
template <typename T>
struct RowPart {
  RowSpan sp;
  const char* zr;
  char* dr;
  const uint4* z16;
  uint4* d16;
  int begin, end, edges, V;
  // rank: which part, of `each` pieces
  __device__ __forceinline__ RowPart(const LossRows& a, long long row, int each, int rank) : sp(row_span<T>(row, a.V)), V(a.V) {
    zr = reinterpret_cast<const char*>(a.z) + row * a.V * (long long)sizeof(T);
    dr = reinterpret_cast<char*>(a.d) + row * a.V * (long long)sizeof(T);
    z16 = reinterpret_cast<const uint4*>(zr + sp.head * (int)sizeof(T));
    d16 = reinterpret_cast<uint4*>(dr + sp.head * (int)sizeof(T));
    begin = min(sp.pieces, rank * each);
    end = min(sp.pieces, begin + each);
    edges = rank == 0 ? sp.head + sp.tail : 0;
  }
  __device__ __forceinline__ int edge(int i) const { return edge_element(sp, i, V); }
  __device__ __forceinline__ bool owned(int e) const {
    constexpr int n = Piece<T>::kN;
    return (e >= sp.head + begin * n && e < sp.head + end * n) || (edges && (e < sp.head || e >= V - sp.tail));
  }
  __device__ __forceinline__ void zeros(int tid, int n) const {
    for (int p = begin + tid; p < end; p += n) d16[p] = make_uint4(0u, 0u, 0u, 0u);
    if (tid < edges) Piece<T>::set(dr, edge(tid), 0.f);
  }
};

// The part's largest entry and sums from differences to it, by one warp: for the rows that RunningSum leaves out.  Slow, one entry a lane at a time and twice over the
// part, while the block waits; a row that is masked as a whole should have the weight 0.  8192 x 32768 bf16 in one call: 191 us without such rows, 790 with one, 2180 with 1024,
// 6420 with 4096; their statistics alone 99, 429, 635, 1173.  2048 x 131072: 231, with one 1320, with 1024 12800; alone 99, 1930, 5560.
template <typename T, int NT>
__device__ __noinline__ void sums_of_differences(const RowPart<T>& part, int lane, const Factors& F, float& m, float& s0, float& s1) {
  constexpr int n = Piece<T>::kN;
  const int first = part.sp.head + part.begin * n, last = part.sp.head + part.end * n;
  auto each = [&](auto f) {
    for (int e = first + lane; e < last; e += 32) f(Piece<T>::one(part.zr, e));
    if (lane < part.edges) f(Piece<T>::one(part.zr, part.edge(lane)));
  };
  m = kLowest;
  each([&](float z) { m = fmaxf(m, z); });
  m = warp_max(m);
  s0 = s1 = 0.f;
  each([&](float z) {
    s0 += ex2(soft_power(NT) * ((z - m) * F.a0));
    if (NT != kOne) s1 += ex2(hard_power(NT) * ((z - m) * (NT == kTwo ? F.a1 : F.a0)));
  });
  s0 = warp_add(s0);
  s1 = warp_add(s1);
}

// ---- one block per row, which walks over it in global memory ---------------------------------------------------------------------
constexpr int kRowWarps = 8;

// pieces [begin, end) of a row, by threads `at` of n, U loads in flight a thread
template <int U, typename F>
__device__ __forceinline__ void walk(const uint4* z16, int begin, int end, int at, int n, F f) {
  for (int p = begin + at; p < end; p += U * n) {
    uint4 u[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (p + i * n < end) u[i] = z16[p + i * n];
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (p + i * n < end) f(p + i * n, u[i]);
  }
}

struct Scratch {
  float m[kRowWarps], s0[kRowWarps], s1[kRowWarps];
  float4 part;                 // this block's sums, for the other blocks of the row
  RowGrad g;
};
static_assert(sizeof(Scratch) % 16 == 0, "the teacher's list lies behind it");

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t in_peer(const void* p, uint32_t rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  return at;
}

// Bound: memory, for all but few rows; then a chain of latencies (the label, the row, its sums, its numbers in 64 bits).  Statistics are one pass with
// a running reference, loads of four pieces ahead; a gradient reads its row again, from the L2 cache where the statistics have just left it.
// 8192 x 32768 bf16: statistics 94 us (5.7 TB/s; the special-function unit is busy for 60), a gradient 157 (6.8); 16 rows in one call 6 us.
// Registers are held to four blocks an SM (teacher's lists: three, other gradients on their own: six): with five 777 f32 rows of 50001 take 72 us in place of 66, with three 69.
//
// A row may be cut into `parts`, a block each.  Where sums are taken (few rows) the blocks are a cluster and read each other's sums.  A gradient on its own
// needs nothing of the other parts: what a block reads of them it has no use for (they may be overwritten already).
// A distillation's teacher is worked out by a warp of its own beside the walk.
template <typename T, int OP, int PASS, int NT>
__global__ void __launch_bounds__((kRowWarps + (OP == mtf::LOSS_DISTILL)) * 32, OP == mtf::LOSS_DISTILL ? 3 : PASS == mtf::LOSS_BACKWARD ? 6 : 4) loss_rows_kernel(const LossRows a, const Factors F, const int parts, const int each) {
  extern __shared__ __align__(128) unsigned char dyn[];
  Scratch& sc = *reinterpret_cast<Scratch*>(dyn);
  const Slots sl(dyn + sizeof(Scratch), a.slots);
  unsigned* const seen = reinterpret_cast<unsigned*>(dyn + sizeof(Scratch) + Slots::bytes(a.slots));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = OP == mtf::LOSS_DISTILL ? blockDim.x - 32 : blockDim.x, warps = n >> 5;      // of the walk
  const bool walks = tid < n, numbers = warp == (OP == mtf::LOSS_DISTILL ? warps : 0);
  const unsigned which = parts == 1 ? blockIdx.x : blockIdx.x / (unsigned)parts;
  const int rank = blockIdx.x - which * parts;
  const long long at = which, row = a.reverse ? a.rows - 1 - at : at;
  constexpr bool kSums = (PASS & mtf::LOSS_FORWARD) != 0;
  const RowPart<T> part(a, row, each, rank);
  if (OP == mtf::LOSS_LOGP && PASS == mtf::LOSS_FORWARD) mtf::chain_wait();      // (the pairs' kernel reads its inputs meanwhile)
  else mtf::chain_wait_only();
  const RowIn in = row_in<OP, PASS>(a, row);
  if (in.skip) {               // (every block of the row)
    if (tid == 0 && rank == 0 && in.bad) atomicExch(&g_bad_id, 1);
    if ((PASS & mtf::LOSS_FORWARD) && tid == 0 && rank == 0) zero_results<OP>(a, row);
    if (PASS & mtf::LOSS_BACKWARD) part.zeros(tid, blockDim.x);
    return;
  }
  RowInputs x = {};
  if (numbers) {
    Fetched f = {};
    if (OP == mtf::LOSS_DISTILL) fetch_slots(a, row, 0, lane, soft_on<OP>(a), f);
    if (OP == mtf::LOSS_DISTILL && (PASS & mtf::LOSS_BACKWARD) && a.slots > 32)
      for (int i = lane; i < kSeenWords; i += 32) seen[i] = 0u;
    x = row_inputs<T, OP>(a, row, part.zr, in.label, f, sl, lane, rank == 0);
    if (OP == mtf::LOSS_DISTILL && PASS != mtf::LOSS_BACKWARD) teacher(a, x, sl, lane);
  }
  // a gradient on its own: the first pieces are on their way while the row's factors are worked out
  uint4 early[4];
  if (PASS == mtf::LOSS_BACKWARD && walks)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (part.begin + tid + i * n < part.end) early[i] = part.z16[part.begin + tid + i * n];

  float m = 0.f, s0 = 1.f, s1 = 1.f;
  if (PASS & mtf::LOSS_FORWARD) {
    RunningSum<NT> rs(F);
    // four pieces' loads in flight while the four before are worked on
    const int first = walks ? part.begin + tid : part.end, fours = first < part.end ? (part.end - first + n - 1) / n / 4 : 0;
    const uint4* z = part.z16 + first;
    uint4 u[4], w[4];
    auto load = [&](uint4* to) {
#pragma unroll
      for (int i = 0; i < 4; ++i) to[i] = z[i * n];
      z += 4 * n;
    };
    if (PASS == mtf::LOSS_FORWARD) {
      if (fours) load(u);
      for (int k = 1; k < fours; k += 2) {
        load(w);
        rs.template add<T, 4>(u, F);
        if (k + 1 < fours) load(u);
        rs.template add<T, 4>(w, F);
      }
      if (fours & 1) rs.template add<T, 4>(u, F);
    } else {
      for (int k = 0; k < fours; ++k) {
        load(u);
        rs.template add<T, 4>(u, F);
      }
    }
    for (; z < part.z16 + part.end; z += n) {
      const uint4 one = *z;
      rs.template add<T, 1>(&one, F);
    }
    if (tid < part.edges) rs.add_one(Piece<T>::one(part.zr, part.edge(tid)), F);
    float t_m, t_0, t_1;
    rs.of_warp(t_m, t_0, t_1, F);
    if (lane == 0 && walks) { sc.m[warp] = t_m; sc.s0[warp] = t_0; sc.s1[warp] = t_1; }
    __syncthreads();
    if (numbers) {
      m = lane < warps ? sc.m[lane] : -F.huge;
      s0 = lane < warps ? sc.s0[lane] : 0.f;
      s1 = lane < warps ? sc.s1[lane] : 0.f;
      warp_join<NT>(m, s0, s1, F);
      if (F.is_huge(m)) sums_of_differences<T, NT>(part, lane, F, m, s0, s1);
      if (lane == 0) sc.part = make_float4(m, s0, s1, 0.f);
    }
  }
  if (kSums && parts > 1) {
    __syncwarp();
    cluster_arrive();
    cluster_wait();            // (from here on a block may overwrite its part of the row)
    if (numbers) {
      m = kLowest;
      s0 = s1 = 0.f;
      if (lane < parts)
        asm volatile("{\n\t.reg .f32 none;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, none}, [%3];\n\t}" : "=f"(m), "=f"(s0), "=f"(s1) : "r"(in_peer(&sc.part, lane)) : "memory");
      warp_join<NT>(m, s0, s1, F);
    }
    __syncwarp();
    cluster_arrive();          // this block has read the others' sums: they may end once all have
  }
  RowNumbers r = {};
  if (numbers) {
    const RowGrad g = row_gradient<OP, PASS, NT>(a, row, in, x, m, s0, s1, F, r);
    if ((PASS & mtf::LOSS_BACKWARD) && lane == 0) sc.g = g;
    if (PASS == mtf::LOSS_FORWARD) row_results<OP, PASS, NT>(a, row, in, x, m, s0, s1, rank == 0 && lane == 0, F, r);
  }
  if (PASS & mtf::LOSS_BACKWARD) {
    __syncthreads();
    const bool zero = sc.g.zero;
    if (zero) {
      part.zeros(tid, blockDim.x);
    } else if (walks) {
      if (sc.g.huge) {
        huge_pieces<T, NT>(part.z16, part.d16, part.begin, part.end, tid, n, sc.g, F);
      } else {
        GradValues<T, NT> v;
        v.set(sc.g);
        int from = part.begin;
        if (PASS == mtf::LOSS_BACKWARD) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (from + tid + i * n < part.end) part.d16[from + tid + i * n] = v.piece(early[i], F);
          from += 4 * n;
        }
        walk<4>(part.z16, from, part.end, tid, n, [&](int p, const uint4& u) { part.d16[p] = v.piece(u, F); });
      }
      if (tid < part.edges) Piece<T>::set(part.dr, part.edge(tid), gradient_of<NT>(Piece<T>::one(part.zr, part.edge(tid)), sc.g, F));
    }
    bool alone = true;
    float fix = 0.f;
    if (numbers) {
      if (PASS & mtf::LOSS_FORWARD) row_results<OP, PASS, NT>(a, row, in, x, m, s0, s1, rank == 0 && lane == 0, F, r);
      if (OP == mtf::LOSS_DISTILL && PASS == mtf::LOSS_BACKWARD) teacher(a, x, sl, lane);
      fix = label_value<OP, NT>(sc.g, r, x.zy, F);
      if (OP == mtf::LOSS_DISTILL) alone = !slot_values<NT>(a, sc.g, r, sl, seen, in.label, lane, F) && hard_on<OP>(a);
    }
    __syncthreads();
    if (numbers && !zero) {
      if (OP == mtf::LOSS_DISTILL) write_slots<T>(a, fix, sl, in.label, alone, part.dr, lane, 32, [&](int e) { return part.owned(e); });
      else if (lane == 0 && part.owned(in.label)) Piece<T>::set(part.dr, in.label, fix);
    }
  }
  if (kSums && parts > 1) {
    __syncwarp();
    cluster_wait();
  }
}

// ---- rows streamed through shared memory: statistics and gradient from one read ------------------------------------------------------
// A block (or a cluster of them, each with a part of every row) takes every n-th row.  One warp keeps a ring of chunks filled by bulk copies.
// Sixteen warps walk over the chunks twice, for the statistics and, `lead` chunks later, for the gradient, taking a chunk of each walk in turn:
// chunks are read, freed and written at one steady rate.  Three more warps work out the rows' numbers, a row each; a row's are wanted `lead`
// chunks behind its first, that is some chunks behind its last.  Rows are numbered by those that are not skipped (o); row o has slot o mod 3.
// Bound: memory, and close behind it the special-function unit: two exponentials an entry are 1020 cycles of the 1600 that a chunk takes.  Measured:
// 8192 x 32768 bf16 184 us (5.85 TB/s, of measured 0.90), with a teacher's 64 words at temperature 2 196 of 7592 rows that count (two powers an entry; with 256 words 334, the numbers);
// 4096 x 32768 f32 168 (6.4); 2048 x 131072 bf16 in pairs of blocks 226, which wait for each other's sums.  Four to six warps for the numbers take
// issue slots from the walks (212 to 223 in place of 210 with a teacher, when its list was searched for equal words by comparing all pairs).
constexpr int kWalkers = 16, kNumberWarps = 3, kStreamThreads = 32 * (1 + kNumberWarps + kWalkers);
constexpr int kChunk = 16384, kChunkPieces = kChunk / 16, kMaxChunks = 13, kMaxParts = 8, kRowSlots = kNumberWarps;
constexpr int kBlockSharedMemory = 227 * 1024;       // what a block may have

struct Stream {
  uint64_t full[kMaxChunks], empty[kMaxChunks];      // a chunk has landed / every walking warp is through with it
  uint64_t sums[kRowSlots];                          // the walking warps' sums of the slot's row are there
  uint64_t ready[kRowSlots];                         // ... its numbers are
  uint64_t done[kRowSlots];                          // ... its gradient is, but for the entries that differ
  uint64_t peers[kRowSlots], heard[kRowSlots];       // the other parts' sums are there; the other blocks have read this one's
  int abort;
  int pad[3];
  float4 sum[kRowSlots][kWalkers];
  float4 peer[kRowSlots][kMaxParts];
  RowGrad g[kRowSlots];
};
static_assert(sizeof(Stream) % 16 == 0, "lists lie behind it");

__device__ __forceinline__ void bar_init(uint64_t* bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint64_t* bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory"); }
__device__ __forceinline__ void bar_expect(uint64_t* bar, uint32_t bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory"); }
__device__ __forceinline__ bool bar_try(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
  return ok != 0;
}
// Gives up after about two seconds: a code for mtf_device_status, and from then on no wait of the block waits (its rows' results are unspecified).
// Warps that then go on only write what is unspecified and arrive at barriers whose phases end with the last of so many arrivals.  What counts bytes, or is another
// block's, needs the waits in front of it: there the copying warp and the numbers' warps leave (given_up), and the other blocks' waits for this one run out in turn.
// (Checks behind the numbers' other waits and a signal left out by a comparison in each row took a step with 64 words at temperature 2 from 198 to 217 us: the rows'
// numbers run at the rate at which their instructions come in.)
__device__ __noinline__ void bar_wait_slow(uint64_t* bar, uint32_t parity, int code, volatile int* abort) {
  const long long t0 = clock64(), limit = g_wait_limit;
  while (!bar_try(bar, parity)) {
    if (*abort) return;
    if (clock64() - t0 > limit) {
      atomicCAS(&g_loss_status, 0, code);
      *abort = 1;
      return;
    }
  }
}
__device__ __forceinline__ void bar_wait(uint64_t* bar, uint32_t parity, int code, int* abort) {
  if (!bar_try(bar, parity)) bar_wait_slow(bar, parity, code, abort);
}
// Whether a wait of the block has been given up, as any lane of the warp sees it (a lane that gave up itself does).
__device__ __forceinline__ bool given_up(const Stream& st) { return __any_sync(0xffffffffu, *(const volatile int*)&st.abort); }
constexpr long long kLandCycles = 200000000LL;       // 0.1 s, for copies in flight
template <typename T, int OP, int NT>
__global__ void __launch_bounds__(kStreamThreads, 1) loss_stream_kernel(const LossRows a, const Factors F, const int parts, const int each, const int chunks, const int lead) {
  constexpr int PASS = mtf::LOSS_STEP;
  extern __shared__ __align__(128) unsigned char dyn[];
  const size_t list = OP == mtf::LOSS_DISTILL ? Slots::bytes(a.slots) : 0;
  uint4* const ring = reinterpret_cast<uint4*>(dyn);
  Stream& st = *reinterpret_cast<Stream*>(dyn + (size_t)chunks * kChunk);
  unsigned char* const lists = dyn + (size_t)chunks * kChunk + sizeof(Stream);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = blockIdx.x % parts;
  const long long first = blockIdx.x / parts, stride = gridDim.x / parts;
  const int n = (int)((a.rows - first + stride - 1) / stride);        // rows of this block, each known by its number i
  auto row_of = [&](int i) { return first + i * stride; };
  if (tid == 0) {
    for (int c = 0; c < chunks; ++c) { bar_init(&st.full[c], 1); bar_init(&st.empty[c], kWalkers); }
    for (int s = 0; s < kRowSlots; ++s) {
      bar_init(&st.sums[s], kWalkers);
      bar_init(&st.ready[s], s == 0 && g_withhold == kNumbersHeld ? 2 : 1);
      bar_init(&st.done[s], kWalkers);
      bar_init(&st.peers[s], s == 0 && g_withhold == kSumsHeld ? 2 : 1);
      bar_init(&st.heard[s], parts);
    }
    st.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (parts > 1) {             // the others' barriers are set up as well
    cluster_arrive();
    cluster_wait();
  }
  mtf::chain_wait_only();

  // Which rows are skipped is found out 32 rows at a time, a row a lane, by every warp for itself.
  uint32_t live = 0u;
  auto look = [&](uint32_t& mask, int i) {
    if ((i & 31) == 0) mask = __ballot_sync(0xffffffffu, i + lane < n && !row_in<OP, PASS>(a, row_of(i + lane)).skip);
    return ((mask >> (i & 31)) & 1u) != 0u;
  };

  if (warp == 0) {
    // ------------------------------- copies -------------------------------
    int slot = 0;
    uint32_t phase = 1u;
    for (int i = 0; i < n; ++i) {
      if (!look(live, i)) continue;
      if (lane == 0) {
        const RowPart<T> part(a, row_of(i), each, rank);
        for (int p = part.begin; p < part.end; p += kChunkPieces) {
          bar_wait(&st.empty[slot], phase, 0xA01, &st.abort);
          if (*(volatile int*)&st.abort) break;      // (a chunk may be on its way into the slot, still)
          const uint32_t bytes = (uint32_t)min(kChunkPieces, part.end - p) * 16u;
          bar_expect(&st.full[slot], bytes);
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                       ::"r"(smem_u32(ring + slot * kChunkPieces)), "l"(part.z16 + p), "r"(bytes), "r"(smem_u32(&st.full[slot])) : "memory");
          if (++slot == chunks) { slot = 0; phase ^= 1u; }
        }
      }
      __syncwarp();
      if (given_up(st)) break;
    }
    // The block does not end in front of its copies, which nobody else waits for once a wait was given up.  (Slots from `slot` on were last filled a turn of the ring
    // before the others, or not yet: then the wait is for the phase before a barrier's first, which is over.)
    if (lane == 0) {
      const long long t0 = clock64();
      for (int c = 0; c < chunks; ++c)
        while (!bar_try(&st.full[c], c < slot ? phase ^ 1u : phase) && clock64() - t0 < kLandCycles) {}
    }
    __syncwarp();
  } else if (warp <= kNumberWarps) {
    // ------------------------------- the rows' numbers -------------------------------
    const int s = warp - 1;
    uint32_t phase = 1u;
    int turn = -1, uses = 0, i = -1;                 // slot of row i; rows of this warp so far
    // to this warp's next row, with the results of skipped rows on the way; false behind the last
    auto next = [&] {
      while (++i < n) {
        if (look(live, i)) {
          if (++turn == kRowSlots) turn = 0;
          if (turn == s) return true;
        } else if (i % kNumberWarps == s && rank == 0 && lane == 0) {
          const long long row = row_of(i);
          if (row_in<OP, PASS>(a, row).bad) atomicExch(&g_bad_id, 1);
          zero_results<OP>(a, row);
        }
      }
      return false;
    };
    // What is read of a row is read while the walks still have the row before in hand: two lists a warp, and the loads a row earlier still.
    RowIn in = {}, in_next = {};
    RowInputs x = {};
    Fetched f = {};
    unsigned* const seen = reinterpret_cast<unsigned*>(lists + 2 * kNumberWarps * list) + s * kSeenWords;
    if (OP == mtf::LOSS_DISTILL)
      for (int k = lane; k < kSeenWords; k += 32) seen[k] = 0u;
    __syncwarp();
    auto list_of = [&](int use) { return Slots(lists + (2 * s + (use & 1)) * list, a.slots); };
    auto fetch = [&] {
      in_next.w = a.weight ? a.weight[row_of(i)] : 1.f;      // (a row that is not skipped: its label is good)
      in_next.label = OP != mtf::LOSS_DISTILL || hard_on<OP>(a) ? a.targets[row_of(i)] : 0;
      if (OP == mtf::LOSS_DISTILL) fetch_slots(a, row_of(i), 0, lane, soft_on<OP>(a), f);
    };
    auto read = [&] {
      in = in_next;
      x = row_inputs<T, OP>(a, row_of(i), RowPart<T>(a, row_of(i), each, rank).zr, in.label, f, list_of(uses), lane, rank == 0);
      if (OP == mtf::LOSS_DISTILL) teacher(a, x, list_of(uses), lane);
    };
    bool more = next();
    if (more) { fetch(); read(); }
    while (more) {
      const long long row = row_of(i);
      const RowPart<T> part(a, row, each, rank);
      more = next();
      if (more) fetch();
      const Slots sl = list_of(uses);
      phase ^= 1u;
      float m = -F.huge, s0 = 0.f, s1 = 0.f;
      bar_wait(&st.sums[s], phase, 0xA02, &st.abort);
      if (lane < kWalkers) { const float4 v = st.sum[s][lane]; m = v.x; s0 = v.y; s1 = v.z; }
      warp_join<NT>(m, s0, s1, F);
      if (F.is_huge(m)) sums_of_differences<T, NT>(part, lane, F, m, s0, s1);
      if (parts > 1) {
        // to every block of the row, and from there
        if (uses) bar_wait(&st.heard[s], phase ^ 1u, 0xA03, &st.abort);
        if (given_up(st)) break;
        if (lane == 0) bar_expect(&st.peers[s], (uint32_t)parts * 16u);
        __syncwarp();
        if (lane < parts)
          asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                       ::"r"(in_peer(&st.peer[s][rank], lane)), "f"(m), "f"(s0), "f"(s1), "f"(0.f), "r"(in_peer(&st.peers[s], lane)) : "memory");
        bar_wait(&st.peers[s], phase, 0xA04, &st.abort);
        if (given_up(st)) break;
        m = kLowest;
        s0 = s1 = 0.f;
        if (lane < parts) { const float4 v = st.peer[s][lane]; m = v.x; s0 = v.y; s1 = v.z; }
        __syncwarp();
        if (lane < parts) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_peer(&st.heard[s], lane)) : "memory");
        warp_join<NT>(m, s0, s1, F);
      }
      RowNumbers r;
      const RowGrad g = row_gradient<OP, PASS, NT>(a, row, in, x, m, s0, s1, F, r);
      __syncwarp();            // (every lane has read the sums)
      if (lane == 0) {
        st.g[s] = g;
        bar_arrive(&st.ready[s]);
      }
      if (rank == 0) row_results<OP, PASS, NT>(a, row, in, x, m, s0, s1, lane == 0, F, r);
      const int label = in.label;
      bool alone = true;
      if (OP == mtf::LOSS_DISTILL) alone = !slot_values<NT>(a, g, r, sl, seen, label, lane, F) && hard_on<OP>(a);
      const float fix = label_value<OP, NT>(g, r, x.zy, F);
      const bool zero = g.zero;
      ++uses;
      if (more) read();
      bar_wait(&st.done[s], phase, 0xA05, &st.abort);
      if (!zero) {
        if (OP == mtf::LOSS_DISTILL) write_slots<T>(a, fix, sl, label, alone, part.dr, lane, 32, [&](int e) { return part.owned(e); });
        else if (lane == 0 && part.owned(label)) Piece<T>::set(part.dr, label, fix);
      }
      __syncwarp();
    }
  } else {
    // ------------------------------- walks -------------------------------
    const int at = tid - 32 * (1 + kNumberWarps);
    constexpr int nt = 32 * kWalkers, kEach = kChunkPieces / nt;
    // Rows whose length is a whole number of pieces all have the same part, without edges.
    const bool aligned = a.V % Piece<T>::kN == 0;
    const int begin0 = min(a.V / Piece<T>::kN, rank * each), end0 = min(a.V / Piece<T>::kN, begin0 + each);
    // the statistics' walk: row i, with slot s1; pieces [p, end) of its part are to come, the next of them in chunk c1
    int i = -1, s1 = -1, p = 0, end = 0, c1 = 0;
    uint32_t phase1 = 0u;
    float edge = 0.f;
    bool has_edge = false;
    RunningSum<NT> rs(F);
    auto next = [&] {                                // to the next row; false behind the last
      do {
        if (++i >= n) return false;
      } while (!look(live, i));
      if (++s1 == kRowSlots) s1 = 0;
      rs = RunningSum<NT>(F);
      p = begin0;
      end = end0;
      if (aligned) return true;
      const RowPart<T> part(a, row_of(i), each, rank);
      p = part.begin;
      end = part.end;
      has_edge = at < part.edges;
      if (has_edge) edge = Piece<T>::one(part.zr, part.edge(at));      // (wanted at the row's end)
      return true;
    };
    auto count = [&] {                               // a chunk
      bar_wait(&st.full[c1], phase1, 0xA11, &st.abort);
      const uint4* const c = ring + c1 * kChunkPieces;
      if (end - p >= kChunkPieces) {
        uint4 u[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) u[k] = c[at + k * nt];
        rs.template add<T, kEach>(u, F);
      } else {
        for (int k = at; k < end - p; k += nt) {
          const uint4 u = c[k];
          rs.template add<T, 1>(&u, F);
        }
      }
      if (++c1 == chunks) { c1 = 0; phase1 ^= 1u; }
      p += kChunkPieces;
    };
    auto finish = [&] {                              // the row's sums are complete
      if (has_edge) rs.add_one(edge, F);
      float t_m, t_0, t_1;
      rs.of_warp(t_m, t_0, t_1, F);
      if (lane == 0) {
        st.sum[s1][warp - 1 - kNumberWarps] = make_float4(t_m, t_0, t_1, 0.f);
        bar_arrive(&st.sums[s1]);
      }
      __syncwarp();
    };
    // the gradient's walk: row j, slot s2; `left` pieces to come, to `to` and behind, from chunk c2
    int j = -1, s2 = -1, left = 0, c2 = 0;
    uint32_t live_j = 0u, phase2 = 1u;
    uint4* to = nullptr;
    float edge_j = 0.f;
    bool has_edge_j = false, no_chunk = false, plain = false;      // plain: neither zeros nor huge logits
    GradValues<T, NT> v;
    auto next_j = [&] {                              // to the next row that is not skipped, writing the zeros of those between; false behind the last
      while (true) {
        if (++j >= n) return false;
        const bool alive = look(live_j, j);
        if (alive) {
          if (++s2 == kRowSlots) s2 = 0;
          if (s2 == 0) phase2 ^= 1u;
          if (aligned) {
            to = reinterpret_cast<uint4*>(reinterpret_cast<char*>(a.d) + row_of(j) * a.V * (long long)sizeof(T)) + begin0;
            left = end0 - begin0;
            no_chunk = left == 0;
            return true;
          }
        }
        const RowPart<T> part(a, row_of(j), each, rank);
        if (!alive) { part.zeros(at, nt); continue; }
        to = part.d16 + part.begin;
        left = part.end - part.begin;
        no_chunk = left == 0;
        has_edge_j = at < part.edges;
        if (has_edge_j) edge_j = Piece<T>::one(part.zr, part.edge(at));
        return true;
      }
    };
    auto put = [&] {                                 // a chunk
      const uint4* const c = ring + c2 * kChunkPieces;
      const int here = min(left, kChunkPieces);
      if (!plain) {
        if (!st.g[s2].zero) huge_pieces<T, NT>(c, to, 0, here, at, nt, st.g[s2], F);
        else
          for (int k = at; k < here; k += nt) to[k] = make_uint4(0u, 0u, 0u, 0u);
      } else if (here == kChunkPieces) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) to[at + k * nt] = v.piece(c[at + k * nt], F);
      } else {
        for (int k = at; k < here; k += nt) to[k] = v.piece(c[k], F);
      }
      __syncwarp();
      if (lane == 0) bar_arrive(&st.empty[c2]);
      if (++c2 == chunks) c2 = 0;
      to += kChunkPieces;
      left -= kChunkPieces;
    };
    auto finish_j = [&] {
      if (has_edge_j) {
        const RowPart<T> part(a, row_of(j), each, rank);
        Piece<T>::set(part.dr, part.edge(at), st.g[s2].zero ? 0.f : gradient_of<NT>(edge_j, st.g[s2], F));
      }
      __syncwarp();
      if (lane == 0) bar_arrive(&st.done[s2]);
    };
    // `ahead`: chunks that the first walk is ahead by.  A row may be without a chunk (fewer entries than a piece): it counts as one.
    int ahead = 0;
    bool more = next(), more_j = next_j(), begun = false;
    while (more_j) {
      if (more && ahead < lead) {
        if (p < end) count();
        ++ahead;
        if (p >= end) { finish(); more = next(); }
        continue;
      }
      if (!begun) {                                  // the row's numbers
        bar_wait(&st.ready[s2], phase2, 0xA12, &st.abort);
        plain = !st.g[s2].zero && !st.g[s2].huge;
        v.set(st.g[s2]);
        begun = true;
      }
      if (more && plain) {
        // both walks at once: their chains of instructions fill each other's waits
        const int both_full = min(end - p, left) / kChunkPieces;
#pragma unroll 1
        for (int c = 0; c < both_full; ++c) {
          bar_wait(&st.full[c1], phase1, 0xA11, &st.abort);
          uint4 u[kEach], w[kEach];
#pragma unroll
          for (int k = 0; k < kEach; ++k) { u[k] = ring[c1 * kChunkPieces + at + k * nt]; w[k] = ring[c2 * kChunkPieces + at + k * nt]; }
          rs.raise(Piece<T>::template largest<kEach>(u), F);
          rs.template add_below<T, kEach>(u, F);
#pragma unroll
          for (int k = 0; k < kEach; ++k) to[at + k * nt] = (k & 1) && Piece<T>::kN == 4 ? v.template piece<2>(w[k], F) : v.piece(w[k], F);
          __syncwarp();
          if (lane == 0) bar_arrive(&st.empty[c2]);
          if (++c1 == chunks) { c1 = 0; phase1 ^= 1u; }
          if (++c2 == chunks) c2 = 0;
          p += kChunkPieces;
          to += kChunkPieces;
          left -= kChunkPieces;
        }
        if (both_full) {
          if (p >= end) { finish(); more = next(); }
          if (left > 0) continue;
        }
      }
      if (left > 0) {
        put();
        --ahead;
      }
      if (left <= 0) {
        if (no_chunk) --ahead;
        finish_j();
        more_j = next_j();
        begun = false;
      }
    }
  }

  if (parts > 1 && *(volatile int*)&st.abort)
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);      // sums on their way to and from other blocks get time to land
  if (parts > 1) {             // nobody leaves while another block may still write to its shared memory
    __syncwarp();
    cluster_arrive();
    cluster_wait();
  }
}

// ---- the pairs of the preference loss ----------------------------------------------------------------------------------------------------
constexpr int kPairThreads = 1024;
// One block per pair: both sequences' log-probabilities added up in a fixed order, in 64 bits, then the loss of the pair and its
// derivative by each of the two sums.  A sum of hundreds of log-probabilities that are each rounded to f32 would be off by more than its
// own rounding (the loss goes by the difference of two): the rows' kernel has left the rest of each in lse's place, and lse itself, the
// label's logit less the log-probability, is written here.
template <typename T>
__global__ void __launch_bounds__(kPairThreads) preference_pairs_kernel(const mtf::PreferencePairs a) {
  __shared__ double red[kPairThreads / 32];
  const long long b = blockIdx.x;
  // half of the threads to each of the two
  constexpr int half = kPairThreads / 2;
  const int side = threadIdx.x / half;
  const long long end = (side * a.pairs + b + 1) * a.length, first = end - a.length + threadIdx.x % half;
  // What the rows' kernel only reads, too, is read while that still runs: the first tokens' weights, targets and labels' logits.  (Blocks of this
  // kernel start when all of that one's have waited for what came before it.)
  constexpr int ahead = 2;
  float w[ahead], z[ahead];
  auto input = [&](long long t, float& wt, float& zt) {
    const int label = a.targets[t];
    const bool good = label >= 0 && label < a.V;
    wt = good ? (a.weight ? a.weight[t] : 1.f) : 0.f;
    zt = good ? Piece<T>::one(a.z, t * a.V + label) : 0.f;
  };
#pragma unroll
  for (int i = 0; i < ahead; ++i) {
    w[i] = 0.f;
    if (first + i * half < end) input(first + i * half, w[i], z[i]);
  }
  mtf::chain_wait();
  double v = 0.0;
  auto add = [&](long long t, float wt, float zt) {
    const float hi = a.logp[t], lo = a.lse[t];
    if (wt == 0.f) return;       // (both 0)
    if (isfinite(hi)) {
      const double logp = (double)hi + (double)lo;
      v += (double)wt * logp;
      a.lse[t] = (float)((double)zt - logp);
    } else {
      v += (double)wt * (double)hi;
    }
  };
#pragma unroll
  for (int i = 0; i < ahead; ++i)
    if (first + i * half < end) add(first + i * half, w[i], z[i]);
  for (long long t = first + ahead * half; t < end; t += half) {
    float wt, zt;
    input(t, wt, zt);
    add(t, wt, zt);
  }
  v = warp_add(v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  double s[2];
  v = red[threadIdx.x];
#pragma unroll
  for (int o = half / 64; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  s[0] = __shfl_sync(0xffffffffu, v, 0);
  s[1] = __shfl_sync(0xffffffffu, v, half / 32);
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

// the first sum is the softened one wherever there is one
template <int NT>
Factors factors(const LossRows& a) {
  if (is_powers(NT)) return Factors(kLog2e / hard_power(NT), kLog2e);
  return Factors(kLog2e * (float)a.inv_tau, kLog2e);
}
template <typename T>
int pieces_each(const LossRows& a, int parts) { return (a.V / Piece<T>::kN + parts - 1) / parts; }

// Clusters of `parts` blocks of the stream kernel, one block to an SM, that the GPU holds at once (the SMs of a cluster lie in one group of
// them, so this is less than SMs / parts); 0 where the driver does not say.
template <typename K>
int resident_clusters(K kernel, const cudaLaunchConfig_t& cfg, mtf::KnownPerDevice& known) {
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess) (void)cudaGetLastError();
  return known.get(device, [&] {
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) { (void)cudaGetLastError(); n = 0; }
    return n;
  });
}

// false: not a launch for this kernel (too long a list or row for the shared memory, no cluster of its size on the device)
template <typename T, int OP, int NT>
bool launch_stream(const LossRows& a, size_t list, cudaLaunchConfig_t cfg, cudaLaunchAttribute* at) {
  const long long pieces = (long long)a.V * (a.bf16 ? 2 : 4) / 16;
  const size_t fixed = sizeof(Stream) + kNumberWarps * (2 * list + (list ? kSeenWords * 4 : 0));
  const int chunks = std::min<int>(kMaxChunks, (int)((kBlockSharedMemory - fixed) / kChunk));
  auto part_chunks = [&](int parts) { return (int)(((pieces + parts - 1) / parts + kChunkPieces - 1) / kChunkPieces); };
  // The ring holds the lead and three chunks on their way; the lead is more than a row's part, and two at most (their slots).
  int parts = 1;
  while (parts < kMaxParts && part_chunks(parts) + 1 > chunks - (parts == 1 ? 4 : 3)) parts *= 2;
  const int lead = std::min(chunks - (parts == 1 ? 4 : 3), 2 * part_chunks(parts));
  if (lead < part_chunks(parts) + 1) return false;
  auto kernel = loss_stream_kernel<T, OP, NT>;
  cfg.dynamicSmemBytes = fixed + (size_t)chunks * kChunk;
  // (the limit is one number for all host threads: always the same, or a call with a shorter list could lower it between another's setting and launch)
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBlockSharedMemory) != cudaSuccess) return true;
  cfg.blockDim = dim3(kStreamThreads, 1, 1);
  long long at_once = mtf::device_sm_count();
  if (parts > 1) {
    static mtf::KnownPerDevice known[kMaxParts + 1];
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)parts; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
    cfg.gridDim = dim3((unsigned)parts, 1, 1);
    at_once = resident_clusters(kernel, cfg, known[parts]);
    if (at_once < 1) return false;
  }
  cfg.gridDim = dim3((unsigned)(std::min(a.rows, at_once) * parts), 1, 1);
  (void)cudaLaunchKernelEx(&cfg, kernel, a, factors<NT>(a), parts, pieces_each<T>(a, parts), chunks, lead);
  return true;
}

template <typename T, int OP, int PASS, int NT>
void launch(const LossRows& b, cudaStream_t st) {
  LossRows a = b;
  a.inv_tau = a.soft != 0.f ? 1.0 / (double)a.temperature : 1.0;
  // (a gradient that is asked for later begins where the statistics ended: those rows are still in the L2 cache)
  a.reverse = PASS == mtf::LOSS_BACKWARD;
  const size_t list = OP == mtf::LOSS_DISTILL ? Slots::bytes(a.slots) : 0;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.stream = st; cfg.attrs = at; cfg.numAttrs = 1;
  const long long bytes = (long long)a.V * (a.bf16 ? 2 : 4), pieces = bytes / 16, sms = mtf::device_sm_count();
  int parts = 1, threads = 32;
  if (PASS == mtf::LOSS_BACKWARD) {
    // Independent blocks of 32 KB (777 f32 rows of 50001, both directions: 66 us, with whole rows 73, blocks of 12 KB 76; 8192 bf16 rows of 32768, half of them
    // skipped: 121, with whole rows 126).  A teacher's list is worked out by every block of its row, so there only with few rows (822 rows of
    // 128 KB with 100 slots: 37 us, in two blocks each 46).
    if (OP != mtf::LOSS_DISTILL) parts = (int)std::min<long long>(64, (bytes + 32767) / 32768);
    while (parts < 64 && a.rows * parts * 2 <= 4 * sms && bytes / parts > 2048) parts *= 2;
    while (threads < kRowWarps * 32 && threads * 8 < pieces / parts) threads *= 2;
  } else {
    // Streamed or a block per row, us in one call: 8192 x 32768 bf16 184 or 217, 4096 x 32768 f32 168 or 248, 2048 x 131072 bf16 226 or 263,
    // 1024 x 32768 bf16 30 or 33; but 512 x 32768 18 or 16, and 16384 x 16384 227 or 212: little that is read twice comes from memory twice, and
    // short rows end too often.
    if constexpr (PASS == mtf::LOSS_STEP)
      if (bytes > 32768 && a.rows * bytes > (48LL << 20) && launch_stream<T, OP, NT>(a, list, cfg, at)) return;
    // Few rows are cut up, as far as the longer way to a row's sums leaves it worth: bf16 rows in one call, uncut / as here, 16 of 8192 4.7 / 4.7 us,
    // 16 of 32768 7.4 / 6.0, 16 of 131072 19.8 / 8.2, 40 of 131072 19.9 / 11.5; their statistics alone 4.6 / 4.6 (32768), 8.4 / 5.8 and 8.4 / 7.5.
    const long long least = PASS == mtf::LOSS_STEP ? 16384 : 32768;
    if (PASS == mtf::LOSS_STEP || bytes > 131072)
      while (parts < kMaxParts && bytes / parts > least &&
             (a.rows * parts * 2 <= (PASS == mtf::LOSS_STEP ? sms : 2 * sms) || (PASS == mtf::LOSS_STEP && bytes / parts > 65536 && a.rows * parts * 2 <= 4 * sms)))
        parts *= 2;
    // pieces a thread, while there are rows enough (statistics of 4389 bf16 rows of 32768 among 8192: 62 us with 128 threads, 72 with 256; 529 f32
    // rows of 50001: 36 with 128, 30 with 256)
    const int each = PASS == mtf::LOSS_STEP ? 16 : a.bf16 ? 32 : 256;
    while (threads < kRowWarps * 32 && (threads * each < pieces / parts || a.rows * parts * threads * 2 <= (PASS == mtf::LOSS_STEP ? 1024 : 2048) * sms)) threads *= 2;
    if (parts > 1) {
      at[1].id = cudaLaunchAttributeClusterDimension;
      at[1].val.clusterDim.x = (unsigned)parts; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
      cfg.numAttrs = 2;
    }
  }
  cfg.blockDim = dim3((unsigned)(threads + (OP == mtf::LOSS_DISTILL ? 32 : 0)), 1, 1);
  cfg.dynamicSmemBytes = sizeof(Scratch) + list + (list && PASS != mtf::LOSS_FORWARD ? kSeenWords * 4 : 0);
  cfg.gridDim = dim3((unsigned)(a.rows * parts), 1, 1);
  (void)cudaLaunchKernelEx(&cfg, loss_rows_kernel<T, OP, PASS, NT>, a, factors<NT>(a), parts, pieces_each<T>(a, parts));
}

// The temperatures that are small whole powers' quotients and the usual choices; each is an instantiation of every kernel, and others (5/4, 5/2, 5) take two exponentials.
template <typename T, int PASS>
void launch_distill(const LossRows& a, cudaStream_t st) {
  if (a.soft == 0.f || a.hard == 0.f || a.temperature == 1.f) launch<T, mtf::LOSS_DISTILL, PASS, kOne>(a, st);
  else if (a.temperature == 1.5f) launch<T, mtf::LOSS_DISTILL, PASS, powers(2, 3)>(a, st);
  else if (a.temperature == 2.f) launch<T, mtf::LOSS_DISTILL, PASS, powers(1, 2)>(a, st);
  else if (a.temperature == 3.f) launch<T, mtf::LOSS_DISTILL, PASS, powers(1, 3)>(a, st);
  else if (a.temperature == 4.f) launch<T, mtf::LOSS_DISTILL, PASS, powers(1, 4)>(a, st);
  else launch<T, mtf::LOSS_DISTILL, PASS, kTwo>(a, st);
}

template <typename T>
void dispatch(mtf::LossOp op, mtf::LossPass pass, const LossRows& a, cudaStream_t st) {
  using namespace mtf;
  if (op == LOSS_DISTILL) {
    if (pass == LOSS_FORWARD) launch_distill<T, LOSS_FORWARD>(a, st);
    else if (pass == LOSS_BACKWARD) launch_distill<T, LOSS_BACKWARD>(a, st);
    else launch_distill<T, LOSS_STEP>(a, st);
  } else if (pass == LOSS_BACKWARD) {
    launch<T, LOSS_LOGP, LOSS_BACKWARD, kOne>(a, st);
  } else if (op == LOSS_LOGP) {
    launch<T, LOSS_LOGP, LOSS_FORWARD, kOne>(a, st);
  } else if (pass == LOSS_FORWARD) {
    launch<T, LOSS_POLICY, LOSS_FORWARD, kOne>(a, st);
  } else {
    launch<T, LOSS_POLICY, LOSS_STEP, kOne>(a, st);
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
  if (a.bf16) dispatch<__nv_bfloat16>(op, pass, a, (cudaStream_t)stream);
  else dispatch<float>(op, pass, a, (cudaStream_t)stream);
  return after("loss_rows_kernel");
}

mtf_status debug_loss_wait_test(long long limit_cycles, int withhold) {
  const long long limit = limit_cycles > 0 ? limit_cycles : kWaitCycles;
  cudaError_t e = cudaMemcpyToSymbol(g_wait_limit, &limit, sizeof(limit));
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_withhold, &withhold, sizeof(int));
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "cudaMemcpyToSymbol: %s", cudaGetErrorString(e));
  return MTF_OK;
}

mtf_status read_loss_status(int* code) {
  int v = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_loss_status, sizeof(int));
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "cudaMemcpyFromSymbol: %s", cudaGetErrorString(e));
  if (v) { int z = 0; cudaMemcpyToSymbol(g_loss_status, &z, sizeof(int)); }
  *code = v;
  return MTF_OK;
}
mtf_status read_loss_bad_id(int* seen) {
  int v = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_bad_id, sizeof(int));
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "cudaMemcpyFromSymbol: %s", cudaGetErrorString(e));
  if (v) { int z = 0; cudaMemcpyToSymbol(g_bad_id, &z, sizeof(int)); }
  *seen = v;
  return MTF_OK;
}

mtf_status launch_preference_pairs(const PreferencePairs& a, void* stream) {
  if (a.bf16) launch_chained(preference_pairs_kernel<__nv_bfloat16>, (unsigned)a.pairs, kPairThreads, 0, (cudaStream_t)stream, a);
  else launch_chained(preference_pairs_kernel<float>, (unsigned)a.pairs, kPairThreads, 0, (cudaStream_t)stream, a);
  return after("preference_pairs_kernel");
}

}  // namespace mtf
