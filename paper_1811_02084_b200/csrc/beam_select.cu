// Beam search's selection: of all (beam i, word v) of a sentence the `slots` best by
//     score[i] + (logits[i, v] - log sum_w exp(logits[i, w])),
// the better ones first, equal ones by the lower i, then the lower v.  A finished beam stands for itself (its end, its score) alone.
//
// One read of the logits (HBM is the bound, close behind it the exponentials' unit) gives the sums, and of every run of 128 16-byte pieces the largest word.  A sentence's best
// words lie in runs whose largest words are among its best: the slots-th largest of the maxima of 64 groups of runs is a value that `slots` words at least
// reach, and a second launch looks only into the runs that reach it, hardly more than `slots` of 2 KB.  So the first launch is a walk and nothing else: its warps are streams of
// their own, with bulk copies into a ring each, and wait for nobody.  (64 x 8 rows of 131072 in bf16, a tenth of them finished, calls in a graph: lists of the best words kept for each part of a row,
// by blocks that stop to sort them, 47 us; by a warp of their own, 82; the walk with as many groups as slots, in 64 bits, 35.2; as it is 29.3, of which the walk is 24.  It
// would take 18.8 without its exponentials; 1 x 4 rows of 32768 take 6.4 us in one launch, 2.3 of them the walk, and the rest is the choice's chain of some ten dependent steps.)
// Runs are the finest groups: where fewer than `slots` of them are live there is no bar, and more than 1024 words then go by counting, one block a sentence.  (16 sentences of 8 beams over 4096 words, 8
// slots: 7.3 us with all beams live, 82 in a search's first step; 12 beams over 1000, 24 slots: 225 in every step.  Finer groups of the few runs would give a bar there; not written.)
//
// What decides between beams is held in 64 bits across runs.  Within one, exponentials relative to its largest word are f32 (of differences that are exact for the words that weigh), are added up in f32
// by the lanes and then across them, and the run's factor is an f32 exponential: a row's sum is off by some 2^-18 at most, and offers of different beams nearer than that may change places.  Which thread takes which word goes by the word's index alone, not by
// how the row is aligned: rows that are equal have equal sums to the bit, and their words tie as they should.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "answer.cuh"
#include "answer.h"
#include "launch.cuh"
#include "row_part.h"

namespace {

using mtf::ex2;
using mtf::kWaitCycles;
using mtf::smem_at;

// (64 x 8 rows of 131072: three blocks of four stages 1.6 us slower; runs of 256 pieces in two stages 0.8 faster, but 0.4 slower for one sentence; the choice by 256 threads
// 4.7 us slower, by 1024 1.0.)
constexpr int kThreads = 256, kWarps = kThreads / 32, kBlocks = 4;      // of the walk; blocks an SM holds
constexpr int kRun = 128;             // 16-byte pieces that a warp takes at a time
constexpr int kStages = 3;            // of a warp's ring, a run each: 50 KB a block
constexpr int kStage = (kRun + 8) * 16, kRing = kWarps * kStages * kStage, kFewRing = 2 * kRing;
constexpr int kChoosers = 512, kChooserWarps = kChoosers / 32;
constexpr int kCluster = 8;           // blocks a sentence, where there are few
constexpr int kList = 1024;           // words that may be looked at again before the choice goes by counting
constexpr int kRuns = 1024;           // runs they may lie in
constexpr int kFirst = 4;             // a sentence's runs that a thread of the choice keeps the largest words of
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 0x1p-20f;    // of values in f32, which are off by some 2^-24

struct Args {
  const void* z;
  int vocab, beams, slots;
  int runs;                                      // of a row
  uint32_t runs_mul;                             // i / runs = (i * runs_mul) >> runs_shift in 64 bits, for i below 2^31
  int runs_shift;
  long long rows;
  const float* scores;
  const int32_t* finished;
  int end_id;
  int32_t *parents, *tokens, *new_finished;
  float* new_scores;
  float2* of_run;                                // [row, run]: the largest word, and the sum of exponentials relative to it
};

// two f32 operations an instruction
__device__ __forceinline__ float2 plus(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 times(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}

// 16 bytes of words
template <typename T> struct Words;
template <> struct Words<__nv_bfloat16> {
  static constexpr int kN = 8;
  static constexpr uint32_t kNone = 0xff80ff80u;           // -infinity twice
  // those that begin `off` words into the 32 bytes lo, hi
  static __device__ __forceinline__ uint4 shifted(const uint4& lo, const uint4& hi, int off) {
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    uint32_t u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t a = w[j], b = w[j + 1];
#pragma unroll
      for (int s = 1; s < 4; ++s) {
        a = off / 2 == s ? w[j + s] : a;
        b = off / 2 == s ? w[j + s + 1 < 8 ? j + s + 1 : 7] : b;
      }
      u[j] = off & 1 ? __funnelshift_r(a, b, 16) : a;
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
  static __device__ __forceinline__ uint4 some(const __nv_bfloat16* p, int n) {
    uint32_t u[4] = {kNone, kNone, kNone, kNone};
    const uint16_t* const h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) u[j / 2] = j & 1 ? (u[j / 2] & 0xffffu) | (uint32_t)h[j] << 16 : (u[j / 2] & 0xffff0000u) | h[j];
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
  static __device__ __forceinline__ void values(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
  // words 2j and 2j + 1, and r to each, in f32
  static __device__ __forceinline__ float2 plus_two(const uint4& v, int j, float r) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float2 s;
    asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tadd.rn.f32.bf16 %0, x, %3;\n\tadd.rn.f32.bf16 %1, y, %3;\n\t}" : "=f"(s.x), "=f"(s.y) : "r"(w[j]), "f"(r));
    return s;
  }
  static __device__ __forceinline__ __nv_bfloat162 two(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
  template <int K>
  static __device__ __forceinline__ float largest(const uint4 (&v)[K]) {          // (NaN are passed over)
    __nv_bfloat162 m = __hmax2(__hmax2(two(v[0].x), two(v[0].y)), __hmax2(two(v[0].z), two(v[0].w)));
#pragma unroll
    for (int e = 1; e < K; ++e) m = __hmax2(m, __hmax2(__hmax2(two(v[e].x), two(v[e].y)), __hmax2(two(v[e].z), two(v[e].w))));
    return fmaxf(__low2float(m), __high2float(m));
  }
};
template <> struct Words<float> {
  static constexpr int kN = 4;
  static constexpr uint32_t kNone = 0xff800000u;
  static __device__ __forceinline__ uint4 shifted(const uint4& lo, const uint4& hi, int off) {
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    uint32_t u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[j] = w[j];
#pragma unroll
      for (int s = 1; s < 4; ++s) u[j] = off == s ? w[j + s] : u[j];
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
  static __device__ __forceinline__ uint4 some(const float* p, int n) {
    uint32_t u[4] = {kNone, kNone, kNone, kNone};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) u[j] = __float_as_uint(p[j]);
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
  static __device__ __forceinline__ void values(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float2 plus_two(const uint4& v, int j, float r) {
    return plus(j ? make_float2(__uint_as_float(v.z), __uint_as_float(v.w)) : make_float2(__uint_as_float(v.x), __uint_as_float(v.y)), make_float2(r, r));
  }
  template <int K>
  static __device__ __forceinline__ float largest(const uint4 (&v)[K]) {
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < K; ++e) {
      float x[4];
      values(v[e], x);
      m = fmaxf(m, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
    }
    return m;
  }
};

template <typename T>
__device__ __noinline__ uint4 load_some(const T* p, int n) { return Words<T>::some(p, n); }

// One part of a row: words [0, n) from `first` on; pieces of kN words, piece p holding words p kN ..  kAligned: rows begin on 16 bytes.  (What only row ends need is kept out of
// line here and below: with it in the loops the warps, each at another place, waited for instructions more than for anything else.)
template <typename T, bool kAligned>
struct Part {
  static constexpr int kN = Words<T>::kN;
  const T* first;
  const uint4* base;           // 16-byte boundary at or in front of `first`
  int off, n;                  // words from there to `first`
  int whole;                   // pieces that come in whole 16-byte loads: all but the row's last, if it is not full, and, where rows may begin anywhere, the logits' last

  __device__ __forceinline__ Part(const T* z, long long at, int count, long long total) {
    first = z + at;
    n = count;
    off = kAligned ? 0 : (int)(at % kN);
    base = reinterpret_cast<const uint4*>(z + (at - off));
    whole = mtf::whole_pieces(at, n, total, kN, kAligned);
  }
  __device__ __forceinline__ int pieces() const { return (n + kN - 1) / kN; }
  // from the 16 bytes that piece p begins in, and those behind
  __device__ __forceinline__ uint4 at(const uint4* p) const { return kAligned ? p[0] : Words<T>::shifted(p[0], p[1], off); }
  __device__ __forceinline__ uint4 load(int p) const { return p < whole ? at(base + p) : load_some(first + p * kN, n - p * kN); }
};

__device__ int g_beam_status = 0;                    // a wait was given up
__constant__ long long g_wait_limit = kWaitCycles;
__constant__ int g_withhold = 0;                     // testing: each warp's first wait asks for a copy that nobody has sent

// e^(from - to), 1 for equal ones (in f32: a run's share of a row's sum is off by 2^-22 at most, and the runs' by less together)
__device__ __forceinline__ double rescale(float from, float to) { return from == to ? 1. : (double)expf(from - to); }
__device__ __noinline__ double log_of(double s) { return log(s); }

// the sum of exponentials of some words relative to ref (from differences, which are exact for the words that weigh)
template <typename T, int K>
__device__ __forceinline__ float2 exponentials(const uint4 (&v)[K], float ref) {
  float2 s = make_float2(0.f, 0.f);
  const float r = ref == -INFINITY ? 0.f : -ref;
#pragma unroll
  for (int e = 0; e < K; ++e) {
#pragma unroll
    for (int j = 0; j < Words<T>::kN / 2; ++j) {
      const float2 d = times(Words<T>::plus_two(v[e], j, r), make_float2(kLog2e, kLog2e));
      s = plus(s, make_float2(ex2(d.x), ex2(d.y)));
    }
  }
  return s;
}

__device__ __forceinline__ bool better(float z, int i, float y, int j) { return z > y || (z == y && i < j); }
// 64 bits in the order of the values
__device__ __forceinline__ unsigned long long order_of(double v) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(v);
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ float warp_max(float m) {                  // (NaN are passed over)
  float top;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(top) : "f"(m));
  return top;
}

// A beam's row, whole
template <typename T, bool kAligned>
__device__ __forceinline__ Part<T, kAligned> row_at(const Args& a, long long row) {
  return Part<T, kAligned>(reinterpret_cast<const T*>(a.z), row * a.vocab, a.vocab, a.rows * a.vocab);
}

__device__ __forceinline__ void ready(uint64_t (&bars)[kStages]) {
  if ((threadIdx.x & 31) == 0) {
    for (int i = 0; i < kStages; ++i) mtf::landing_init(&bars[i]);
    mtf::landing_ready();
  }
  __syncwarp();
}

// One of `all` warps' walk over the runs of rows [begin, rows), one behind another, every warp the next one: all of them have as many, wherever beams lie that are not to be read.
template <typename T, bool kAligned>
__device__ __forceinline__ void walk(const Args& a, const uint8_t* ring, uint64_t (&bars)[kStages], int first, int all, int begin, int rows) {
  constexpr int kDeep = kRun / 32;
  const int lane = threadIdx.x & 31, some_rows = all / a.runs, some_runs = all - some_rows * a.runs;
  struct Place {
    int row, run;
  };
  auto onward = [&](Place& p) {
    p.row += some_rows;
    p.run += some_runs;
    if (p.run >= a.runs) {
      p.run -= a.runs;
      ++p.row;
    }
  };
  // whether a row is to be read (a beam that is finished, or none, is not): asked for a step before it is needed
  struct Asked {
    float score;
    int done;
  };
  auto ask = [&](const Place& p) {
    const bool in = p.row < rows;
    Asked q;
    q.score = in ? a.scores[p.row] : INFINITY;
    q.done = in && a.finished ? a.finished[p.row] : 0;
    return q;
  };
  Place now = {begin + first / a.runs, first % a.runs}, ahead = now;
  uint32_t read = 0, flying = 0;                     // of the stages: the run is to be read, and is being copied
  auto fetch = [&](int stage, const Place& p, const Asked& q) {
    const bool live = fabsf(q.score) < INFINITY && !q.done;
    read = (read & ~(1u << stage)) | (live ? 1u : 0u) << stage;
    flying &= ~(1u << stage);
    if (!live) return;
    const Part<T, kAligned> w = row_at<T, kAligned>(a, p.row);
    if ((p.run + 1) * kRun > w.whole) return;        // (a row's last words: by loads)
    flying |= 1u << stage;
    if (lane == 0) {
      const uint32_t bar = smem_at(&bars[stage]), bytes = (kRun + (w.off ? 1 : 0)) * 16;
      mtf::expect(bar, bytes);
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_at(ring) + stage * kStage), "l"(w.base + (long long)p.run * kRun),
                   "r"(bytes), "r"(bar)
                   : "memory");
    }
  };
  {
    Place p = now;
    Asked q[kStages];
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
      q[i] = ask(p);
      onward(p);
    }
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
      fetch(i, ahead, q[i]);
      onward(ahead);
    }
  }
  Asked next = ask(ahead);
  uint32_t phases = 0;                               // of the stages' barriers
  for (int stage = 0; now.row < rows; stage = stage + 1 == kStages ? 0 : stage + 1) {
    if (read >> stage & 1) {
      const Part<T, kAligned> w = row_at<T, kAligned>(a, now.row);
      uint4 v[kDeep];
      if (flying >> stage & 1) {
        const uint32_t bar = smem_at(&bars[stage]), phase = phases >> stage & 1;
        if (!mtf::landed(bar, phase, g_wait_limit) || (g_withhold && !mtf::landed(bar, phase ^ 1, g_wait_limit))) {
          if (lane == 0) atomicCAS(&g_beam_status, 0, 0xB11);
          // given up: what is under way gets a little more time
          for (int i = 0; i < kStages; ++i)
            if (flying >> i & 1) mtf::landed_late(smem_at(&bars[i]), phases >> i & 1, mtf::kLandCycles);
          return;
        }
        phases ^= 1u << stage;
        const uint4* const at = reinterpret_cast<const uint4*>(ring + stage * kStage) + lane;
#pragma unroll
        for (int e = 0; e < kDeep; ++e) v[e] = w.at(at + e * 32);
      } else {
#pragma unroll 1
        for (int e = 0; e < kDeep; ++e) {
          const int q = now.run * kRun + e * 32 + lane;
          const uint4 u = q < w.pieces() ? w.load(q) : make_uint4(Words<T>::kNone, Words<T>::kNone, Words<T>::kNone, Words<T>::kNone);
          if (e == 0) v[0] = u;
          else if (e == 1) v[1] = u;
          else if (e == 2) v[2] = u;
          else v[3] = u;
        }
      }
      const float top = warp_max(Words<T>::largest(v));
      __syncwarp();                                  // (every lane has its words)
      fetch(stage, ahead, next);
      onward(ahead);
      next = ask(ahead);
      const float2 s2 = exponentials<T>(v, top);
      float s = s2.x + s2.y;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == 0) a.of_run[(long long)now.row * a.runs + now.run] = make_float2(top, s);
    } else {
      fetch(stage, ahead, next);
      onward(ahead);
      next = ask(ahead);
    }
    onward(now);
  }
}

template <typename T, bool kAligned>
__global__ void __launch_bounds__(kThreads, kBlocks) beam_rows_kernel(const Args a) {
  __shared__ uint64_t bars[kWarps][kStages];
  extern __shared__ __align__(128) uint8_t dyn[];
  const int warp = threadIdx.x >> 5;
  ready(bars[warp]);
  mtf::chain_wait();
  walk<T, kAligned>(a, dyn + warp * kStages * kStage, bars[warp], blockIdx.x * kWarps + warp, gridDim.x * kWarps, 0, (int)a.rows);
}

// What a sentence's choice is made from.
struct Room {
  unsigned long long key[kList];       // words that may be among the best: their values in order, beams, logits and numbers (and counters, before)
  float z[kList];
  int word[kList], beam[kList];
  int runs[kRuns];
  unsigned long long group[kChooserWarps][32];
  float near_group[kChooserWarps][32], near_bar;
  double base[mtf::kMaxBeams];         // a word's value is base + (logit - ref)
  float ref[mtf::kMaxBeams], low[mtf::kMaxBeams];
  float off[mtf::kMaxBeams], slack[mtf::kMaxBeams];    // in f32: a word's value is logit + off, give or take slack / 2
  signed char state[mtf::kMaxBeams];   // 0: offers nothing, 1: its words, 2: its end
  int count, n_runs, far, below[kChooserWarps];       // far: off is none in f32
};

__device__ __forceinline__ unsigned long long value_key(const Room& m, int b, float z) { return order_of(m.base[b] + ((double)z - (double)m.ref[b]) + 0.); }
// a logit that no word of value v or more lies below: a little under v - base + ref, which is rounded
__device__ __forceinline__ float lowest(double v, double base, float ref) {
  const double at = v - base + (double)ref;
  return v > -INFINITY ? (float)(at - (fabs(at) * 1e-6 + (fabs(v) + fabs(base)) * 1e-15)) : -INFINITY;
}
__device__ __forceinline__ double value_of(unsigned long long key) { return __longlong_as_double((long long)(key >> 63 ? key & 0x7fffffffffffffffull : ~key)); }

__device__ __forceinline__ int beam_of(const Args& a, int i) { return (int)((unsigned long long)(uint32_t)i * a.runs_mul >> a.runs_shift); }

// The runs (of all beams of the sentence, one behind another) that `noted` has, into the room's list; `first`: the largest words of the thread's first.  Behind it, a barrier.
template <typename N>
__device__ __forceinline__ void note_runs(const Args& a, long long row0, Room& m, const float (&first)[kFirst], N noted) {
  const int tid = threadIdx.x;
  auto note = [&](int i, float top) {
    const int b = beam_of(a, i);
    if (m.state[b] != 1 || !(top > -INFINITY) || !noted(b, top)) return;
    const int at = atomicAdd(&m.n_runs, 1);
    if (at < kRuns) m.runs[at] = i;
  };
#pragma unroll
  for (int e = 0; e < kFirst; ++e)
    if (tid + e * kChoosers < a.beams * a.runs) note(tid + e * kChoosers, first[e]);
  for (int i = tid + kFirst * kChoosers; i < a.beams * a.runs; i += kChoosers) note(i, a.of_run[row0 * a.runs + i].x);
  __syncthreads();
}
// The words of these runs that are low(b) at least, and whose values `wanted` has, into the list of words: a warp a run.  Behind it, a barrier.
template <typename T, bool kAligned, typename L, typename W>
__device__ __forceinline__ void list_words(const Args& a, long long row0, Room& m, L low_of, W wanted) {
  constexpr int kN = Words<T>::kN, kDeep = kRun / 32;
  const int lane = threadIdx.x & 31, n = m.n_runs;
  for (int i = threadIdx.x >> 5; i < n; i += kChooserWarps) {
    const int at_run = m.runs[i], b = beam_of(a, at_run), run = at_run - b * a.runs;
    const Part<T, kAligned> w = row_at<T, kAligned>(a, row0 + b);
    const float low = low_of(b);
    uint4 v[kDeep];
#pragma unroll
    for (int e = 0; e < kDeep; ++e) {
      const int q = run * kRun + e * 32 + lane;
      v[e] = q < w.pieces() ? w.load(q) : make_uint4(Words<T>::kNone, Words<T>::kNone, Words<T>::kNone, Words<T>::kNone);
    }
    uint32_t have = 0;
#pragma unroll
    for (int e = 0; e < kDeep; ++e) {
      const uint4 u[1] = {v[e]};
      have |= (Words<T>::largest(u) >= low ? 1u : 0u) << e;
    }
    for (; have; have &= have - 1) {
      const int e = __ffs(have) - 1;
      const uint4 u = e == 0 ? v[0] : e == 1 ? v[1] : e == 2 ? v[2] : v[3];
      float x[kN];
      Words<T>::values(u, x);
      uint32_t those = 0;
#pragma unroll
      for (int j = 0; j < kN; ++j) those |= (x[j] >= low && x[j] > -INFINITY ? 1u : 0u) << j;
      for (; those; those &= those - 1) {
        const int j = __ffs(those) - 1;
        float z = x[0];
#pragma unroll
        for (int k = 1; k < kN; ++k) z = j == k ? x[k] : z;
        const unsigned long long k = value_key(m, b, z);
        if (!wanted(k)) continue;
        const int at = atomicAdd(&m.count, 1);
        if (at < kList) {
          m.key[at] = k;
          m.z[at] = z;
          m.word[at] = (run * kRun + e * 32 + lane) * kN + j;
          m.beam[at] = b;
        }
      }
    }
  }
  __syncthreads();
}
// The ends of finished beams, into the list (which has room for them: they come first).
template <typename W>
__device__ __forceinline__ void list_ends(const Args& a, Room& m, W wanted) {
  const int b = threadIdx.x;
  if (b >= a.beams || m.state[b] != 2) return;
  const unsigned long long k = order_of(m.base[b] + 0.);
  if (!wanted(k)) return;
  const int at = atomicAdd(&m.count, 1);
  m.key[at] = k;
  m.z[at] = 0.f;
  m.word[at] = a.end_id;
  m.beam[at] = b;
}

// The words whose value is above thr, and such ends.  All threads.  Returns how many there are: over kList where that is more than the list holds, or where they lie in too many runs.
template <typename T, bool kAligned>
__device__ __noinline__ int gather_above(const Args& a, long long row0, Room& m, unsigned long long thr, const float (&first)[kFirst]) {
  const int tid = threadIdx.x;
  auto above = [&](unsigned long long k) { return k > thr; };
  __syncthreads();
  if (tid == 0) m.count = m.n_runs = 0;
  if (tid < a.beams) m.low[tid] = thr ? lowest(value_of(thr), m.base[tid], m.ref[tid]) : -INFINITY;
  __syncthreads();
  list_ends(a, m, above);
  note_runs(a, row0, m, first, [&](int b, float top) { return above(value_key(m, b, top)); });
  if (m.n_runs > kRuns) return kList + 1;
  list_words<T, kAligned>(a, row0, m, [&](int b) { return m.low[b]; }, above);
  return m.count;
}

// Where too many words reach the bar to be sorted (rows of equal words, or masked by a finite value).  In 64 bits: thr = the least of the largest words of as many groups of runs as
// there are slots (the next power of two), which `slots` words at least reach; those above it, and the first of those equal to it.  Where those above are
// too many, too, thr becomes the slots-th largest value, by counting its bytes from the highest on.  Returns how many the list holds.  All threads.
template <typename T, bool kAligned>
__device__ __noinline__ int narrowed(const Args& a, long long row0, Room& m, const float (&first)[kFirst]) {
  constexpr int kN = Words<T>::kN;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  unsigned long long best = 0;
  auto better_of = [&](int i, float top) {
    const int b = beam_of(a, i);
    if (m.state[b] == 1 && top > -INFINITY) best = max(best, value_key(m, b, top));
  };
#pragma unroll
  for (int e = 0; e < kFirst; ++e)
    if (tid + e * kChoosers < a.beams * a.runs) better_of(tid + e * kChoosers, first[e]);
  for (int i = tid + kFirst * kChoosers; i < a.beams * a.runs; i += kChoosers) better_of(i, a.of_run[row0 * a.runs + i].x);
  if (tid < a.beams && m.state[tid] == 2) best = max(best, order_of(m.base[tid] + 0.));
  int groups = 1;
  while (groups < min(a.slots, 32)) groups *= 2;
  for (int o = groups; o < 32; o *= 2) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
  m.group[warp][lane] = best;
  __syncthreads();
  unsigned long long even = m.group[0][lane], odd = m.group[1][lane];
#pragma unroll
  for (int i = 2; i < kChooserWarps; i += 2) {
    even = max(even, m.group[i][lane]);
    odd = max(odd, m.group[i + 1][lane]);
  }
  unsigned long long thr = a.slots > 32 ? min(even, odd) : max(even, odd);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) thr = min(thr, __shfl_xor_sync(0xffffffffu, thr, o));
  int above = gather_above<T, kAligned>(a, row0, m, thr, first);
  if (above > kList) {
    int* const counts = reinterpret_cast<int*>(m.key);
    unsigned long long prefix = 0;
    int want = a.slots;                            // of those that share the prefix
    for (int byte = 7; byte >= 0; --byte) {
      __syncthreads();
      if (tid < 256) counts[tid] = 0;
      __syncthreads();
      auto note = [&](unsigned long long k) {
        if (byte == 7 || k >> (8 * byte + 8) == prefix) atomicAdd(&counts[k >> (8 * byte) & 255], 1);
      };
      for (int b = 0; b < a.beams; ++b) {
        if (m.state[b] == 2 && tid == 0) note(order_of(m.base[b] + 0.));
        if (m.state[b] != 1) continue;
        const Part<T, kAligned> w = row_at<T, kAligned>(a, row0 + b);
        for (int q = tid; q < w.pieces(); q += kChoosers) {
          float x[kN];
          Words<T>::values(w.load(q), x);
#pragma unroll 1
          for (int j = 0; j < kN; ++j)
            if (x[j] > -INFINITY) note(value_key(m, b, x[j]));
        }
      }
      __syncthreads();
      int over = 0, d = 255;
      while (d > 0 && over + counts[d] < want) over += counts[d--];
      want -= over;
      prefix = prefix << 8 | (unsigned)d;
    }
    thr = prefix;
    above = gather_above<T, kAligned>(a, row0, m, thr, first);              // fewer than `slots`, in runs of which there are no more
  }
  // equal ones: by the lower beam, of a beam's the larger logits (the sums may have lost what tells them apart), of these the lower words; as long as there is need of them
  int at = above;
  for (int b = 0; b < a.beams && at < a.slots; ++b) {
    if (m.state[b] == 2 && order_of(m.base[b] + 0.) == thr) {
      __syncthreads();
      if (tid == 0) { m.key[at] = thr; m.z[at] = 0.f; m.word[at] = a.end_id; m.beam[at] = b; }
      ++at;
    }
    if (m.state[b] != 1) continue;
    const Part<T, kAligned> w = row_at<T, kAligned>(a, row0 + b);
    for (float below = INFINITY; at < a.slots;) {
      // the largest logit under `below` whose value is thr
      float z = -INFINITY;
      for (int q = tid; q < w.pieces(); q += kChoosers) {
        float x[kN];
        Words<T>::values(w.load(q), x);
#pragma unroll
        for (int j = 0; j < kN; ++j)
          if (x[j] < below && x[j] > z && value_key(m, b, x[j]) == thr) z = x[j];
      }
      z = warp_max(z);
      __syncthreads();
      if (lane == 0) m.low[warp] = z;
      __syncthreads();
      for (int i = 0; i < kChooserWarps; ++i) z = fmaxf(z, m.low[i]);
      if (z == -INFINITY) break;
      below = z;
      for (int q0 = 0; q0 < w.pieces() && at < a.slots; q0 += kChoosers) {
        const int q = q0 + tid;
        float x[kN];
        int same = 0;
        if (q < w.pieces()) {
          Words<T>::values(w.load(q), x);
#pragma unroll
          for (int j = 0; j < kN; ++j) same += x[j] == z;
        }
        int upto = same;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const int y = __shfl_up_sync(0xffffffffu, upto, d);
          if (lane >= d) upto += y;
        }
        __syncthreads();
        if (lane == 31) m.below[warp] = upto;
        __syncthreads();
        int to = at + upto - same, all = 0;
        for (int i = 0; i < kChooserWarps; ++i) {
          if (i < warp) to += m.below[i];
          all += m.below[i];
        }
        if (q < w.pieces())
#pragma unroll
          for (int j = 0; j < kN; ++j)
            if (x[j] == z) {
              if (to < a.slots) { m.key[to] = thr; m.z[to] = z; m.word[to] = q * kN + j; m.beam[to] = b; }
              ++to;
            }
        at = min(a.slots, at + all);
      }
    }
  }
  __syncthreads();
  return max(above, at);
}

// A sentence's choice.  All threads of a block; the room's counters are 0.
template <typename T, bool kAligned>
__device__ __forceinline__ void choose(const Args& a, Room& m, long long sentence) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row0 = sentence * a.beams;
  float first[kFirst];
#pragma unroll
  for (int e = 0; e < kFirst; ++e) first[e] = tid + e * kChoosers < a.beams * a.runs ? a.of_run[row0 * a.runs + tid + e * kChoosers].x : -INFINITY;
  // ---- a warp a beam: its sum, joined in 64 bits in a fixed order
  for (int b = warp; b < a.beams; b += kChooserWarps) {
    const long long row = row0 + b;
    const float2* const runs = a.of_run + row * a.runs;
    constexpr int kMine = 4;                         // that a lane keeps
    float2 r[kMine];                                 // (of a beam that was not looked at anything)
#pragma unroll
    for (int e = 0; e < kMine; ++e) r[e] = lane + e * 32 < a.runs ? runs[lane + e * 32] : make_float2(-INFINITY, 0.f);
    const float score = a.scores[row];
    const int done = a.finished ? a.finished[row] : 0;
    int state = fabsf(score) < INFINITY ? done ? 2 : 1 : 0;
    float top = 0.f;
    double at = score;
    if (state == 1) {
      top = -INFINITY;
#pragma unroll
      for (int e = 0; e < kMine; ++e) top = fmaxf(top, r[e].x);
      for (int i = lane + kMine * 32; i < a.runs; i += 32) top = fmaxf(top, runs[i].x);
      top = warp_max(top);
      // (a run without a finite word: 0 times its sum, 0 or NaN)
      double s = 0.;
#pragma unroll
      for (int e = 0; e < kMine; ++e)
        if (lane + e * 32 < a.runs) s += r[e].y * rescale(r[e].x, top);
      for (int i = lane + kMine * 32; i < a.runs; i += 32) s += runs[i].y * rescale(runs[i].x, top);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (!(s > 0. && s < INFINITY && fabsf(top) < INFINITY)) state = 0;
      at -= log_of(s);
    }
    if (lane == 0) {
      m.state[b] = (signed char)state;
      m.base[b] = at;
      m.ref[b] = top;
      const double off = at - top;
      const float slack = (float)(fabs(off) * kSlack + (fabs(at) + fabsf(top)) * 1e-14);
      const bool near = fabs(off) < 1e38 && slack < 1e38f;
      m.off[b] = near ? (float)off : 0.f;
      m.slack[b] = near ? slack : 0.f;
      if (state && !near) m.far = 1;
    }
  }
  __syncthreads();
  // ---- the largest words of 64 groups of runs, in f32 and a little too low: the slots-th largest of them is a bar that `slots` words at least reach, and hardly more runs than
  // those have to be looked into.  A group is the lanes that are alike modulo their number, of the even warps or of the odd ones.
  float best = -INFINITY;
  auto better_of = [&](int i, float top) {
    const int b = beam_of(a, i);
    const float v = top + m.off[b];
    if (m.state[b] == 1 && top > -INFINITY) best = fmaxf(best, v - (m.slack[b] + fabsf(v) * kSlack));
  };
#pragma unroll
  for (int e = 0; e < kFirst; ++e)
    if (tid + e * kChoosers < a.beams * a.runs) better_of(tid + e * kChoosers, first[e]);
  for (int i = tid + kFirst * kChoosers; i < a.beams * a.runs; i += kChoosers) better_of(i, a.of_run[row0 * a.runs + i].x);
  if (tid < a.beams && m.state[tid] == 2) best = fmaxf(best, m.off[tid] - m.slack[tid]);
  m.near_group[warp][lane] = best;
  __syncthreads();
  float even = m.near_group[0][lane], odd = m.near_group[1][lane];
#pragma unroll
  for (int i = 2; i < kChooserWarps; i += 2) {
    even = fmaxf(even, m.near_group[i][lane]);
    odd = fmaxf(odd, m.near_group[i + 1][lane]);
  }
  constexpr int kPlaces = 64 / kChooserWarps;      // groups whose place among all a warp finds
#pragma unroll
  for (int e = 0; e < kPlaces; ++e) {
    const int c = warp * kPlaces + e;
    const float v = __shfl_sync(0xffffffffu, c < 32 ? even : odd, c & 31);
    const int place = __popc(__ballot_sync(0xffffffffu, even > v || (even == v && lane < c))) + __popc(__ballot_sync(0xffffffffu, odd > v || (odd == v && lane + 32 < c)));
    if (lane == 0 && place == a.slots - 1) m.near_bar = m.far ? -INFINITY : v;
  }
  __syncthreads();
  // ---- the words that may reach it (all that do, and some a little below), and their places among each other: a warp a word
  const float bar = m.near_bar;
  auto low_of = [&](int b) { return bar - m.off[b] - (m.slack[b] + (fabsf(bar) + fabsf(m.off[b])) * kSlack); };
  auto any = [](unsigned long long) { return true; };
  list_ends(a, m, any);
  note_runs(a, row0, m, first, [&](int b, float top) { return top >= low_of(b); });
  if (m.n_runs <= kRuns) list_words<T, kAligned>(a, row0, m, low_of, any);
  int n = m.n_runs <= kRuns ? m.count : kList + 1;
  if (n > kList) n = narrowed<T, kAligned>(a, row0, m, first);
  for (int i = warp; i < n; i += kChooserWarps) {
    const unsigned long long k = m.key[i];
    const int b = m.beam[i], word = m.word[i];
    const float z = m.z[i];
    int place = 0;
    for (int j = lane; j < n; j += 32)
      place += m.key[j] > k || (m.key[j] == k && (m.beam[j] < b || (m.beam[j] == b && better(m.z[j], m.word[j], z, word))));
    place = __reduce_add_sync(0xffffffffu, place);
    if (lane == 0 && place < a.slots) {
      const long long at = sentence * a.slots + place;
      a.parents[at] = b;
      a.tokens[at] = word;
      a.new_scores[at] = (float)value_of(k);
      if (a.new_finished) a.new_finished[at] = word == a.end_id || m.state[b] == 2 ? 1 : 0;
    }
  }
  // slots without an offer
  for (int i = n + tid; i < a.slots; i += kChoosers) {
    const long long at = sentence * a.slots + i;
    a.parents[at] = 0;
    a.tokens[at] = a.end_id;
    a.new_scores[at] = -INFINITY;
    if (a.new_finished) a.new_finished[at] = 1;
  }
}

// A block a sentence.
template <typename T, bool kAligned>
__global__ void __launch_bounds__(kChoosers, 1) beam_choose_kernel(const Args a) {
  __shared__ Room m;
  if (threadIdx.x == 0) m.count = m.n_runs = m.far = 0;
  __syncthreads();
  mtf::chain_wait_only();
  choose<T, kAligned>(a, m, blockIdx.x);
}

// Few and short rows: a cluster of blocks a sentence, which walk over its rows, and one of which chooses.  (launch_beam_select has the rule.)
template <typename T, bool kAligned>
__global__ void __launch_bounds__(kChoosers, 1) beam_few_kernel(const Args a) {
  __shared__ uint64_t bars[kChooserWarps][kStages];
  __shared__ Room m;
  extern __shared__ __align__(128) uint8_t dyn[];
  const int warp = threadIdx.x >> 5, sentence = blockIdx.x / kCluster, rank = blockIdx.x - sentence * kCluster;
  if (threadIdx.x == 0) m.count = m.n_runs = m.far = 0;
  ready(bars[warp]);
  mtf::chain_wait();
  walk<T, kAligned>(a, dyn + warp * kStages * kStage, bars[warp], rank * kChooserWarps + warp, kCluster * kChooserWarps, sentence * a.beams, (sentence + 1) * a.beams);
  __syncwarp();
  mtf::cluster_barrier();                            // (all runs' sums are written)
  if (rank == 0) choose<T, kAligned>(a, m, sentence);
}

int runs_of(int vocab, bool bf16) {
  const int words = kRun * (bf16 ? 8 : 4);
  return (vocab + words - 1) / words;
}

}  // namespace

namespace mtf {

size_t beam_select_workspace(long long sentences, int beams, int vocab, int bf16) { return (size_t)sentences * beams * runs_of(vocab, bf16) * sizeof(float2); }

mtf_status launch_beam_select(const BeamSelect& b, void* stream) {
  Args a = {};
  a.z = b.logits;
  a.vocab = b.vocab;
  a.beams = b.beams;
  a.slots = b.slots;
  a.rows = b.sentences * b.beams;
  a.runs = runs_of(b.vocab, b.bf16);
  // with 2^n >= runs > 2^(n - 1) the factor ceil(2^(31 + n) / runs) is below 2^32 and off by less than 2^n in 2^(31 + n): exact for i < 2^31
  int log2_runs = 0;
  while ((1LL << log2_runs) < a.runs) ++log2_runs;
  a.runs_mul = (uint32_t)(((1ULL << (31 + log2_runs)) + a.runs - 1) / a.runs);
  a.runs_shift = 31 + log2_runs;
  a.scores = b.scores;
  a.finished = b.finished;
  a.end_id = b.end_id;
  a.parents = b.parents;
  a.tokens = b.tokens;
  a.new_finished = b.new_finished;
  a.new_scores = b.new_scores;
  a.of_run = reinterpret_cast<float2*>(b.workspace);
  // (rows, with a step of the grid beyond the last, and a sentence's words are counted in 32 bits: the entry's checks keep them below 2^31)
  cudaStream_t st = (cudaStream_t)stream;
  const bool aligned = (long long)b.vocab * (b.bf16 ? 2 : 4) % 16 == 0;
  static KnownPerDevice limits[2][4];
  // One launch instead of two where a cluster's warps have at most a run each and half of the SMs hold the clusters: it saves the host 2.5 us a call, and costs the GPU what a cluster
  // is slower than the whole of it.  (Calls in a row / in a graph, two launches -> one: 1 x 4 rows of 32768 in bf16 9.5 / 6.5 -> 7.0 / 6.8 us, 8 x 4 9.5 / 6.8 -> 7.2 / 7.0, 16 x 4
  // 9.6 / 7.0 -> 9.6 / 9.6; two runs a warp, 1 x 8 rows, 9.5 / 6.9 -> 8.0 / 7.9; eight, 1 x 8 of 131072, 9.6 / 7.3 -> 13.8 / 13.8.)
  const bool few = b.sentences * kCluster * 2 <= device_sm_count() && a.beams * a.runs <= kCluster * kChooserWarps;
  const auto walking = few ? (b.bf16 ? (aligned ? beam_few_kernel<__nv_bfloat16, true> : beam_few_kernel<__nv_bfloat16, false>) : (aligned ? beam_few_kernel<float, true> : beam_few_kernel<float, false>))
                           : (b.bf16 ? (aligned ? beam_rows_kernel<__nv_bfloat16, true> : beam_rows_kernel<__nv_bfloat16, false>) : (aligned ? beam_rows_kernel<float, true> : beam_rows_kernel<float, false>));
  const cudaError_t set = shared_memory_limit(limits[few][(b.bf16 ? 2 : 0) + (aligned ? 1 : 0)], walking, few ? kFewRing : kRing);
  if (set != cudaSuccess) return fail(MTF_ERR_CUDA, "beam_select kernels: %s", cudaGetErrorString(set));
  count_launch();
  if (few) {
    launch_clusters(walking, dim3((unsigned)(b.sentences * kCluster)), kChoosers, kFewRing, kCluster, st, a);
  } else {
    const auto choosing = b.bf16 ? (aligned ? beam_choose_kernel<__nv_bfloat16, true> : beam_choose_kernel<__nv_bfloat16, false>)
                                 : (aligned ? beam_choose_kernel<float, true> : beam_choose_kernel<float, false>);
    const long long blocks = (a.rows * a.runs + kWarps - 1) / kWarps;
    launch_chained(walking, (unsigned)std::min<long long>(blocks, (long long)device_sm_count() * kBlocks), kThreads, kRing, st, a);
    count_launch();
    launch_chained(choosing, (unsigned)b.sentences, kChoosers, 0, st, a);
  }
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "beam_select kernels: %s", cudaGetErrorString(e));
  return MTF_OK;
}

mtf_status debug_beam_wait_test(long long limit_cycles, int withhold) {
  const long long limit = limit_cycles > 0 ? limit_cycles : kWaitCycles;
  cudaError_t e = cudaMemcpyToSymbol(g_wait_limit, &limit, sizeof(limit));
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_withhold, &withhold, sizeof(int));
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "cudaMemcpyToSymbol: %s", cudaGetErrorString(e));
  return MTF_OK;
}
mtf_status read_beam_status(int* code) {
  int v = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_beam_status, sizeof(int));
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "cudaMemcpyFromSymbol: %s", cudaGetErrorString(e));
  if (v) { int z = 0; cudaMemcpyToSymbol(g_beam_status, &z, sizeof(int)); }
  *code = v;
  return MTF_OK;
}

}  // namespace mtf
