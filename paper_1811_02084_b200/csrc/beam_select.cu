// Beam search's selection: of all (beam i, word v) of a sentence the `slots` best by
//     score[i] + (logits[i, v] - log sum_w exp(logits[i, w])),
// the better ones first, equal ones by the lower i, then the lower v.  A finished beam stands for itself (its end, its score) alone.
//
// A beam can only give its own `slots` best words, and which these are its logits say.  So one read of the logits (HBM is the bound) serves both
// the sum of exponentials and the choice: while a block of threads walks over its part of a row, each thread keeps its sum and its own maximum.  The
// slots-th largest of the threads' maxima is a value that at least `slots` words reach; only the threads whose maximum reaches it hold words that do, so
// their pieces alone, about `slots` in 256 of them, are looked at again (they are in L2), by all threads.  A second launch joins a sentence's parts and
// takes the best of the sorted lists.
//
// What decides between beams is held in 64 bits: sums of a thread are f32 sums of f32 exponentials relative to an entry of its own, so that
// the entries that weigh are exact or nearly so; they are joined in 64 bits.  Which thread takes which word goes by the word's index alone, not by
// how the row is aligned: rows that are equal have equal sums to the bit, and their words tie as they should.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "answer.h"
#include "launch.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kList = 1024;           // words that may be looked at again before the choice goes by counting
constexpr int kMostBlocks = 8;        // of a cluster
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 20.f;        // a thread's reference is raised where an entry lies e^20 above it

struct Args {
  const void* z;
  int vocab, beams, slots, parts, part;          // part: words of one, a multiple of 8
  int cluster;                                   // a sentence's parts are one cluster's, which also joins them; else they are left in the workspace
  long long rows;
  const float* scores;
  const int32_t* finished;
  int end_id;
  int32_t *parents, *tokens, *new_finished;
  float* new_scores;
  float* tops;                                   // [row, part]: maximum
  double* sums;                                  // ... and the sum of exponentials relative to it
  float* best_z;                                 // [row, part, slots], sorted; index -1 behind the last
  int* best_i;
};

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

// One part of a row: words [0, n) from `first` on; pieces of kN words, piece p holding words p kN ..
template <typename T>
struct Part {
  static constexpr int kN = Words<T>::kN;
  const T* first;
  const uint4* base;           // 16-byte boundary at or in front of `first`
  int off, n;                  // words from there to `first`
  int whole;                   // pieces that come in whole 16-byte loads: all but the row's last, if it is not full, and, off the boundaries, the logits' last

  __device__ __forceinline__ Part(const T* z, long long at, int count, long long total) {
    first = z + at;
    n = count;
    off = (int)(at % kN);
    base = reinterpret_cast<const uint4*>(z + (at - off));
    const long long left = (total - (at - off)) / kN - (off ? 1 : 0);
    whole = (int)min((long long)(n / kN), max(left, 0LL));
  }
  __device__ __forceinline__ int pieces() const { return (n + kN - 1) / kN; }
  __device__ __forceinline__ uint4 load(int p) const {
    if (p < whole) return off == 0 ? base[p] : Words<T>::shifted(base[p], base[p + 1], off);
    return Words<T>::some(first + p * kN, n - p * kN);
  }
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
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A thread's sum of exponentials relative to `ref`, an entry of the part (from differences, which are exact for the entries that weigh), and its largest entry.
struct Sum {
  float ref, top = -INFINITY;
  float2 s = make_float2(0.f, 0.f);
  template <typename T, int K>
  __device__ __forceinline__ void add(const uint4 (&v)[K]) {
    const float m = Words<T>::largest(v);
    top = fmaxf(top, m);
    if (m > ref + kSlack || (ref == -INFINITY && m > -INFINITY)) {
      const float f = ref == -INFINITY ? 0.f : exp2f((ref - m) * kLog2e);
      s = times(s, make_float2(f, f));               // (a sum of 0, or NaN, where there was no reference)
      ref = m;
    }
    const float r = ref == -INFINITY ? 0.f : -ref;
#pragma unroll
    for (int e = 0; e < K; ++e) {
      float x[Words<T>::kN];
      Words<T>::values(v[e], x);
#pragma unroll
      for (int j = 0; j < Words<T>::kN; j += 2) {
        const float2 d = times(plus(make_float2(x[j], x[j + 1]), make_float2(r, r)), make_float2(kLog2e, kLog2e));
        s = plus(s, make_float2(ex2(d.x), ex2(d.y)));
      }
    }
  }
};

__device__ __forceinline__ bool better(float z, int i, float y, int j) { return z > y || (z == y && i < j); }
// 32 bits in the order of the values, -0 as 0; NaN does not come here
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// What a block knows, and what joins the lists of a sentence.
struct Room {
  float list_z[kList];
  int list_i[kList];
  float sorted_z[mtf::kMaxSlots];
  int sorted_i[mtf::kMaxSlots];
  double red_s[kThreads / 32];
  float red_m[kThreads / 32], red_r[kThreads / 32];
  int chosen[kThreads], counts[256];
  int count, n_chosen, taken;
  float top;
  double sum;
};

// A list's first word.  The words of a beam go by their logits (a score far from 0 may leave nothing of those in the sum), equal ones by the lower word.
struct Offer {
  double value = -INFINITY;
  float z = 0.f;
  int beam = 0x7fffffff, word = 0, list = 0;
  __device__ __forceinline__ bool before(const Offer& o) const {
    return value > o.value || (value == o.value && (beam < o.beam || (beam == o.beam && better(z, word, o.z, o.word))));
  }
};

// One warp: the best of a sentence's lists, one after the other.  All in shared memory: per list (beam, part) its maximum and sum, its words z, index (sorted; an index
// below 0 behind the last); per beam two numbers, per list one, of this warp's own.
__device__ __forceinline__ void merge_lists(const Args& a, long long sentence, const float* tops, const double* sums, const float* z, int* index, double* base, double* maxima, int* head) {
  const int lane = threadIdx.x & 31, lists = a.beams * a.parts;
  const long long row0 = sentence * a.beams;
  for (int b = lane; b < a.beams; b += 32) {
    const float score = a.scores[row0 + b];
    const bool done = a.finished && a.finished[row0 + b];
    bool live = fabsf(score) < INFINITY;
    base[b] = score;
    maxima[b] = 0.;
    if (live && !done) {
      float top = -INFINITY;
      for (int p = 0; p < a.parts; ++p) top = fmaxf(top, tops[b * a.parts + p]);
      double s = 0.;
      for (int p = 0; p < a.parts; ++p) {
        const float m = tops[b * a.parts + p];
        const double x = sums[b * a.parts + p];
        s += m == top ? x : x * exp((double)m - (double)top);      // (a part without a finite word: 0 times its sum, 0 or NaN)
      }
      live = s > 0. && s < INFINITY && fabsf(top) < INFINITY;
      base[b] = (double)score - log(s);
      maxima[b] = top;
    }
    if (!live) base[b] = -INFINITY;
    // what a finished beam offers, and one that offers nothing
    if (!live || done)
      for (int p = 0; p < a.parts; ++p) index[(b * a.parts + p) * a.slots] = -1;
    if (live && done) {
      index[b * a.parts * a.slots] = a.end_id;
      if (a.slots > 1) index[b * a.parts * a.slots + 1] = -1;
    }
  }
  for (int l = lane; l < lists; l += 32) head[l] = 0;
  __syncwarp();
  for (int slot = 0; slot < a.slots; ++slot) {
    Offer best;
    for (int l = lane; l < lists; l += 32) {
      const int i = l * a.slots + head[l];
      if (head[l] >= a.slots || index[i] < 0) continue;
      const int b = l / a.parts;
      const bool done = a.finished && a.finished[row0 + b];
      const float y = done ? 0.f : z[i];
      const Offer o = {base[b] + ((double)y - maxima[b]), y, b, index[i], l};
      if (o.before(best)) best = o;
    }
    // the largest value of the warp; where several lanes have it, the first of them by the other rules
    double top = best.value;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmax(top, __shfl_xor_sync(0xffffffffu, top, d));
    uint32_t those = __ballot_sync(0xffffffffu, best.value == top && top > -INFINITY);
    int from = those ? __ffs(those) - 1 : 0;
    for (those &= those - 1; those; those &= those - 1) {
      const int other = __ffs(those) - 1;
      const int b0 = __shfl_sync(0xffffffffu, best.beam, from), b1 = __shfl_sync(0xffffffffu, best.beam, other);
      const int w0 = __shfl_sync(0xffffffffu, best.word, from), w1 = __shfl_sync(0xffffffffu, best.word, other);
      const float z0 = __shfl_sync(0xffffffffu, best.z, from), z1 = __shfl_sync(0xffffffffu, best.z, other);
      if (b1 < b0 || (b1 == b0 && better(z1, w1, z0, w0))) from = other;
    }
    const bool any = top > -INFINITY;
    if (lane == from) {
      if (any) ++head[best.list];
      const long long at = sentence * a.slots + slot;
      const int parent = any ? best.beam : 0, token = any ? best.word : a.end_id;
      a.parents[at] = parent;
      a.tokens[at] = token;
      a.new_scores[at] = any ? (float)top : -INFINITY;
      if (a.new_finished) a.new_finished[at] = token == a.end_id || (any && a.finished && a.finished[row0 + parent]) ? 1 : 0;
    }
    __syncwarp();
  }
}

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t in_block(uint32_t at, int rank) {
  uint32_t x;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(x) : "r"(at), "r"(rank));
  return x;
}
__device__ __forceinline__ uint32_t far(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ double far_double(uint32_t at) {
  double x;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A part's maximum, sum and sorted best words, into room.
template <typename T>
__device__ __forceinline__ void part_of_row(const Args& a, long long row, int c0, int n, Room& m) {
  constexpr int kN = Words<T>::kN, kDeep = 4, kWarps = kThreads / 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Part<T> w(reinterpret_cast<const T*>(a.z), row * a.vocab + c0, n, a.rows * a.vocab);
  const int pieces = w.pieces();
  const uint4 none = make_uint4(Words<T>::kNone, Words<T>::kNone, Words<T>::kNone, Words<T>::kNone);

  // ---- one walk: sum and maximum.  All threads begin with the same reference, the largest of the first pieces, so that their sums can be added as they are.
  Sum sum;
  uint4 v[kDeep];
  int p = tid;
  auto load = [&](int first, uint4 (&to)[kDeep]) {
    if (first + (kDeep - 1) * kThreads < w.whole && w.off == 0) {
#pragma unroll
      for (int e = 0; e < kDeep; ++e) to[e] = w.base[first + e * kThreads];
    } else {
#pragma unroll
      for (int e = 0; e < kDeep; ++e) to[e] = first + e * kThreads < pieces ? w.load(first + e * kThreads) : none;
    }
  };
  load(p, v);
  float top = Words<T>::largest(v);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) m.red_m[warp] = top;
  if (tid == 0) { m.count = 0; m.n_chosen = 0; }
  __syncthreads();
  top = m.red_m[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) top = fmaxf(top, m.red_m[i]);
  sum.ref = top;
  for (; p < pieces; p += kDeep * kThreads) {
    uint4 next[kDeep];
    if (p + kDeep * kThreads < pieces) load(p + kDeep * kThreads, next);
    sum.add<T>(v);
#pragma unroll
    for (int e = 0; e < kDeep; ++e) v[e] = next[e];
  }

  // ---- the largest, and a value that `slots` words at least reach: the least of the maxima of as many groups of threads (the next power of two)
  float group = sum.top, ref = sum.ref;
  int groups = 1;
  while (groups < a.slots) groups *= 2;
  const int width = kThreads / groups;                       // threads of a group
  for (int o = 1; o < min(width, 32); o *= 2) group = fmaxf(group, __shfl_xor_sync(0xffffffffu, group, o));
  float low = group;
  top = group;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, o));
  }
  __syncthreads();
  if (lane == 0) {
    m.red_m[warp] = top;
    m.red_r[warp] = ref;
    m.chosen[warp] = __float_as_int(low);
  }
  __syncthreads();
  top = m.red_m[0];
  ref = m.red_r[0];
  float thr = INFINITY;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    top = fmaxf(top, m.red_m[i]);
    ref = fmaxf(ref, m.red_r[i]);
    thr = fminf(thr, __int_as_float(m.chosen[i]));
  }
  if (width > 32) {                                          // groups of whole warps
    thr = INFINITY;
    const int warps = width / 32;
    for (int g = 0; g < kWarps; g += warps) {
      float x = m.red_m[g];
      for (int i = 1; i < warps; ++i) x = fmaxf(x, m.red_m[g + i]);
      thr = fminf(thr, x);
    }
  }
  // ---- the threads' sums, joined in 64 bits in a fixed order
  double s = (double)sum.s.x + (double)sum.s.y;
  if (sum.ref != ref && sum.ref != -INFINITY) s *= exp((double)sum.ref - (double)ref);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) m.red_s[warp] = s;
  __syncthreads();                                           // (the maxima have been read, too)
  if (tid == 0) {
    double all = m.red_s[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) all += m.red_s[i];
    m.top = top;
    m.sum = top == ref || top == -INFINITY ? all : all * exp((double)ref - (double)top);
  }
  if (sum.top >= thr && sum.top > -INFINITY) m.chosen[atomicAdd(&m.n_chosen, 1)] = tid;
  __syncthreads();

  // ---- the words that reach it, from the pieces of the threads that have some
  const int per = (pieces + kThreads - 1) / kThreads, again = m.n_chosen * per;
  for (int i = tid; i < again; i += kThreads) {
    const int which = i / per, q = m.chosen[which] + (i - which * per) * kThreads;
    if (q >= pieces) continue;
    float x[kN];
    Words<T>::values(w.load(q), x);
#pragma unroll
    for (int j = 0; j < kN; ++j)
      if (x[j] >= thr && x[j] > -INFINITY) {
        const int at = atomicAdd(&m.count, 1);
        if (at < kList) { m.list_z[at] = x[j]; m.list_i[at] = c0 + q * kN + j; }
      }
  }
  __syncthreads();
  int found = m.count;
  if (found > kList) {
    // Too many to be sorted (a row of equal words, or masked by a finite value): the slots-th largest value by counting its bytes from the highest on,
    // then all words above it, fewer than `slots`, and of those equal to it the first.
    uint32_t prefix = 0;
    int want = a.slots;                            // of those that share the prefix
    for (int byte = 3; byte >= 0; --byte) {
      __syncthreads();
      m.counts[tid] = 0;
      __syncthreads();
      for (int q = tid; q < pieces; q += kThreads) {
        float x[kN];
        Words<T>::values(w.load(q), x);
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const uint32_t k = key_of(x[j]);
          if (x[j] > -INFINITY && (byte == 3 || (k >> (8 * byte + 8)) == prefix)) atomicAdd(&m.counts[k >> (8 * byte) & 255], 1);
        }
      }
      __syncthreads();
      int above = 0, b = 255;
      while (b > 0 && above + m.counts[b] < want) above += m.counts[b--];
      want -= above;
      prefix = prefix << 8 | (uint32_t)b;
    }
    __syncthreads();
    if (tid == 0) { m.count = 0; m.taken = 0; }
    __syncthreads();
    for (int q0 = 0; q0 < pieces; q0 += kThreads) {
      const int q = q0 + tid;
      float x[kN];
      int same = 0;
      if (q < pieces) {
        Words<T>::values(w.load(q), x);
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const uint32_t k = key_of(x[j]);
          if (x[j] > -INFINITY && k > prefix) {
            const int at = atomicAdd(&m.count, 1);
            m.list_z[at] = x[j];
            m.list_i[at] = c0 + q * kN + j;
          }
          same += x[j] > -INFINITY && k == prefix;
        }
      }
      // equal ones in the order of their index, as long as there is need of them
      if (m.taken < want) {                        // (the same for all threads: it is written between barriers)
        int upto = same;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
          const int y = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += y;
        }
        if (lane == 31) m.counts[warp] = upto;
        __syncthreads();
        int at = m.taken + upto - same, all = m.taken;
        for (int i = 0; i < kWarps; ++i) {
          if (i < warp) at += m.counts[i];
          all += m.counts[i];
        }
        if (q < pieces)
#pragma unroll
          for (int j = 0; j < kN; ++j)
            if (x[j] > -INFINITY && key_of(x[j]) == prefix) {
              if (at < want) {
                const int to = kList - 1 - at;     // from the other end
                m.list_z[to] = x[j];
                m.list_i[to] = c0 + q * kN + j;
              }
              ++at;
            }
        __syncthreads();
        if (tid == 0) m.taken = min(all, want);
        __syncthreads();
      }
    }
    __syncthreads();
    const int over = m.count, equal = m.taken;
    if (tid < equal) { m.list_z[over + tid] = m.list_z[kList - 1 - tid]; m.list_i[over + tid] = m.list_i[kList - 1 - tid]; }
    found = over + equal;
    __syncthreads();
  }

  // ---- in order
  for (int i = tid; i < found; i += kThreads) {
    const float z = m.list_z[i];
    const int at = m.list_i[i];
    int place = 0;
    for (int j = 0; j < found; ++j) place += better(m.list_z[j], m.list_i[j], z, at);
    if (place < a.slots) { m.sorted_z[place] = z; m.sorted_i[place] = at; }
  }
  for (int i = found + tid; i < a.slots; i += kThreads) m.sorted_i[i] = -1;
  __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kThreads) beam_rows_kernel(const Args a) {
  __shared__ __align__(16) Room m;
  mtf::chain_wait();
  const int tid = threadIdx.x;
  const long long row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x - row * a.parts);
  const float score = a.scores[row];
  // (a beam that is finished, or none, is not looked at behind this either)
  const bool live = fabsf(score) < INFINITY && !(a.finished && a.finished[row]);
  if (live) part_of_row<T>(a, row, part * a.part, max(0, min(a.part, a.vocab - part * a.part)), m);
  if (!a.cluster) {
    if (!live) return;
    if (tid == 0) {
      a.tops[blockIdx.x] = m.top;
      a.sums[blockIdx.x] = m.sum;
    }
    if (tid < a.slots) {
      a.best_z[(long long)blockIdx.x * a.slots + tid] = m.sorted_z[tid];
      a.best_i[(long long)blockIdx.x * a.slots + tid] = m.sorted_i[tid];
    }
    return;
  }
  // a sentence's parts are this cluster's blocks: the first takes what the others have
  cluster_barrier();
  const int lists = a.cluster, rank = blockIdx.x % lists;
  __shared__ float tops[kMostBlocks];
  __shared__ double sums[kMostBlocks], base[kMostBlocks], maxima[kMostBlocks];
  __shared__ int head[kMostBlocks];
  if (rank == 0) {
    for (int i = tid; i < lists * a.slots; i += kThreads) {
      const int l = i / a.slots, j = i - l * a.slots;
      m.list_z[i] = __uint_as_float(far(in_block(smem_at(&m.sorted_z[j]), l)));
      m.list_i[i] = (int)far(in_block(smem_at(&m.sorted_i[j]), l));
    }
    if (tid < lists) {
      tops[tid] = __uint_as_float(far(in_block(smem_at(&m.top), tid)));
      sums[tid] = far_double(in_block(smem_at(&m.sum), tid));
    }
  }
  cluster_barrier();                               // (from here on a block may leave)
  if (rank == 0 && tid < 32) merge_lists(a, blockIdx.x / lists, tops, sums, m.list_z, m.list_i, base, maxima, head);
}

// A sentence's parts from the workspace.
__global__ void __launch_bounds__(128) beam_merge_kernel(const Args a) {
  extern __shared__ __align__(16) uint8_t room[];
  mtf::chain_wait_only();
  const int tid = threadIdx.x, lists = a.beams * a.parts, n = lists * a.slots;
  double* const sums = reinterpret_cast<double*>(room);
  double* const base = sums + lists;
  double* const maxima = base + a.beams;
  float* const z = reinterpret_cast<float*>(maxima + a.beams);
  int* const index = reinterpret_cast<int*>(z + n);
  float* const tops = reinterpret_cast<float*>(index + n);
  int* const head = reinterpret_cast<int*>(tops + lists);
  // (the lists of beams that were not looked at hold anything, and are not used)
  const long long list0 = (long long)blockIdx.x * lists;
  for (int i = tid; i < n; i += 128) {
    index[i] = a.best_i[list0 * a.slots + i];
    z[i] = a.best_z[list0 * a.slots + i];
  }
  for (int i = tid; i < lists; i += 128) {
    tops[i] = a.tops[list0 + i];
    sums[i] = a.sums[list0 + i];
  }
  __syncthreads();
  if (tid < 32) merge_lists(a, blockIdx.x, tops, sums, z, index, base, maxima, head);
}

// How a row is cut, and whether a sentence's parts are a cluster that joins them itself.
struct Cut {
  int parts, cluster;
};
Cut cut_of(long long sentences, int beams, int slots, int vocab) {
  const long long rows = sentences * beams, sms = mtf::device_sm_count();
  if (beams <= kMostBlocks && rows <= sms * 2) {
    int parts = 1;
    while (beams * parts * 2 <= kMostBlocks && rows * parts * 2 <= sms * 2 && vocab / (parts * 2) >= 4096) parts *= 2;
    return {parts, beams * parts};
  }
  // parts of at least 4096 words, so many that every SM has some blocks, and so few that a sentence's lists fit shared memory
  const long long wanted = std::max(1LL, (sms * 8 + rows - 1) / rows);
  const long long most = std::max(1LL, std::min<long long>(vocab / 4096, 4096 / ((long long)beams * slots)));
  return {(int)std::min(wanted, most), 0};
}
size_t merge_room(int beams, int slots, int parts) {
  return (size_t)beams * (2 + parts) * sizeof(double) + (size_t)beams * parts * slots * 8 + (size_t)beams * parts * 8;
}
size_t up16(size_t n) { return (n + 15) / 16 * 16; }

}  // namespace

namespace mtf {

size_t beam_select_workspace(long long sentences, int beams, int slots, int vocab) {
  const Cut c = cut_of(sentences, beams, slots, vocab);
  if (c.cluster) return 0;
  const size_t lists = (size_t)sentences * beams * c.parts;
  return up16(lists * sizeof(double)) + up16(lists * sizeof(float)) + up16(lists * slots * 4) + lists * slots * 4;
}

mtf_status launch_beam_select(const BeamSelect& b, void* stream) {
  Args a = {};
  a.z = b.logits;
  a.vocab = b.vocab;
  a.beams = b.beams;
  a.slots = b.slots;
  a.rows = b.sentences * b.beams;
  const Cut c = cut_of(b.sentences, b.beams, b.slots, b.vocab);
  a.parts = c.parts;
  a.cluster = c.cluster;
  a.part = ((b.vocab + a.parts - 1) / a.parts + 7) / 8 * 8;
  a.scores = b.scores;
  a.finished = b.finished;
  a.end_id = b.end_id;
  a.parents = b.parents;
  a.tokens = b.tokens;
  a.new_finished = b.new_finished;
  a.new_scores = b.new_scores;
  const size_t lists = (size_t)a.rows * a.parts;
  uint8_t* w = reinterpret_cast<uint8_t*>(b.workspace);
  a.sums = reinterpret_cast<double*>(w);
  w += up16(lists * sizeof(double));
  a.tops = reinterpret_cast<float*>(w);
  w += up16(lists * sizeof(float));
  a.best_z = reinterpret_cast<float*>(w);
  w += up16(lists * a.slots * 4);
  a.best_i = reinterpret_cast<int*>(w);
  cudaStream_t st = (cudaStream_t)stream;
  if (a.rows * a.parts > 0x7fffffffLL) return fail(MTF_ERR_UNSUPPORTED, "beam_select: at most 2^31 parts of rows");
  if (a.cluster) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = a.cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(a.rows * a.parts), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    (void)cudaLaunchKernelEx(&cfg, b.bf16 ? beam_rows_kernel<__nv_bfloat16> : beam_rows_kernel<float>, a);
    count_launch();
  } else {
    if (b.bf16) launch_chained(beam_rows_kernel<__nv_bfloat16>, (unsigned)(a.rows * a.parts), kThreads, 0, st, a);
    else launch_chained(beam_rows_kernel<float>, (unsigned)(a.rows * a.parts), kThreads, 0, st, a);
    count_launch();
    launch_chained(beam_merge_kernel, (unsigned)b.sentences, 128, merge_room(a.beams, a.slots, a.parts), st, a);
    count_launch();
  }
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "beam_select kernels: %s", cudaGetErrorString(e));
  return MTF_OK;
}

}  // namespace mtf
