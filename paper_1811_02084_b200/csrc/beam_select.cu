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
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 20.f;        // a thread's reference is raised where an entry lies e^20 above it

struct Args {
  const void* z;
  int vocab, beams, slots, parts, part;          // part: words of one, a multiple of 8
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

template <typename T> struct Words;
template <> struct Words<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  // 8 words from the 32 bytes lo, hi, beginning at byte 2 `off`
  static __device__ __forceinline__ void spread(const uint4& lo, const uint4& hi, int off, float (&x)[8]) {
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    uint32_t u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t a = w[j], b = w[j + 1];           // words off / 2 + j and the next
#pragma unroll
      for (int s = 1; s < 4; ++s) {
        a = off / 2 == s ? w[j + s] : a;
        b = off / 2 == s ? w[j + s + 1 < 8 ? j + s + 1 : 7] : b;
      }
      u[j] = off & 1 ? __funnelshift_r(a, b, 16) : a;
    }
    whole(make_uint4(u[0], u[1], u[2], u[3]), x);
  }
  static __device__ __forceinline__ void whole(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
};
template <> struct Words<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ void spread(const uint4& lo, const uint4& hi, int off, float (&x)[4]) {
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t a = w[j];
#pragma unroll
      for (int s = 1; s < 4; ++s) a = off == s ? w[j + s] : a;
      x[j] = __uint_as_float(a);
    }
  }
  static __device__ __forceinline__ void whole(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
};

// One part of a row: words [0, n) from `first` on; pieces of kN words.
template <typename T>
struct Part {
  static constexpr int kN = Words<T>::kN;
  const T* first;
  const uint4* base;           // 16-byte boundary at or in front of `first`
  int off, n;                  // words from there to `first`
  long long left;              // whole 16-byte pieces from `base` to the end of all logits

  __device__ __forceinline__ Part(const T* z, long long at, int count, long long total) {
    first = z + at;
    n = count;
    off = (int)(at % kN);
    base = reinterpret_cast<const uint4*>(z + (at - off));
    left = (total - (at - off)) / kN;
  }
  __device__ __forceinline__ int pieces() const { return (n + kN - 1) / kN; }
  // whether piece p comes in whole 16-byte loads; the others are the row's last and, off the boundaries, the logits' last
  __device__ __forceinline__ bool whole(int p) const { return (p + 1) * kN <= n && p + (off ? 2 : 1) <= left; }
  // piece p; what lies behind the part is -infinity
  __device__ __forceinline__ void load(int p, float (&x)[kN]) const {
    if (whole(p)) {
      if (off == 0) Words<T>::whole(base[p], x);
      else Words<T>::spread(base[p], base[p + 1], off, x);
    } else {
#pragma unroll
      for (int j = 0; j < kN; ++j) x[j] = p * kN + j < n ? Words<T>::one(first + p * kN + j) : -INFINITY;
    }
  }
};

// a sum of exponentials relative to `ref`, and the largest entry
struct Sum {
  float ref = -INFINITY, top = -INFINITY, s = 0.f;
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N]) {
    float m = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) m = fmaxf(m, x[j]);
    if (m > ref + kSlack || ref == -INFINITY) {
      if (m > ref) {
        s *= exp2f((ref - m) * kLog2e);                  // (ref -infinity: 0, of a sum that is 0 or NaN)
        ref = m;
      }
    }
    top = fmaxf(top, m);
    const float r = ref == -INFINITY ? 0.f : ref;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float e;
      asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"((x[j] - r) * kLog2e));
      s += e;
    }
  }
};

__device__ __forceinline__ bool better(float z, int i, float y, int j) { return z > y || (z == y && i < j); }
// 32 bits in the order of the values, -0 as 0; NaN does not come here
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) beam_rows_kernel(const Args a) {
  constexpr int kN = Words<T>::kN;
  __shared__ __align__(16) float tops[kThreads];
  __shared__ int chosen[kThreads];
  __shared__ float list_z[kList];
  __shared__ int list_i[kList];
  __shared__ double red_s[kThreads / 32];
  __shared__ float red_m[kThreads / 32];
  __shared__ int count, n_chosen, taken, counts[256];
  __shared__ float threshold;
  mtf::chain_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x - row * a.parts);
  const float score = a.scores[row];
  if (!(fabsf(score) < INFINITY) || (a.finished && a.finished[row])) return;      // (not looked at behind this launch either)
  const int c0 = part * a.part, n = max(0, min(a.part, a.vocab - c0));
  const Part<T> w(reinterpret_cast<const T*>(a.z), row * a.vocab + c0, n, a.rows * a.vocab);
  const int pieces = w.pieces();

  // ---- one walk: sum and maximum
  Sum sum;
  int p = tid;
  constexpr int kDeep = 4;
  if (w.off == 0) {
    const int full = (int)min((long long)(n / kN), w.left);
    for (; p + (kDeep - 1) * kThreads < full; p += kDeep * kThreads) {
      uint4 v[kDeep];
#pragma unroll
      for (int e = 0; e < kDeep; ++e) v[e] = w.base[p + e * kThreads];
#pragma unroll
      for (int e = 0; e < kDeep; ++e) {
        float x[kN];
        Words<T>::whole(v[e], x);
        sum.add(x);
      }
    }
  } else {
    for (; p + (kDeep - 1) * kThreads < pieces && w.whole(p + (kDeep - 1) * kThreads); p += kDeep * kThreads) {
      uint4 v[kDeep], u[kDeep];
#pragma unroll
      for (int e = 0; e < kDeep; ++e) { v[e] = w.base[p + e * kThreads]; u[e] = w.base[p + e * kThreads + 1]; }
#pragma unroll
      for (int e = 0; e < kDeep; ++e) {
        float x[kN];
        Words<T>::spread(v[e], u[e], w.off, x);
        sum.add(x);
      }
    }
  }
  for (; p < pieces; p += kThreads) {
    float x[kN];
    w.load(p, x);
    sum.add(x);
  }

  // ---- the threads' sums, joined in 64 bits in a fixed order; the maxima
  float top = sum.top;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) red_m[warp] = top;
  tops[tid] = sum.top;
  if (tid == 0) { count = 0; n_chosen = 0; }
  __syncthreads();
  top = red_m[0];
#pragma unroll
  for (int i = 1; i < kThreads / 32; ++i) top = fmaxf(top, red_m[i]);
  double s = sum.ref == -INFINITY ? (double)sum.s : (double)sum.s * exp((double)sum.ref - (double)top);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) red_s[warp] = s;
  // how many threads' maxima come in front of this one's
  int rank = 0;
  for (int i = 0; i < kThreads; i += 4) {
    const float4 t = *reinterpret_cast<const float4*>(&tops[i]);
    rank += better(t.x, i, sum.top, tid) + better(t.y, i + 1, sum.top, tid) + better(t.z, i + 2, sum.top, tid) + better(t.w, i + 3, sum.top, tid);
  }
  if (rank == a.slots - 1) threshold = sum.top;
  __syncthreads();
  if (tid == 0) {
    double all = red_s[0];
#pragma unroll
    for (int i = 1; i < kThreads / 32; ++i) all += red_s[i];
    a.tops[row * a.parts + part] = top;
    a.sums[row * a.parts + part] = all;
  }
  const float thr = threshold;
  if (sum.top >= thr && sum.top > -INFINITY) chosen[atomicAdd(&n_chosen, 1)] = tid;
  __syncthreads();

  // ---- the words that reach the threshold, from the pieces of the threads that have some
  const int per = (pieces + kThreads - 1) / kThreads, again = n_chosen * per;
  for (int i = tid; i < again; i += kThreads) {
    const int q = chosen[i / per] + i % per * kThreads;
    if (q >= pieces) continue;
    float x[kN];
    w.load(q, x);
#pragma unroll
    for (int j = 0; j < kN; ++j)
      if (x[j] >= thr && x[j] > -INFINITY) {
        const int at = atomicAdd(&count, 1);
        if (at < kList) { list_z[at] = x[j]; list_i[at] = c0 + q * kN + j; }
      }
  }
  __syncthreads();
  int found = count;
  if (found > kList) {
    // Too many to be sorted (a row of equal words, or masked by a finite value): the slots-th largest value by counting its bytes from the highest on,
    // then all words above it, fewer than `slots`, and of those equal to it the first.
    uint32_t prefix = 0;
    int want = a.slots;                            // of those that share the prefix
    for (int byte = 3; byte >= 0; --byte) {
      __syncthreads();
      counts[tid] = 0;
      __syncthreads();
      for (int q = tid; q < pieces; q += kThreads) {
        float x[kN];
        w.load(q, x);
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const uint32_t k = key_of(x[j]);
          if (x[j] > -INFINITY && (byte == 3 || (k >> (8 * byte + 8)) == prefix)) atomicAdd(&counts[k >> (8 * byte) & 255], 1);
        }
      }
      __syncthreads();
      int above = 0, b = 255;
      while (b > 0 && above + counts[b] < want) above += counts[b--];
      want -= above;
      prefix = prefix << 8 | (uint32_t)b;
    }
    __syncthreads();
    if (tid == 0) { count = 0; taken = 0; }
    __syncthreads();
    for (int q0 = 0; q0 < pieces; q0 += kThreads) {
      const int q = q0 + tid;
      float x[kN];
      int same = 0;
      if (q < pieces) {
        w.load(q, x);
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const uint32_t k = key_of(x[j]);
          if (x[j] > -INFINITY && k > prefix) {
            const int at = atomicAdd(&count, 1);
            list_z[at] = x[j];
            list_i[at] = c0 + q * kN + j;
          }
          same += x[j] > -INFINITY && k == prefix;
        }
      }
      // equal ones in the order of their index, as long as there is need of them
      if (taken < want) {                          // (the same for all threads: it is written between barriers)
        int upto = same;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
          const int y = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += y;
        }
        if (lane == 31) counts[warp] = upto;
        __syncthreads();
        int at = taken + upto - same, all = taken;
        for (int i = 0; i < kThreads / 32; ++i) {
          if (i < warp) at += counts[i];
          all += counts[i];
        }
        if (q < pieces)
#pragma unroll
          for (int j = 0; j < kN; ++j)
            if (x[j] > -INFINITY && key_of(x[j]) == prefix) {
              if (at < want) {
                const int to = kList - 1 - at;     // from the other end
                list_z[to] = x[j];
                list_i[to] = c0 + q * kN + j;
              }
              ++at;
            }
        __syncthreads();
        if (tid == 0) taken = min(all, want);
        __syncthreads();
      }
    }
    __syncthreads();
    const int over = count, equal = taken;
    if (tid < equal) { list_z[over + tid] = list_z[kList - 1 - tid]; list_i[over + tid] = list_i[kList - 1 - tid]; }
    found = over + equal;
    __syncthreads();
  }

  // ---- in order
  float* const to_z = a.best_z + (row * a.parts + part) * a.slots;
  int* const to_i = a.best_i + (row * a.parts + part) * a.slots;
  for (int i = tid; i < found; i += kThreads) {
    const float z = list_z[i];
    const int at = list_i[i];
    int place = 0;
    for (int j = 0; j < found; ++j) place += better(list_z[j], list_i[j], z, at);
    if (place < a.slots) { to_z[place] = z; to_i[place] = at; }
  }
  for (int i = found + tid; i < a.slots; i += kThreads) to_i[i] = -1;
}

// A list's first word.  The words of a beam go by their logits (a score far from 0 may leave nothing of those in the sum), equal ones by the lower word.
struct Offer {
  double value = -INFINITY;
  float z = 0.f;
  int beam = 0x7fffffff, word = 0, list = 0;
  __device__ __forceinline__ bool before(const Offer& o) const {
    return value > o.value || (value == o.value && (beam < o.beam || (beam == o.beam && better(z, word, o.z, o.word))));
  }
};

// One warp a sentence: the best of its beams' parts' lists, one after the other.
__global__ void __launch_bounds__(32) beam_merge_kernel(const Args a) {
  extern __shared__ __align__(16) uint8_t room[];
  mtf::chain_wait_only();
  const int lane = threadIdx.x, lists = a.beams * a.parts, n = lists * a.slots;
  double* const base = reinterpret_cast<double*>(room);            // [beam]: score - log of the sum - maximum is added to a word's logit in two steps
  double* const maxima = base + a.beams;
  float* const z = reinterpret_cast<float*>(maxima + a.beams);
  int* const index = reinterpret_cast<int*>(z + n);
  int* const head = index + n;
  const long long sentence = blockIdx.x, row0 = sentence * a.beams;
  for (int b = lane; b < a.beams; b += 32) {
    const float score = a.scores[row0 + b];
    bool live = fabsf(score) < INFINITY;
    base[b] = score;
    maxima[b] = 0.;
    if (live && !(a.finished && a.finished[row0 + b])) {
      float top = -INFINITY;
      for (int p = 0; p < a.parts; ++p) top = fmaxf(top, a.tops[(row0 + b) * a.parts + p]);
      double s = 0.;
      for (int p = 0; p < a.parts; ++p) {
        const float m = a.tops[(row0 + b) * a.parts + p];
        const double x = a.sums[(row0 + b) * a.parts + p];
        s += m == top ? x : x * exp((double)m - (double)top);      // (a part without a finite word: 0 times its sum, 0 or NaN)
      }
      live = s > 0. && s < INFINITY && fabsf(top) < INFINITY;
      base[b] = (double)score - log(s);
      maxima[b] = top;
    }
    if (!live) base[b] = -INFINITY;
  }
  __syncwarp();
  for (int i = lane; i < n; i += 32) {
    const int list = i / a.slots, b = list / a.parts;
    const bool done = a.finished && a.finished[row0 + b];
    const bool live = base[b] > -INFINITY;
    index[i] = -1;
    if (!live) continue;
    if (done) {
      if (i == list * a.slots && list == b * a.parts) { index[i] = a.end_id; z[i] = 0.f; }
    } else {
      const long long at = row0 * a.parts * a.slots + i;
      index[i] = a.best_i[at];
      z[i] = a.best_z[at];
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
      const Offer o = {base[b] + ((double)z[i] - maxima[b]), z[i], b, index[i], l};
      if (o.before(best)) best = o;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const Offer o = {__shfl_xor_sync(0xffffffffu, best.value, d), __shfl_xor_sync(0xffffffffu, best.z, d), __shfl_xor_sync(0xffffffffu, best.beam, d),
                       __shfl_xor_sync(0xffffffffu, best.word, d), __shfl_xor_sync(0xffffffffu, best.list, d)};
      if (o.before(best)) best = o;
    }
    const bool any = best.value > -INFINITY;
    if (any && (best.list & 31) == lane) ++head[best.list];
    __syncwarp();
    if (lane == 0) {
      const long long at = sentence * a.slots + slot;
      const int parent = any ? best.beam : 0, token = any ? best.word : a.end_id;
      a.parents[at] = parent;
      a.tokens[at] = token;
      a.new_scores[at] = any ? (float)best.value : -INFINITY;
      if (a.new_finished) a.new_finished[at] = token == a.end_id || (any && a.finished && a.finished[row0 + parent]) ? 1 : 0;
    }
  }
}

// Parts of a row: so many that every SM has some blocks, each of at least 4096 words, and so few that a sentence's lists fit shared memory.
int parts_of(long long rows, int beams, int slots, int vocab) {
  const long long wanted = std::max(1LL, ((long long)mtf::device_sm_count() * 8 + rows - 1) / rows);
  const long long most = std::max(1LL, std::min<long long>(vocab / 4096, 4096 / ((long long)beams * slots)));
  return (int)std::min(wanted, most);
}
size_t merge_room(int beams, int slots, int parts) {
  return (size_t)beams * 2 * sizeof(double) + (size_t)beams * parts * slots * 8 + (size_t)beams * parts * 4;
}
size_t up16(size_t n) { return (n + 15) / 16 * 16; }

}  // namespace

namespace mtf {

size_t beam_select_workspace(long long sentences, int beams, int slots, int vocab) {
  const long long rows = sentences * beams;
  const size_t lists = (size_t)rows * parts_of(rows, beams, slots, vocab);
  return up16(lists * sizeof(double)) + up16(lists * sizeof(float)) + up16(lists * slots * 4) + lists * slots * 4;
}

mtf_status launch_beam_select(const BeamSelect& b, void* stream) {
  Args a = {};
  a.z = b.logits;
  a.vocab = b.vocab;
  a.beams = b.beams;
  a.slots = b.slots;
  a.rows = b.sentences * b.beams;
  a.parts = parts_of(a.rows, b.beams, b.slots, b.vocab);
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
  if (b.bf16) launch_chained(beam_rows_kernel<__nv_bfloat16>, (unsigned)(a.rows * a.parts), kThreads, 0, st, a);
  else launch_chained(beam_rows_kernel<float>, (unsigned)(a.rows * a.parts), kThreads, 0, st, a);
  count_launch();
  launch_chained(beam_merge_kernel, (unsigned)b.sentences, 32, merge_room(a.beams, a.slots, a.parts), st, a);
  count_launch();
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "beam_select kernels: %s", cudaGetErrorString(e));
  return MTF_OK;
}

}  // namespace mtf
