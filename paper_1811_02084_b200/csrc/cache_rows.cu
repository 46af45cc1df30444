// A paged cache's rows: written from dense ones, read back as dense ones, and reordered behind a step of beam search; and the reordering of
// dense states.
//
// An 8-bit cache holds a row of d values as e4m3 and one scale: the smallest power of two by which the row's largest finite value is at most 448,
// e4m3's largest.  A power of two divides exactly, so a value is rounded once, to e4m3's 4 significant bits, and nothing about the result
// depends on how a quotient is rounded; the finer scale amax / 448 would gain nothing, since a floating-point format's steps are relative.
// NaN and infinities are stored as NaN.  A row of zeros has scale 1.
//
// All of it is copying (a row is read once and written once): HBM is the bound.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "answer.cuh"
#include "answer.h"
#include "launch.cuh"

namespace {

__device__ int g_bad_place = 0;                  // a position or page outside the cache, or a parent outside the beams, was seen

// n / d for n < 2^31
struct Divide {
  uint32_t mul;
  int shift, d;
};
Divide divide_by(int d) {
  int n = 0;
  while ((1LL << n) < d) ++n;
  return {(uint32_t)(((1ULL << (31 + n)) + d - 1) / d), 31 + n, d};      // off by less than 2^n in 2^(31 + n)
}
__device__ __forceinline__ int over(int n, const Divide& d) { return (int)((unsigned long long)(uint32_t)n * d.mul >> d.shift); }

struct RowsArgs {
  uint8_t* pool[2];                              // K, V
  float* scale[2];
  uint8_t* dense[2];
  int d[2];
  const int32_t *table, *starts, *counts;
  long long length;
  int units;                                     // sequences * length
  long long items;                               // units * passes over the heads
  int heads, slots, pages, per_sequence, rows_page, row_slot, row_head;
  Divide by_length, by_slots, by_passes;
};

__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t two_bf16(float x, float y) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// e4m3 of two values of magnitude up to 448 or NaN; x in the low byte
__device__ __forceinline__ uint32_t two_e4m3(float x, float y) {
  uint32_t v;
  asm("{\n\t.reg .b16 t;\n\tcvt.rn.satfinite.e4m3x2.f32 t, %2, %1;\n\tcvt.u32.u16 %0, t;\n\t}" : "=r"(v) : "f"(x), "f"(y));
  return v;
}
__device__ __forceinline__ float2 of_e4m3(uint32_t two) {
  uint32_t h;
  asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}" : "=r"(h) : "r"(two));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Position `unit` = (sequence, index) of the dense rows: its first row in the pool (head 0), -1 where the rows are not meant, -2 where there is no place for them.
__device__ __forceinline__ int place(const RowsArgs& a, int unit) {
  const int s = over(unit, a.by_length), at = unit - s * (int)a.length;
  const int count = a.counts ? a.counts[s] : (int)a.length;
  const long long m = (long long)(a.starts ? a.starts[s] : 0) + at;
  if (at >= count) return -1;
  if (m < 0 || m >= (long long)a.per_sequence * a.slots) return -2;
  const int index = over((int)m, a.by_slots), page = a.table[(long long)s * a.per_sequence + index];
  if (page < 0 || page >= a.pages) return -2;
  return page * a.rows_page + ((int)m - index * a.slots) * a.row_slot;
}

// A position's rows of all heads are together in the dense tensor, and their place is one look at the table.  kLanes lanes take a head, 8 or 16 values each (d up to as many times kLanes); the
// 32 / kLanes heads of a warp are an item, and a warp has kEach items' loads under way at once: of one position, or of several where it has few heads.  Their places
// are looked up by a lane each, those of the next items while these ones' rows are under way.  blockIdx.y: K or V.
// (A look at the table a row, whole calls: 32 x 512 prompts of 16 heads of 64 written in e4m3 and read back 63 us, 8 x 16384 positions of 8 heads of 128 read back 138; this way 36 and 120, 4.9 and 5.8 TB/s.  Reading is near
// HBM's rate; writing waits for its loads and spends issue slots, 62 % of them, on finding the rows' largest values and on the conversions, of 16 values a lane with some spills: 64 registers are what
// four blocks an SM leave a thread.)
constexpr int kRowBlocks = 4;          // an SM holds; K's come first
template <int kEach>
struct Items {
  int unit, head, row;                 // of item lane % kEach: position, first head, place (below 0: none)
  __device__ __forceinline__ void look(const RowsArgs& a, long long first, int heads) {
    const long long j = first + (threadIdx.x & (kEach - 1));
    unit = -1;
    row = -1;
    if (j < a.items) {
      unit = over((int)j, a.by_passes);
      head = ((int)j - unit * a.by_passes.d) * heads;
      row = place(a, unit);
    }
  }
};

template <int kLanes, int kValues, bool kBf16, bool kE4m3, int kEach>
__global__ void __launch_bounds__(256, kRowBlocks) cache_write_kernel(const RowsArgs a) {
  mtf::chain_wait();
  const int side = blockIdx.y, d = a.d[side], lane = threadIdx.x & 31, col = lane % kLanes * kValues, group = lane / kLanes;
  constexpr int kHeads = 32 / kLanes, kPieces = kValues * (kBf16 ? 2 : 4) / 16;
  const long long step = (long long)gridDim.x * 8 * kEach;
  long long first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * kEach;
  Items<kEach> next;
  next.look(a, first, kHeads);
  for (; first < a.items; first += step) {
    const Items<kEach> now = next;
    if (now.row == -2 && lane < kEach) atomicExch(&g_bad_place, 1);
    uint4 w[kEach][kPieces];
    int row[kEach];                                  // -1: nothing to be done by this lane
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int unit = __shfl_sync(0xffffffffu, now.unit, e), head = __shfl_sync(0xffffffffu, now.head, e) + group, here = __shfl_sync(0xffffffffu, now.row, e);
      row[e] = here >= 0 && head < a.heads && col < d ? here + head * a.row_head : -1;
      const uint4* const p = reinterpret_cast<const uint4*>(a.dense[side] + (((long long)unit * a.heads + head) * d + col) * (kBf16 ? 2 : 4));
#pragma unroll
      for (int i = 0; i < kPieces; ++i) w[e][i] = row[e] >= 0 ? p[i] : make_uint4(0u, 0u, 0u, 0u);
    }
    next.look(a, first + step, kHeads);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const long long at = (long long)row[e] * d + col;
      uint32_t u[4 * kPieces];
#pragma unroll
      for (int i = 0; i < kPieces; ++i) { u[4 * i] = w[e][i].x; u[4 * i + 1] = w[e][i].y; u[4 * i + 2] = w[e][i].z; u[4 * i + 3] = w[e][i].w; }
      float x[kValues];
#pragma unroll
      for (int j = 0; j < kValues; ++j) x[j] = kBf16 ? (j & 1 ? hi16(u[j / 2]) : lo16(u[j / 2])) : __uint_as_float(u[j]);
      if (!kE4m3) {
        if (row[e] >= 0)
          *reinterpret_cast<uint4*>(a.pool[side] + at * 2) = kBf16 ? w[e][0] : make_uint4(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7]));
        continue;
      }
      // the row's largest magnitude as bits, in whose order infinities and NaN come last
      uint32_t top = 0;
      if (kBf16) {
#pragma unroll
        for (int i = 0; i < 4 * kPieces; ++i) top = __vmaxu2(top, u[i] & 0x7fff7fffu);
        top = max(top << 16, top & 0xffff0000u);
      } else {
#pragma unroll
        for (int j = 0; j < kValues; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
      }
#pragma unroll
      for (int o = kLanes / 2; o > 0; o /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (__any_sync(0xffffffffu, top >= 0x7f800000u)) {
        // NaN and infinities: all to NaN, and the largest of the others
        top = 0;
#pragma unroll
        for (int j = 0; j < kValues; ++j) {
          const uint32_t m = __float_as_uint(x[j]) & 0x7fffffffu;
          if (m < 0x7f800000u) top = max(top, m);
          else x[j] = __uint_as_float(0x7fc00000u);
        }
#pragma unroll
        for (int o = kLanes / 2; o > 0; o /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      }
      // 448 = 1.75 2^8: scale 2^(e - 8) for a largest value m 2^e with m up to 1.75, else 2^(e - 7); not below 2^-126, so that it is a normal number, too, and so is its inverse
      int field = max((int)((top + 0x1fffffu) >> 23) - 8, 1);
      if (top == 0) field = 127;
      if (row[e] < 0) continue;
      const float up = __uint_as_float((uint32_t)(254 - field) << 23);
      uint32_t four[kValues / 4];
#pragma unroll
      for (int i = 0; i < kValues / 4; ++i) four[i] = two_e4m3(x[4 * i] * up, x[4 * i + 1] * up) | two_e4m3(x[4 * i + 2] * up, x[4 * i + 3] * up) << 16;
      if constexpr (kValues == 16) *reinterpret_cast<uint4*>(a.pool[side] + at) = make_uint4(four[0], four[1], four[2], four[3]);
      else *reinterpret_cast<uint2*>(a.pool[side] + at) = make_uint2(four[0], four[1]);
      if (col == 0) a.scale[side][row[e]] = __uint_as_float((uint32_t)field << 23);
    }
  }
}

template <int kLanes, int kValues, bool kBf16, bool kE4m3, int kEach>
__global__ void __launch_bounds__(256, kRowBlocks) cache_read_kernel(const RowsArgs a) {
  mtf::chain_wait();
  const int side = blockIdx.y, d = a.d[side], lane = threadIdx.x & 31, col = lane % kLanes * kValues, group = lane / kLanes;
  constexpr int kHeads = 32 / kLanes;
  const long long step = (long long)gridDim.x * 8 * kEach;
  long long first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * kEach;
  Items<kEach> next;
  next.look(a, first, kHeads);
  for (; first < a.items; first += step) {
    const Items<kEach> now = next;
    if (now.row == -2 && lane < kEach) atomicExch(&g_bad_place, 1);
    uint4 w[kEach];
    float scale[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int head = __shfl_sync(0xffffffffu, now.head, e) + group, here = __shfl_sync(0xffffffffu, now.row, e);
      w[e] = make_uint4(0u, 0u, 0u, 0u);             // (zeros in e4m3 as well)
      scale[e] = 0.f;
      if (here < 0 || head >= a.heads || col >= d) continue;
      const int row = here + head * a.row_head;
      const long long at = (long long)row * d + col;
      if (kE4m3 && kValues == 8) {
        const uint2 v = *reinterpret_cast<const uint2*>(a.pool[side] + at);
        w[e].x = v.x;
        w[e].y = v.y;
      } else {
        w[e] = *reinterpret_cast<const uint4*>(a.pool[side] + at * (kE4m3 ? 1 : 2));
      }
      if (kE4m3) scale[e] = a.scale[side][row];
    }
    next.look(a, first + step, kHeads);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int unit = __shfl_sync(0xffffffffu, now.unit, e), head = __shfl_sync(0xffffffffu, now.head, e) + group;
      if (unit < 0 || head >= a.heads || col >= d) continue;
      uint4* const p = reinterpret_cast<uint4*>(a.dense[side] + (((long long)unit * a.heads + head) * d + col) * (kBf16 ? 2 : 4));
      if (!kE4m3 && kBf16) { p[0] = w[e]; continue; }
      const uint32_t u[4] = {w[e].x, w[e].y, w[e].z, w[e].w};
      float x[kValues];
      if (kE4m3) {
#pragma unroll
        for (int j = 0; j < kValues / 2; ++j) {
          const float2 v = of_e4m3(u[j / 2] >> (16 * (j & 1)));
          x[2 * j] = v.x * scale[e];
          x[2 * j + 1] = v.y * scale[e];
        }
      } else {
#pragma unroll
        for (int j = 0; j < kValues; ++j) x[j] = j & 1 ? hi16(u[j / 2]) : lo16(u[j / 2]);
      }
#pragma unroll
      for (int i = 0; i < kValues * (kBf16 ? 2 : 4) / 16; ++i) {
        if constexpr (kBf16) p[i] = make_uint4(two_bf16(x[8 * i], x[8 * i + 1]), two_bf16(x[8 * i + 2], x[8 * i + 3]), two_bf16(x[8 * i + 4], x[8 * i + 5]), two_bf16(x[8 * i + 6], x[8 * i + 7]));
        else p[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
      }
    }
  }
}

struct ReorderArgs {
  uint8_t* pool[2];
  float* scale[2];
  int row_bytes[2];
  const int32_t *table, *parents, *lengths, *fresh;
  int32_t *new_table, *new_lengths;
  int beams, out, heads, slots, pages, per_sequence, rows_page, row_slot, row_head;
};

// Block (x, y): answer x = (group, i); the y-th share of what is copied for it.  A chain of parent, length, table entry and rows, each a load behind the one before: 32 x 8 beams, pages
// of 16 of 16 heads of 64 in bf16, 15 MB, take 7.7 us a call (6.2 in a graph), of which the bytes are 2.3; with K's and V's pieces one after the other 8.5.
__global__ void __launch_bounds__(256) cache_reorder_kernel(const ReorderArgs a) {
  mtf::chain_wait();
  const int x = blockIdx.x, group = x / a.out, parent = a.parents[x];
  const int tid = blockIdx.y * 256 + threadIdx.x, threads = gridDim.y * 256;
  int32_t* const to = a.new_table + (long long)x * a.per_sequence;
  if (parent < 0 || parent >= a.beams) {             // no such beam: an answer without positions
    if (tid == 0) { atomicExch(&g_bad_place, 1); a.new_lengths[x] = 0; }
    for (int i = tid; i < a.per_sequence; i += threads) to[i] = -1;
    return;
  }
  const int from = group * a.beams + parent;
  const int32_t* const of = a.table + (long long)from * a.per_sequence;
  const int length = a.lengths[from], n = min(max(length, 0), a.per_sequence * a.slots), whole = n / a.slots, used = n - whole * a.slots;      // (positions that the table has pages for)
  const int page = used ? of[whole] : 0, fresh = used ? a.fresh[x] : 0;
  const bool source = page >= 0 && page < a.pages, there = source && fresh >= 0 && fresh < a.pages;
  if (tid == 0) {
    a.new_lengths[x] = n;
    if (n != length || !there) atomicExch(&g_bad_place, 1);
  }
  // (a last page that is none stays one: what is left out goes on being left out)
  for (int i = tid; i < a.per_sequence; i += threads) to[i] = i == whole && used && source ? fresh : of[i];
  if (!used || !there) return;
  // Rows in use of the page that goes on, `used` slots of every head, K's and V's as one range of 16-byte pieces, four under way a thread.  The inner one of slot and head is
  // contiguous: slots of a head (used of them), or all heads of a slot.
  const int rows = used * a.heads, run = a.row_slot == 1 ? used : a.heads, gap = a.row_slot == 1 ? a.row_head : a.row_slot;
  const int pieces_k = a.row_bytes[0] / 16, pieces_v = a.row_bytes[1] / 16, total_k = rows * pieces_k, total = total_k + rows * pieces_v;
  const long long src = (long long)page * a.rows_page, dst = (long long)fresh * a.rows_page;
  constexpr int kDeep = 4;
  for (int i0 = tid; i0 < total; i0 += kDeep * threads) {
    uint4 v[kDeep];
    uint4* to[kDeep];
#pragma unroll
    for (int e = 0; e < kDeep; ++e) {
      const int i = i0 + e * threads;
      to[e] = nullptr;
      if (i >= total) continue;
      const int side = i >= total_k, j = side ? i - total_k : i, pieces = side ? pieces_v : pieces_k;
      const int inner = run * pieces, n = j / inner, at = n * gap * pieces + (j - n * inner);
      uint4* const pool = reinterpret_cast<uint4*>(a.pool[side]);
      to[e] = pool + dst * pieces + at;
      v[e] = pool[src * pieces + at];
    }
#pragma unroll
    for (int e = 0; e < kDeep; ++e)
      if (to[e]) *to[e] = v[e];
  }
  if (a.scale[0])
    for (int i = tid; i < 2 * rows; i += threads) {
      float* const scale = a.scale[i >= rows];
      const int j = i >= rows ? i - rows : i, n = j / run, at = n * gap + (j - n * run);
      scale[dst + at] = scale[src + at];
    }
}

// out[x, :] = in[group(x), parents[x], :]; rows of `pieces` pieces of type T, the widest that addresses and rows allow.  16 x 4 rows of 1 MB: 11.2 us, 6.0 TB/s.
template <typename T>
__global__ void __launch_bounds__(256) beam_reorder_kernel(const int32_t* __restrict__ parents, const T* __restrict__ in, T* __restrict__ out, int beams, int slots,
                                                           long long pieces) {
  mtf::chain_wait();
  const long long x = blockIdx.x;
  const int parent = parents[x];
  const bool there = parent >= 0 && parent < beams;
  if (!there && threadIdx.x == 0 && blockIdx.y == 0) atomicExch(&g_bad_place, 1);
  const T* const src = in + (x / slots * beams + (there ? parent : 0)) * pieces;
  T* const dst = out + x * pieces;
  const long long step = (long long)gridDim.y * 256;
  long long i = (long long)blockIdx.y * 256 + threadIdx.x;
  for (; i + 3 * step < pieces; i += 4 * step) {
    T v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = there ? src[i + e * step] : T();
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[i + e * step] = v[e];
  }
  for (; i < pieces; i += step) dst[i] = there ? src[i] : T();
}

RowsArgs rows_args(const mtf::CachePool& c, const mtf::CacheRows& r) {
  RowsArgs a = {};
  a.pool[0] = reinterpret_cast<uint8_t*>(c.k);
  a.pool[1] = reinterpret_cast<uint8_t*>(c.v);
  a.scale[0] = c.ks;
  a.scale[1] = c.vs;
  a.dense[0] = reinterpret_cast<uint8_t*>(r.k);
  a.dense[1] = reinterpret_cast<uint8_t*>(r.v);
  a.d[0] = c.dk;
  a.d[1] = c.dv;
  a.table = c.table;
  a.starts = r.starts;
  a.counts = r.counts;
  a.length = r.length;
  a.heads = c.heads;
  a.slots = c.slots;
  a.pages = c.pages;
  a.per_sequence = c.per_sequence;
  a.rows_page = c.rows_page;
  a.row_slot = c.row_slot;
  a.row_head = c.row_head;
  a.units = (int)(c.sequences * r.length);
  a.by_length = divide_by((int)r.length);
  a.by_slots = divide_by(c.slots);
  return a;
}

template <int kLanes, int kValues, bool kBf16, bool kE4m3>
void rows_launch(RowsArgs a, bool write, cudaStream_t st) {
  const int passes = (a.heads + 32 / kLanes - 1) / (32 / kLanes);
  // items at once: 16 to 32 registers of what is loaded.  (Half as many: prompts 37.8 us for 35.5, the long read 127 for 120; twice as many 39.7 and 132.)
  constexpr int kWrite = kValues == 16 && !kBf16 ? 2 : 4, kRead = kValues == 8 && kE4m3 ? 8 : 4;
  const int each = write ? kWrite : kRead;
  a.items = (long long)a.units * passes;
  a.by_passes = divide_by(passes);
  const long long blocks = std::min<long long>((a.items + 8 * each - 1) / (8 * each), (long long)mtf::device_sm_count() * kRowBlocks);
  mtf::launch_clusters(write ? cache_write_kernel<kLanes, kValues, kBf16, kE4m3, kWrite> : cache_read_kernel<kLanes, kValues, kBf16, kE4m3, kRead>, dim3((unsigned)blocks, 2, 1), 256, 0, 1, st, a);
}
template <bool kBf16, bool kE4m3>
void rows_lanes(const RowsArgs& a, bool write, cudaStream_t st) {
  const int d = std::max(a.d[0], a.d[1]), lanes = d <= 64 ? 8 : d <= 128 ? 16 : 32;
  // 8-bit rows: 16 values a lane where that saves a pass over the heads, 8 where lanes would stand idle.  (8 -> 16 values, rows of 64: written and read back, 2 heads 19.6 -> 24.9 us, 4 12.0 -> 15.1,
  // 6 15.1 -> 12.5, 8 12.1 -> 11.5, 16 heads of 32 x 512 positions 39.6 -> 35.5; read, 8 x 16384 positions of 4 heads 32 -> 41, of 6 60 -> 46, of 8 65 -> 63.)
  if constexpr (kE4m3)
    if (a.heads > 32 / lanes) {
      if (lanes == 8) rows_launch<4, 16, kBf16, true>(a, write, st);
      else if (lanes == 16) rows_launch<8, 16, kBf16, true>(a, write, st);
      else rows_launch<16, 16, kBf16, true>(a, write, st);
      return;
    }
  if (lanes == 8) rows_launch<8, 8, kBf16, kE4m3>(a, write, st);
  else if (lanes == 16) rows_launch<16, 8, kBf16, kE4m3>(a, write, st);
  else rows_launch<32, 8, kBf16, kE4m3>(a, write, st);
}
mtf_status after(const char* what) {
  mtf::count_launch();
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return mtf::fail(MTF_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
  return MTF_OK;
}
mtf_status cache_rows(const mtf::CachePool& c, const mtf::CacheRows& r, bool write, void* stream) {
  const RowsArgs a = rows_args(c, r);
  cudaStream_t st = (cudaStream_t)stream;
  if (r.bf16) c.e4m3 ? rows_lanes<true, true>(a, write, st) : rows_lanes<true, false>(a, write, st);
  else c.e4m3 ? rows_lanes<false, true>(a, write, st) : rows_lanes<false, false>(a, write, st);
  return after(write ? "cache_write_kernel" : "cache_read_kernel");
}

template <typename T>
void reorder_launch(const int32_t* parents, const void* in, void* out, long long rows, int beams, int slots, long long bytes, cudaStream_t st) {
  const long long pieces = bytes / (long long)sizeof(T);
  const long long shares = std::max(1LL, std::min((pieces + 1023) / 1024, std::max(1LL, (long long)mtf::device_sm_count() * 16 / rows)));
  mtf::launch_clusters(beam_reorder_kernel<T>, dim3((unsigned)rows, (unsigned)std::min(shares, 65535LL), 1), 256, 0, 1, st, parents, reinterpret_cast<const T*>(in), reinterpret_cast<T*>(out), beams, slots, pieces);
}

}  // namespace

namespace mtf {

mtf_status launch_cache_write(const CachePool& c, const CacheRows& r, void* stream) { return cache_rows(c, r, true, stream); }
mtf_status launch_cache_read(const CachePool& c, const CacheRows& r, void* stream) { return cache_rows(c, r, false, stream); }

mtf_status launch_cache_reorder(const CachePool& c, const CacheReorder& r, void* stream) {
  ReorderArgs a = {};
  a.pool[0] = reinterpret_cast<uint8_t*>(c.k);
  a.pool[1] = reinterpret_cast<uint8_t*>(c.v);
  a.scale[0] = c.ks;
  a.scale[1] = c.vs;
  a.row_bytes[0] = c.dk * (c.e4m3 ? 1 : 2);
  a.row_bytes[1] = c.dv * (c.e4m3 ? 1 : 2);
  a.table = c.table;
  a.parents = r.parents;
  a.lengths = r.lengths;
  a.fresh = r.fresh;
  a.new_table = r.table;
  a.new_lengths = r.new_lengths;
  a.beams = r.beams;
  a.out = r.out;
  a.heads = c.heads;
  a.slots = c.slots;
  a.pages = c.pages;
  a.per_sequence = c.per_sequence;
  a.rows_page = c.rows_page;
  a.row_slot = c.row_slot;
  a.row_head = c.row_head;
  const long long rows = r.groups * r.out, page_bytes = (long long)c.rows_page * (a.row_bytes[0] + a.row_bytes[1]);
  // a share of a page's copy that is worth a block, as long as the GPU has room for more of them
  const long long shares = std::max(1LL, std::min({(page_bytes + 32767) / 32768, (long long)device_sm_count() * 8 / rows + 1, 64LL}));
  mtf::launch_clusters(cache_reorder_kernel, dim3((unsigned)rows, (unsigned)shares, 1), 256, 0, 1, (cudaStream_t)stream, a);
  return after("cache_reorder_kernel");
}

mtf_status launch_beam_reorder(const int32_t* parents, const void* in, void* out, long long groups, int beams, int slots, long long bytes, void* stream) {
  const uintptr_t low = reinterpret_cast<uintptr_t>(in) | reinterpret_cast<uintptr_t>(out) | (uintptr_t)bytes;
  const cudaStream_t st = (cudaStream_t)stream;
  const long long rows = groups * slots;
  if (low % 16 == 0) reorder_launch<uint4>(parents, in, out, rows, beams, slots, bytes, st);
  else if (low % 4 == 0) reorder_launch<uint32_t>(parents, in, out, rows, beams, slots, bytes, st);
  else if (low % 2 == 0) reorder_launch<uint16_t>(parents, in, out, rows, beams, slots, bytes, st);
  else reorder_launch<uint8_t>(parents, in, out, rows, beams, slots, bytes, st);
  return after("beam_reorder_kernel");
}

// 1 when a position, page or parent outside its range was met since the last call; resets the flag
mtf_status read_cache_bad_place(int* seen) {
  int v = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_bad_place, sizeof(int));
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "cudaMemcpyFromSymbol: %s", cudaGetErrorString(e));
  if (v) { int z = 0; cudaMemcpyToSymbol(g_bad_place, &z, sizeof(int)); }
  *seen = v;
  return MTF_OK;
}

}  // namespace mtf
