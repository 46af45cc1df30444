// Attention of one new token a sequence over a paged cache:
//     o[s, h, g, :] = sum_m p_m v[m, h, :],   p = softmax over m < n_s of scale * q[s, h, g, :] . k[m, h, :]
// where position m of sequence s lies in page table[s][m / slots], slot m % slots.
//
// Every row of the cache is read once and used for `group` heads of queries, 2 to 4 flops a byte and head: HBM is the bound, and the
// products only have to keep out of its way.  So a warp is a stream of its own: it loads a chunk of 16 (or 32, 64) rows of K and of V straight into
// the registers that matrix instructions want them in, and loads the next chunk of either as soon as the current one is used up; there is
// no shared memory and no barrier in the loop, and each warp keeps its own running maximum and sums.  With the rows of the cache as the
// instruction's 16 rows and the heads as its 8 columns, eight heads of queries cost no more than one and nothing is padded to 16:
//     S^T [16 keys x 8 heads] = K [16 x d] q^T [d x 8],   O^T [d x 8 heads] += V^T [d x 16 keys] P^T [16 keys x 8]
// The order of a sum's terms is free, so the lanes take d in the order in which 16-byte loads leave it (K), and the rows of O^T are the d that
// a lane's load holds (V, whose pairs of keys are put together by byte permutes).
//
// The work is cut evenly: the keys of all (sequence, head) items are laid end to end in units of some rows a warp, and every block takes an equal
// run of them, whatever the lengths.  Items that cross a block's edge are left as partial sums and joined behind the launch, in order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "answer.h"
#include "launch.cuh"

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kPlanned = 2048;        // sequences whose units a block adds up by itself
constexpr int kLeastUnits = 2;        // a block's run
constexpr float kLog2e = 1.4426950408889634f;
// The running maximum is raised only where a logit lies 2^6 above it: otherwise every chunk would pay for a maximum across lanes.
constexpr float kSlack = 6.f;
// e4m3: the weights are f16, and a weight of 1 is held as 2^9, so that with the slack they stay below 2^16 and those of 2^-23 keep all of f16's digits.
constexpr float kLift = 9.f;

struct Args {
  const __nv_bfloat16* q;
  const uint8_t *k, *v;
  const float *ks, *vs;
  const int32_t *table, *lengths;
  __nv_bfloat16* o;
  int n_seq, heads, group, chunks, dk, dv;       // chunks: of the group, 8 NT heads each
  int pages, slots, per_sequence, rows_page, row_slot, row_head;
  uint32_t slots_mul;                            // m / slots = (m * slots_mul) >> slots_shift in 64 bits, for m below 2^31
  int slots_shift;
  float scale_log2;
  int balanced;
  float* part_o;                                 // [block][2][8 NT][DC]
  float* part_s;                                 // [block][2][8 NT][4]: reference of l, l, reference of o
  int4* pieces;                                  // [block]: of the item that starts last in it and goes on: sequence, head and chunk, its last block, slot
};

__device__ int g_bad_page = 0;                   // a page id outside the pool, or a length beyond the table, was seen

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t s) { return __byte_perm(a, b, s); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint4 load16(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load8(const uint8_t* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
// two e4m3 values as f16 (exact)
__device__ __forceinline__ uint32_t halves(uint32_t two) {
  uint32_t h;
  asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}" : "=r"(h) : "r"(two));
  return h;
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool kHalf>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (kHalf)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word(const uint2& v, int i) { return i == 0 ? v.x : v.y; }

template <bool kE4m3, int DC>
struct Shape {
  static constexpr int kElt = kE4m3 ? 1 : 2;
  static constexpr int kTiles = DC * kElt <= 64 ? 4 : DC * kElt <= 128 ? 2 : 1;     // 16-key tiles of a chunk: 4 to 8 KB of K and of V a warp (d = 256: 8)
  static constexpr int kKeys = 16 * kTiles;
  static constexpr int kTB = 16 / kElt;              // K: values of a lane's 16 bytes
  static constexpr int kKP = DC / (4 * kTB);         // ... pieces of a row
  static constexpr int kSteps = kTB / 4;             // ... products of a piece, 16 deep
  static constexpr int kVB = kE4m3 && DC == 64 ? 8 : kTB;   // V: values of a lane's piece (8 lanes a row)
  static constexpr int kVP = DC / (8 * kVB);
  static constexpr int kIndexes = (kKeys + 31) / 32;
};
template <int kBytes> struct Piece { using T = uint4; };
template <> struct Piece<8> { using T = uint2; };

// first unit of block c, of `units` over `blocks`
__device__ __forceinline__ long long first_unit(long long units, int blocks, int c) { return units * c / blocks; }

template <bool kE4m3, int DC, int NT>
__global__ void __launch_bounds__(kThreads, DC == 256 || (NT > 1 && DC == 128) ? 2 : 3) attention_decode_kernel(const Args a) {
  using S = Shape<kE4m3, DC>;
  using VT = typename Piece<S::kVB * S::kElt>::T;
  constexpr int kUnit = kWarps * S::kKeys, kHeads = 8 * NT, kMT = DC / 16;
  __shared__ __align__(16) float so[kWarps][kHeads][DC + 4];      // (read and written two at a time)
  __shared__ int cum[kPlanned + 1];
  __shared__ int warp_total[kWarps];
  __shared__ float ss[kWarps][kHeads][3];
  mtf::chain_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, t = lane & 3;
  const int H = a.heads * a.chunks;
  const int capacity = (int)min((long long)a.per_sequence * a.slots, 0x7fffffffLL);
  auto length_of = [&](int s) {
    const int n = a.lengths[s];
    if ((n < 0 || n > capacity)) atomicExch(&g_bad_page, 1);
    return min(max(n, 0), capacity);
  };

  // ---- this block's run of units
  long long u0, u1, units = 0;
  int blocks = gridDim.x;
  if (a.balanced) {
    const int each = (a.n_seq + kThreads - 1) / kThreads, s0 = tid * each;
    int sum = 0;
    for (int i = 0; i < each; ++i)
      if (s0 + i < a.n_seq) sum += (length_of(s0 + i) + kUnit - 1) / kUnit;
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) warp_total[warp] = upto;
    __syncthreads();
    int before = upto - sum;
    for (int w = 0; w < warp; ++w) before += warp_total[w];
    for (int i = 0; i < each; ++i)
      if (s0 + i < a.n_seq) {
        cum[s0 + i] = before;
        before += (length_of(s0 + i) + kUnit - 1) / kUnit;
        if (s0 + i == a.n_seq - 1) cum[a.n_seq] = before;
      }
    __syncthreads();
    units = (long long)cum[a.n_seq] * H;
    // (no block without a unit among those that share them: a join goes from block to block)
    blocks = (int)min((long long)blocks, max(1LL, units / kLeastUnits));
    u0 = u1 = 0;
    if ((int)blockIdx.x < blocks) {
      u0 = first_unit(units, blocks, blockIdx.x);
      u1 = first_unit(units, blocks, blockIdx.x + 1);
    }
    if (tid == 0) a.pieces[blockIdx.x] = make_int4(-1, 0, 0, 0);
    // sequences without a position
    for (int s = blockIdx.x; s < a.n_seq; s += gridDim.x)
      if (cum[s + 1] == cum[s])
        for (long long i = tid; i < (long long)a.heads * a.group * a.dv; i += kThreads) a.o[(long long)s * a.heads * a.group * a.dv + i] = __float2bfloat16(0.f);
  } else {
    u0 = 0;
    u1 = 1;
  }

  for (long long u = u0; u < u1;) {
    // ---- the item, and the part of it that is this block's
    int seq, hc, j0, j1, n;
    bool whole;
    int slot = 0;
    if (a.balanced) {
      const int x = (int)(u / H);                   // (units of a sequence's heads lie one behind another)
      int lo = 0, hi = a.n_seq;                     // the last sequence with cum <= x
      while (hi - lo > 1) {
        const int m = (lo + hi) / 2;
        if (cum[m] <= x) lo = m; else hi = m;
      }
      seq = lo;
      const int each = cum[seq + 1] - cum[seq];
      const long long in = u - (long long)cum[seq] * H;
      hc = (int)(in / each);
      j0 = (int)(in - (long long)hc * each);
      j1 = (int)min((long long)each, j0 + (u1 - u));
      whole = j0 == 0 && j1 == each;
      slot = 2 * blockIdx.x + (u == u0 ? 0 : 1);
      if (tid == 0 && j0 == 0 && !whole) {
        const long long end = u + each;              // behind the item's last unit
        const int last = (int)((end * blocks - 1) / units);
        a.pieces[blockIdx.x] = make_int4(seq, hc, last, slot);
      }
      n = length_of(seq);
      u += j1 - j0;
    } else {
      const long long item = blockIdx.x;
      seq = (int)(item / H);
      hc = (int)(item - (long long)seq * H);
      n = length_of(seq);
      j0 = 0;
      j1 = (n + kUnit - 1) / kUnit;
      whole = true;
      u = 1;
    }
    const int head = hc / a.chunks, g0 = (hc - head * a.chunks) * kHeads;
    const int here = min(kHeads, a.group - g0);      // heads of queries in this chunk

    // ---- queries, in the order in which the lanes hold K
    uint32_t qf[NT][S::kKP * S::kSteps][2];
    float factor[NT][2];                             // of the products of the lane's two heads
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int g = nt * 8 + r;
      const __nv_bfloat16* const row = a.q + (((long long)seq * a.heads + head) * a.group + g0 + g) * a.dk;
      float top = 0.f;
#pragma unroll
      for (int p = 0; p < S::kKP; ++p)
#pragma unroll
        for (int j = 0; j < S::kSteps; ++j) {
          const int d = p * 4 * S::kTB + t * S::kTB + j * 4;
          uint2 x = make_uint2(0u, 0u);
          if (g < here && d < a.dk) x = *reinterpret_cast<const uint2*>(row + d);
          qf[nt][p * S::kSteps + j][0] = x.x;
          qf[nt][p * S::kSteps + j][1] = x.y;
          if (kE4m3) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t w = e ? x.y : x.x;
              const float lo = fabsf(__uint_as_float(w << 16)), hi = fabsf(__uint_as_float(w & 0xffff0000u));
              if (lo < INFINITY) top = fmaxf(top, lo);
              if (hi < INFINITY) top = fmaxf(top, hi);
            }
          }
        }
      float f = a.scale_log2;
      if (kE4m3) {
        // f16 for the products with e4m3 keys (exact in it): a row of q times a power of two that brings its largest value to 2^14
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = max((int)(__float_as_uint(top) >> 23), 14) - 127;    // (subnormal rows: as the smallest normal ones, whose 2^(14 - e) is still a float)
        const float up = __uint_as_float((uint32_t)(min(14 - e, 127) + 127) << 23);
#pragma unroll
        for (int i = 0; i < S::kKP * S::kSteps; ++i)
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint32_t x = qf[nt][i][w];
            const __half2 h = __floats2half2_rn(__uint_as_float(x << 16) * up, __uint_as_float(x & 0xffff0000u) * up);
            qf[nt][i][w] = *reinterpret_cast<const uint32_t*>(&h);
          }
        f = 1.f / up;
      }
      // the lane's results are those of heads 2t and 2t + 1
      factor[nt][0] = kE4m3 ? a.scale_log2 * __shfl_sync(0xffffffffu, f, 8 * t) : f;
      factor[nt][1] = kE4m3 ? a.scale_log2 * __shfl_sync(0xffffffffu, f, 8 * t + 4) : f;
    }

    float o[NT][kMT][4], ml[NT][2], mo[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < kMT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
      ml[nt][0] = ml[nt][1] = mo[nt][0] = mo[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
    }

    const int32_t* const pages = a.table + (long long)seq * a.per_sequence;
    // rows of a chunk's keys, key i with lane i % 32; -1: not there
    auto rows_of = [&](int step, int (&row)[S::kIndexes]) {
#pragma unroll
      for (int i = 0; i < S::kIndexes; ++i) {
        const int m = (step * kWarps + warp) * S::kKeys + i * 32 + lane;
        row[i] = -1;
        if (step < j1 && m < n && (S::kKeys >= 32 || lane < S::kKeys)) {
          const int index = (int)((unsigned long long)(uint32_t)m * a.slots_mul >> a.slots_shift);
          const int page = pages[index];
          if (page >= 0 && page < a.pages) row[i] = page * a.rows_page + (m - index * a.slots) * a.row_slot + head * a.row_head;
          else atomicExch(&g_bad_page, 1);
        }
      }
    };
    uint4 kr[S::kTiles][2][S::kKP];
    VT vr[S::kTiles][4][S::kVP];
    float ksr[S::kTiles][2], vsr[S::kTiles][2];
    auto load_k = [&](const int (&row)[S::kIndexes]) {
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = c * 16 + e * 8;
          const int x = __shfl_sync(0xffffffffu, row[key / 32], key % 32 + r);
          const uint8_t* const p = a.k + (long long)x * a.dk * S::kElt + t * 16;
#pragma unroll
          for (int i = 0; i < S::kKP; ++i) {
            kr[c][e][i] = make_uint4(0u, 0u, 0u, 0u);
            if (x >= 0 && (i * 4 + t) * S::kTB < a.dk) kr[c][e][i] = load16(p + i * 64);
          }
          if (kE4m3) ksr[c][e] = x >= 0 ? a.ks[x] : 0.f;
        }
    };
    auto load_v = [&](const int (&row)[S::kIndexes]) {
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = c * 16 + (e >> 1) * 8 + (e & 1);
          const int x = __shfl_sync(0xffffffffu, row[key / 32], key % 32 + 2 * t);
          const uint8_t* const p = a.v + ((long long)x * a.dv + r * S::kVB) * S::kElt;
#pragma unroll
          for (int i = 0; i < S::kVP; ++i) {
            const bool in = x >= 0 && (i * 8 + r) * S::kVB < a.dv;
            if constexpr (sizeof(VT) == 16) {
              vr[c][e][i] = make_uint4(0u, 0u, 0u, 0u);
              if (in) vr[c][e][i] = load16(p + i * 128);
            } else {
              vr[c][e][i] = make_uint2(0u, 0u);
              if (in) vr[c][e][i] = load8(p + i * 64);
            }
          }
        }
      if (kE4m3)
#pragma unroll
        for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int key = c * 16 + e * 8;
            const int x = __shfl_sync(0xffffffffu, row[key / 32], key % 32 + r);
            vsr[c][e] = x >= 0 ? a.vs[x] : 0.f;
          }
    };

    int row[S::kIndexes], next[S::kIndexes];
    rows_of(j0, row);
    load_k(row);
    load_v(row);
    rows_of(j0 + 1, next);
    for (int step = j0; step < j1; ++step) {
      // ---- logits
      float s[S::kTiles][NT][4];
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[c][nt][0] = s[c][nt][1] = s[c][nt][2] = s[c][nt][3] = 0.f;
#pragma unroll
        for (int p = 0; p < S::kKP; ++p)
#pragma unroll
          for (int j = 0; j < S::kSteps; ++j) {
            uint32_t a0, a1, a2, a3;
            if (kE4m3) {
              const uint32_t x = word(kr[c][0][p], j), y = word(kr[c][1][p], j);
              a0 = halves(x); a2 = halves(x >> 16);
              a1 = halves(y); a3 = halves(y >> 16);
            } else {
              a0 = word(kr[c][0][p], 2 * j); a2 = word(kr[c][0][p], 2 * j + 1);
              a1 = word(kr[c][1][p], 2 * j); a3 = word(kr[c][1][p], 2 * j + 1);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma<kE4m3>(s[c][nt], a0, a1, a2, a3, qf[nt][p * S::kSteps + j][0], qf[nt][p * S::kSteps + j][1]);
          }
      }
      // in the scale of exp2; keys that are not there -infinity
      float tv[S::kTiles][2];                        // e4m3: log2 of the scale of V's row
      float xl[NT][2], xo[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) xl[nt][0] = xl[nt][1] = xo[nt][0] = xo[nt][1] = -INFINITY;
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = c * 16 + e * 8;
          const bool in = __shfl_sync(0xffffffffu, row[key / 32], key % 32 + r) >= 0;
          if (kE4m3) tv[c][e] = __log2f(vsr[c][e]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float x = s[c][nt][2 * e + h] * factor[nt][h];
              if (kE4m3) x *= ksr[c][e];
              if (!in) x = -INFINITY;
              s[c][nt][2 * e + h] = x;
              xl[nt][h] = fmaxf(xl[nt][h], x);
              if (kE4m3) xo[nt][h] = fmaxf(xo[nt][h], in ? x + tv[c][e] : -INFINITY);
            }
        }
      load_k(next);                                  // K of this chunk is used up
      bool rise = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          rise |= xl[nt][h] > ml[nt][h] + kSlack;
          if (kE4m3) rise |= xo[nt][h] > mo[nt][h] + kSlack;
        }
      if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float x = xl[nt][h], y = xo[nt][h];
#pragma unroll
            for (int w = 4; w < 32; w *= 2) {
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, w));
              if (kE4m3) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, w));
            }
            const float m = fmaxf(ml[nt][h], x);
            const float f = ml[nt][h] == -INFINITY ? 0.f : ex2(ml[nt][h] - m);
            l[nt][h] *= f;
            ml[nt][h] = m;
            float g = f;
            if (kE4m3) {
              const float w = fmaxf(mo[nt][h], y);
              g = mo[nt][h] == -INFINITY ? 0.f : ex2(mo[nt][h] - w);
              mo[nt][h] = w;
            }
#pragma unroll
            for (int i = 0; i < kMT; ++i) {
              o[nt][i][h] *= g;
              o[nt][i][2 + h] *= g;
            }
          }
      }
      // ---- weights
      uint32_t pb[S::kTiles][NT][2];
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float x = s[c][nt][2 * e + h], m = ml[nt][h] == -INFINITY ? 0.f : ml[nt][h];
              float w = ex2(x - m);
              l[nt][h] += w;
              if (kE4m3) {
                const float m2 = mo[nt][h] == -INFINITY ? 0.f : mo[nt][h];
                w = x == -INFINITY ? 0.f : ex2(x + tv[c][e] - m2 + kLift);
              }
              p[2 * e + h] = w;
            }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t two;
            if (kE4m3) {
              const __half2 x = __floats2half2_rn(p[2 * e], p[2 * e + 1]);
              two = *reinterpret_cast<const uint32_t*>(&x);
            } else {
              const __nv_bfloat162 x = __floats2bfloat162_rn(p[2 * e], p[2 * e + 1]);
              two = *reinterpret_cast<const uint32_t*>(&x);
            }
            pb[c][nt][e] = transposed(two);
          }
        }
      // ---- weights . v
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
        for (int p = 0; p < S::kVP; ++p)
#pragma unroll
          for (int w = 0; w < (int)sizeof(VT) / 4; ++w) {
            const uint32_t x0 = word(vr[c][0][p], w), x1 = word(vr[c][1][p], w), x2 = word(vr[c][2][p], w), x3 = word(vr[c][3][p], w);
#pragma unroll
            for (int i = 0; i < (kE4m3 ? 2 : 1); ++i) {
              uint32_t y0 = x0, y1 = x1, y2 = x2, y3 = x3;
              if (kE4m3) { y0 = halves(x0 >> (16 * i)); y1 = halves(x1 >> (16 * i)); y2 = halves(x2 >> (16 * i)); y3 = halves(x3 >> (16 * i)); }
              const uint32_t a0 = prmt(y0, y1, 0x5410), a1 = prmt(y0, y1, 0x7632), a2 = prmt(y2, y3, 0x5410), a3 = prmt(y2, y3, 0x7632);
              const int tile = p * (S::kVB / 2) + w * (kE4m3 ? 2 : 1) + i;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma<kE4m3>(o[nt][tile], a0, a1, a2, a3, pb[c][nt][0], pb[c][nt][1]);
            }
          }
      load_v(next);
#pragma unroll
      for (int i = 0; i < S::kIndexes; ++i) row[i] = next[i];
      rows_of(step + 2, next);
    }

    // ---- the four warps' sums, in order
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x = l[nt][h];
#pragma unroll
        for (int w = 4; w < 32; w *= 2) x += __shfl_xor_sync(0xffffffffu, x, w);
        const int g = nt * 8 + 2 * t + h;
        if (r == 0) {
          ss[warp][g][0] = ml[nt][h];
          ss[warp][g][1] = x;
          ss[warp][g][2] = kE4m3 ? mo[nt][h] - kLift : ml[nt][h];
        }
#pragma unroll
        for (int i = 0; i < kMT; ++i) {
          constexpr int kHalfPiece = S::kVB / 2;
          const int d = (i / kHalfPiece) * 8 * S::kVB + r * S::kVB + (i % kHalfPiece) * 2;
          *reinterpret_cast<float2*>(&so[warp][g][d]) = make_float2(o[nt][i][h], o[nt][i][2 + h]);
        }
      }
    __syncthreads();
    for (int i = tid; i < kHeads * (DC / 2); i += kThreads) {
      const int g = i / (DC / 2), d = 2 * (i % (DC / 2));
      float top_l = -INFINITY, top_o = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        top_l = fmaxf(top_l, ss[w][g][0]);
        top_o = fmaxf(top_o, ss[w][g][2]);
      }
      float sum = 0.f, x = 0.f, y = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (ss[w][g][0] != -INFINITY || ss[w][g][1] != 0.f) sum += ss[w][g][1] * (ss[w][g][0] == top_l ? 1.f : ex2(ss[w][g][0] - top_l));
        const float f = ss[w][g][2] == top_o ? 1.f : ex2(ss[w][g][2] - top_o);
        const float2 v = *reinterpret_cast<const float2*>(&so[w][g][d]);
        x += v.x * f;
        y += v.y * f;
      }
      if (whole) {
        if (g < here && d < a.dv) {
          const float f = sum == 0.f ? 0.f : (kE4m3 ? ex2(top_o - top_l) : 1.f) / sum;
          __nv_bfloat162* const to = reinterpret_cast<__nv_bfloat162*>(a.o + ((((long long)seq * a.heads + head) * a.group + g0 + g) * a.dv + d));
          *to = __floats2bfloat162_rn(sum == 0.f ? 0.f : x * f, sum == 0.f ? 0.f : y * f);
        }
      } else {
        *reinterpret_cast<float2*>(a.part_o + ((long long)slot * kHeads + g) * DC + d) = make_float2(x, y);
        if (d == 0) *reinterpret_cast<float4*>(a.part_s + ((long long)slot * kHeads + g) * 4) = make_float4(top_l, sum, top_o, 0.f);
      }
    }
    __syncthreads();
  }
}

// Joins the parts of the item that starts last in block b and goes on behind it: one in b, and the first of every block up to the item's last.
template <int kHeads, int DC>
__global__ void __launch_bounds__(256) attention_decode_join_kernel(const Args a) {
  mtf::chain_wait_only();
  const int4 piece = a.pieces[blockIdx.x];
  if (piece.x < 0) return;
  const int head = piece.y / a.chunks, g0 = (piece.y - head * a.chunks) * kHeads;
  const int here = min(kHeads, a.group - g0);
  for (int i = threadIdx.x; i < here * (a.dv / 2); i += 256) {
    const int g = i / (a.dv / 2), d = 2 * (i % (a.dv / 2));
    float top_l = -INFINITY, top_o = -INFINITY, sum = 0.f, x = 0.f, y = 0.f;
    for (int b = blockIdx.x; b <= piece.z; ++b) {
      const long long at = (long long)(b == (int)blockIdx.x ? piece.w : 2 * b) * kHeads + g;
      const float4 s = *reinterpret_cast<const float4*>(a.part_s + at * 4);
      const float2 v = *reinterpret_cast<const float2*>(a.part_o + at * DC + d);
      const float ml = fmaxf(top_l, s.x), mo = fmaxf(top_o, s.z);
      const float f0 = top_l == ml ? 1.f : ex2(top_l - ml), f1 = s.x == ml ? 1.f : ex2(s.x - ml);
      const float e0 = top_o == mo ? 1.f : ex2(top_o - mo), e1 = s.z == mo ? 1.f : ex2(s.z - mo);
      sum = sum * f0 + s.y * f1;
      x = x * e0 + v.x * e1;
      y = y * e0 + v.y * e1;
      top_l = ml;
      top_o = mo;
    }
    const float f = sum == 0.f ? 0.f : (top_o == top_l ? 1.f : ex2(top_o - top_l)) / sum;
    __nv_bfloat162* const to = reinterpret_cast<__nv_bfloat162*>(a.o + ((((long long)piece.x * a.heads + head) * a.group + g0 + g) * a.dv + d));
    *to = __floats2bfloat162_rn(sum == 0.f ? 0.f : x * f, sum == 0.f ? 0.f : y * f);
  }
}

int width_class(const mtf::CachePool& c) {
  const int d = std::max(c.dk, c.dv);
  return d <= 64 ? 64 : d <= 128 ? 128 : 256;
}
int tiles_of_heads(const mtf::CachePool& c, int group) { return group > 8 && width_class(c) < 256 ? 2 : 1; }
int blocks_an_sm(int dc, int nt) { return dc == 256 || (nt > 1 && dc == 128) ? 2 : 3; }

// Items of at most this many positions are not cut: a block takes one whole.
constexpr long long kWholeItem = 256;

int unit_keys(const mtf::CachePool& c) {
  const int row = width_class(c) * (c.e4m3 ? 1 : 2);
  return kWarps * 16 * (row <= 64 ? 4 : row <= 128 ? 2 : 1);
}
// (the sum of all sequences' units is kept in 32 bits)
bool balanced(const mtf::CachePool& c) {
  const long long most = (long long)c.per_sequence * c.slots;
  return c.sequences <= kPlanned && most > kWholeItem && c.sequences * (most / unit_keys(c) + 1) < (1LL << 31);
}
int grid_of(const mtf::CachePool& c, int group) {
  const int nt = tiles_of_heads(c, group), chunks = (group + 8 * nt - 1) / (8 * nt);
  const long long most = (long long)mtf::device_sm_count() * blocks_an_sm(width_class(c), nt);
  const long long units = c.sequences * c.heads * chunks * (((long long)c.per_sequence * c.slots + unit_keys(c) - 1) / unit_keys(c));
  return (int)std::max(1LL, std::min(most, units / kLeastUnits));
}

template <bool kE4m3, int DC, int NT>
void launch(const Args& a, int grid, cudaStream_t st) {
  mtf::launch_chained(attention_decode_kernel<kE4m3, DC, NT>, (unsigned)grid, kThreads, 0, st, a);
  mtf::count_launch();
  if (a.balanced && grid > 1) {
    mtf::launch_chained(attention_decode_join_kernel<8 * NT, DC>, (unsigned)grid - 1, 256, 0, st, a);
    mtf::count_launch();
  }
}
template <bool kE4m3>
void dispatch(const Args& a, int dc, int nt, int grid, cudaStream_t st) {
  if (dc == 256) launch<kE4m3, 256, 1>(a, grid, st);
  else if (dc == 128) nt == 1 ? launch<kE4m3, 128, 1>(a, grid, st) : launch<kE4m3, 128, 2>(a, grid, st);
  else nt == 1 ? launch<kE4m3, 64, 1>(a, grid, st) : launch<kE4m3, 64, 2>(a, grid, st);
}

}  // namespace

namespace mtf {

size_t attention_decode_workspace(const CachePool& c, int group) {
  if (!balanced(c)) return 0;
  const size_t grid = grid_of(c, group), heads = 8 * tiles_of_heads(c, group);
  return grid * 2 * heads * (width_class(c) + 4) * sizeof(float) + grid * sizeof(int4);
}

mtf_status launch_attention_decode(const CachePool& c, const DecodeCall& d, void* stream) {
  const int dc = width_class(c), nt = tiles_of_heads(c, d.group);
  Args a = {};
  a.q = reinterpret_cast<const __nv_bfloat16*>(d.q);
  a.k = reinterpret_cast<const uint8_t*>(c.k);
  a.v = reinterpret_cast<const uint8_t*>(c.v);
  a.ks = c.ks;
  a.vs = c.vs;
  a.table = c.table;
  a.lengths = d.lengths;
  a.o = reinterpret_cast<__nv_bfloat16*>(d.o);
  a.n_seq = (int)c.sequences;
  a.heads = c.heads;
  a.group = d.group;
  a.chunks = (d.group + 8 * nt - 1) / (8 * nt);
  a.dk = c.dk;
  a.dv = c.dv;
  a.pages = c.pages;
  a.slots = c.slots;
  a.per_sequence = c.per_sequence;
  a.rows_page = c.rows_page;
  a.row_slot = c.row_slot;
  a.row_head = c.row_head;
  // with 2^n >= slots > 2^(n - 1) the factor ceil(2^(31 + n) / slots) is below 2^32 and off by less than 2^n in 2^(31 + n): exact for m < 2^31
  int n = 0;
  while ((1LL << n) < c.slots) ++n;
  a.slots_mul = (uint32_t)(((1ULL << (31 + n)) + c.slots - 1) / c.slots);
  a.slots_shift = 31 + n;
  a.scale_log2 = d.scale * kLog2e;
  a.balanced = balanced(c);
  long long grid = a.balanced ? grid_of(c, d.group) : c.sequences * c.heads * a.chunks;
  if (grid > 0x7fffffffLL) return fail(MTF_ERR_UNSUPPORTED, "attention_decode: at most 2^31 heads of sequences");
  if (a.balanced) {
    const size_t heads = 8 * nt;
    a.pieces = reinterpret_cast<int4*>(d.workspace);
    a.part_s = reinterpret_cast<float*>(a.pieces + grid);
    a.part_o = a.part_s + (size_t)grid * 2 * heads * 4;
  }
  if (c.e4m3) dispatch<true>(a, dc, nt, (int)grid, (cudaStream_t)stream);
  else dispatch<false>(a, dc, nt, (int)grid, (cudaStream_t)stream);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "attention_decode_kernel: %s", cudaGetErrorString(e));
  return MTF_OK;
}

// 1 when a page outside the pool or a length beyond the table was met since the last call; resets the flag
mtf_status read_decode_bad_page(int* seen) {
  int v = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_bad_page, sizeof(int));
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "cudaMemcpyFromSymbol: %s", cudaGetErrorString(e));
  if (v) { int z = 0; cudaMemcpyToSymbol(g_bad_page, &z, sizeof(int)); }
  *seen = v;
  return MTF_OK;
}

}  // namespace mtf
