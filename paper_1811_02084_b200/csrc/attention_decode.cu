// Attention of one new token a sequence over a paged cache:
//     o[s, h, g, :] = sum_m p_m v[m, h, :],   p = softmax over m < n_s of scale * q[s, h, g, :] . k[m, h, :]
// where position m of sequence s lies in page table[s][m / slots], slot m % slots.
//
// Every row of the cache is read once and used for up to 16 heads of queries (8 for rows of more than 128 values; a larger group's further heads read it again, where L2 may still have it), 2 to 4 flops a
// byte and head: HBM is the bound, and the products only have to keep out of its way.  So a warp is a stream of its own: it has chunks of 16 (or 32, 64) rows of K and of V, 8 KB, copied by TMA into a
// ring of its own and waits for nobody but them; there is no block barrier in the loop, and each warp keeps its own running maximum and sums.  With the
// rows of the cache as the instruction's 16 rows and the heads as its 8 columns, eight heads of queries cost no more than one and nothing is padded to 16:
//     S^T [16 keys x 8 heads] = K [16 x d] q^T [d x 8],   O^T [d x 8 heads] += V^T [d x 16 keys] P^T [16 keys x 8]
// The order of a sum's terms is free, so a lane reads 16 bytes of a row at a time and what it has of d, and of the keys, is what it multiplies; V's pairs of keys are put together by
// byte permutes.  (64 sequences of up to 4096 positions in bf16, 1.1 GB, whole call: loads into registers 252 us, copies by the lanes into shared memory 244, TMA 199,
// of warps that look the pages up a step ahead and join in fours 180: 6.2 TB/s.  4 sequences of up to 65536 in e4m3, 0.4 GB: 74 to 77, half of the issue slots used, a third of them to
// make f16 of e4m3, and 5 for joining.)
//
// What is shared out are units, 64 to 256 keys of an item (a sequence's head) that the block's warps take a chunk each: a block or a cluster of blocks an item, or, where sequences may be
// long, the units of all items end to end and an equal run of them for every block, whatever the lengths (plan_of has the rule and what was measured).  Items that cross a block's edge are left
// as partial sums then, and joined behind the launch, in order.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <mutex>

#include "answer.cuh"
#include "answer.h"
#include "launch.cuh"

namespace {

using mtf::cluster_barrier;
using mtf::ex2;
using mtf::far;
using mtf::far2;
using mtf::in_block;
using mtf::kLandCycles;
using mtf::kWaitCycles;
using mtf::landed;
using mtf::landed_late;
using mtf::smem_at;

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kPlanned = 1024;        // sequences whose units a block adds up by itself, eight a thread; more of them have items enough for a block each
constexpr int kFewSteps = 8, kLoneSteps = 11;      // units a block of a cluster, and one by itself: plan_of
constexpr int kMostBlocks = 8;        // of a cluster
constexpr int kOver = 3;              // units that an item costs beside its own: first loads, joining
constexpr int kLeastCost = 5;         // a block's run
constexpr float kLog2e = 1.4426950408889634f;
// The running maximum is raised only where a logit lies 2^6 above it: otherwise every chunk would pay for a maximum across lanes.
constexpr float kSlack = 6.f;
// e4m3: the weights are f16, and a weight of 1 is held as 2^9, so that with the slack they stay below 2^16 and those of 2^-23 keep all of f16's digits.
constexpr float kLift = 9.f;

struct Args {
  const __nv_bfloat16* q;
  const float *ks, *vs;
  const int32_t *table, *lengths;
  __nv_bfloat16* o;
  int n_seq, heads, group, chunks, dk, dv;       // chunks: of the group, 8 NT heads each
  int pages, slots, per_sequence, rows_page, row_slot, row_head;
  uint32_t slots_mul;                            // m / slots = (m * slots_mul) >> slots_shift in 64 bits, for m below 2^31
  int slots_shift;
  float scale_log2;
  int box_rows;                                  // keys of a copied box: a power of two up to 16 that divides a page's slots
  int balanced;                                  // all blocks share all units evenly; else an item is one cluster's
  int cluster;
  float* part_o;                                 // [block][2][8 NT][DC]
  float* part_s;                                 // [block][2][8 NT][4]: reference of l, l, reference of o
  int4* pieces;                                  // [block]: of the item that starts last in it and goes on: sequence, head and chunk, its last block, slot
};

__device__ int g_bad_page = 0;                   // a page id outside the pool, or a length beyond the table, was seen

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t s) { return __byte_perm(a, b, s); }
// four e4m3 values as f16 (exact), two and two
__device__ __forceinline__ void halves(uint32_t four, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(four));
}
// (neither these nor the products touch memory, and no lane leaves the loop early: the compiler may move them)
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool kHalf>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (kHalf)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word(const uint2& v, int i) { return i == 0 ? v.x : v.y; }

template <bool kE4m3, int DC>
struct Shape {
  static constexpr int kElt = kE4m3 ? 1 : 2;
  static constexpr int kTiles = DC * kElt <= 64 ? 4 : DC * kElt <= 128 ? 2 : 1;     // 16-key tiles of a chunk: 4 KB of K and of V (bf16 rows of 256: 8)
  static constexpr int kKeys = 16 * kTiles;
  static constexpr int kIndexes = (kKeys + 31) / 32;
  static constexpr int kTB = 16 / kElt;              // K: values of a lane's 16 bytes
  static constexpr int kKP = DC / (4 * kTB);         // ... pieces of a row
  static constexpr int kSteps = kTB / 4;             // ... products of a piece, 16 deep
  static constexpr int kVB = kE4m3 && DC == 64 ? 8 : kTB;   // V: values of a lane's piece (8 lanes a row)
  static constexpr int kVP = DC / (8 * kVB);
  static constexpr int kRow = DC * kElt < 128 ? DC * kElt : 128;      // bytes of a box's rows
  static constexpr int kBoxes = DC * kElt / kRow;    // ... beside each other for a whole row
  static constexpr int kSide = kTiles * kBoxes * 16 * kRow;           // bytes of a chunk of K, and of V
  static constexpr int kStage = 2 * kSide;
  static constexpr int kStages = kStage > 8192 ? 3 : 2;
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr int kBlocks = kStage > 8192 ? 1 : 3;               // an SM holds
};
template <int kBytes> struct Piece { using T = uint4; };
template <> struct Piece<8> { using T = uint2; };

// Which key of a tile is the i-th row of a product, and which 16 bytes of V's 128 are lane group r's: free choices, since the order of a sum's terms and of the
// results' rows is, made so that the lanes that shared memory serves together find their pieces in different banks.  A copy puts piece j of row k at j ^ (k % 8)
// (rows of 64 bytes: at j ^ (k / 2 % 4)).  K: lanes (r, t) of two neighbouring r read pieces t of rows key(r), which have to differ in bit 2 (64 bytes: in bit
// 0); V: they read pieces piece(r) of the rows key(2t).
template <int kRow>
__device__ __forceinline__ int key_of_row(int i) {
  return kRow == 128 ? (i & 8) | (i & 1) << 2 | (i >> 1 & 3) : (i & 8) | (((i >> 1 & 1) << 2 | (i >> 2 & 1)) ^ (i & 1 ? 3 : 0));
}
template <int kRow>
__device__ __forceinline__ int swizzled(int key, int piece) { return kRow == 128 ? piece ^ (key & 7) : piece ^ (key >> 1 & 3); }

__device__ int g_decode_status = 0;                  // a wait was given up
__constant__ long long g_wait_limit = kWaitCycles;
__constant__ int g_withhold = 0;                     // testing: each warp's first wait asks for a copy that nobody has sent
__device__ __forceinline__ void copy_box(uint32_t to, const CUtensorMap* map, int d, int slot, int head, int page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to), "l"(map), "r"(d), "r"(slot),
               "r"(head), "r"(page), "r"(bar)
               : "memory");
}

// What a weighted sum relative to 2^top_o is multiplied by, one factor after the other, where the weights' sum is relative to 2^top_l.  8-bit rows of V may have scales down to the smallest float, and
// the reference lies 2^-9 below them (kLift), where ex2 gives 0: what lies below 2^-60 is a factor of its own.  (bf16: the references are equal, and the factors 1 / sum and 1.)
__device__ __forceinline__ float2 last_factors(float top_o, float top_l, float sum) {
  constexpr float kFar = -60.f;                    // (1 / sum is above 2^-40)
  const float e = top_o == top_l ? 0.f : top_o - top_l;
  return make_float2(ex2(fmaxf(e, kFar)) / sum, ex2(fminf(e - kFar, 0.f)));
}

// first unit of block c, of `units` over `blocks`
__device__ __forceinline__ long long first_unit(long long units, int blocks, int c) { return units * c / blocks; }

template <bool kE4m3, int DC, int NT>
__global__ void __launch_bounds__(kThreads, Shape<kE4m3, DC>::kBlocks) attention_decode_kernel(const Args a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = Shape<kE4m3, DC>;
  using VT = typename Piece<S::kVB * S::kElt>::T;
  constexpr int kUnit = kWarps * S::kKeys, kHeads = 8 * NT, kMT = DC / 16;
  extern __shared__ uint8_t room[];
  uint8_t* const ring = room + (-smem_at(room) & 1023);      // each warp's stages; behind the loop, the warps' results
  float(*const so)[kHeads][DC + 4] = reinterpret_cast<float(*)[kHeads][DC + 4]>(ring);
  __shared__ float ring_scale[kE4m3 ? kWarps : 1][S::kStages][2][kE4m3 ? S::kKeys : 1];
  __shared__ __align__(8) uint64_t bars[kWarps][S::kStages];
  __shared__ int cum[kPlanned + 1];
  __shared__ int warp_total[kWarps];
  __shared__ float ss[kWarps + 1][kHeads][3];        // (the last: the block's)
  float(*const block_o)[DC + 4] = so[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, t = lane & 3;
  if (lane == 0) {
    for (int i = 0; i < S::kStages; ++i) mtf::landing_init(&bars[warp][i]);
    mtf::landing_ready();
  }
  __syncwarp();
  mtf::chain_wait();
  const int H = a.heads * a.chunks;
  const int capacity = (int)min((long long)a.per_sequence * a.slots, 0x7fffffffLL);
  auto cost_of = [&](int n) { return n ? (n + kUnit - 1) / kUnit + kOver : 0; };
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
      if (s0 + i < a.n_seq) sum += cost_of(length_of(s0 + i));
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
        before += cost_of(length_of(s0 + i));
        if (s0 + i == a.n_seq - 1) cum[a.n_seq] = before;
      }
    __syncthreads();
    units = (long long)cum[a.n_seq] * H;
    // (no block without a unit among those that share them: a join goes from block to block)
    blocks = (int)min((long long)blocks, max(1LL, units / kLeastCost));
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

  // where this warp reads: its lanes' rows of K, its pieces of V's even and odd rows
  const uint8_t* const mine = ring + warp * S::kStages * S::kStage;
  const int key_r = key_of_row<S::kRow>(r);
  const int at_k = key_r * S::kRow + swizzled<S::kRow>(key_r, t) * 16;
  const int piece = S::kRow == 128 ? (r & 1) << 2 | r >> 1 : r;
  int at_v[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int key = key_of_row<S::kRow>(2 * t + e);
    at_v[e] = key * S::kRow + (sizeof(VT) == 16 ? swizzled<S::kRow>(key, piece) * 16 : swizzled<S::kRow>(key, piece >> 1) * 16 + (piece & 1) * 8);
  }
  uint32_t into = 0, from = 0;                       // the stage that is filled next, and the one that is used next; bit 8: the parity of its barrier's phase
  bool gone = false;                                 // a wait was given up: no keys from there on
  auto onward = [](uint32_t x) { return (x & 255) + 1 == S::kStages ? (x & 256) ^ 256 : x + 1; };

  for (long long u = u0; u < u1;) {
    // ---- the item, and the part of it that is this block's
    int seq, hc, j0, j1, n;
    bool whole;
    int slot = 0;
    if (a.balanced) {
      const int x = (int)(u / H);                   // (units of a sequence's heads lie one behind another: 182 us; of a head's sequences: 184)
      int lo = 0, hi = a.n_seq;                     // the last sequence with cum <= x
      while (hi - lo > 1) {
        const int m = (lo + hi) / 2;
        if (cum[m] <= x) lo = m; else hi = m;
      }
      seq = lo;
      const int each = cum[seq + 1] - cum[seq];
      const long long in = u - (long long)cum[seq] * H;
      hc = (int)(in / each);
      const int x0 = (int)(in - (long long)hc * each), x1 = (int)min((long long)each, x0 + (u1 - u));
      j0 = max(0, x0 - kOver);
      j1 = max(0, x1 - kOver);
      whole = j0 == 0 && j1 == each - kOver;
      slot = 2 * blockIdx.x + (u == u0 ? 0 : 1);
      const long long end = u - x0 + each;           // behind the item
      u += x1 - x0;
      if (j0 == j1) continue;
      if (tid == 0 && j0 == 0 && !whole) a.pieces[blockIdx.x] = make_int4(seq, hc, (int)((end * blocks - 1) / units), slot);
      n = length_of(seq);
    } else {
      const int item = blockIdx.x / a.cluster, rank = blockIdx.x - item * a.cluster;
      seq = item / H;
      hc = item - seq * H;
      n = length_of(seq);
      const long long each = (n + kUnit - 1) / kUnit;
      j0 = (int)(each * rank / a.cluster);
      j1 = (int)(each * (rank + 1) / a.cluster);
      whole = a.cluster == 1;
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
        // f16 for the products with e4m3 keys, which are exact in it: a row of q times a power of two that brings its largest value to 2^14.  (bf16's digits all fit for values down to 2^-31 of the
        // largest; what is smaller loses some of them, 2^-39 of the largest at most.)
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
      // (a factor beyond f32 stays finite: a product of 0 stays 0, and others are as far apart as weights can tell)
      if (kE4m3)
#pragma unroll
        for (int h = 0; h < 2; ++h) factor[nt][h] = fminf(fmaxf(factor[nt][h], -FLT_MAX), FLT_MAX);
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
    auto page_of = [&](int m) { return (int)((unsigned long long)(uint32_t)m * a.slots_mul >> a.slots_shift); };
    // The keys of a step's chunk, key i with lane i % 32: their pages' ids, asked for a step before they are needed.
    auto ask_pages = [&](int step, int (&page)[S::kIndexes]) {
#pragma unroll
      for (int i = 0; i < S::kIndexes; ++i) {
        const int m = (step * kWarps + warp) * S::kKeys + i * 32 + lane;
        page[i] = 0;
        if (step < j1 && m < n && (S::kKeys >= 32 || lane < S::kKeys)) page[i] = pages[page_of(m)];
      }
    };
    // Chunks come as boxes of box_rows keys by kRow bytes, which no page's end cuts; lane i asks for boxes i, i + 32, ..  Keys without a place (behind the
    // last, or of a page that is none) come as zeros, from a page behind the pool, and have no bit in the mask.
    const int boxes = S::kKeys / a.box_rows * 2 * S::kBoxes;
    auto fetch = [&](int step, const int (&asked)[S::kIndexes], uint32_t (&there)[S::kIndexes]) {
      const uint32_t bar = smem_at(&bars[warp][into & 255]), to = smem_at(mine) + (into & 255) * S::kStage;
      const int m0 = (step * kWarps + warp) * S::kKeys;
      int page[S::kIndexes];
#pragma unroll
      for (int i = 0; i < S::kIndexes; ++i) {
        bool in = m0 + i * 32 + lane < n && (S::kKeys >= 32 || lane < S::kKeys);
        if (in && (uint32_t)asked[i] >= (uint32_t)a.pages) {
          atomicExch(&g_bad_page, 1);
          in = false;
        }
        page[i] = in ? asked[i] : a.pages;
        there[i] = __ballot_sync(0xffffffffu, in);
      }
      if (lane == 0) mtf::expect(bar, S::kStage);
      __syncwarp();
      for (int i0 = 0; i0 < boxes; i0 += 32) {
        const int i = min(i0 + lane, boxes - 1), key = i / (2 * S::kBoxes) * a.box_rows, side = i / S::kBoxes & 1, box = i % S::kBoxes;
        int pg = __shfl_sync(0xffffffffu, page[0], key & 31);
        if (S::kIndexes > 1) {
          const int pg1 = __shfl_sync(0xffffffffu, page[S::kIndexes - 1], key & 31);
          pg = key >= 32 ? pg1 : pg;
        }
        const int m = m0 + key;
        if (i0 + lane < boxes)
          copy_box(to + side * S::kSide + (((key >> 4) * S::kBoxes + box) * 16 + (key & 15)) * S::kRow, side ? &map_v : &map_k, box * (S::kRow / S::kElt),
                   m - page_of(m) * a.slots, head, pg, bar);
      }
      if (kE4m3) {
        // scales, a key a lane
#pragma unroll
        for (int i = 0; i < S::kIndexes; ++i)
          if (S::kKeys >= 32 || lane < S::kKeys) {
            const int key = i * 32 + lane, m = m0 + key;
            const bool in = there[i] >> lane & 1;
            const int row = in ? page[i] * a.rows_page + (m - page_of(m) * a.slots) * a.row_slot + head * a.row_head : 0;
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_at(&ring_scale[warp][into & 255][0][key])), "l"(a.ks + row), "r"(in ? 4 : 0) : "memory");
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_at(&ring_scale[warp][into & 255][1][key])), "l"(a.vs + row), "r"(in ? 4 : 0) : "memory");
          }
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
      into = onward(into);
    };
    int page[S::kIndexes];
    uint32_t there[S::kStages][S::kIndexes];         // of the stages, the oldest first
    if (!gone) {
      int first[S::kStages][S::kIndexes];
#pragma unroll
      for (int i = 0; i < S::kStages; ++i) ask_pages(j0 + i, first[i]);
#pragma unroll
      for (int i = 0; i < S::kStages; ++i)
        if (j0 + i < j1) fetch(j0 + i, first[i], there[i]);
        else if (kE4m3) asm volatile("cp.async.commit_group;" ::: "memory");
      ask_pages(j0 + S::kStages, page);
    }
    for (int step = j0; step < j1 && !gone; ++step) {
      const uint32_t bar = smem_at(&bars[warp][from & 255]), phase = from >> 8;
      if (!landed(bar, phase, g_wait_limit) || (g_withhold && !landed(bar, phase ^ 1, g_wait_limit))) {
        if (lane == 0) atomicCAS(&g_decode_status, 0, 0xB01);
        gone = true;
        for (uint32_t i = from; i != into; i = onward(i)) landed_late(smem_at(&bars[warp][i & 255]), i >> 8, kLandCycles);
        break;
      }
      if (kE4m3) {
        asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 1) : "memory");
        __syncwarp();
      }
      uint8_t* const stage = ring + warp * S::kStages * S::kStage + (from & 255) * S::kStage;
      bool here_all = true;                          // no key is left out
#pragma unroll
      for (int i = 0; i < S::kIndexes; ++i) here_all &= there[0][i] == (S::kKeys < 32 ? (1u << (S::kKeys & 31)) - 1u : 0xffffffffu);
      if (!here_all) {
        // slots behind the last position may hold anything: zeros in their rows of V, which weights of 0 leave as they are
        for (int i = lane; i < S::kSide / 16; i += 32) {
          const int row = i / (S::kRow / 16), key = row / (16 * S::kBoxes) * 16 + row % 16;
          if (!(there[0][S::kIndexes > 1 ? key / 32 : 0] >> (key & 31) & 1)) *reinterpret_cast<uint4*>(stage + S::kSide + i * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        __syncwarp();
      }
      // ---- logits; two sums where one would be a long chain
      constexpr int kChains = S::kTiles * NT == 1 ? 2 : 1;
      float s[S::kTiles][NT][4], s2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[c][nt][0] = s[c][nt][1] = s[c][nt][2] = s[c][nt][3] = 0.f;
#pragma unroll
        for (int p = 0; p < S::kKP; ++p) {
          // piece 4p + t of the row: of box p / 2, its first or second half (rows of 64 bytes: all of it)
          const int in_box = S::kRow == 128 ? p & 1 : 0, block = (c * S::kBoxes + (S::kRow == 128 ? p / 2 : 0)) * 16 * S::kRow;
          const uint8_t* const from_k = stage + block + (at_k ^ (in_box * 64));
          const uint4 k0 = *reinterpret_cast<const uint4*>(from_k);
          const uint4 k1 = *reinterpret_cast<const uint4*>(from_k + 8 * S::kRow);
#pragma unroll
          for (int j = 0; j < S::kSteps; ++j) {
            uint32_t a0, a1, a2, a3;
            if (kE4m3) {
              halves(word(k0, j), a0, a2);
              halves(word(k1, j), a1, a3);
            } else {
              a0 = word(k0, 2 * j); a2 = word(k0, 2 * j + 1);
              a1 = word(k1, 2 * j); a3 = word(k1, 2 * j + 1);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              mma<kE4m3>(kChains == 2 && (p & 1) ? s2 : s[c][nt], a0, a1, a2, a3, qf[nt][p * S::kSteps + j][0], qf[nt][p * S::kSteps + j][1]);
          }
        }
      }
      if (kChains == 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[0][0][i] += s2[i];
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
          float ks = 1.f;
          if (kE4m3) {
            ks = ring_scale[warp][from & 255][0][key + key_r];
            tv[c][e] = __log2f(ring_scale[warp][from & 255][1][key + key_r]);
          }
          bool in = true;
          if (!here_all) in = there[0][key / 32] >> (key % 32 + key_r) & 1;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float x = s[c][nt][2 * e + h] * factor[nt][h];
              if (kE4m3) x *= ks;
              if (!in) x = -INFINITY;
              s[c][nt][2 * e + h] = x;
              xl[nt][h] = fmaxf(xl[nt][h], x);
              if (kE4m3) xo[nt][h] = fmaxf(xo[nt][h], in ? x + tv[c][e] : -INFINITY);
            }
        }
      bool rise = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          rise |= xl[nt][h] > ml[nt][h] + kSlack;
          if (kE4m3) rise |= xo[nt][h] > mo[nt][h] + kSlack;
        }
      if (__any_sync(0xffffffffu, rise)) {
        if (kE4m3) {
          // Rows of zeros of V take part in the sum of weights alone: their scale, which is 1 where they were written, would else put the reference so far above rows of small values
          // that these have no digits left.  Looked at where a reference rises, the only place where it matters.
          uint32_t zeros[S::kIndexes];
#pragma unroll
          for (int i = 0; i < S::kIndexes; ++i) {
            const int key = S::kKeys < 32 ? lane & (S::kKeys - 1) : i * 32 + lane;
            uint32_t any = 0;
#pragma unroll
            for (int box = 0; box < S::kBoxes; ++box)
#pragma unroll
              for (int j = 0; j < S::kRow / 16; ++j) {
                const uint4 x = *reinterpret_cast<const uint4*>(stage + S::kSide + (((key >> 4) * S::kBoxes + box) * 16 + (key & 15)) * S::kRow + ((j + lane) & (S::kRow / 16 - 1)) * 16);
                any |= x.x | x.y | x.z | x.w;
              }
            zeros[i] = __ballot_sync(0xffffffffu, (any & 0x7f7f7f7fu) == 0);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) xo[nt][0] = xo[nt][1] = -INFINITY;
#pragma unroll
          for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int key = c * 16 + e * 8;
              if (zeros[key / 32] >> (key % 32 + key_r) & 1 && tv[c][e] < INFINITY) tv[c][e] = -INFINITY;      // (0 times a scale that is none is NaN)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int h = 0; h < 2; ++h) xo[nt][h] = fmaxf(xo[nt][h], s[c][nt][2 * e + h] + tv[c][e]);
            }
        }
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
      // ---- weights.  bf16: two pieces, the bits in front and the nearest value of what they leave, so that a weight is off by 2^-16 of itself at most.  The first is the next value below even where
      // that would leave nothing: both are above 0, and what they make of an infinity in V is one.  (One piece, 2^-8, puts the results of the 64 sequences above 2^-9.6 of their size from
      // those of f32 weights, as far as their own rounding; two 2^-13.  The second costs 0.7 us of 181, 1 of 82 with 16 heads of queries a head.)
      // e4m3: one f16 piece, 2^-11, which leaves 2^-12; a second would leave 2^-13.7 and cost 75 -> 77 us for the 4 sequences above, 62 -> 72 with 16 heads of queries to each of 4 heads.
      constexpr int kPieces = kE4m3 ? 1 : 2;
      uint32_t pb[S::kTiles][NT][kPieces][2];
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
            if (kE4m3) {
              const __half2 x = __floats2half2_rn(p[2 * e], p[2 * e + 1]);
              pb[c][nt][0][e] = transposed(*reinterpret_cast<const uint32_t*>(&x));
            } else {
              const uint32_t f0 = max(__float_as_uint(p[2 * e]), 1u) - 1u, f1 = max(__float_as_uint(p[2 * e + 1]), 1u) - 1u;
              const __nv_bfloat162 x = __floats2bfloat162_rn(p[2 * e] - __uint_as_float(f0 & 0xffff0000u), p[2 * e + 1] - __uint_as_float(f1 & 0xffff0000u));
              pb[c][nt][0][e] = transposed(prmt(f0, f1, 0x7632));
              pb[c][nt][kPieces - 1][e] = transposed(*reinterpret_cast<const uint32_t*>(&x));
            }
          }
        }
      // ---- weights . v
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
        for (int p = 0; p < S::kVP; ++p) {
          VT v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const VT*>(stage + S::kSide + (c * S::kBoxes + p) * 16 * S::kRow + at_v[e & 1] + (e >> 1) * 8 * S::kRow);
#pragma unroll
          for (int w = 0; w < (int)sizeof(VT) / 4; ++w) {
            const uint32_t x0 = word(v[0], w), x1 = word(v[1], w), x2 = word(v[2], w), x3 = word(v[3], w);
            for (int i = 0; i < (kE4m3 ? 2 : 1); ++i) {
              // pairs of keys (2t, 2t + 1), (2t + 8, 2t + 9) of one column, two columns
              uint32_t a0, a1, a2, a3;
              if (kE4m3) {
                halves(prmt(x0, x1, i ? 0x7362 : 0x5140), a0, a1);
                halves(prmt(x2, x3, i ? 0x7362 : 0x5140), a2, a3);
              } else {
                a0 = prmt(x0, x1, 0x5410); a1 = prmt(x0, x1, 0x7632);
                a2 = prmt(x2, x3, 0x5410); a3 = prmt(x2, x3, 0x7632);
              }
              const int tile = p * (S::kVB / 2) + w * (kE4m3 ? 2 : 1) + i;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < kPieces; ++j) mma<kE4m3>(o[nt][tile], a0, a1, a2, a3, pb[c][nt][j][0], pb[c][nt][j][1]);
            }
          }
        }
      // ---- the stage is used up: the chunk behind those under way
      from = onward(from);
#pragma unroll
      for (int i = 0; i + 1 < S::kStages; ++i)
#pragma unroll
        for (int j = 0; j < S::kIndexes; ++j) there[i][j] = there[i + 1][j];
      if (step + S::kStages < j1) {
        if (!here_all) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (zeros were written there)
        __syncwarp();                                // every lane has read it
        fetch(step + S::kStages, page, there[S::kStages - 1]);
        ask_pages(step + S::kStages + 1, page);
      } else if (kE4m3) {
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
    }
    __syncthreads();                                 // (the results below lie over all warps' stages)

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
          const int d = (i / kHalfPiece) * 8 * S::kVB + piece * S::kVB + (i % kHalfPiece) * 2;
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
          const float2 f = last_factors(top_o, top_l, sum);
          __nv_bfloat162* const to = reinterpret_cast<__nv_bfloat162*>(a.o + ((((long long)seq * a.heads + head) * a.group + g0 + g) * a.dv + d));
          *to = __floats2bfloat162_rn(sum == 0.f ? 0.f : x * f.x * f.y, sum == 0.f ? 0.f : y * f.x * f.y);
        }
      } else if (a.balanced) {
        *reinterpret_cast<float2*>(a.part_o + ((long long)slot * kHeads + g) * DC + d) = make_float2(x, y);
        if (d == 0) *reinterpret_cast<float4*>(a.part_s + ((long long)slot * kHeads + g) * 4) = make_float4(top_l, sum, top_o, 0.f);
      } else {
        *reinterpret_cast<float2*>(&block_o[g][d]) = make_float2(x, y);
        if (d == 0) { ss[kWarps][g][0] = top_l; ss[kWarps][g][1] = sum; ss[kWarps][g][2] = top_o; }
      }
    }
    if (!whole && !a.balanced) {
      // ---- the blocks' sums, in order, each block its share of the columns
      cluster_barrier();
      const int rank = blockIdx.x % a.cluster;
      for (int i = rank * kThreads + tid; i < here * (DC / 2); i += a.cluster * kThreads) {
        const int g = i / (DC / 2), d = 2 * (i % (DC / 2));
        if (d >= a.dv) continue;
        const uint32_t at_s = smem_at(&ss[kWarps][g][0]), at_o = smem_at(&block_o[g][d]);
        float bl[kMostBlocks], bs[kMostBlocks], bo[kMostBlocks], top_l = -INFINITY, top_o = -INFINITY, sum = 0.f, x = 0.f, y = 0.f;
        float2 v[kMostBlocks];
#pragma unroll
        for (int c = 0; c < kMostBlocks; ++c) {
          const int of = min(c, a.cluster - 1);
          const uint32_t p = in_block(at_s, of);
          bl[c] = far(p);
          bs[c] = far(p + 4);
          bo[c] = far(p + 8);
          v[c] = far2(in_block(at_o, of));
          top_l = fmaxf(top_l, bl[c]);
          top_o = fmaxf(top_o, bo[c]);
        }
#pragma unroll
        for (int c = 0; c < kMostBlocks; ++c)
          if (c < a.cluster) {
            sum += bs[c] * (bl[c] == top_l ? 1.f : ex2(bl[c] - top_l));
            const float f = bo[c] == top_o ? 1.f : ex2(bo[c] - top_o);
            x += v[c].x * f;
            y += v[c].y * f;
          }
        const float2 f = last_factors(top_o, top_l, sum);
        __nv_bfloat162* const to = reinterpret_cast<__nv_bfloat162*>(a.o + ((((long long)seq * a.heads + head) * a.group + g0 + g) * a.dv + d));
        *to = __floats2bfloat162_rn(sum == 0.f ? 0.f : x * f.x * f.y, sum == 0.f ? 0.f : y * f.x * f.y);
      }
      cluster_barrier();                             // (no block leaves while others read what it has)
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // (copies may come over the results from here on)
    __syncthreads();
  }
}

// Joins the parts of the item that starts last in block b and goes on behind it: one in b, and the first of every block up to the item's last.  Each part's
// factor is worked out once; then a thread adds up four columns of a head, in the parts' order, with some loads under way at once.
constexpr int kJoined = 64;                          // parts at a time
template <int kHeads, int DC>
__global__ void __launch_bounds__(256, 4) attention_decode_join_kernel(const Args a) {
  __shared__ float factor[kHeads][kJoined];
  __shared__ float tops[kHeads][2], sums[kHeads], again[kHeads];
  mtf::chain_wait_only();
  const int4 piece = a.pieces[blockIdx.x];
  if (piece.x < 0) return;
  const int head = piece.y / a.chunks, g0 = (piece.y - head * a.chunks) * kHeads, here = min(kHeads, a.group - g0);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, parts = piece.z - (int)blockIdx.x + 1;
  auto place = [&](int i) { return (long long)(i == 0 ? piece.w : 2 * ((int)blockIdx.x + i)) * kHeads; };
  if (tid < kHeads) {
    tops[tid][0] = tops[tid][1] = -INFINITY;
    sums[tid] = 0.f;
  }
  constexpr int kFours = (kHeads * DC / 4 + 255) / 256;        // of a thread
  float4 sum[kFours];
#pragma unroll
  for (int j = 0; j < kFours; ++j) sum[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = 0; i0 < parts; i0 += kJoined) {
    const int some = min(kJoined, parts - i0);
    __syncthreads();
    for (int g = warp; g < here; g += 8) {           // a warp a head
      float4 s[kJoined / 32];
      float ml = tops[g][0], mo = tops[g][1];
#pragma unroll
      for (int j = 0; j < kJoined / 32; ++j) {
        s[j] = make_float4(-INFINITY, 0.f, -INFINITY, 0.f);
        if (j * 32 + lane < some) s[j] = *reinterpret_cast<const float4*>(a.part_s + (place(i0 + j * 32 + lane) + g) * 4);
        ml = fmaxf(ml, s[j].x);
        mo = fmaxf(mo, s[j].z);
      }
#pragma unroll
      for (int w = 16; w > 0; w /= 2) {
        ml = fmaxf(ml, __shfl_xor_sync(0xffffffffu, ml, w));
        mo = fmaxf(mo, __shfl_xor_sync(0xffffffffu, mo, w));
      }
      float l = 0.f;
#pragma unroll
      for (int j = 0; j < kJoined / 32; ++j) {
        l += s[j].y * (s[j].x == ml ? 1.f : ex2(s[j].x - ml));
        factor[g][j * 32 + lane] = s[j].z == mo ? 1.f : ex2(s[j].z - mo);
      }
#pragma unroll
      for (int w = 16; w > 0; w /= 2) l += __shfl_xor_sync(0xffffffffu, l, w);
      if (lane == 0) {
        again[g] = tops[g][1] == mo ? 1.f : ex2(tops[g][1] - mo);
        sums[g] = sums[g] * (tops[g][0] == ml ? 1.f : ex2(tops[g][0] - ml)) + l;
        tops[g][0] = ml;
        tops[g][1] = mo;
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kFours; ++j) {
      const int at = (j * 256 + tid) * 4, g = at / DC, d = at % DC;
      if (g >= here || d >= a.dv) continue;
      const float f = again[g];
      sum[j] = make_float4(sum[j].x * f, sum[j].y * f, sum[j].z * f, sum[j].w * f);
      constexpr int kDeep = 8;                       // under way at once
      for (int i = 0; i < some; i += kDeep) {
        float4 v[kDeep];
#pragma unroll
        for (int e = 0; e < kDeep; ++e) v[e] = *reinterpret_cast<const float4*>(a.part_o + (place(i0 + min(i + e, some - 1)) + g) * DC + d);
#pragma unroll
        for (int e = 0; e < kDeep; ++e)
          if (i + e < some) {
            const float w = factor[g][i + e];
            sum[j].x += v[e].x * w;
            sum[j].y += v[e].y * w;
            sum[j].z += v[e].z * w;
            sum[j].w += v[e].w * w;
          }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kFours; ++j) {
    const int at = (j * 256 + tid) * 4, g = at / DC, d = at % DC;
    if (g >= here || d >= a.dv) continue;
    const float l = sums[g];
    const float2 f = last_factors(tops[g][1], tops[g][0], l);
    __nv_bfloat162* const to = reinterpret_cast<__nv_bfloat162*>(a.o + ((((long long)piece.x * a.heads + head) * a.group + g0 + g) * a.dv + d));
    to[0] = __floats2bfloat162_rn(l == 0.f ? 0.f : sum[j].x * f.x * f.y, l == 0.f ? 0.f : sum[j].y * f.x * f.y);
    to[1] = __floats2bfloat162_rn(l == 0.f ? 0.f : sum[j].z * f.x * f.y, l == 0.f ? 0.f : sum[j].w * f.x * f.y);
  }
}

int width_class(const mtf::CachePool& c) {
  const int d = std::max(c.dk, c.dv);
  // (rows of 64 bytes are copied two at least at a time, to where 128 bytes begin: a page of an odd number of slots has wider ones)
  if (d <= 64) return c.e4m3 && c.slots % 2 ? 128 : 64;
  return d <= 128 ? 128 : 256;
}
int tiles_of_heads(const mtf::CachePool& c, int group) { return group > 8 && width_class(c) < 256 ? 2 : 1; }
int blocks_an_sm(const mtf::CachePool& c) { return width_class(c) == 256 && !c.e4m3 ? Shape<false, 256>::kBlocks : Shape<false, 128>::kBlocks; }

int unit_keys(const mtf::CachePool& c) {
  const int row = width_class(c) * (c.e4m3 ? 1 : 2);
  return kWarps * 16 * (row <= 64 ? 4 : row <= 128 ? 2 : 1);
}

// How a call's items (a head, or as many heads of queries as a block takes, of a sequence) are shared out: to a block each, to a cluster of blocks each, which join their sums
// through their shared memory, or, cut into units, evenly to all blocks of the GPU, which leave parts for a second launch.  The host knows how many positions a sequence may have, not how
// many it has.  A unit takes a block 0.7 us; the cluster's joining 1.2, and its blocks start the later the more there are beyond one an SM; the even cut pays 5 to 6 for its sums over the
// lengths and its second launch, and is the only one of the three whose time does not go by the longest sequence.  Hence
//   - clusters as long as they are no more blocks than SMs, and cut something off: not for 2 units;
//   - beyond that, up to what the SMs hold at once, where a block has more than 8 units left;
//   - the even cut where it still has (a block by itself: more than 11).
// Measured (bf16, d 128 unless said; us for a block an item / clusters of 2 / 4 / 8 / the even cut):
//   1 x 16 heads, 512 positions of d 64 (4 units)  6.8  6.1  5.6  5.6  10.3;  256 positions (2 units)  4.9  5.6  5.3  5.7  6.8
//   4 x 8, 512 (8 units)                          10.8  8.9  7.6  8.2  12.6;  26 x 8, 300 (5)          9.2 11.1 18.7 33.4  14.5
//   40 x 5, up to 777 (13)                        15.5 13.0 18.0 33.1  14.8;  80 x 5, 700 (11)        28.5 35.4 47.7 73.4  33.2
//   16 x 8, up to 1500 (24)                       24.4 17.6 19.2 23.9  14.8;  all of 1500             25.9 20.8 26.6 29.8  20.1
//   64 x 16, up to 4096 (64)                       179  169  182  257   176;  all of 4096              322  310  319  383   335
// (In the last line clusters of two are ahead, but where one sequence in 64 has 4096 positions and the others few they take three times as long as the even cut.)
struct Plan {
  bool balanced;
  int cluster;
  long long grid;
};
Plan plan_of(const mtf::CachePool& c, int group) {
  const int nt = tiles_of_heads(c, group), chunks = (group + 8 * nt - 1) / (8 * nt);
  const long long items = c.sequences * c.heads * chunks, units = ((long long)c.per_sequence * c.slots + unit_keys(c) - 1) / unit_keys(c);
  const long long sms = mtf::device_sm_count(), most = sms * blocks_an_sm(c);
  int cluster = 1;
  while (cluster < kMostBlocks && ((units > std::max(2, cluster) && items * cluster * 2 <= sms) || (units > kFewSteps * cluster && items * cluster * 2 <= most))) cluster *= 2;
  // (the sum of all sequences' units is kept in 32 bits)
  const bool balanced = units > (cluster > 1 ? kFewSteps * cluster : kLoneSteps) && c.sequences <= kPlanned && c.sequences * (units + kOver) < (1LL << 31);
  if (balanced) return {true, 1, std::max(1LL, std::min(most, items * (units + kOver) / kLeastCost))};
  return {false, cluster, items * cluster};
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encoder() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess) fn = reinterpret_cast<EncodeTiledFn>(p);
  });
  return fn;
}
// a pool as [page][head][slot][d], whichever of slot and head lies inside; boxes of `rows` slots of a head, `row` bytes wide
mtf_status pool_map(CUtensorMap* m, const void* pool, const mtf::CachePool& c, int width, int rows, int row) {
  EncodeTiledFn enc = encoder();
  if (!enc) return mtf::fail(MTF_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const cuuint64_t elt = c.e4m3 ? 1 : 2, bytes = width * elt;
  const cuuint64_t d[4] = {(cuuint64_t)width, (cuuint64_t)c.slots, (cuuint64_t)c.heads, (cuuint64_t)c.pages};
  const cuuint64_t s[3] = {bytes * c.row_slot, bytes * c.row_head, bytes * c.rows_page};
  const cuuint32_t box[4] = {(cuuint32_t)(row / elt), (cuuint32_t)rows, 1, 1}, es[4] = {1, 1, 1, 1};
  const CUresult r = mtf::in_context([&] { return enc(m, c.e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), d, s, box, es,
                                                      CU_TENSOR_MAP_INTERLEAVE_NONE, row == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                                      CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE); });
  return r == CUDA_SUCCESS ? MTF_OK : mtf::fail(MTF_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d", (int)r);
}

template <bool kE4m3, int DC, int NT>
mtf_status launch(const Args& a, const mtf::CachePool& c, int grid, cudaStream_t st) {
  using S = Shape<kE4m3, DC>;
  CUtensorMap map_k, map_v;
  mtf_status ok = pool_map(&map_k, c.k, c, c.dk, a.box_rows, S::kRow);
  if (ok != MTF_OK || (ok = pool_map(&map_v, c.v, c, c.dv, a.box_rows, S::kRow)) != MTF_OK) return ok;
  constexpr int kResults = (kWarps + 1) * 8 * NT * (DC + 4) * 4, kRoom = 1024 + (S::kRing > kResults ? S::kRing : kResults);
  static mtf::KnownPerDevice limit;
  const cudaError_t e = mtf::shared_memory_limit(limit, attention_decode_kernel<kE4m3, DC, NT>, kRoom);
  if (e != cudaSuccess) return mtf::fail(MTF_ERR_CUDA, "attention_decode_kernel: %s", cudaGetErrorString(e));
  mtf::launch_clusters(attention_decode_kernel<kE4m3, DC, NT>, dim3((unsigned)grid), kThreads, kRoom, a.cluster, st, a, map_k, map_v);
  mtf::count_launch();
  if (a.balanced && grid > 1) {
    mtf::launch_chained(attention_decode_join_kernel<8 * NT, DC>, (unsigned)grid - 1, 256, 0, st, a);
    mtf::count_launch();
  }
  return MTF_OK;
}
template <bool kE4m3>
mtf_status dispatch(const Args& a, const mtf::CachePool& c, int dc, int nt, int grid, cudaStream_t st) {
  if (dc == 256) return launch<kE4m3, 256, 1>(a, c, grid, st);
  if (dc == 128) return nt == 1 ? launch<kE4m3, 128, 1>(a, c, grid, st) : launch<kE4m3, 128, 2>(a, c, grid, st);
  return nt == 1 ? launch<kE4m3, 64, 1>(a, c, grid, st) : launch<kE4m3, 64, 2>(a, c, grid, st);
}

}  // namespace

namespace mtf {

size_t attention_decode_workspace(const CachePool& c, int group) {
  const Plan p = plan_of(c, group);
  if (!p.balanced) return 0;
  const size_t heads = 8 * tiles_of_heads(c, group);
  return p.grid * 2 * heads * (width_class(c) + 4) * sizeof(float) + p.grid * sizeof(int4);
}

mtf_status launch_attention_decode(const CachePool& c, const DecodeCall& d, void* stream) {
  const int dc = width_class(c), nt = tiles_of_heads(c, d.group);
  Args a = {};
  a.q = reinterpret_cast<const __nv_bfloat16*>(d.q);
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
  // (16 keys a copy where a page has a multiple of 16; of an odd number each key is a copy of its own: 64 x 16 heads of up to 4096, pages of 17 slots instead of 16, 321 us for 184 in bf16, 218 for 113 in e4m3)
  a.box_rows = 16;
  while (c.slots % a.box_rows) a.box_rows /= 2;
  a.scale_log2 = d.scale * kLog2e;
  const Plan p = plan_of(c, d.group);
  const long long grid = p.grid;
  a.balanced = p.balanced;
  a.cluster = p.cluster;
  if (grid > 0x7fffffffLL) return fail(MTF_ERR_UNSUPPORTED, "attention_decode: at most 2^31 heads of sequences");
  if (a.balanced) {
    const size_t heads = 8 * nt;
    a.pieces = reinterpret_cast<int4*>(d.workspace);
    a.part_s = reinterpret_cast<float*>(a.pieces + grid);
    a.part_o = a.part_s + (size_t)grid * 2 * heads * 4;
  }
  const mtf_status st = c.e4m3 ? dispatch<true>(a, c, dc, nt, (int)grid, (cudaStream_t)stream) : dispatch<false>(a, c, dc, nt, (int)grid, (cudaStream_t)stream);
  if (st != MTF_OK) return st;
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

mtf_status debug_decode_wait_test(long long limit_cycles, int withhold) {
  const long long limit = limit_cycles > 0 ? limit_cycles : kWaitCycles;
  cudaError_t e = cudaMemcpyToSymbol(g_wait_limit, &limit, sizeof(limit));
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_withhold, &withhold, sizeof(int));
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "cudaMemcpyToSymbol: %s", cudaGetErrorString(e));
  return MTF_OK;
}
mtf_status read_decode_status(int* code) {
  int v = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_decode_status, sizeof(int));
  if (e != cudaSuccess) return fail(MTF_ERR_CUDA, "cudaMemcpyFromSymbol: %s", cudaGetErrorString(e));
  if (v) { int z = 0; cudaMemcpyToSymbol(g_decode_status, &z, sizeof(int)); }
  *code = v;
  return MTF_OK;
}

}  // namespace mtf
