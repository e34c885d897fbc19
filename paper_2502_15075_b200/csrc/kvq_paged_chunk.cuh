// Paged attention of many query rows on the fifth-generation tensor cores: softmax(q K^T / sqrt(d)) V (App. A.1) over a paged packed cache,
// with a causal mask, a sliding window and first tokens that stay visible.
//
// A tile is 256 (query row, head) pairs of one sequence and KV head - the query heads of a KV head are rows of one product - against pages of 128
// tokens.  One CTA per SM:
//  * warps 16-23 (keys) and 24-27 (values) turn a page into 16-bit tiles in shared memory: codes become fp16 by a mask under the bits of 1024 and
//    an exact operation, scale and zero-point enter by a fused one (one rounding, 2^-11 of the value at most).  Their packed words were
//    loaded a page ahead, straight into registers.  The order of channels (keys) and of tokens (both) is the one in which codes lie in the
//    page; queries and the weights follow it, so that nothing is transposed.
//  * one thread of warp 28 issues tcgen05.mma (kind f16, M 128, fp32 accumulators in tensor memory): S = Q K^T of both halves of the tile
//    in turn, and O += P V with P read from tensor memory, where it takes the place of S.
//  * warps 0-7 and 8-15 take the two halves, two threads per row: row maximum, p = 2^(x - reference), fp16 weights back to tensor memory;
//    sums in fp32.  While one half's softmax runs, the tensor cores have the other half's products.  The reference moves only when a logit
//    passes the largest one before by kHeadroom bits; then the row's outputs are rescaled in tensor memory.
// The loss against fp32 is the rounding of the weights (see kLift) and of the tiles (2^-11 of an element) to fp16; all sums are fp32.
// bf16 queries are scaled by a power of two per row.  A token with a group that reaches beyond the fp16 range enters its tile times 2^-(B + 1), which
// brings the largest B-bit group into it; its logit (keys) or its weight (values) is made as much larger.  Other tokens of its page are as exact as
// without it.
//
// The (tile, page) pairs of a call lie on one axis that is cut into equal shares, one per CTA, so that a long prompt, a ragged batch and a few
// drafted rows behind a long context all fill the GPU.  A tile that falls to several CTAs leaves partials (m, l, o); the CTA that comes last
// merges them by log-sum-exp, in a fixed order.
//
// 8B shape K4V2, a prompt of 8,192 tokens against its own cache 749 us (550 GFLOP: 734 TFLOP/s, 0.45 of the measured bf16 rate; with a scaled token in every
// page 924 to 949, with nothing else 2,250 to 3,420); two chunks of up to 700 rows behind 16,001 tokens with a window of 4,096 160 us.  Bound by the chain softmax - product - softmax of a half: both products of a half
// are 1,024 cycles, its softmax about 2,000, and the other half's work covers only part of that.  (Of 830 us at one thread per row 579 were left
// without the softmax, 733 without the conversion of pages, 494 without both.)  Not gained by: every fourth power of two by a cubic instead of the
// special-function unit (850 against 833), the next columns loaded ahead of the arithmetic (850), products issued by a lone thread (861).
// Every wait is bounded; on expiry the kernel sets KVQ_STATUS_DEVICE_TIMEOUT, goes on without waiting (nothing that it then reads is out of range) and
// frees its tensor memory.
#pragma once

#include <type_traits>

#include "kvq_paged.cuh"
#include "kvq_tcgen05.cuh"

namespace kvq {
namespace chunk {

using namespace mma;

constexpr int kThreads = 32 * 32;          // warps 0-15 softmax, 16-23 keys, 24-27 values, 28 products (29-31 complete its warpgroup)
// Registers per thread at launch, and of the roles: 512 softmax threads, 384 that make tiles, 128 more.
constexpr int kRegsLaunch = 64, kRegsSoftmax = 80, kRegsTiles = 48, kRegsRest = 48;
static_assert(512 * kRegsSoftmax + 384 * kRegsTiles + 128 * kRegsRest <= kThreads * kRegsLaunch, "an increase waits for registers that the others gave up");
constexpr int kGrid = 148;
constexpr int kTile = 256;                 // (query row, head) pairs of a tile
// What a tile costs besides its pages (queries, a first product that nothing overlaps, outputs), in pages: the prompt above with 2 870 us, 3 788, 4 749,
// 6 746; the chunks 156, 157, 160, 157.
constexpr int kGap = 5;
// Weights are 2^(logit - reference), the reference `lift` bits below the largest logit when it moves; it moves when a logit passes it by lift +
// kHeadroom.  So the largest weight of a row is between 2^11 and 2^15, and a weight is off by 2^-11 of it or, below 2^-14 in fp16, by 2^-36 of the
// largest (131,072 tokens of that kind: 2^-19).  Of logits x of millions of bits fp32 rounds x and the reference by up to 2^-24 x each: the
// lift leaves room for that.
constexpr float kHeadroom = 4.0f, kLift = 11.0f;
__device__ __forceinline__ float lift_at(float x) { return fmaxf(fmaf(fabsf(x), -2.3841858e-7f, kLift), 0.0f); }      // kLift - |x| 2^-22
__host__ __device__ constexpr float big_up(int bits) { return (float)(2 << bits); }      // of tokens beyond the fp16 range, see above
constexpr uint32_t FULL = 0xffffffffu;
// tensor memory: S of the two halves (columns 0-31 and 64-95 of each take P), then O of the two halves
constexpr uint32_t kColS = 0, kColO = 256, kTmemCols = 512;
// fp16 operands, fp32 accumulate, both K-major, M 128
__host__ __device__ constexpr uint32_t idesc(int n) { return (1u << 4) | ((uint32_t)(n / 8) << 17) | (8u << 24); }

// Shared memory.  Operands lie in 8 x 16-byte core matrices: rows 16 bytes apart, octets of rows 128, chunks of eight k `lb` apart; eight
// neighbouring lanes write one core matrix.
template <int D> struct Tiles {
  static constexpr int kLbQ = 128 * 16, kLbK = 128 * 16, kLbV = D * 16;
  static constexpr int kQ = D / 8 * kLbQ, kK = D / 8 * kLbK, kV = 16 * kLbV;      // bytes of a query half, a key and a value tile
};
struct Smem { int q, k, v, bars, misc, rows, pref, seq, total; };
template <int D>
__host__ __device__ inline Smem smem_of(int batch) {
  using T = Tiles<D>;
  Smem s;
  s.q = 0;
  s.k = 2 * T::kQ;
  s.v = s.k + 2 * T::kK;
  s.bars = s.v + 2 * T::kV;
  s.misc = s.bars + 32 * 8;
  s.rows = s.misc + 160;                     // per row of the tile: what its two threads tell each other, for two pages in turn
  s.pref = s.rows + 2 * kTile * 2 * 4;
  s.seq = s.pref + (batch + 1) * 8;
  s.total = s.seq + 3 * batch * 4;
  return s;
}

// Workspace: per CTA two partials of `cap` rows (o [D], then (m, l) of all of them), then two count words.
__host__ __device__ inline int row_cap(int pairs) { return pairs < kTile ? pairs : kTile; }
__host__ __device__ inline size_t ml_offset_floats(int cap, int D) { return (size_t)2 * kGrid * cap * D; }
__host__ __device__ inline size_t count_offset_floats(int cap, int D) { return ml_offset_floats(cap, D) + (size_t)2 * kGrid * cap * 2; }
__host__ __device__ inline size_t workspace_bytes(int cap, int D) { return count_offset_floats(cap, D) * 4 + (size_t)2 * kGrid * 8; }

// ------------------------------------------------------------------ PTX wrappers
// D (+)= A B.  a, b: low words of the descriptors (start address, leading offset), their high words are the same for all operands here.  The
// one thread that issues them has few instructions between two products: the descriptors' parts are added up from constants.
constexpr uint32_t kDescHigh = (128u >> 4) | (1u << 14);       // octets of rows 128 bytes apart, version 1, no swizzle
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t lb) { return ((addr >> 4) & 0x3FFFu) | ((lb >> 4) << 16); }
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
template <bool ACC>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t id) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b), "r"(id), "n"(ACC ? 1 : 0), "n"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t id, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 y, {%2, %5};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b), "r"(id), "r"(acc), "n"(kDescHigh) : "memory");
}
#define KVQ_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define KVQ_W8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define KVQ_S8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : KVQ_R8(r, 0), KVQ_R8(r, 8) : "r"(addr) : "memory");
}
// Waits for this thread's loads from tensor memory; the registers go through it, so that nothing is computed from them before.
__device__ __forceinline__ void wait_ld(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : KVQ_W8(r, 0), KVQ_W8(r, 8)::"memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(addr), KVQ_S8(r, 0), KVQ_S8(r, 8) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), KVQ_S8(r, 0) : "memory");
}
// One column, there at once.
__device__ __forceinline__ uint32_t tmem_ld1(uint32_t addr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=r"(r) : "r"(addr) : "memory");
  return r;
}
__device__ __forceinline__ void tmem_st1(uint32_t addr, uint32_t r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(addr), "r"(r) : "memory");
}
__device__ __forceinline__ float max3(float a, uint32_t b, uint32_t c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
  return d;
}
// Token of a page's block of 32 that stands at place k of its 32 columns: codes of four tokens share a word, those of two halves a load.
__host__ __device__ constexpr int token_at(int k) { return 16 * ((k & 7) >> 2) + 2 * (k >> 3) + (k & 1) + 8 * ((k >> 1) & 1); }

// Its inverse: the place of token u.
__host__ __device__ constexpr int place_of(int u) { return 8 * ((u & 7) >> 1) + (u & 1) + 2 * ((u >> 3) & 1) + 4 * (u >> 4); }
constexpr bool places_match() {
  for (int k = 0; k < 32; ++k)
    if (place_of(token_at(k)) != k) return false;
  return true;
}
static_assert(places_match(), "columns of single tokens");
// Of the tokens marked in two blocks' words (the same for the whole warp): what to do with each one's column.
template <typename F>
__device__ __forceinline__ void for_tokens(uint32_t first, uint32_t second, F&& each) {
#pragma unroll 1
  for (int base = 0; base < 64; base += 32) {
#pragma unroll 1
    for (uint32_t bits = base == 0 ? first : second; bits; bits &= bits - 1) each(base + place_of(__ffs(bits) - 1));
  }
}

// Two codes of a field of a word's bytes 0 and 2 (of w >> 8: bytes 1 and 3) as fp16 numbers times scale plus zero-point, one rounding.  The
// field stays where it stands: under the bits of 1024 it reads 1024 + code 2^(B f), which one operation makes the code, exactly.
// The constants are held in registers (the compiler would make them again for every use).
template <int B>
struct Codes {
  static constexpr int F = 8 / B;
  uint32_t magic, up[F], bias[F];
  __device__ __forceinline__ Codes() {
    asm volatile("mov.b32 %0, 0x64006400;" : "=r"(magic));
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const uint32_t u = as_u32(__float2half2_rn(1.0f / (float)(1 << (B * f)))), v = as_u32(__float2half2_rn(-1024.0f / (float)(1 << (B * f))));
      asm volatile("mov.b32 %0, %1;" : "=r"(up[f]) : "r"(u));
      asm volatile("mov.b32 %0, %1;" : "=r"(bias[f]) : "r"(v));
    }
  }
  __device__ __forceinline__ uint32_t values(uint32_t w, int f, __half2 s, __half2 z) const {
    const uint32_t mask = (((1u << B) - 1u) << (B * f)) * 0x00010001u;
    const __half2 raw = as_h2((w & mask) | magic);
    const __half2 code = f == 0 ? __hadd2(raw, as_h2(bias[0])) : __hfma2(raw, as_h2(up[f]), as_h2(bias[f]));
    return as_u32(__hfma2(code, s, z));
  }
};

// A tile: its rows, and the pages that they see.
struct Tile {
  int b, h, i;                 // sequence, KV head, tile of the sequence's (row, head) pairs
  int n, rows, first, pairs;   // of the sequence
  SeenPages seen;
};

template <int D, int KB, int VB>
__global__ void __launch_bounds__(kThreads, 1)
chunk_kernel(Geom g, Paged p, const uint16_t* __restrict__ q, float c1, float* __restrict__ ws, int cap, void* __restrict__ out,
             int out_dtype, unsigned long long call_id, unsigned long long wait_ns, long long skip_x) {
  using T = Tiles<D>;
  constexpr int KW = D * KB / 128;            // words of a lane's quarter of a key row
  constexpr int FPB = 8 / VB, NMW = D / 16 / FPB;      // value codes per byte, quads of value words per lane and block
  constexpr int NI = D / 32;
  extern __shared__ __align__(128) uint8_t smem[];
  const Smem sl = smem_of<D>(g.B);
  long long* sPref = reinterpret_cast<long long*>(smem + sl.pref);      // (tile, page) pairs and gaps in front of every sequence
  int* sSeq = reinterpret_cast<int*>(smem + sl.seq);                    // tokens, rows, first row
  int* sMisc = reinterpret_cast<int*>(smem + sl.misc);                  // [0] abort [1] tensor memory [2, 3] counts returned [4..7] share [8..39] tokens that are scaled
  volatile int* abort_flag = sMisc;
  // which tokens are scaled: a bit per token; four pages in turn, two sides of 64 tokens, their two blocks' keys, then values
  const uint32_t sScaled = smem_u32(sMisc + 8);
  auto get_scaled = [&](int it, int side) {
    uint4 b;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "r"(sScaled + 16 * (2 * (it & 3) + side)) : "memory");
    return b;
  };
  auto set_scaled = [&](int it, int blk, int of_values, uint32_t bits) {
    asm volatile("st.shared.u32 [%0], %1;" ::"r"(sScaled + 16 * (2 * (it & 3) + (blk >> 1)) + 8 * of_values + 4 * (blk & 1)), "r"(bits) : "memory");
  };
  const int tid_ = threadIdx.x, lane = tid_ & 31, warp = __shfl_sync(FULL, tid_ >> 5, 0);
  const int B = g.B, G = g.G, Hkv = g.Hkv;
  const uint32_t inv_g = G > 1 ? 0xFFFFFFFFu / (uint32_t)G + 1u : 0u;
  auto by_g = [&](int x) { return G > 1 ? (int)__umulhi((uint32_t)x, inv_g) : x; };      // x / G, exact up to 2^29
  // barriers: key tile full / empty [2], value tile full / empty [2], queries [2], S [2], P [2], O [2], drain
  const uint32_t bar = smem_u32(smem + sl.bars);
  const uint32_t bKF = bar, bKE = bar + 16, bVF = bar + 32, bVE = bar + 48, bQ = bar + 64, bS = bar + 80, bP = bar + 96, bO = bar + 112, bDrain = bar + 128;

  if (tid_ == 0) {
    sMisc[0] = 0;
    for (int k = 0; k < 2; ++k) {
      mbar_init(bKF + 8 * k, 8); mbar_init(bKE + 8 * k, 1); mbar_init(bVF + 8 * k, 4); mbar_init(bVE + 8 * k, 1);
      mbar_init(bQ + 8 * k, 8); mbar_init(bS + 8 * k, 1); mbar_init(bP + 8 * k, 8); mbar_init(bO + 8 * k, 1);
    }
    mbar_init(bDrain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  begin_after_predecessor();
  if (warp == 28) {
    tc::tmem_alloc(smem_u32(&sMisc[1]), kTmemCols);
    tc::tmem_relinquish();
  }
  // ---- plan: (tile, page) pairs per sequence, this CTA's share
  auto seen_by = [&](int n, int rows, int pairs, int i) {
    return seen_pages(n - rows + by_g(i * kTile), n - rows + by_g(min(i * kTile + kTile, pairs) - 1), p.window, p.sinks);
  };
  for (int b = warp; b < B; b += kThreads / 32) {
    bool bad;
    const SeqRows s = seq_rows(p, b, g.capacity, p.max_rows, bad);
    if (bad && lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
    const int pairs = s.rows * G;
    long long sum = 0;
    for (int i = lane; i * kTile < pairs; i += 32) sum += seen_by(s.n, s.rows, pairs, i).count + kGap;
    for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(FULL, sum, off);
    if (lane == 0) {
      sPref[b + 1] = sum * Hkv;
      sSeq[3 * b] = s.n; sSeq[3 * b + 1] = s.rows; sSeq[3 * b + 2] = s.first;
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sMisc[1]);
  if (warp == 0) {
    if (lane == 0) sPref[0] = 0;
    long long carry = 0;
    for (int base = 0; base < B; base += 32) {
      const int i = base + lane;
      long long v = i < B ? sPref[i + 1] : 0;
      for (int off = 1; off < 32; off <<= 1) {
        const long long u = __shfl_up_sync(FULL, v, off);
        if (lane >= off) v += u;
      }
      if (i < B) sPref[i + 1] = v + carry;
      carry += __shfl_sync(FULL, v, 31);
    }
  }
  __syncthreads();
  FlatPlan plan;
  plan.N = sPref[B];
  plan.c_eff = plan.N < (long long)gridDim.x ? (int)plan.N : (int)gridDim.x;
  const bool on = (int)blockIdx.x < plan.c_eff;
  const long long x_lo = on ? plan.lo(blockIdx.x) : 0, x_hi = on ? plan.lo(blockIdx.x + 1) : 0;
  if (warp == 0 && on) {
    int lo = 0, hi = B - 1;                          // the last sequence that starts at or before x_lo
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sPref[mid] <= x_lo) lo = mid; else hi = mid - 1;
    }
    const int n = sSeq[3 * lo], rows = sSeq[3 * lo + 1], pairs = rows * G;
    const long long per_head = (sPref[lo + 1] - sPref[lo]) / Hkv;
    const int h = (int)((x_lo - sPref[lo]) / per_head);
    long long rest = x_lo - sPref[lo] - h * per_head;
    int i0 = 0, tile = 0;
    bool found = false;
    for (; !found && i0 * kTile < pairs; i0 += 32) {
      const int i = i0 + lane;
      const long long own = i * kTile < pairs ? seen_by(n, rows, pairs, i).count + kGap : 0;
      long long v = own;
      for (int off = 1; off < 32; off <<= 1) {
        const long long u = __shfl_up_sync(FULL, v, off);
        if (lane >= off) v += u;
      }
      const uint32_t beyond = __ballot_sync(FULL, v > rest);
      if (beyond) {
        const int src = __ffs(beyond) - 1;
        rest -= __shfl_sync(FULL, v - own, src);
        tile = i0 + src;
        found = true;
      } else {
        rest -= __shfl_sync(FULL, v, 31);
      }
    }
    if (lane == 0) { sMisc[4] = lo; sMisc[5] = h; sMisc[6] = tile; sMisc[7] = (int)rest; }
  }
  __syncthreads();

  auto tile_of = [&](int b, int h, int i) {
    Tile t;
    t.b = b; t.h = h; t.i = i;
    t.n = sSeq[3 * b]; t.rows = sSeq[3 * b + 1]; t.first = sSeq[3 * b + 2];
    t.pairs = t.rows * G;
    t.seen = seen_by(t.n, t.rows, t.pairs, i);
    return t;
  };
  auto next_tile = [&](const Tile& t) {
    int b = t.b, h = t.h, i = t.i + 1;
    if (i * kTile >= t.pairs) {
      i = 0;
      if (++h == Hkv) {
        h = 0;
        do { ++b; } while (b < B - 1 && sSeq[3 * b + 1] == 0);
      }
    }
    return tile_of(min(b, B - 1), h, i);
  };
  // The share, segment by segment: pages page .. end - 1 of tile t, which starts at xs on the axis (a gap, then its pages).
  struct Cursor { Tile t; long long xs; int page, end; bool on; };
  auto settle = [&](Cursor& c) {                     // on to the first tile from c.t on of which a page lies in the share
    while (true) {
      const long long lo = x_lo - c.xs - kGap, hi = x_hi - c.xs - kGap;
      c.page = lo > 0 ? (int)lo : 0;
      c.end = hi < c.t.seen.count ? (int)hi : c.t.seen.count;
      c.on = c.end > c.page;
      if (c.on) return;
      c.xs += kGap + c.t.seen.count;
      if (c.xs + kGap >= x_hi) return;
      c.t = next_tile(c.t);
    }
  };
  auto start = [&]() {
    Cursor c;
    c.on = false;
    if (x_lo >= x_hi) return c;
    c.t = tile_of(sMisc[4], sMisc[5], sMisc[6]);
    c.xs = x_lo - sMisc[7];
    settle(c);
    return c;
  };
  auto advance = [&](Cursor& c) {                    // to the next segment
    c.xs += kGap + c.t.seen.count;
    c.on = c.xs + kGap < x_hi;
    if (c.on) {
      c.t = next_tile(c.t);
      settle(c);
    }
  };
  bool aborted = false;
  // A wait of a whole warp; after a time-out the role goes on without waiting.  Most waits are long: a look costs three instructions, the clock
  // and the other roles' failure are looked at now and then.
  auto wait_warp = [&](uint32_t b, uint32_t parity) {
    if (aborted) return;
    if (__all_sync(FULL, mbar_try_wait(b, parity))) return;
    bool got = false;
    const unsigned long long t0 = globaltimer_ns();
    while (true) {
#pragma unroll 1
      for (int n = 0; n < 32 && !got; ++n) got = mbar_try_wait_hint(b, parity, 1000u);
      if (got || *abort_flag || globaltimer_ns() - t0 > wait_ns) break;
    }
    if (!__all_sync(FULL, got)) {
      aborted = true;
      *abort_flag = 1;
      if (lane == 0) atomicOr(p.status, KVQ_STATUS_DEVICE_TIMEOUT);
      __syncwarp();
    }
  };

  if (warp < 16) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // =========================================================== softmax: half w of the tile, two threads per row, each with a side of 64 of the
    // page's columns and half of the channels (the softmax's latency is what the products wait for; one thread per row, both at a gap of 2 pages: the
    // prompt 831 us against 873, whose shares were less even, the chunks 170 against 156)
    const int w = warp >> 3, side = (warp >> 2) & 1, row = 32 * (warp & 3) + lane;
    const uint32_t tS = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + kColS + 128 * w + 64 * side;
    const uint32_t tO = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + kColO + 128 * w + D / 2 * side;
    uint8_t* sq = smem + sl.q + w * T::kQ + row * 16 + side * (D / 16) * T::kLbQ;
    volatile float* sRow = reinterpret_cast<float*>(smem + sl.rows) + (128 * w + row) * 2;      // [page parity][row][side]
    const unsigned long long id40 = (call_id & 0xFFFFFFFFFFull) ? (call_id & 0xFFFFFFFFFFull) : 1ull;
    unsigned long long* counts = reinterpret_cast<unsigned long long*>(ws + count_offset_floats(cap, D));
    // a value for the row's other thread, and its
    uint32_t turn = 0;
    auto exchange = [&](float x) {
      volatile float* at = sRow + turn * (2 * kTile);
      turn ^= 1;
      at[side] = x;
      named_bar_sync(1 + w, 256);
      return at[side ^ 1];
    };
    int it = 0, done = 0, seg = 0;                   // pages of the share so far, those that this half had, segments it had
#pragma unroll 1
    for (Cursor c = start(); c.on; advance(c)) {
      const Tile& t = c.t;
      const int page0 = c.page, pages = c.end - c.page;
      const int pair0 = t.i * kTile + 128 * w;
      if (pair0 >= t.pairs) { it += pages; continue; }
      // ---- the row's query: fp16 in the order of the key tiles' channels; rows of bf16 scaled to a largest element from 1 to below 2
      const int pair = pair0 + row, r = by_g(min(pair, t.pairs - 1));
      const bool real = pair < t.pairs;
      float f = c1;
      {
        const uint16_t* src = q + ((size_t)(t.first + r) * g.Hq + (size_t)t.h * G + (pair - r * G)) * D;
        uint32_t qw[D / 4];                          // (this side's channels at once: one wait for memory)
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (real) v = *reinterpret_cast<const uint4*>(src + side * (D / 2) + 8 * k);
          qw[4 * k] = v.x; qw[4 * k + 1] = v.y; qw[4 * k + 2] = v.z; qw[4 * k + 3] = v.w;
        }
        // |q| has the order of its 16-bit pattern: bf16 rows are scaled to bring the exponent of the largest to that of one
        if (g.in_dtype == KVQ_BF16) {
          uint32_t top = 0;
#pragma unroll
          for (int k = 0; k < D / 4; ++k) top = __vmaxu2(top, qw[k] & 0x7FFF7FFFu);
#pragma unroll 4
          for (int k = 0; k < D / 16; ++k) {         // (the other side's)
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (real) v = *reinterpret_cast<const uint4*>(src + (side ^ 1) * (D / 2) + 8 * k);
            top = __vmaxu2(__vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)), top);
          }
          const int e = (int)(max(top & 0xFFFFu, top >> 16) >> 7);
          const int shift = e == 0 ? 0 : min(max(127 - e, -126), 126);
          const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
          f = c1 * __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll
          for (int k = 0; k < D / 4; ++k)
            qw[k] = as_u32(__floats2half2_rn(__uint_as_float(qw[k] << 16) * up, __uint_as_float(qw[k] & 0xFFFF0000u) * up));
        }
        // chunk 4 i + ch: channels 32 i + 4 ch + {0, 2, 1, 3}, then those 16 further
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const int i = k >> 2, ch = k & 3, a = (32 * i + 4 * ch) / 2;
          *reinterpret_cast<uint4*>(sq + k * T::kLbQ) = make_uint4(prmt(qw[a], qw[a + 1], 0x5410u), prmt(qw[a], qw[a + 1], 0x7632u),
                                                                   prmt(qw[a + 8], qw[a + 9], 0x5410u), prmt(qw[a + 8], qw[a + 9], 0x7632u));
        }
      }
      tc::fence_async_smem();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bQ + 8 * w);
      // the next tile's queries come to L2 meanwhile
      if (pair + kTile < t.pairs) {
        const int rn = by_g(pair + kTile);
        asm volatile("prefetch.global.L2 [%0];" ::"l"(q + ((size_t)(t.first + rn) * g.Hq + (size_t)t.h * G + (pair + kTile - rn * G)) * D + side * (D / 2)));
      }
      // ---- what the rows see
      const int pos = t.n - t.rows + r, lim = pos + 1, low = p.window > 0 ? max(lim - p.window, 0) : 0;
      const int r_first = by_g(pair0), r_last = by_g(min(pair0 + 128, t.pairs) - 1);
      const int lim_all = t.n - t.rows + r_first + 1, low_all = p.window > 0 ? max(t.n - t.rows + r_last + 1 - p.window, 0) : 0;
      float m = -INFINITY;
      f32x2 l2 = pack2(0.f, 0.f);
      int j = 0;
      // Page j: S to weights.  SCALED: of this side's tokens some are scaled.
      auto soften = [&](auto scaled_tag) {
        constexpr bool SCALED = decltype(scaled_tag)::value;
        const int tok = t.seen.logical(page0 + j) * kPageTokens;
        const bool open = tok + kPageTokens <= lim_all && (tok >= low_all || tok + kPageTokens <= p.sinks);       // every row sees the whole page
        const int lim_t = lim - tok, low_t = low - tok, sink_t = p.sinks - tok;
        uint32_t a[16];
        if (!open) {
          // what a row does not see becomes -infinity where it stands (pages at a mask's edge; the code below has no conditions)
#pragma unroll 1
          for (int c = 0; c < 64; c += 32) {
#pragma unroll
            for (int h = 0; h < 32; h += 16) {
              tmem_ld16(tS + c + h, a);
              wait_ld(a);
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                const int u = 64 * side + c + token_at(h + k);
                const bool hidden = (u >= lim_t) | ((u < low_t) & (u >= sink_t));    // (no branches)
                a[k] = hidden ? 0xFF800000u : a[k];
              }
              tmem_st16(tS + c + h, a);
            }
          }
          tc::tc_wait_st();
        }
        float top = -INFINITY;
        [[maybe_unused]] float top_big = -INFINITY;
        if constexpr (SCALED) {
          // logits of tokens whose keys are scaled: as much larger; what those count whose values are scaled (their weights have to fit too)
          const uint4 b = get_scaled(it, side);
          for_tokens(b.x, b.y, [&](int column) {
            tmem_st1(tS + column, __float_as_uint(__uint_as_float(tmem_ld1(tS + column)) * big_up(KB)));
            tc::tc_wait_st();
          });
          for_tokens(b.z, b.w, [&](int column) { top_big = fmaxf(top_big, fmaf(__uint_as_float(tmem_ld1(tS + column)), f, (float)(VB + 1))); });
        }
#pragma unroll 1
        for (int c = 0; c < 64; c += 16) {
          tmem_ld16(tS + c, a);
          wait_ld(a);
          float t0 = max3(top, a[0], a[1]), t1 = max3(__uint_as_float(a[2]), a[3], a[4]);
#pragma unroll
          for (int k = 5; k < 13; k += 4) { t0 = max3(t0, a[k], a[k + 1]); t1 = max3(t1, a[k + 2], a[k + 3]); }
          top = max3(max3(t0, a[13], a[14]), __float_as_uint(t1), a[15]);
        }
        top *= f;
        if constexpr (SCALED) top = fmaxf(top, top_big);
        top = fmaxf(top, exchange(top));
        // ---- the reference moves when a logit passes it by the headroom
        const bool move = top > m + (lift_at(m) + kHeadroom);       // (m = -inf: any logit at all)
        if (__any_sync(FULL, move)) {
          const float nm = move ? top - lift_at(top) : m;
          const float keep = m == -INFINITY ? 0.f : ex2(m - nm);         // (no logit yet: nothing but zeros in O)
          if (j > 0) {
            // (nobody writes O now: this page's product has not been asked for, and S arrived behind the last one's)
#pragma unroll 1
            for (int c = 0; c < D / 2; c += 16) {
              tmem_ld16(tO + c, a);
              wait_ld(a);
#pragma unroll
              for (int k = 0; k < 16; ++k) a[k] = __float_as_uint(__uint_as_float(a[k]) * keep);
              tmem_st16(tO + c, a);
            }
          }
          l2 = mul2(l2, pack2(keep, keep));
          m = nm;
        }
        // ---- weights: 2^(x - m), fp16, where S was (columns that this warp has read)
        const float base = m == -INFINITY ? 0.f : m;
        const f32x2 f2 = pack2(f, f), nb = pack2(-base, -base);
        f32x2 sum = pack2(0.f, 0.f);
        auto weigh = [&](const uint32_t (&s)[16], uint32_t to) {
          uint32_t w16[8];
#pragma unroll
          for (int k = 0; k < 16; k += 2) {
            const float2 e = unpack2(fma2(pack2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), f2, nb));
            const float2 pr = make_float2(ex2(e.x), ex2(e.y));
            sum = add2(sum, pack2(pr.x, pr.y));
            w16[k / 2] = as_u32(__floats2half2_rn(pr.x, pr.y));
          }
          tmem_st8(to, w16);
        };
#pragma unroll 1
        for (int c = 0; c < 64; c += 16) {
          tmem_ld16(tS + c, a);
          wait_ld(a);
          weigh(a, tS + (c >> 1));
        }
        l2 = add2(l2, sum);
        if constexpr (SCALED) {
          // weights of tokens whose values are scaled: as much larger
          tc::tc_wait_st();
          const uint4 b = get_scaled(it, side);
          for_tokens(b.z, b.w, [&](int column) {
            const uint32_t at = tS + (column >> 1), both = tmem_ld1(at), up = as_u32(__float2half2_rn(big_up(VB)));
            tmem_st1(at, as_u32(__hmul2(as_h2(both), as_h2(column & 1 ? (up & 0xFFFF0000u) | 0x3C00u : (up & 0xFFFFu) | 0x3C000000u))));
            tc::tc_wait_st();
          });
        }
        tc::tc_wait_st();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bP + 8 * w);
        ++j; ++it; ++done;
      };
      // (pages with scaled tokens leave the loop over the others: within it their code, never reached, made the prompt 2 to 4 % slower)
#pragma unroll 1
      while (true) {
#pragma unroll 1
        while (true) {
          if (j == pages) goto pages_done;
          wait_warp(bS + 8 * w, done & 1);
          tc::tc_fence_after();
          wait_warp(bVF + 8 * (it & 1), (it >> 1) & 1);          // (there by now: the values' tile and what of it is scaled)
          const uint4 b = get_scaled(it, side);
          if (__any_sync(FULL, (b.x | b.y | b.z | b.w) != 0)) break;
          soften(std::false_type{});
        }
        soften(std::true_type{});
      }
    pages_done:
      // ---- the tile's outputs, or its partial
      wait_warp(bO + 8 * w, seg & 1);
      ++seg;
      tc::tc_fence_after();
      float l = unpack2(l2).x + unpack2(l2).y;
      {
        const float other = exchange(l);
        l = side == 0 ? l + other : other + l;       // (the same sum in both)
      }
      const bool whole = page0 == 0 && pages == t.seen.count;
      const float inv = whole ? (l > 0.f ? 1.0f / l : 0.f) : 1.0f;
      const int slot = 2 * (int)blockIdx.x + (page0 == 0 ? 1 : 0), cr = 128 * w + row;      // (page0 > 0: the tile started in another share)
      // Rows leave through the warp's part of the query tile (done with), so that a store covers whole rows: piece k of 16 bytes of row r
      // goes to place (r + k) % 32 of its 32, which neither the rows' nor the pieces' order makes collide.
      {
        const long long out_row = (long long)(t.first + r) * g.Hq + (long long)t.h * G + (pair - r * G);
        const int wr = row & ~31, rows_here = min(32, t.pairs - pair0 - wr);         // (may be none)
        constexpr int NP = D / 16;                   // pieces of a row, side and round
        uint8_t* stage = smem + sl.q + w * T::kQ + wr * 16 + side * NP * T::kLbQ;
        const bool wide = !whole || out_dtype == KVQ_FP32;                           // 4 bytes a channel: two rounds
        const int step = wide ? D / 4 : D / 2;
#pragma unroll 1
        for (int c0 = 0; c0 < D / 2; c0 += step) {
#pragma unroll 1
          for (int cc = 0; cc < step; cc += 16) {
            uint32_t a[16];
            tmem_ld16(tO + c0 + cc, a);
            wait_ld(a);
            if (wide) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int piece = cc / 4 + k;
                *reinterpret_cast<float4*>(stage + piece * T::kLbQ + ((lane + piece) & 31) * 16) =
                    make_float4(__uint_as_float(a[4 * k]) * inv, __uint_as_float(a[4 * k + 1]) * inv, __uint_as_float(a[4 * k + 2]) * inv, __uint_as_float(a[4 * k + 3]) * inv);
              }
            } else {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const int piece = cc / 8 + k;
                uint32_t o4[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  o4[e] = (uint32_t)f32_to_bits16(__uint_as_float(a[8 * k + 2 * e]) * inv, out_dtype) |
                          ((uint32_t)f32_to_bits16(__uint_as_float(a[8 * k + 2 * e + 1]) * inv, out_dtype) << 16);
                *reinterpret_cast<uint4*>(stage + piece * T::kLbQ + ((lane + piece) & 31) * 16) = make_uint4(o4[0], o4[1], o4[2], o4[3]);
              }
            }
          }
          __syncwarp();
          const int ch0 = side * (D / 2) + c0;       // first channel of the round
          // (all lanes go round as often: they ask each other where a row goes)
#pragma unroll 4
          for (int i = 0; i < rows_here * NP; i += 32) {
            const int idx = min(i + lane, rows_here * NP - 1);
            const int rr = idx / NP, piece = idx % NP;
            const uint4 v = *reinterpret_cast<const uint4*>(stage + piece * T::kLbQ + ((rr + piece) & 31) * 16);
            uint8_t* dst;
            const long long orow = __shfl_sync(FULL, out_row, rr);
            if (whole) dst = static_cast<uint8_t*>(out) + (orow * D + ch0) * (wide ? 4 : 2);
            else dst = reinterpret_cast<uint8_t*>(ws + ((size_t)slot * cap + 128 * w + wr + rr) * D + ch0);
            *reinterpret_cast<uint4*>(dst + 16 * piece) = v;
          }
          __syncwarp();
        }
      }
      tc::tc_fence_before();
      if (whole) continue;
      if (real && side == 0) *reinterpret_cast<float2*>(ws + ml_offset_floats(cap, D) + ((size_t)slot * cap + cr) * 2) = make_float2(m, l);
      const int first = plan.cta_of(c.xs + kGap), parts = plan.cta_of(c.xs + kGap + t.seen.count - 1) - first + 1;
      __threadfence();
      named_bar_sync(1 + w, 256);
      if (row == 0 && side == 0) const_cast<volatile int*>(sMisc)[2 + w] = (int)tagged_count(counts + 2 * first + w, id40);
      named_bar_sync(1 + w, 256);
      if (const_cast<volatile int*>(sMisc)[2 + w] == parts) {
        __threadfence();
        const int rows_w = min(128, t.pairs - pair0);
        const float2* mls = reinterpret_cast<const float2*>(ws + ml_offset_floats(cap, D));
        // the parts' places: the tile starts in the second one of its first CTA, goes on in the first one of those behind
        auto place = [&](int j) { return (size_t)(2 * (first + j) + (j == 0 ? 1 : 0)) * cap + 128 * w; };
        // a thread per 16 bytes of a row, four parts in flight at a time
        constexpr int NP = D / 4;
#pragma unroll 1
        for (int idx = row + 128 * side; idx < rows_w * NP; idx += 256) {
          const int rr = idx / NP, piece = idx & (NP - 1);
          float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
          float ms = -INFINITY, den = 0.f;
#pragma unroll 1
          for (int j = 0; j < parts; j += 4) {
            float2 ml[4];
            float4 o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const size_t at = place(min(j + e, parts - 1)) + rr;
              ml[e] = __ldcg(mls + at);
              o[e] = __ldcg(reinterpret_cast<const float4*>(ws + at * D) + piece);
              if (j + e >= parts) ml[e].x = -INFINITY;
            }
            const float mb = fmaxf(ms, fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)));
            if (mb == -INFINITY) continue;           // (parts without a token for this row: their o is zero, their sum too)
            const float w0 = ms == -INFINITY ? 0.f : ex2(ms - mb);
            den *= w0; num.x *= w0; num.y *= w0; num.z *= w0; num.w *= w0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float wt = ml[e].x == -INFINITY ? 0.f : ex2(ml[e].x - mb);
              den = fmaf(wt, ml[e].y, den);
              num.x = fmaf(wt, o[e].x, num.x); num.y = fmaf(wt, o[e].y, num.y);
              num.z = fmaf(wt, o[e].z, num.z); num.w = fmaf(wt, o[e].w, num.w);
            }
            ms = mb;
          }
          const float iv = den > 0.f ? 1.0f / den : 0.f;
          const int rw = by_g(pair0 + rr);
          const size_t at = ((size_t)(t.first + rw) * g.Hq + (size_t)t.h * G + (pair0 + rr - rw * G)) * D + 4 * piece;
          if (out_dtype == KVQ_FP32) {
            *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(num.x * iv, num.y * iv, num.z * iv, num.w * iv);
          } else {
            uint2 v;
            v.x = (uint32_t)f32_to_bits16(num.x * iv, out_dtype) | ((uint32_t)f32_to_bits16(num.y * iv, out_dtype) << 16);
            v.y = (uint32_t)f32_to_bits16(num.z * iv, out_dtype) | ((uint32_t)f32_to_bits16(num.w * iv, out_dtype) << 16);
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = v;
          }
        }
        if (row == 0 && side == 0) counts[2 * first + w] = 0ull;
      }
      named_bar_sync(1 + w, 256);
    }
  } else if (warp < 28) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsTiles));
    // =========================================================== pages to 16-bit tiles: by blocks of 32 tokens
    const int blk = warp & 3;
    const int ngk = D / g.gk, ngv = D / g.gv;
    // The page to load is one ahead of the one that is written, its number was read a page earlier still.
    const uint8_t* page_ptr = nullptr;
    Cursor nc = start();
    int nid = 0, tokens = 0;                         // of the page at page_ptr: tokens of this warp's block that the sequence holds
    auto look_up = [&]() { if (nc.on) nid = p.table[(long long)nc.t.b * p.table_stride + nc.t.seen.logical(nc.page)]; };
    auto to_next = [&]() {                           // address of the page whose number is there, and on to the number of the one behind
      int id = nid;
      if ((unsigned)id >= (unsigned)p.n_pool) {      // outside the pool: another page is read in its place
        if (lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
        id = 0;
      }
      page_ptr = p.pages + ((size_t)id * Hkv + nc.t.h) * (size_t)g.page_bytes;
      tokens = nc.t.n - nc.t.seen.logical(nc.page) * kPageTokens - 32 * blk;
      if (++nc.page == nc.end) advance(nc);
      look_up();
    };
    look_up();
    // Scales and zero-points of the lane's token, a word per group; nothing of tokens that the sequence does not hold (their bytes are
    // anything).  True where a value may pass the fp16 range (zero-points are in it).
    auto load_meta = [&](uint32_t (&m)[4], int off, int count) {
      const uint32_t* src = reinterpret_cast<const uint32_t*>(page_ptr + off) + (32 * blk + lane) * count;
#pragma unroll
      for (int e = 0; e < NI; ++e) if (e < count) m[e] = src[e];
    };
    auto check_meta = [&](uint32_t (&m)[4], int count, float qmax, bool there) {
      bool wide = false;
#pragma unroll
      for (int e = 0; e < NI; ++e) {
        if (e < count) {
          if (!there) m[e] = 0u;
          const float2 sz = __half22float2(as_h2(m[e]));
          wide |= fmaf(sz.x, qmax, sz.y) > 65504.0f;
        }
      }
      return wide;
    };
    auto scale_meta = [&](uint32_t (&m)[4], int count, float down) {
#pragma unroll
      for (int e = 0; e < NI; ++e) if (e < count) m[e] = as_u32(__hmul2(as_h2(m[e]), __float2half2_rn(down)));
    };
    int it = 0;
    if (warp < 24) {
      // ------------------------------------------------------------ keys: two warps a block, half of the passes of eight tokens each
      const int half = (warp >> 2) & 1;
      const int tl = lane & 7, ch = lane >> 3;       // token of a pass of eight (neighbours in place), quarter of its row
      constexpr int KCB = (KW < 4 ? KW : 4) * 4;
      const Codes<KB> kc;
      uint32_t kw[2][KW], km[4] = {0u, 0u, 0u, 0u};
      auto load = [&]() {
#pragma unroll
        for (int k = 0; k < 2; ++k) load_words<KW>(page_ptr + (32 * blk + token_at(8 * k + 16 * half + tl)) * (D * KB / 8) + ch * KCB, 64, kw[k]);
        load_meta(km, g.k_meta_off, ngk);
      };
      bool more = nc.on;
      if (more) { to_next(); load(); }
#pragma unroll 1
      for (; more; ++it) {
          const int buf = it & 1;
          const bool there = lane < tokens;
          const bool wide = check_meta(km, ngk, (float)((1 << KB) - 1), there);
          if (wide) scale_meta(km, ngk, 1.0f / big_up(KB));
          const uint32_t big = __ballot_sync(FULL, wide);
          if (it >= 2) wait_warp(bKE + 8 * buf, ((it >> 1) - 1) & 1);
          if (half == 0 && lane == 0) set_scaled(it, blk, 0, big);
          uint8_t* dst = smem + sl.k + buf * T::kK;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int u = token_at(8 * k + 16 * half + tl);
            uint8_t* row = dst + (4 * blk + 2 * half + k) * 128 + tl * 16;
            __half2 s, z;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
              if (i == 0 || ((32 * i) & (g.gk - 1)) == 0) {      // a new group (the same for all lanes)
                const int e = (32 * i) / g.gk;
                const uint32_t meta = __shfl_sync(FULL, e == 0 ? km[0] : e == 1 ? km[1 % NI] : e == 2 ? km[2 % NI] : km[3 % NI], u);
                s = __low2half2(as_h2(meta)); z = __high2half2(as_h2(meta));
              }
              // slots 2 i and 2 i + 1: fields of a word, or words
              constexpr int FPK = 8 / KB;
              const uint32_t w0 = kw[k][(2 * i) / FPK], w1 = kw[k][(2 * i + 1) / FPK];
              const int f0 = (2 * i) % FPK, f1 = (2 * i + 1) % FPK;
              *reinterpret_cast<uint4*>(row + (4 * i + ch) * T::kLbK) = make_uint4(kc.values(w0, f0, s, z), kc.values(w0 >> 8, f0, s, z),
                                                                                   kc.values(w1, f1, s, z), kc.values(w1 >> 8, f1, s, z));
            }
          }
          tc::fence_async_smem();
          __syncwarp();
          if (lane == 0 && it != skip_x) mbar_arrive(bKF + 8 * buf);      // (skip_x: test hook - a page that never arrives)
          more = nc.on;
          if (more) { to_next(); load(); }
      }
    } else {
      // ------------------------------------------------------------ values
      const int vl = lane & 7, tq = lane >> 3;       // channel of eight, place of the chunk
      uint32_t vm[4] = {0u, 0u, 0u, 0u};
      uint4 vw[NMW];
      const Codes<VB> vc;
      auto load = [&]() {
        const uint8_t* v = page_ptr + g.v_codes_off + blk * (4 * D * VB) + (4 * vl + tq) * 16;
#pragma unroll
        for (int mw = 0; mw < NMW; ++mw) vw[mw] = *reinterpret_cast<const uint4*>(v + 512 * mw);
        load_meta(vm, g.v_meta_off, ngv);
      };
      bool more = nc.on;
      if (more) { to_next(); load(); }
#pragma unroll 1
      for (; more; ++it) {
          const int buf = it & 1;
          const bool there = lane < tokens;
          const bool wide = check_meta(vm, ngv, (float)((1 << VB) - 1), there);
          if (wide) scale_meta(vm, ngv, 1.0f / big_up(VB));
          const uint32_t big = __ballot_sync(FULL, wide);
          if (it >= 2) wait_warp(bVE + 8 * buf, ((it >> 1) - 1) & 1);
          if (lane == 0) set_scaled(it, blk, 1, big);
          uint8_t* dst = smem + sl.v + buf * T::kV + vl * 16 + (4 * blk + tq) * T::kLbV;
          __half2 s[2][2], z[2][2];                  // [half][pair of tokens]
#pragma unroll
          for (int mw = 0; mw < NMW; ++mw) {
#pragma unroll
            for (int f = 0; f < FPB; ++f) {
              const int m16 = mw * FPB + f;          // channels 16 m16 .. 16 m16 + 15
              if (m16 == 0 || ((16 * m16) & (g.gv - 1)) == 0) {
                const int e = 16 * m16 / g.gv;
                const uint32_t own = e == 0 ? vm[0] : e == 1 ? vm[1 % NI] : e == 2 ? vm[2 % NI] : vm[3 % NI];
#pragma unroll
                for (int kh = 0; kh < 2; ++kh) {
#pragma unroll
                  for (int pr = 0; pr < 2; ++pr) {
                    const uint32_t m0 = __shfl_sync(FULL, own, 16 * kh + 2 * tq + 8 * pr), m1 = __shfl_sync(FULL, own, 16 * kh + 2 * tq + 8 * pr + 1);
                    s[kh][pr] = as_h2(prmt(m0, m1, 0x5410u));
                    z[kh][pr] = as_h2(prmt(m0, m1, 0x7632u));
                  }
                }
              }
              // words (row half, token half): bytes 0, 2 are tokens 2 tq, 2 tq + 1 of the half, bytes 1, 3 those eight further
              *reinterpret_cast<uint4*>(dst + 2 * m16 * 128) = make_uint4(vc.values(vw[mw].x, f, s[0][0], z[0][0]), vc.values(vw[mw].x >> 8, f, s[0][1], z[0][1]),
                                                                          vc.values(vw[mw].y, f, s[1][0], z[1][0]), vc.values(vw[mw].y >> 8, f, s[1][1], z[1][1]));
              *reinterpret_cast<uint4*>(dst + (2 * m16 + 1) * 128) = make_uint4(vc.values(vw[mw].z, f, s[0][0], z[0][0]), vc.values(vw[mw].z >> 8, f, s[0][1], z[0][1]),
                                                                                vc.values(vw[mw].w, f, s[1][0], z[1][0]), vc.values(vw[mw].w >> 8, f, s[1][1], z[1][1]));
            }
          }
          tc::fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bVF + 8 * buf);
          more = nc.on;
          if (more) { to_next(); load(); }
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRest));
    if (warp == 28) {
    // =========================================================== products
    // The whole warp goes along on values that it shares (counts come from one lane), so that descriptors are made on the uniform path: a
    // product per 64 cycles leaves the one thread that issues it few instructions.
    const uint32_t dk = desc_low(smem_u32(smem + sl.k), T::kLbK), dv = desc_low(smem_u32(smem + sl.v), T::kLbV), dq = desc_low(smem_u32(smem + sl.q), T::kLbQ);
    const uint32_t tm = __shfl_sync(FULL, tmem, 0);
    auto keys = [&](int w, int buf) {                // S = Q K^T
      const uint32_t a = dq + w * (T::kQ >> 4), b = dk + buf * (T::kK >> 4), d = tm + kColS + 128 * w;
      if (elect_one()) {
        mma_ss<false>(d, a, b, idesc(128));
#pragma unroll
        for (int k = 1; k < D / 16; ++k) mma_ss<true>(d, a + k * (2 * T::kLbQ >> 4), b + k * (2 * T::kLbK >> 4), idesc(128));
        tc::tc_commit(bS + 8 * w);
      }
      __syncwarp();
    };
    auto values = [&](int w, int buf, uint32_t add) {  // O += P V
      const uint32_t a = tm + kColS + 128 * w, b = dv + buf * (T::kV >> 4), d = tm + kColO + 128 * w;
      if (elect_one()) {
        mma_ts(d, a, b, idesc(D), add);
#pragma unroll
        for (int k = 1; k < 8; ++k) mma_ts(d, a + 8 * k + (k >= 4 ? 32 : 0), b + k * (2 * T::kLbV >> 4), idesc(D), 1u);
      }
      __syncwarp();
    };
    auto commit = [&](uint32_t b) {
      if (elect_one()) tc::tc_commit(b);
      __syncwarp();
    };
    uint32_t it = 0, done = 0, seg = 0;              // pages; phases of P (page 2^w) and of the queries, a bit per half
#pragma unroll 1
    for (Cursor c = start(); c.on; advance(c)) {
      const int halves = __shfl_sync(FULL, c.t.i * kTile + 128 < c.t.pairs ? 2 : 1, 0), pages = __shfl_sync(FULL, c.end - c.page, 0);
      // step 0: the first page's S of both halves; then, page by page and half by half: O of this page, S of the next
#pragma unroll 1
      for (int j = -1; j < pages; ++j) {
        const uint32_t buf = it & 1, nbuf = (it + (j >= 0)) & 1;
        if (j >= 0) wait_warp(bVF + 8 * buf, (it >> 1) & 1);
#pragma unroll 1
        for (int w = 0; w < halves; ++w) {
          if (j >= 0) {
            wait_warp(bP + 8 * w, (done >> w) & 1);
            done ^= 1u << w;
            tc::tc_fence_after();
            if (!aborted) values(w, buf, j > 0);
            if (w == halves - 1) commit(bVE + 8 * buf);
          } else {
            wait_warp(bQ + 8 * w, (seg >> w) & 1);
            seg ^= 1u << w;
          }
          if (j + 1 < pages) {
            if (w == 0) wait_warp(bKF + 8 * nbuf, ((it + (j >= 0)) >> 1) & 1);
            tc::tc_fence_after();
            if (!aborted) keys(w, nbuf);
            if (w == halves - 1) commit(bKE + 8 * nbuf);
          } else {
            commit(bO + 8 * w);
          }
        }
        if (j >= 0) ++it;
      }
    }
    // nothing of this CTA's may still run on the tensor cores when its tensor memory is freed
    commit(bDrain);
    if (lane == 0) mbar_wait(bDrain, 0, wait_ns);
    __syncwarp();
    }
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (warp == 28) tc::tmem_dealloc(tmem, kTmemCols);
}

template <int D, int KB, int VB>
int launch_chunk_inst(const Geom& g, const Paged& p, const void* q, float c1, float* ws, void* out, int out_dtype, unsigned long long call_id,
                      unsigned long long wait_ns, long long skip_x, cudaStream_t stream) {
  const Smem sl = smem_of<D>(g.B);
  auto kern = chunk_kernel<D, KB, VB>;
  // (an increase of registers waits for ever where the block was launched with fewer than the roles take together)
  static const bool fits = [&] {
    cudaFuncAttributes a;
    return cudaFuncGetAttributes(&a, kern) == cudaSuccess && a.numRegs >= kRegsLaunch;
  }();
  if (!fits) return KVQ_ERR_CUDA_LAUNCH;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, sl.total) != cudaSuccess) return KVQ_ERR_CUDA_LAUNCH;
  const long long pairs = (long long)p.max_rows * g.G;
  const cudaError_t e = launch_dependent(kern, dim3(kGrid), kThreads, sl.total, stream, 1, g, p, static_cast<const uint16_t*>(q), c1, ws,
                                         row_cap(pairs > kTile ? kTile : (int)pairs), out, out_dtype, call_id, wait_ns, skip_x);
  return e == cudaSuccess ? KVQ_OK : KVQ_ERR_CUDA_LAUNCH;
}

}  // namespace chunk
}  // namespace kvq
