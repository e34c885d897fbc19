// Paged attention of many query rows on the fifth-generation tensor cores: softmax(q K^T / sqrt(d)) V (App. A.1) over a paged packed cache,
// with a causal mask, a sliding window and first tokens that stay visible.
//
// A tile is 256 (query row, head) pairs of one sequence and KV head - the query heads of a KV head are rows of one product - against pages of 128
// tokens.  One CTA per SM:
//  * warps 8-11 turn a page into 16-bit tiles in shared memory: codes become fp16 by a byte permute and an exact subtraction, scale and
//    zero-point enter by one fused operation (one rounding, 2^-11 of the value at most).  Their packed words were loaded a page ahead, straight
//    into registers.  The order of channels (keys) and of tokens (both) is the one in which codes lie in the page; queries and the weights
//    follow it, so that nothing is transposed.
//  * one thread of warp 12 issues tcgen05.mma (kind f16, M 128, fp32 accumulators in tensor memory): S = Q K^T of both halves of the tile
//    in turn, and O += P V with P read from tensor memory, where it takes the place of S.
//  * warps 0-3 and 4-7 take the two halves, a thread per row: row maximum, p = 2^(x - reference), fp16 weights back to tensor memory;
//    sums in fp32.  While one half's softmax runs, the tensor cores have the other half's products.  The reference moves only when a logit
//    passes it by kHeadroom bits; then the row's outputs are rescaled in tensor memory.
// The order of the fp16 weights' rounding (2^-11 of a weight at most) and of the tiles' is the loss against fp32; all sums are fp32.
// bf16 queries are scaled by a power of two per row, pages whose values pass half the fp16 range by 2^-10 (undone in fp32 and in P).
//
// The (tile, page) pairs of a call lie on one axis that is cut into equal shares, one per CTA, so that a long prompt, a ragged batch and a few
// drafted rows behind a long context all fill the GPU.  A tile that falls to several CTAs leaves partials (m, l, o); the CTA that comes last
// merges them by log-sum-exp, in a fixed order.
// Every wait is bounded; on expiry the kernel sets KVQ_STATUS_DEVICE_TIMEOUT, goes on without waiting (nothing that it then reads is out of range) and
// frees its tensor memory.
#pragma once

#include "kvq_paged.cuh"
#include "kvq_tcgen05.cuh"

namespace kvq {
namespace chunk {

using namespace mma;
using tc::smem_desc;

constexpr int kThreads = 13 * 32;
constexpr int kGrid = 148;
constexpr int kTile = 256;                 // (query row, head) pairs of a tile
constexpr float kHeadroom = 4.0f;
constexpr float kBigDown = 9.765625e-4f, kBigUp = 1024.0f;      // 2^-10 for pages whose values pass half the fp16 range, and back
constexpr uint32_t FULL = 0xffffffffu;
// tensor memory: S of the two halves (their first 64 columns take P), then O of the two halves
constexpr uint32_t kColS = 0, kColO = 256, kTmemCols = 512;
// fp16 operands, fp32 accumulate, both K-major, M 128
__host__ __device__ constexpr uint32_t idesc(int n) { return (1u << 4) | ((uint32_t)(n / 8) << 17) | (8u << 24); }

// Shared memory.  Operands lie in 8 x 16-byte core matrices: rows 16 bytes apart, octets of rows 128, chunks of eight k `lb` apart (keys and
// values 32 bytes more than dense, which spreads the writers' lanes over the banks).
template <int D> struct Tiles {
  static constexpr int kLbQ = 128 * 16, kLbK = 128 * 16 + 32, kLbV = D * 16 + 32;
  static constexpr int kQ = D / 8 * kLbQ, kK = D / 8 * kLbK, kV = 16 * kLbV;      // bytes of a query half, a key and a value tile
};
struct Smem { int q, k, v, bars, misc, pref, seq, total; };
template <int D>
__host__ __device__ inline Smem smem_of(int batch) {
  using T = Tiles<D>;
  Smem s;
  s.q = 0;
  s.k = 2 * T::kQ;
  s.v = s.k + 2 * T::kK;
  s.bars = s.v + 2 * T::kV;
  s.misc = s.bars + 32 * 8;
  s.pref = s.misc + 64;
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
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(id), "r"(acc) : "memory");
}
#define KVQ_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define KVQ_W8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define KVQ_S8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : KVQ_R8(r, 0), KVQ_R8(r, 8), KVQ_R8(r, 16), KVQ_R8(r, 24) : "r"(addr) : "memory");
}
// Waits for this thread's loads from tensor memory; the registers go through it, so that nothing is computed from them before.
__device__ __forceinline__ void wait_ld(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : KVQ_W8(r, 0), KVQ_W8(r, 8), KVQ_W8(r, 16), KVQ_W8(r, 24)::"memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(addr), KVQ_S8(r, 0), KVQ_S8(r, 8), KVQ_S8(r, 16), KVQ_S8(r, 24) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(addr), KVQ_S8(r, 0), KVQ_S8(r, 8) : "memory");
}
__device__ __forceinline__ uint32_t permute(uint32_t a, uint32_t b, uint32_t sel) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(sel));
  return d;
}
__device__ __forceinline__ bool bar_any(int id, int nthreads, bool p) {
  uint32_t r;
  __syncwarp();
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"((uint32_t)p), "r"(id), "r"(nthreads) : "memory");
  return r != 0;
}

// Token of a page's block of 32 that stands at place k of its 32 columns: codes of four tokens share a word, those of two halves a load.
__host__ __device__ constexpr int token_at(int k) { return 16 * ((k & 7) >> 2) + 2 * (k >> 3) + ((k & 3) >> 1) + 8 * (k & 1); }
__host__ __device__ constexpr int place_of(int u) { return 8 * ((u & 7) >> 1) + 4 * (u >> 4) + 2 * (u & 1) + ((u >> 3) & 1); }

// Code bytes lo, hi of a word as fp16 numbers times scale plus zero-point, one rounding (byte -> 0x64bb = 1024 + code, minus 1024: exact).
__device__ __forceinline__ uint32_t values2(uint32_t bytes, uint32_t sel, __half2 s, __half2 z) {
  const __half2 code = __hsub2(as_h2(permute(bytes, 0x64646464u, sel)), __half2half2(__ushort_as_half(0x6400)));
  return as_u32(__hfma2(code, s, z));
}

// A tile: its rows, and the pages that they see.
struct Tile {
  int b, h, i;                 // sequence, KV head, tile of the sequence's (row, head) pairs
  int n, rows, first, pairs;   // of the sequence
  SeenPages seen;
};
struct Share { long long lo, hi; int b, h, i, page; };       // of a CTA: positions on the axis, tile and page of the first

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
  long long* sPref = reinterpret_cast<long long*>(smem + sl.pref);      // (tile, page) pairs in front of every sequence
  int* sSeq = reinterpret_cast<int*>(smem + sl.seq);                    // tokens, rows, first row
  int* sMisc = reinterpret_cast<int*>(smem + sl.misc);                  // [0] abort [1] tensor memory [2, 3] counts returned [4..7] pages of big values [8..11] share
  volatile int* abort_flag = sMisc;
  volatile int* sBig = sMisc + 4;
  const int tid_ = threadIdx.x, lane = tid_ & 31, warp = __shfl_sync(FULL, tid_ >> 5, 0);
  const int B = g.B, G = g.G, Hkv = g.Hkv;
  // barriers: key tile full / empty [2], value tile full / empty [2], queries [2], S [2], P [2], O [2], drain
  const uint32_t bar = smem_u32(smem + sl.bars);
  const uint32_t bKF = bar, bKE = bar + 16, bVF = bar + 32, bVE = bar + 48, bQ = bar + 64, bS = bar + 80, bP = bar + 96, bO = bar + 112, bDrain = bar + 128;

  if (tid_ == 0) {
    sMisc[0] = 0;
    for (int k = 0; k < 2; ++k) {
      mbar_init(bKF + 8 * k, 4); mbar_init(bKE + 8 * k, 1); mbar_init(bVF + 8 * k, 4); mbar_init(bVE + 8 * k, 1);
      mbar_init(bQ + 8 * k, 4); mbar_init(bS + 8 * k, 1); mbar_init(bP + 8 * k, 4); mbar_init(bO + 8 * k, 1);
    }
    mbar_init(bDrain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  begin_after_predecessor();
  if (warp == 12) {
    tc::tmem_alloc(smem_u32(&sMisc[1]), kTmemCols);
    tc::tmem_relinquish();
  }
  // ---- plan: (tile, page) pairs per sequence, this CTA's share
  auto seen_by = [&](int n, int rows, int pairs, int i) {
    const int r0 = i * kTile / G, r1 = min(i * kTile + kTile, pairs) - 1;
    return seen_pages(n - rows + r0, n - rows + r1 / G, p.window, p.sinks);
  };
  for (int b = warp; b < B; b += kThreads / 32) {
    bool bad;
    const SeqRows s = seq_rows(p, b, g.capacity, p.max_rows, bad);
    if (bad && lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
    const int pairs = s.rows * G;
    long long sum = 0;
    for (int i = lane; i * kTile < pairs; i += 32) sum += seen_by(s.n, s.rows, pairs, i).count;
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
    int i0 = 0, page = 0, tile = 0;
    bool found = false;
    for (; !found && i0 * kTile < pairs; i0 += 32) {
      const int i = i0 + lane;
      const long long own = i * kTile < pairs ? seen_by(n, rows, pairs, i).count : 0;
      long long v = own;
      for (int off = 1; off < 32; off <<= 1) {
        const long long u = __shfl_up_sync(FULL, v, off);
        if (lane >= off) v += u;
      }
      const uint32_t beyond = __ballot_sync(FULL, v > rest);
      if (beyond) {
        const int src = __ffs(beyond) - 1;
        page = (int)(rest - __shfl_sync(FULL, v - own, src));
        tile = i0 + src;
        found = true;
      } else {
        rest -= __shfl_sync(FULL, v, 31);
      }
    }
    if (lane == 0) { sMisc[8] = lo; sMisc[9] = h; sMisc[10] = tile; sMisc[11] = page; }
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
  // Segments: the pages of one tile that lie in the share.  each(tile, first page, pages).
  auto segments = [&](auto&& each) {
    if (x_lo >= x_hi) return;
    Tile t = tile_of(sMisc[8], sMisc[9], sMisc[10]);
    int page = sMisc[11];
    for (long long x = x_lo; x < x_hi;) {
      const int pages = (int)min((long long)(t.seen.count - page), x_hi - x);
      each(t, page, pages, x);
      x += pages;
      page = 0;
      if (x < x_hi) t = next_tile(t);
    }
  };
  bool aborted = false;
  // A wait of a whole warp; after a time-out the role goes on without waiting.
  auto wait_warp = [&](uint32_t b, uint32_t parity) {
    if (aborted) return;
    if (__all_sync(FULL, mbar_try_wait(b, parity))) return;
    const bool got = tc::wait_or_abort(b, parity, wait_ns, abort_flag);
    if (!__all_sync(FULL, got)) {
      aborted = true;
      *abort_flag = 1;
      if (lane == 0) atomicOr(p.status, KVQ_STATUS_DEVICE_TIMEOUT);
      __syncwarp();
    }
  };

  if (warp < 8) {
    // =========================================================== softmax: half w of the tile, a thread per row
    const int w = warp >> 2, row = tid_ & 127;
    const uint32_t tS = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + kColS + 128 * w, tO = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + kColO + 128 * w;
    uint8_t* sq = smem + sl.q + w * T::kQ + (row >> 3) * 128 + (row & 7) * 16;
    const unsigned long long id40 = (call_id & 0xFFFFFFFFFFull) ? (call_id & 0xFFFFFFFFFFull) : 1ull;
    unsigned long long* counts = reinterpret_cast<unsigned long long*>(ws + count_offset_floats(cap, D));
    int it = 0, done = 0, seg = 0;                   // pages of the share so far, those that this half had, segments it had
    segments([&](const Tile& t, int page0, int pages, long long x) {
      const int pair0 = t.i * kTile + 128 * w;
      if (pair0 >= t.pairs) { it += pages; return; }
      // ---- the row's query: fp16 in the order of the key tiles' channels, scaled to at most 2^15 in size
      const int pair = pair0 + row, r = min(pair, t.pairs - 1) / G;
      const bool real = pair < t.pairs;
      float f = c1;
      {
        const uint16_t* src = q + ((size_t)(t.first + r) * g.Hq + (size_t)t.h * G + (pair - r * G)) * D;
        uint32_t qw[D / 2];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (real) v = *reinterpret_cast<const uint4*>(src + 8 * k);
          qw[4 * k] = v.x; qw[4 * k + 1] = v.y; qw[4 * k + 2] = v.z; qw[4 * k + 3] = v.w;
          top = __vmaxu2(__vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)), top);
        }
        if (g.in_dtype == KVQ_BF16) {
          // |q| has the exponent of its 16-bit pattern: bring the largest to 2^0 .. 2^1
          const int e = (int)(max(top & 0xFFFFu, top >> 16) >> 7);
          const int shift = e == 0 ? 0 : min(max(127 - e, -126), 126);
          const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
          f = c1 * __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll
          for (int k = 0; k < D / 2; ++k)
            qw[k] = as_u32(__floats2half2_rn(__uint_as_float(qw[k] << 16) * up, __uint_as_float(qw[k] & 0xFFFF0000u) * up));
        }
        // chunk 4 i + ch: channels 32 i + 4 ch + {0..3}, then those 16 further
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          const int i = k >> 2, ch = k & 3, a = (32 * i + 4 * ch) / 2;
          *reinterpret_cast<uint4*>(sq + k * T::kLbQ) = make_uint4(qw[a], qw[a + 1], qw[a + 8], qw[a + 9]);
        }
      }
      tc::fence_async_smem();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bQ + 8 * w);
      // ---- what the rows see
      const int pos = t.n - t.rows + r, lim = pos + 1, low = p.window > 0 ? max(lim - p.window, 0) : 0;
      const int r_first = pair0 / G, r_last = (min(pair0 + 128, t.pairs) - 1) / G;
      const int lim_all = t.n - t.rows + r_first + 1, low_all = p.window > 0 ? max(t.n - t.rows + r_last + 1 - p.window, 0) : 0;
      float m = -INFINITY;
      f32x2 l2 = pack2(0.f, 0.f);
#pragma unroll 1
      for (int j = 0; j < pages; ++j, ++it, ++done) {
        wait_warp(bS + 8 * w, done & 1);
        tc::tc_fence_after();
        const bool big = sBig[it & 3] != 0;
        const float fs = big ? f * kBigUp : f;
        const int tok = t.seen.logical(page0 + j) * kPageTokens;
        const bool open = tok + kPageTokens <= lim_all && (tok >= low_all || tok + kPageTokens <= p.sinks);       // every row sees the whole page
        const int lim_t = lim - tok, low_t = low - tok, sink_t = p.sinks - tok;
        auto sees = [&](int c, int k) {              // column 32 c + k
          const int u = 32 * c + token_at(k);
          return u < lim_t && (u >= low_t || u < sink_t);
        };
        auto page_pass = [&](auto masked_tag) {
          constexpr bool MASKED = decltype(masked_tag)::value;
          uint32_t a[32], b[32];
          float top = -INFINITY;
          auto max_of = [&](const uint32_t (&s)[32], int c) {
            float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              float x0 = __uint_as_float(s[k]), x1 = __uint_as_float(s[k + 1]);
              if (MASKED) { if (!sees(c, k)) x0 = -INFINITY; if (!sees(c, k + 1)) x1 = -INFINITY; }
              t0 = fmaxf(t0, x0); t1 = fmaxf(t1, x1);
            }
            top = fmaxf(top, fmaxf(t0, t1));
          };
          tmem_ld32(tS, a);
          wait_ld(a);
          tmem_ld32(tS + 32, b);
          max_of(a, 0);
          wait_ld(b);
          tmem_ld32(tS + 64, a);
          max_of(b, 1);
          wait_ld(a);
          tmem_ld32(tS + 96, b);
          max_of(a, 2);
          wait_ld(b);
          tmem_ld32(tS, a);                          // the second pass's first columns are on their way
          max_of(b, 3);
          top *= fs;
          // ---- the reference moves when a logit passes it by the headroom
          const bool move = top > m + kHeadroom;     // (m = -inf: any logit at all)
          if (__any_sync(FULL, move)) {
            const float nm = move ? top : m;
            const float keep = m == -INFINITY ? 0.f : ex2(m - nm);       // (no logit yet: nothing but zeros in O)
            if (j > 0) {
              // (nobody writes O now: this page's product has not been asked for, and S arrived behind the last one's.  a is waited for first.)
              wait_ld(a);
#pragma unroll 1
              for (int c = 0; c < D / 32; ++c) {
                tmem_ld32(tO + 32 * c, b);
                wait_ld(b);
#pragma unroll
                for (int k = 0; k < 32; ++k) b[k] = __float_as_uint(__uint_as_float(b[k]) * keep);
                tmem_st32(tO + 32 * c, b);
              }
            }
            l2 = mul2(l2, pack2(keep, keep));
            m = nm;
          }
          // ---- weights: 2^(x - m), fp16, where S was (columns that this warp has read); pages of big values carry P times 2^10
          const float base = m == -INFINITY ? 0.f : m;
          const f32x2 f2 = pack2(fs, fs), nb = pack2(-base, -base);
          f32x2 sum = pack2(0.f, 0.f);
          auto weigh = [&](const uint32_t (&s)[32], int c) {
            uint32_t w16[16];
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              const float2 e = unpack2(fma2(pack2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), f2, nb));
              float2 pr = make_float2(ex2(e.x), ex2(e.y));
              if (MASKED) { if (!sees(c, k)) pr.x = 0.f; if (!sees(c, k + 1)) pr.y = 0.f; }
              sum = add2(sum, pack2(pr.x, pr.y));
              if (big) { pr.x *= kBigUp; pr.y *= kBigUp; }
              w16[k / 2] = as_u32(__floats2half2_rn(pr.x, pr.y));
            }
            tmem_st16(tS + 16 * c, w16);
          };
          wait_ld(a);
          tmem_ld32(tS + 32, b);
          weigh(a, 0);
          wait_ld(b);
          tmem_ld32(tS + 64, a);
          weigh(b, 1);
          wait_ld(a);
          tmem_ld32(tS + 96, b);
          weigh(a, 2);
          wait_ld(b);
          weigh(b, 3);
          l2 = add2(l2, sum);
        };
        if (open) page_pass(std::false_type{});
        else page_pass(std::true_type{});
        tc::tc_wait_st();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bP + 8 * w);
      }
      // ---- the tile's outputs, or its partial
      wait_warp(bO + 8 * w, seg & 1);
      ++seg;
      tc::tc_fence_after();
      const float l = unpack2(l2).x + unpack2(l2).y;
      const long long xs = x - page0;                // where the tile starts on the axis
      const bool whole = page0 == 0 && pages == t.seen.count;
      const float inv = whole ? (l > 0.f ? 1.0f / l : 0.f) : 1.0f;
      const size_t oi = ((size_t)(t.first + r) * g.Hq + (size_t)t.h * G + (pair - r * G)) * D;
      const int slot = 2 * (int)blockIdx.x + (page0 == 0 ? 1 : 0), cr = 128 * w + row;      // (page0 > 0: the tile started in another share)
      float* po = ws + ((size_t)slot * cap + cr) * D;
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t a[32];
        tmem_ld32(tO + 32 * c, a);
        wait_ld(a);
        if (!real) continue;
        if (whole && out_dtype != KVQ_FP32) {
#pragma unroll
          for (int k = 0; k < 32; k += 8) {
            uint32_t o4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o4[e] = (uint32_t)f32_to_bits16(__uint_as_float(a[k + 2 * e]) * inv, out_dtype) |
                      ((uint32_t)f32_to_bits16(__uint_as_float(a[k + 2 * e + 1]) * inv, out_dtype) << 16);
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + oi + 32 * c + k) = make_uint4(o4[0], o4[1], o4[2], o4[3]);
          }
        } else {
          float* dst = whole ? static_cast<float*>(out) + oi : po;
#pragma unroll
          for (int k = 0; k < 32; k += 4)
            *reinterpret_cast<float4*>(dst + 32 * c + k) = make_float4(__uint_as_float(a[k]) * inv, __uint_as_float(a[k + 1]) * inv,
                                                                       __uint_as_float(a[k + 2]) * inv, __uint_as_float(a[k + 3]) * inv);
        }
      }
      tc::tc_fence_before();
      if (whole) return;
      if (real) *reinterpret_cast<float2*>(ws + ml_offset_floats(cap, D) + ((size_t)slot * cap + cr) * 2) = make_float2(m, l);
      const int first = plan.cta_of(xs), parts = plan.cta_of(xs + t.seen.count - 1) - first + 1;
      __threadfence();
      named_bar_sync(1 + w, 128);
      if (row == 0) const_cast<volatile int*>(sMisc)[2 + w] = (int)tagged_count(counts + 2 * first + w, id40);
      named_bar_sync(1 + w, 128);
      if (const_cast<volatile int*>(sMisc)[2 + w] == parts) {
        __threadfence();
        const int rows_w = min(128, t.pairs - pair0);
        for (int idx = row; idx < rows_w * (D / 4); idx += 128) {
          const int rr = idx / (D / 4), c4 = idx % (D / 4), pr = pair0 + rr;
          float ms = -INFINITY, den = 0.f;
          float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int j0 = 0; j0 < parts; j0 += 8) {
            float2 ml[8];
            float4 o[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int j = min(j0 + u, parts - 1);
              const size_t at = (size_t)(2 * (first + j) + (j == 0 ? 1 : 0)) * cap + 128 * w + rr;
              ml[u] = __ldcg(reinterpret_cast<const float2*>(ws + ml_offset_floats(cap, D)) + at);
              o[u] = __ldcg(reinterpret_cast<const float4*>(ws + at * D) + c4);
              if (j0 + u >= parts) ml[u].x = -INFINITY;
            }
            float mb = ms;
#pragma unroll
            for (int u = 0; u < 8; ++u) mb = fmaxf(mb, ml[u].x);
            if (mb == -INFINITY) continue;
            const float keep = ms == -INFINITY ? 0.f : ex2(ms - mb);
            den *= keep; num.x *= keep; num.y *= keep; num.z *= keep; num.w *= keep;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const float wt = ml[u].x == -INFINITY ? 0.f : ex2(ml[u].x - mb);
              if (wt != 0.f) {
                den = fmaf(wt, ml[u].y, den);
                num.x = fmaf(wt, o[u].x, num.x); num.y = fmaf(wt, o[u].y, num.y);
                num.z = fmaf(wt, o[u].z, num.z); num.w = fmaf(wt, o[u].w, num.w);
              }
            }
            ms = mb;
          }
          const float iv = den > 0.f ? 1.0f / den : 0.f;
          const size_t at = ((size_t)(t.first + pr / G) * g.Hq + (size_t)t.h * G + pr % G) * D + 4 * c4;
          if (out_dtype == KVQ_FP32) {
            *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(num.x * iv, num.y * iv, num.z * iv, num.w * iv);
          } else {
            uint2 v;
            v.x = (uint32_t)f32_to_bits16(num.x * iv, out_dtype) | ((uint32_t)f32_to_bits16(num.y * iv, out_dtype) << 16);
            v.y = (uint32_t)f32_to_bits16(num.z * iv, out_dtype) | ((uint32_t)f32_to_bits16(num.w * iv, out_dtype) << 16);
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = v;
          }
        }
        if (row == 0) counts[2 * first + w] = 0ull;
      }
      named_bar_sync(1 + w, 128);
    });
  } else if (warp < 12) {
    // =========================================================== pages to 16-bit tiles: warp `blk` takes a block of 32 tokens
    const int blk = warp - 8;
    const int ngk = D / g.gk, ngv = D / g.gv;
    const int tl = lane >> 2, ch = lane & 3;         // keys: token of a pass, quarter of its row
    constexpr int KCB = (KW < 4 ? KW : 4) * 4;
    uint32_t kw[4][KW], km[4], vm[4];
    uint4 vw[NMW];
    // token (of 32) that lane group tl of pass k takes: neighbours in place, for writes without bank conflicts
    auto pass_token = [&](int k) { return (tl >> 1) + 8 * (tl & 1) + 4 * (k & 1) + 16 * (k >> 1); };
    const uint8_t* page_ptr = nullptr;
    auto find = [&](const Tile& t, int i) {          // the page's address
      int id = pool_page(p, t.b, t.seen.logical(i));
      if (id < 0) {
        if (lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
        id = 0;
      }
      page_ptr = p.pages + ((size_t)id * Hkv + t.h) * (size_t)g.page_bytes;
    };
    auto load_keys = [&]() {
#pragma unroll
      for (int k = 0; k < 4; ++k) load_words<KW>(page_ptr + (size_t)(32 * blk + pass_token(k)) * (D * KB / 8) + ch * KCB, 64, kw[k]);
      const uint32_t* m = reinterpret_cast<const uint32_t*>(page_ptr + g.k_meta_off) + (32 * blk + lane) * ngk;
#pragma unroll
      for (int j = 0; j < NI; ++j) if (j < ngk) km[j] = m[j];
    };
    auto load_values = [&]() {
      const uint8_t* v = page_ptr + g.v_codes_off + blk * (4 * D * VB) + lane * 16;
#pragma unroll
      for (int mw = 0; mw < NMW; ++mw) vw[mw] = *reinterpret_cast<const uint4*>(v + 512 * mw);
      const uint32_t* m = reinterpret_cast<const uint32_t*>(page_ptr + g.v_meta_off) + (32 * blk + lane) * ngv;
#pragma unroll
      for (int j = 0; j < NI; ++j) if (j < ngv) vm[j] = m[j];
    };
    // The next page to load: one ahead of the one that is written.
    Tile nt{};
    int npage = 0;
    long long nx = x_lo;
    auto step = [&]() {                              // to the page behind
      ++nx;
      if (++npage == nt.seen.count) {
        npage = 0;
        if (nx < x_hi) nt = next_tile(nt);
      }
      if (nx < x_hi) find(nt, npage);
    };
    if (x_lo < x_hi) {
      nt = tile_of(sMisc[8], sMisc[9], sMisc[10]);
      npage = sMisc[11];
      find(nt, npage);
      load_keys();
      load_values();
    }
    int it = 0;
    segments([&](const Tile& t, int page0, int pages, long long x) {
#pragma unroll 1
      for (int j = 0; j < pages; ++j, ++it) {
        const int buf = it & 1, tok = t.seen.logical(page0 + j) * kPageTokens + 32 * blk;
        // scales and zero-points of this lane's token; nothing of tokens that the sequence does not hold (their bytes are anything)
        bool wide = false;
        auto checked = [&](uint32_t (&m)[4], int count, float qmax) {
#pragma unroll
          for (int e = 0; e < NI; ++e) {
            if (e < count) {
              if (tok + lane >= t.n) m[e] = 0u;
              const float2 sz = __half22float2(as_h2(m[e]));
              wide |= fabsf(sz.y) > 32752.0f || sz.x * qmax > 32752.0f;
            }
          }
        };
        checked(km, ngk, (float)((1 << KB) - 1));
        checked(vm, ngv, (float)((1 << VB) - 1));
        const bool big = bar_any(3, 128, wide);
        if (big) {
          const __half2 down = __float2half2_rn(kBigDown);
#pragma unroll
          for (int e = 0; e < NI; ++e) {
            if (e < ngk) km[e] = as_u32(__hmul2(as_h2(km[e]), down));
            if (e < ngv) vm[e] = as_u32(__hmul2(as_h2(vm[e]), down));
          }
        }
        if (it >= 2) wait_warp(bKE + 8 * buf, ((it >> 1) - 1) & 1);
        if (warp == 8 && lane == 0) sBig[it & 3] = big;
        {
          uint8_t* dst = smem + sl.k + buf * T::kK;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int u = pass_token(k), n = 32 * blk + place_of(u);
            uint8_t* row = dst + (n >> 3) * 128 + (n & 7) * 16;
            uint32_t meta = __shfl_sync(FULL, km[0], u);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
              if (i > 0 && ((32 * i) & (g.gk - 1)) == 0) {       // a new group (the same for all lanes); group (32 i) / gk
                const int e = (32 * i) / g.gk;
                meta = __shfl_sync(FULL, e == 1 ? km[1 % NI] : e == 2 ? km[2 % NI] : km[3 % NI], u);
              }
              const __half2 s = __low2half2(as_h2(meta)), z = __high2half2(as_h2(meta));
              const uint32_t c0 = key_slot<KB, KW>(kw[k], 2 * i), c1_ = key_slot<KB, KW>(kw[k], 2 * i + 1);
              *reinterpret_cast<uint4*>(row + (4 * i + ch) * T::kLbK) =
                  make_uint4(values2(c0, 0x4140u, s, z), values2(c0, 0x4342u, s, z), values2(c1_, 0x4140u, s, z), values2(c1_, 0x4342u, s, z));
            }
          }
        }
        tc::fence_async_smem();
        __syncwarp();
        if (lane == 0 && x + j != skip_x) mbar_arrive(bKF + 8 * buf);      // (skip_x: test hook - a page that never arrives)
        step();
        if (nx < x_hi) load_keys();
        if (it >= 2) wait_warp(bVE + 8 * buf, ((it >> 1) - 1) & 1);
        {
          const int vl = lane >> 2, tq = lane & 3;   // channel of eight, place of the chunk
          uint8_t* dst = smem + sl.v + buf * T::kV + vl * 16 + (4 * blk + tq) * T::kLbV;
          __half2 s[2][2], z[2][2];                  // [half][pair of tokens]
#pragma unroll
          for (int mw = 0; mw < NMW; ++mw) {
            const uint32_t ww[4] = {vw[mw].x, vw[mw].y, vw[mw].z, vw[mw].w};
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
                    const uint32_t m0 = __shfl_sync(FULL, own, 16 * kh + 2 * tq + pr), m1 = __shfl_sync(FULL, own, 16 * kh + 2 * tq + pr + 8);
                    s[kh][pr] = as_h2(permute(m0, m1, 0x5410u));
                    z[kh][pr] = as_h2(permute(m0, m1, 0x7632u));
                  }
                }
              }
#pragma unroll
              for (int rh = 0; rh < 2; ++rh) {
                constexpr uint32_t M = ((1u << VB) - 1u) * 0x01010101u;
                const uint32_t c0 = (ww[2 * rh] >> (VB * f)) & M, c1_ = (ww[2 * rh + 1] >> (VB * f)) & M;
                *reinterpret_cast<uint4*>(dst + (2 * m16 + rh) * 128) =
                    make_uint4(values2(c0, 0x4140u, s[0][0], z[0][0]), values2(c0, 0x4342u, s[0][1], z[0][1]),
                               values2(c1_, 0x4140u, s[1][0], z[1][0]), values2(c1_, 0x4342u, s[1][1], z[1][1]));
              }
            }
          }
        }
        tc::fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bVF + 8 * buf);
        if (nx < x_hi) load_values();
      }
    });
  } else if (lane == 0) {
    // =========================================================== products
    const uint32_t sk = smem_u32(smem + sl.k), sv = smem_u32(smem + sl.v), sqa = smem_u32(smem + sl.q);
    bool ok = true;
    auto wait = [&](uint32_t b, uint32_t parity) {
      if (ok && !tc::wait_or_abort(b, parity, wait_ns, abort_flag)) {
        ok = false;
        *abort_flag = 1;
        atomicOr(p.status, KVQ_STATUS_DEVICE_TIMEOUT);
      }
      return ok;
    };
    auto keys = [&](int w, int buf) {                // S = Q K^T
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
        mma_ss(tmem + kColS + 128 * w, smem_desc(sqa + w * T::kQ + 2 * k * T::kLbQ, T::kLbQ, 128), smem_desc(sk + buf * T::kK + 2 * k * T::kLbK, T::kLbK, 128),
               idesc(128), k > 0);
      tc::tc_commit(bS + 8 * w);
    };
    auto values = [&](int w, int buf, bool fresh) {  // O += P V
#pragma unroll
      for (int k = 0; k < 8; ++k)
        mma_ts(tmem + kColO + 128 * w, tmem + kColS + 128 * w + 8 * k, smem_desc(sv + buf * T::kV + 2 * k * T::kLbV, T::kLbV, 128), idesc(D), k > 0 || !fresh);
    };
    int it = 0, done[2] = {0, 0}, seg[2] = {0, 0};
    segments([&](const Tile& t, int page0, int pages, long long x) {
      const int halves = t.i * kTile + 128 < t.pairs ? 2 : 1;
      // the first page's S of both halves
      for (int w = 0; w < halves && ok; ++w) {
        if (!wait(bQ + 8 * w, seg[w] & 1)) break;
        ++seg[w];
        if (w == 0 && !wait(bKF + 8 * (it & 1), (it >> 1) & 1)) break;
        tc::tc_fence_after();
        keys(w, it & 1);
      }
      if (ok) tc::tc_commit(bKE + 8 * (it & 1));
      // then, page by page and half by half: O of this page, S of the next
      for (int j = 0; j < pages && ok; ++j, ++it) {
        const int buf = it & 1, nbuf = buf ^ 1;
        if (!wait(bVF + 8 * buf, (it >> 1) & 1)) break;
        for (int w = 0; w < halves && ok; ++w) {
          if (!wait(bP + 8 * w, done[w] & 1)) break;
          ++done[w];
          tc::tc_fence_after();
          values(w, buf, j == 0);
          if (w == halves - 1) tc::tc_commit(bVE + 8 * buf);
          if (j + 1 < pages) {
            if (w == 0 && !wait(bKF + 8 * nbuf, ((it + 1) >> 1) & 1)) break;
            tc::tc_fence_after();
            keys(w, nbuf);
            if (w == halves - 1) tc::tc_commit(bKE + 8 * nbuf);
          } else {
            tc::tc_commit(bO + 8 * w);
          }
        }
      }
    });
    // nothing of this CTA's may still run on the tensor cores when its tensor memory is freed
    tc::tc_commit(bDrain);
    mbar_wait(bDrain, 0, wait_ns);
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (warp == 12) tc::tmem_dealloc(tmem, kTmemCols);
}

template <int D, int KB, int VB>
int launch_chunk_inst(const Geom& g, const Paged& p, const void* q, float c1, float* ws, void* out, int out_dtype, unsigned long long call_id,
                      unsigned long long wait_ns, long long skip_x, cudaStream_t stream) {
  const Smem sl = smem_of<D>(g.B);
  auto kern = chunk_kernel<D, KB, VB>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, sl.total) != cudaSuccess) return KVQ_ERR_CUDA_LAUNCH;
  const long long pairs = (long long)p.max_rows * g.G;
  const cudaError_t e = launch_dependent(kern, dim3(kGrid), kThreads, sl.total, stream, 1, g, p, static_cast<const uint16_t*>(q), c1, ws,
                                         row_cap(pairs > kTile ? kTile : (int)pairs), out, out_dtype, call_id, wait_ns, skip_x);
  return e == cudaSuccess ? KVQ_OK : KVQ_ERR_CUDA_LAUNCH;
}

}  // namespace chunk
}  // namespace kvq
