// What the kernels of the paged cache share: its pointers, the checks of everything that comes from device memory, and the pages that a
// sequence's rows see under a sliding window with first tokens that stay visible.
#pragma once

#include "kvq_internal.h"

namespace kvq {

// A paged cache and a ragged call on it (device memory).
struct Paged {
  uint8_t* pages;            // [n_pool][Hkv][page_bytes]
  const int32_t* table;      // pool page of tokens 128 i .. of sequence b: table[b * table_stride + i]
  long long table_stride;
  const int32_t* seq_len;    // [B], the call's tokens counted in
  const int32_t* cu;         // [B + 1]
  uint32_t* status;
  int n_pool, n_rows;
  int max_rows, window, sinks;      // attention only (window 0: none)
  int from;                         // decode kernel: the launch serves each sequence's rows from .. from + g.rows - 1
};

struct RopeArgs { const float *cos, *sin; int n_positions, half, interleaved; };      // half: rotary_dim / 2, 0 without a rotation

// The rows of a sequence in a call: rows first .. first + rows - 1 are the last `rows` of its n tokens.
struct SeqRows { int n, rows, first; };

// ... of sequence b, checked; `rows` is 0 where something is out of range (then `bad` says so).
__device__ __forceinline__ SeqRows seq_rows(const Paged& p, int b, int limit, int max_rows, bool& bad) {
  const int c0 = p.cu[b], c1 = p.cu[b + 1], n = p.seq_len[b];
  bad = c0 < 0 || c1 < c0 || c1 > p.n_rows || n < 0 || n > limit;
  bad = bad || c1 - c0 > n || c1 - c0 > max_rows;
  return SeqRows{bad ? 0 : n, bad ? 0 : c1 - c0, bad ? 0 : c0};
}

// Says what is out of range in a call (one warp of it), of sequences without rows too: those are nobody's task.
__device__ __forceinline__ void report_bad_input(const Paged& p, int B, int limit, int lane) {
  for (int b = lane; b < B; b += 32) {
    bool bad;
    seq_rows(p, b, limit, p.n_rows, bad);
    if (bad) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
  }
}

// Rows from .. from + most - 1 of a sequence alone: as a call of just these tokens.
__device__ __forceinline__ SeqRows part_of(const SeqRows& s, int from, int most) {
  const int rows = min(max(s.rows - from, 0), most);
  return SeqRows{rows > 0 ? s.n - (s.rows - from - rows) : s.n, rows, s.first + from};
}

// The sequence of row i: the number of ends cu[1 ..] at or below it.  The whole warp asks for the same row.  (Offsets out of order lead to some
// sequence, here and by blocks below; looking at all of them first costs appends and read-backs 3 %.)
__device__ __forceinline__ int sequence_of(const int32_t* cu, int B, int i, int lane) {
  int lo = 0, len = B;                           // the answer is in lo .. lo + len - 1 (or B, which the caller's check finds out)
  while (len > 32) {
    const int step = (len + 31) >> 5, at = lo + lane * step;            // first entries of up to 32 pieces
    const bool below = at < lo + len && cu[at] <= i;                    // (cu[b] <= i for the answer b and all before it)
    const int k = __popc(__ballot_sync(0xffffffffu, below));
    const int piece = k > 0 ? k - 1 : 0, end = lo + len;
    lo += piece * step;
    len = min(step, end - lo);
  }
  const bool passed = lane < len && cu[lo + lane + 1] <= i;
  return min(lo + __popc(__ballot_sync(0xffffffffu, passed)), B - 1);
}

// The rows of a call by aligned blocks of `span` tokens of their sequences (a power of two): block `slot` of at most block_tasks(...) of them.
// Sequence b has the slots from cu[b] / span + 2 b on: r rows touch at most r / span + 2 blocks.
struct BlockTask { int b, t0, lo, hi; long long row0; };      // tokens t0 + lo .. t0 + hi - 1 of sequence b are rows row0 + lo .. (lo >= hi: none)
__host__ __device__ inline long long block_tasks(int n_rows, int B, int span) { return n_rows / span + 2ll * B; }
__device__ __forceinline__ BlockTask block_task(const Paged& p, int B, int slot, int span, int limit, int max_rows, int lane) {
  int lo = 0, len = B;                           // the last sequence whose slots start at or below this one, in pieces as in sequence_of
  while (len > 1) {
    const int step = (len + 31) >> 5, at = lo + lane * step;
    const bool below = at < lo + len && p.cu[at] / span + 2 * at <= slot;
    const int k = __popc(__ballot_sync(0xffffffffu, below));
    const int piece = k > 0 ? k - 1 : 0, end = lo + len;
    lo += piece * step;
    len = min(step, end - lo);
  }
  bool bad;
  const SeqRows s = seq_rows(p, lo, limit, max_rows, bad);
  BlockTask t{lo, 0, 0, 0, 0};
  if (s.rows == 0) return t;
  const int start = s.n - s.rows, skipped = slot - (s.first / span + 2 * lo);
  if (skipped < 0) return t;
  const long long t0 = (long long)(start / span) * span + (long long)skipped * span;
  if (t0 >= s.n) return t;
  t.t0 = (int)t0;
  t.lo = max(start - t.t0, 0);
  t.hi = min(s.n - t.t0, span);
  t.row0 = (long long)s.first - start + t.t0;
  return t;
}

// Pool page of logical page `page` of sequence b, or -1 (outside the pool).
__device__ __forceinline__ int pool_page(const Paged& p, int b, int page) {
  const int id = p.table[(long long)b * p.table_stride + page];
  return (unsigned)id < (unsigned)p.n_pool ? id : -1;
}

// Logical pages that tokens of positions p0 .. p1 see (p0 <= p1, rows of a call): `first` pages from the sequence's start, then those
// from page `low` on; `count` in all.  Page i of them is logical page i < first ? i : i + skip.
struct SeenPages {
  int count, first, skip;
  __host__ __device__ __forceinline__ int logical(int i) const { return i < first ? i : i + skip; }
};
__host__ __device__ __forceinline__ SeenPages seen_pages(int p0, int p1, int window, int sinks) {
  const int reach = p0 - window + 1;                                    // first token that the window of the earliest row holds
  const int low = window > 0 && reach > 0 ? reach >> 7 : 0;
  const int first = min((int)(((unsigned)sinks + 127u) >> 7), low);
  return SeenPages{(p1 >> 7) + 1 - low + first, first, low - first};
}

int launch_paged_append(const Geom& g, const Paged& p, const void* k, const void* v, int64_t kv_row, int64_t kv_head,
                        const RopeArgs& rope, const void* q, int64_t q_row, int64_t q_head, void* q_out, cudaStream_t stream);
int launch_paged_dequantize(const Geom& g, const Paged& p, void* k_out, void* v_out, cudaStream_t stream);
// few rows (g.rows: the most rows of a sequence), where it serves the call; bytes of workspace behind the count words for any window
bool paged_decode_serves(const Geom& g, const Paged& p);
int paged_decode_launches(const Geom& g, const Paged& p);      // 0 where it does not
size_t paged_decode_workspace_bytes(const Geom& g);
int launch_paged_decode(const Geom& g, const Paged& p, const void* q, void* out, int out_dtype, float scale_log2e, float* ws,
                        const DecodeDebug& dbg, cudaStream_t stream);
// any number of rows
size_t paged_chunk_workspace_bytes(const Geom& g);
int launch_paged_chunk(const Geom& g, const Paged& p, const void* q, void* out, int out_dtype, float scale_log2e, float* ws,
                       const DecodeDebug& dbg, cudaStream_t stream);

}  // namespace kvq
