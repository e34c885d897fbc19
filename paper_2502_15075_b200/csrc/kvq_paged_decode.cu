// Paged attention of few rows: dispatch of the decode kernel's paged instantiations, which serve up to eight (row, head) pairs per KV head.
#include "kvq_decode_mma_kernel.cuh"

namespace kvq {
namespace mma {

// Instantiation units (kvq_paged_decode_inst_*.cu).
#define KVQ_PAGED_DECL(D, KB, VB, NGK, NGV, NH, MINB)                                                               \
  extern template int launch_paged_inst<D, KB, VB, NGK, NGV, NH, MINB>(                                             \
      const Geom&, const Paged&, const void*, float, float*, int, void*, int, unsigned long long,                   \
      unsigned long long, long long, cudaStream_t);
#include "kvq_paged_decode_list.inc"
#undef KVQ_PAGED_DECL

}  // namespace mma

namespace {

// The instantiation for this geometry; launches it unless `probe`.
int pick_paged(const Geom& g, const Paged& p, const void* q, float c1, float* ws, void* out, int out_dtype, const DecodeDebug& dbg,
               cudaStream_t stream, bool probe) {
  if (g.rows > kMaxGroupHeads || g.G * g.rows > kMaxGroupHeads) return KVQ_ERR_UNSUPPORTED;
  const int ngk = g.D / g.gk, ngv = g.D / g.gv, nh = g.G * g.rows <= 4 ? 1 : 2;
#define KVQ_PAGED_DECL(D_, KB_, VB_, NGK_, NGV_, NH_, MINB_)                                                        \
  if (g.D == D_ && g.kb == KB_ && g.vb == VB_ && ngk == NGK_ && ngv == NGV_ && NH_ == nh) {                         \
    if (mma::ring_stages(g, NH_, NGV_, false, MINB_, 5) < 2) return KVQ_ERR_UNSUPPORTED;                            \
    if (probe) return KVQ_OK;                                                                                       \
    return mma::launch_paged_inst<D_, KB_, VB_, NGK_, NGV_, NH_, MINB_>(                                            \
        g, p, q, c1, ws, flat_slot_cap(g), out, out_dtype, next_call_id(),                                          \
        dbg.wait_us ? 1000ull * dbg.wait_us : mma::kWaitTimeoutNs, dbg.skip_page, stream);                          \
  }
#include "kvq_paged_decode_list.inc"
#undef KVQ_PAGED_DECL
  return KVQ_ERR_UNSUPPORTED;
}

// Rows that one launch takes, 0 where the chunk kernel serves the call.  A launch reads every page that its rows see, up to eight pairs at
// a time, where the chunk kernel reads it once and turns it into 16-bit tiles whatever the number of pairs.  Per launch 9 us and 0.5 us for each page
// that a SM has to read, against 13 us and 2.6 us.  Measured (8B shape, 4 heads a KV head, K4V2; launches | chunk kernel): 16 sequences x 32,767
// tokens, 1 row 75 | 575 us, 2 rows 114 | 575, 4 rows 228 | 577, 6 rows 342 | 579, 8 rows 455 | 581; 64 x 2,000, 4 rows 90 | 194, 8 rows 180 | 199;
// 8 x 4,096 under a window of 1,000, 2 rows 16 | 31, 4 rows 30 | 32, 6 rows 45 | 34; 1 x 32,767, 4 rows 44 | 56, 6 rows 66 | 61; 2 x 300, 2 rows 9 | 15,
// 4 rows 18 | 16.  (The line is drawn through all of these: 1 x 32,767 with 6 rows lies on the wrong side of it.)  The lengths are not known here: the
// capacity and the window stand for them, so that short sequences in a large capacity pay for several launches.
int rows_per_launch(const Geom& g, const Paged& p) {
  const long long tokens = p.window > 0 && (long long)p.window + p.sinks < g.capacity ? (long long)p.window + p.sinks : g.capacity;
  const long long per_stream = (tokens + kPageTokens - 1) / kPageTokens + (tokens < g.capacity), pages = per_stream * g.B * g.Hkv;
  // (its prefixes over the batch are 32 bits; sequences may share pool pages, so memory does not bound them.  24: a stream's gap, and the
  // pages at a window's and the first tokens' ends)
  if ((per_stream + 24) * g.B * g.Hkv > 0x7FFFFFFFll) return 0;
  for (int pairs = kMaxGroupHeads; pairs >= 4; pairs -= 4) {
    Geom part = g;
    part.rows = g.rows < pairs / g.G ? g.rows : pairs / g.G;
    if (part.rows < 1) continue;
    const long long launches = ((long long)g.rows + part.rows - 1) / part.rows;
    if (launches > 5 || (launches > 1 && launches * (9 * 1480 + 5 * pages) >= 13 * 1480 + 26 * pages)) continue;      // (26 / 5: six never win)
    if (pick_paged(part, p, nullptr, 0.f, nullptr, nullptr, 0, DecodeDebug{}, nullptr, true) == KVQ_OK) return part.rows;
  }
  return 0;
}

}  // namespace

bool paged_decode_serves(const Geom& g, const Paged& p) { return rows_per_launch(g, p) > 0; }

int paged_decode_launches(const Geom& g, const Paged& p) {
  const int step = rows_per_launch(g, p);
  return step > 0 ? (g.rows + step - 1) / step : 0;      // (a few: rows_per_launch sees to it)
}

size_t paged_decode_workspace_bytes(const Geom& g) {
  Geom part = g;
  part.rows = g.rows < kMaxGroupHeads / g.G ? g.rows : kMaxGroupHeads / g.G;
  return part.rows > 0 ? flat_workspace_bytes(part) : 0;
}

int launch_paged_decode(const Geom& g, const Paged& p, const void* q, void* out, int out_dtype, float c1, float* ws,
                        const DecodeDebug& dbg, cudaStream_t stream) {
  const int step = rows_per_launch(g, p);
  Geom part = g;
  Paged rows = p;
  for (; rows.from < g.rows; rows.from += step) {
    part.rows = g.rows - rows.from < step ? g.rows - rows.from : step;
    const int rc = pick_paged(part, rows, q, c1, ws, out, out_dtype, dbg, stream, false);
    if (rc != KVQ_OK) return rc;
  }
  return KVQ_OK;
}

}  // namespace kvq
