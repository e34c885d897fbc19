// Paged attention of up to eight (row, head) pairs per KV head: dispatch of the decode kernel's paged instantiations.
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

}  // namespace

bool paged_decode_supported(const Geom& g) {
  return pick_paged(g, Paged{}, nullptr, 0.f, nullptr, nullptr, 0, DecodeDebug{}, nullptr, true) == KVQ_OK;
}

int launch_paged_decode(const Geom& g, const Paged& p, const void* q, void* out, int out_dtype, float c1, float* ws,
                        const DecodeDebug& dbg, cudaStream_t stream) {
  return pick_paged(g, p, q, c1, ws, out, out_dtype, dbg, stream, false);
}

}  // namespace kvq
