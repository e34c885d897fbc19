// Paged attention of many query rows: dispatch of the chunk kernel.
#include "kvq_paged_chunk.cuh"

namespace kvq {
namespace chunk {

// Instantiation units (kvq_paged_chunk_inst_*.cu).
#define KVQ_CHUNK_DECL(D, KB, VB)                                                                                         \
  extern template int launch_chunk_inst<D, KB, VB>(const Geom&, const Paged&, const void*, float, float*, void*, int,     \
                                                   unsigned long long, unsigned long long, long long, cudaStream_t);
#include "kvq_paged_chunk_list.inc"
#undef KVQ_CHUNK_DECL

}  // namespace chunk

size_t paged_chunk_workspace_bytes(const Geom& g) {
  const long long pairs = (long long)g.rows * g.G;
  return chunk::workspace_bytes(chunk::row_cap(pairs > chunk::kTile ? chunk::kTile : (int)pairs), g.D);
}

int launch_paged_chunk(const Geom& g, const Paged& p, const void* q, void* out, int out_dtype, float c1, float* ws,
                       const DecodeDebug& dbg, cudaStream_t stream) {
#define KVQ_CHUNK_DECL(D_, KB_, VB_)                                                                                      \
  if (g.D == D_ && g.kb == KB_ && g.vb == VB_)                                                                            \
    return chunk::launch_chunk_inst<D_, KB_, VB_>(g, p, q, c1, ws, out, out_dtype, next_call_id(),                        \
                                                  dbg.wait_us ? 1000ull * dbg.wait_us : mma::kWaitTimeoutNs, dbg.skip_page, stream);
#include "kvq_paged_chunk_list.inc"
#undef KVQ_CHUNK_DECL
  return KVQ_ERR_UNSUPPORTED;
}

}  // namespace kvq
