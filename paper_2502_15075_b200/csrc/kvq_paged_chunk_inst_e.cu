// Explicit instantiations of the chunk kernel (split over several files to compile in parallel).
#include "kvq_paged_chunk.cuh"

namespace kvq {
namespace chunk {
#define KVQ_CHUNK_DECL(D, KB, VB)                                                                                  \
  template int launch_chunk_inst<D, KB, VB>(const Geom&, const Paged&, const void*, float, float*, void*, int,     \
                                            unsigned long long, unsigned long long, long long, cudaStream_t);
KVQ_CHUNK_DECL(64, 2, 2)
KVQ_CHUNK_DECL(64, 2, 4)
KVQ_CHUNK_DECL(64, 2, 8)
#undef KVQ_CHUNK_DECL
}  // namespace chunk
}  // namespace kvq
