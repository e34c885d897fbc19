// Explicit instantiations of the decode kernel for paged caches (split over several files to compile in parallel).
#include "kvq_decode_mma_kernel.cuh"

namespace kvq {
namespace mma {
#define KVQ_PAGED_DECL(D, KB, VB, NGK, NGV, NH, MINB)                                                               \
  template int launch_paged_inst<D, KB, VB, NGK, NGV, NH, MINB>(                                                    \
      const Geom&, const Paged&, const void*, float, float*, int, void*, int, unsigned long long,                   \
      unsigned long long, long long, cudaStream_t);
KVQ_PAGED_DECL(64, 4, 2, 1, 1, 2, 2)
KVQ_PAGED_DECL(64, 4, 2, 2, 2, 2, 2)
#undef KVQ_PAGED_DECL
}  // namespace mma
}  // namespace kvq
