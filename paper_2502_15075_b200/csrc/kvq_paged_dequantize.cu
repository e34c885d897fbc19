// kvq_paged_dequantize: x^ = fmaf(code, scale, zero) rounded to the 16-bit input type, for the rows of a ragged call.
#include "kvq_paged.cuh"

namespace kvq {

namespace {

constexpr int kThreads = 256;

__global__ void __launch_bounds__(kThreads) paged_dequant_kernel(Geom g, Paged p, uint16_t* k_out, uint16_t* v_out) {
  const int lane = threadIdx.x & 31;
  const long long task = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  begin_after_predecessor();
  const int row = (int)(task / g.Hkv), h = (int)(task % g.Hkv);
  if (row >= p.n_rows) return;
  const int b = sequence_of(p.cu, g.B, row, lane);
  bool bad;
  const SeqRows s = seq_rows(p, b, g.capacity, p.n_rows, bad);
  if (bad && lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
  if (row < s.first || row >= s.first + s.rows) return;
  const int t = s.n - s.rows + (row - s.first), id = pool_page(p, b, t >> 7);
  if (id < 0) {
    if (lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
    return;
  }
  const uint8_t* pg = p.pages + ((size_t)id * g.Hkv + h) * g.page_bytes;
  const int tp = t & 127;
  const size_t at = ((size_t)row * g.Hkv + h) * g.D;
  for (int d = lane; d < g.D; d += 32) {
    for (int is_v = 0; is_v < 2; ++is_v) {
      uint16_t* out = is_v ? v_out : k_out;
      if (!out) continue;
      const int bits = is_v ? g.vb : g.kb, gs = is_v ? g.gv : g.gk;
      const uint32_t m = reinterpret_cast<const uint32_t*>(pg + (is_v ? g.v_meta_off : g.k_meta_off))[tp * (g.D / gs) + d / gs];
      const float code = (float)load_code_any(pg + (is_v ? g.v_codes_off : 0), is_v, tp, d, g.D, bits);
      const float2 sz = __half22float2(*reinterpret_cast<const __half2*>(&m));
      out[at + d] = f32_to_bits16(fmaf(code, sz.x, sz.y), g.in_dtype);
    }
  }
}

}  // namespace

int launch_paged_dequantize(const Geom& g, const Paged& p, void* k_out, void* v_out, cudaStream_t stream) {
  const long long ctas = ((long long)p.n_rows * g.Hkv + kThreads / 32 - 1) / (kThreads / 32);
  if (ctas > 0x7FFFFFFFll) return KVQ_ERR_INVALID_ARG;
  const cudaError_t e = launch_dependent(paged_dequant_kernel, dim3((unsigned)ctas), kThreads, 0, stream, 1, g, p,
                                         static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out));
  return e == cudaSuccess ? KVQ_OK : KVQ_ERR_CUDA_LAUNCH;
}

}  // namespace kvq
